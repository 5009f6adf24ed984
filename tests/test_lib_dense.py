"""CPU: the dense block's entry points refuse what they do not take, before anything is launched (the pointers are never followed)."""
import ctypes as C

import pytest
import torch

import paper_2107_00961_amd as R
from paper_2107_00961_amd import binding as B

P = 256   # an aligned address that nothing reads
EINVAL, ESHAPE, EWORKSPACE = -1, -2, -3


def ln_fwd(M=4, N=8, dt=0, x=P, ldx=0, gamma=P, beta=P, eps=1e-5, y=P, ldy=0, mean=P, rstd=P):
    return R.lib().resist_layernorm_forward(M, N, dt, x, ldx, gamma, beta, eps, y, ldy, mean, rstd, None)


def ln_bwd(M=4, N=8, dt=0, dy=P, lddy=0, x=P, ldx=0, gamma=P, mean=P, rstd=P, addend=None, lda=0, dx=P, lddx=0, dg=P, db=P, ws=P, n=1 << 30):
    return R.lib().resist_layernorm_backward(M, N, dt, dy, lddy, x, ldx, gamma, mean, rstd, addend, lda, dx, lddx, dg, db, ws, n, None)


def drop_fwd(M=4, N=8, dt=0, x=P, ldx=0, p=0.1, rng=P, res=None, ldr=0, y=P, ldy=0):
    return R.lib().resist_dropout_forward(M, N, dt, x, ldx, p, rng, res, ldr, y, ldy, None)


def drop_bwd(M=4, N=8, dt=0, dy=P, lddy=0, p=0.1, rng=P, act=2, z=P, ldz=0, dx=P, lddx=0):
    return R.lib().resist_dropout_backward(M, N, dt, dy, lddy, p, rng, act, z, ldz, dx, lddx, None)


@pytest.mark.parametrize("call", [ln_fwd, ln_bwd, drop_fwd, drop_bwd])
@pytest.mark.parametrize("kw,rc", [(dict(dt=2), EINVAL), (dict(dt=-1), EINVAL), (dict(M=-1), ESHAPE), (dict(M=1 << 31), ESHAPE),
                                   (dict(N=0), ESHAPE), (dict(N=-3), ESHAPE), (dict(N=(1 << 24) + 1), ESHAPE)])
def test_row_operators_sizes(call, kw, rc):
    assert call(**kw) == rc and R.lib().resist_last_error()


@pytest.mark.parametrize("call,names", [(ln_fwd, ["x", "y"]), (ln_bwd, ["dy", "x", "dx", "mean", "rstd", "ws"]), (drop_fwd, ["x", "y", "rng"]),
                                        (drop_bwd, ["dy", "z", "dx", "rng"])])
def test_row_operators_pointers(call, names):
    for n in names:
        assert call(**{n: None}) == EINVAL, n
        assert call(**{n: P + 4}) == EINVAL, n


def test_row_operators_optional_pointers_are_aligned():
    for n in ("gamma", "beta", "mean", "rstd"):
        assert ln_fwd(**{n: P + 4}) == EINVAL
    for n in ("gamma", "addend", "dg", "db"):
        assert ln_bwd(**{n: P + 8}) == EINVAL
    assert drop_fwd(res=P + 2) == EINVAL


@pytest.mark.parametrize("call,names", [(ln_fwd, ["ldx", "ldy"]), (ln_bwd, ["lddy", "ldx", "lddx"]), (drop_fwd, ["ldx", "ldy"]),
                                        (drop_bwd, ["lddy", "ldz", "lddx"])])
def test_row_operators_strides(call, names):
    for n in names:
        assert call(**{n: 7}) == ESHAPE, n
        assert call(**{n: -8}) == ESHAPE, n
        assert call(**{n: 1 << 41}) == ESHAPE, n


def test_row_operators_values():
    for eps in (-1e-9, float("nan")):
        assert ln_fwd(eps=eps) == EINVAL
    for p in (-0.1, 1.0, 1.5, float("nan"), 1 - 1e-12):
        assert drop_fwd(p=p) == EINVAL and drop_bwd(p=p) == EINVAL
    assert drop_bwd(act=5) == EINVAL and drop_bwd(act=-1) == EINVAL
    n = C.c_int64()
    assert R.lib().resist_layernorm_workspace_bytes(1000, 512, C.byref(n)) == 0 and n.value > 0
    assert ln_bwd(M=1000, N=512, n=n.value - 1) == EWORKSPACE
    assert R.lib().resist_layernorm_workspace_bytes(1000, 512, None) == EINVAL
    assert R.lib().resist_layernorm_workspace_bytes(-1, 512, C.byref(n)) == ESHAPE


def test_no_rows_is_no_work():
    """Without rows there is nothing to read or write: no pointer is needed, and nothing is launched."""
    assert ln_fwd(M=0, x=None, y=None, mean=None, rstd=None) == 0
    assert ln_bwd(M=0, dy=None, x=None, dx=None, mean=None, rstd=None, dg=None, db=None, ws=None, n=0) == 0
    assert drop_fwd(M=0, x=None, y=None) == 0 and drop_bwd(M=0, dy=None, z=None, dx=None) == 0
    assert linear(0, M=0, x=None, w=None, y=None) == 0 and linear(1, M=0, x=None, w=None, y=None) == 0


def linear(op, M=4, K=8, N=8, ldx=0, ldy=0, dt=0, x=P, w=P, y=P, dw=P, db=P, ws=P, n=1 << 40, **e):
    L, sh = R.lib(), B._LinearShape(M, K, N, ldx, ldy, dt)
    if op == 0:
        ep = B._LinearEpilogue(e.get("bias", P), e.get("act", 0), e.get("p", 0.0), e.get("rng"), e.get("residual"), e.get("ldr", 0), e.get("z"), e.get("ldz", 0))
        return L.resist_linear_forward(C.byref(sh), x, w, C.byref(ep), y, ws, n, None)
    if op == 1:
        th = B._LinearThrough(e.get("act", 0), e.get("z"), e.get("ldz", 0), e.get("p", 0.0), e.get("rng"))
        return L.resist_linear_dgrad(C.byref(sh), x, w, C.byref(th), y, ws, n, None)
    return L.resist_linear_wgrad(C.byref(sh), x, y, dw, db, ws, n, None)


@pytest.mark.parametrize("op", [0, 1, 2])
@pytest.mark.parametrize("kw,rc", [(dict(dt=3), EINVAL), (dict(M=-1), ESHAPE), (dict(M=1 << 31), ESHAPE), (dict(K=0), ESHAPE), (dict(N=0), ESHAPE),
                                   (dict(K=(1 << 20) + 1), ESHAPE), (dict(N=(1 << 20) + 1), ESHAPE), (dict(ldx=7), ESHAPE), (dict(ldy=7), ESHAPE),
                                   (dict(ldx=(1 << 20) + 1), ESHAPE), (dict(ldy=-1), ESHAPE), (dict(x=None), EINVAL), (dict(y=None), EINVAL),
                                   (dict(x=P + 8), EINVAL), (dict(y=P + 2), EINVAL)])
def test_linear_refusals(op, kw, rc):
    assert linear(op, **kw) == rc and R.lib().resist_last_error()


def test_linear_epilogue_refusals():
    for op in (0, 1):
        assert linear(op, w=None) == EINVAL and linear(op, w=P + 4) == EINVAL
        assert linear(op, act=5, z=P) == EINVAL and linear(op, p=1.0, rng=P) == EINVAL and linear(op, p=0.5) == EINVAL
        assert linear(op, p=0.5, rng=P + 4) == EINVAL
        assert linear(op, act=2, z=P, ldz=7) == ESHAPE and linear(op, act=2, z=P + 2) == EINVAL
    assert linear(0, bias=P + 4) == EINVAL and linear(0, residual=P + 4) == EINVAL and linear(0, residual=P, ldr=7) == ESHAPE
    assert linear(1, act=2) == EINVAL                                      # an activation's gradient without z
    assert linear(2, dw=P + 4) == EINVAL and linear(2, db=P + 4) == EINVAL and linear(2, dw=None) == EINVAL and linear(2, M=0, dw=None) == EINVAL
    n = C.c_int64()
    sh = B._LinearShape(4, 8, 8, 0, 0, 0)
    L = R.lib()
    assert L.resist_linear_workspace_bytes(C.byref(sh), 3, C.byref(n)) == EINVAL and L.resist_linear_workspace_bytes(C.byref(sh), -1, C.byref(n)) == EINVAL
    assert L.resist_linear_workspace_bytes(C.byref(sh), 0, None) == EINVAL and L.resist_linear_workspace_bytes(None, 0, C.byref(n)) == EINVAL
    assert L.resist_linear_forward(None, P, P, None, P, None, 0, None) == EINVAL


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("op", [0, 1, 2])
def test_linear_workspace_is_asked_for(op, dt):
    """Where a shape needs a workspace, a smaller one, a misaligned one or none is refused."""
    n = C.c_int64()
    for M, K, N in ((1, 4096, 4096), (333, 1000, 2051), (2000, 1024, 1024), (130, 257, 129)):
        sh = B._LinearShape(M, K, N, 0, 0, dt)
        assert R.lib().resist_linear_workspace_bytes(C.byref(sh), op, C.byref(n)) == 0 and n.value >= 0
        if n.value:
            assert linear(op, M, K, N, dt=dt, n=n.value - 1) == EWORKSPACE
            assert linear(op, M, K, N, dt=dt, ws=None) == EINVAL and linear(op, M, K, N, dt=dt, ws=P + 8) == EINVAL


def test_binding_refusals_need_no_gpu():
    x = torch.zeros(4, 8)
    for call in (lambda: R.layernorm_forward(x), lambda: R.layernorm_backward(x, x, None, x[:, 0], x[:, 0]), lambda: R.dropout_forward(x, 0.1, None),
                 lambda: R.dropout_backward(x, 0.1, None), lambda: R.linear_forward(x, x), lambda: R.linear_dgrad(x, x), lambda: R.linear_wgrad(x, x)):
        with pytest.raises(R.ResistError, match="device tensors"):
            call()
    with pytest.raises(R.ResistError, match="matrix"):
        B._matrix(x[0], "x")
    with pytest.raises(R.ResistError, match="shape"):
        B._matrix(x, "x", x, (4, 9))
    with pytest.raises(R.ResistError, match="beside"):
        B._matrix(x.double(), "x", x)
    with pytest.raises(R.ResistError, match="without elements"):
        B._matrix(x[:, :0], "x")
    with pytest.raises(R.ResistError, match="gamma"):
        B._vector(x[0].double(), "gamma", 8, x)
    with pytest.raises(R.ResistError, match="gamma"):
        B._vector(x[0], "gamma", 9, x)
    with pytest.raises(R.ResistError, match="rng"):
        B._rng_ptr(None, 0.5, x)
    for bad in (torch.zeros(3, dtype=torch.int64), torch.zeros(2), torch.zeros(4, dtype=torch.int64)[::2]):
        with pytest.raises(R.ResistError, match="rng"):
            B._rng_ptr(bad, 0.5, x)
    with pytest.raises(R.ResistError, match="act"):
        B._activation("tanh")
    with pytest.raises(R.ResistError, match="w:"):
        B._weights(torch.zeros(3, 7), x, K=8)


def test_rows_the_library_cannot_take_are_copied():
    x = torch.arange(80.0).reshape(8, 10)
    assert B._matrix(x[:, :4], "x").data_ptr() == x.data_ptr() and B._ld(x[:, :4]) == 10     # apart, as they are
    for v in (x[:, 1:5], x.t(), x[:1].expand(3, 10), x[:, ::2]):
        c = B._matrix(v, "x")
        assert c.is_contiguous() and c.data_ptr() % 16 == 0 and torch.equal(c, v)
    assert B._ld(x[:1, :4]) == 0
