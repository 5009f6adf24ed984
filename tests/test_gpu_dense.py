"""GPU parity: layer norm, dropout, dense layers and their gradients against the float64 oracle, element by element.

Tolerances, U = 2^-24 (half a step of fp32): a sum of n terms in fp32 is off by about sqrt(n) U times the sum of their magnitudes S
(the roundings of its steps are independent), 4 sqrt(n) + 4 leaves a factor of four and the roundings of the terms; sums taken in a tree
(rows of a layer norm: at most 4 vectors of 8 a thread, or N/2048 of them, then 8 levels) get the number of their steps instead.
Activations and derivatives: 16 U times max(1, |z|), what an argument rounded a few times and a correctly rounded function of it
leave.  A stored bf16 is off by half a step, 2^-8 relative."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2107_00961_amd as R
from oracle import dense as D
from paper_2107_00961_amd import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": U, "bf16": 2.0 ** -8}
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def dev(a, dt="f32"):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda").to(DT[dt])


def host(t):
    return t.detach().double().cpu().numpy()


def rounded(a, dt):
    """-> (device tensor, its values in float64)."""
    t = dev(a, dt)
    return t, host(t)


def apart(a, dt, extra):
    """The same as rows of a wider matrix whose other columns are NaN."""
    m, n = a.shape
    wide = torch.full((m, n + extra), float("nan"), dtype=DT[dt], device="cuda")
    wide[:, :n] = dev(a, dt)
    return wide[:, :n], host(wide[:, :n])


def near(got, want, tol, what):
    got, want, tol = host(got) if torch.is_tensor(got) else got, np.asarray(want), np.broadcast_to(tol, np.shape(want))
    assert got.shape == want.shape, what
    assert np.isfinite(got).all(), f"{what}: not finite"
    err = np.abs(got - want)
    if (err > tol).any():
        i = np.unravel_index(np.argmax(err / tol), err.shape)
        raise AssertionError(f"{what}: {(err > tol).sum()} of {err.size} off; worst at {i}: {got[i]:.9g} for {want[i]:.9g}, tolerance {tol[i]:.3g}")


def rng_tensor(seed, offset):
    return torch.tensor([seed, offset], dtype=torch.int64, device="cuda")


# ---- layer norm ----------------------------------------------------------------------------------------------------
ROWS = [(1, 1), (3, 2), (5, 7), (4, 8), (1, 4096), (9, 63), (70, 512), (33, 513), (7, 1024), (6, 1025), (5, 2049), (3, 4100), (2, 8192), (3, 8193), (2, 20001),
        (1500, 64), (1100, 1040)]


def row_steps(n):
    return 48 + n / 2048


def ln_data(m, n, seed, dt):
    g = np.random.default_rng(seed)
    x = (g.standard_normal((m, n)) * g.uniform(0.2, 5, (m, 1)) + g.standard_normal((m, 1)) * 4).astype(np.float32)
    return x, (1 + 0.3 * g.standard_normal(n)).astype(np.float32), (0.3 * g.standard_normal(n)).astype(np.float32), g.standard_normal((m, n)).astype(np.float32)


def check_ln_fwd(x, gamma, beta, eps, out, dt, what):
    y, mean, rstd = D.layernorm(x, gamma, beta, eps)
    steps = row_steps(x.shape[1])
    e_mean = steps * U * np.abs(x).mean(1)
    var = 1 / rstd ** 2
    rel = (steps + 8) * U + e_mean ** 2 / var
    near(out[1], mean, e_mean + U * np.abs(mean) + 1e-45, f"{what} mean")
    near(out[2], rstd, rel * rstd, f"{what} rstd")
    g = np.ones(x.shape[1]) if gamma is None else np.abs(gamma)
    xhat = np.abs((x - mean[:, None]) * rstd[:, None])
    tol = g * (e_mean[:, None] * rstd[:, None] * (1 + rel[:, None]) + xhat * (rel[:, None] + 6 * U)) + 4 * U * np.abs(y) + HALF[dt] * np.abs(y) * 1.01
    if beta is not None:
        tol = tol + 2 * U * np.abs(beta)
    near(out[0], y, tol + 1e-38, f"{what} y")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("m,n", ROWS)
def test_layernorm_forward(m, n, dt):
    print("layernorm_forward", m, n, dt, flush=True)
    x, gamma, beta, _ = ln_data(m, n, n, dt)
    xd, x64 = rounded(x, dt)
    check_ln_fwd(x64, gamma.astype(np.float64), beta.astype(np.float64), 1e-5, R.layernorm_forward(xd, dev(gamma), dev(beta)), dt, "affine")
    xd, x64 = apart(x, dt, 3)
    check_ln_fwd(x64, None, None, 1e-3, R.layernorm_forward(xd, eps=1e-3), dt, "plain, rows apart")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_layernorm_rows_of_one_value_and_not_finite(dt):
    x = np.ones((6, 1030), np.float32) * np.array([0, 1, -3, 1000, 2, 0.5], np.float32)[:, None]
    x[4, 7], x[5, 1029] = np.inf, np.nan
    xd, x64 = rounded(x, dt)
    y, mean, rstd = R.layernorm_forward(xd)
    check_ln_fwd(x64[:4], None, None, 1e-5, (y[:4], mean[:4], rstd[:4]), dt, "constant rows")
    assert not torch.isfinite(y[4]).any() and torch.isnan(y[5]).all()       # and no other row


def check_ln_bwd(dy, x, gamma, mean, rstd, addend, out, dt, what):
    dx, dg, db = D.layernorm_backward(dy, x, gamma, mean, rstd, addend)
    h = np.abs((x - mean[:, None]) * rstd[:, None])
    g = np.abs(dy if gamma is None else dy * gamma)
    steps = row_steps(x.shape[1]) + 6
    s1, s2 = g.mean(1, keepdims=True), (g * h).mean(1, keepdims=True)
    tol = rstd[:, None] * (8 * U * (g + s1 + h * s2) + steps * U * (s1 + h * s2)) + 2 * U * np.abs(dx) + HALF[dt] * np.abs(dx) * 1.01
    if addend is not None:
        tol = tol + 2 * U * np.abs(addend)
    near(out[0], dx, tol + 1e-38, f"{what} dx")
    cols = x.shape[0] / 128 + 12
    near(out[1], dg, cols * U * (np.abs(dy) * h).sum(0) + 1e-38, f"{what} dgamma")
    near(out[2], db, cols * U * np.abs(dy).sum(0) + 1e-38, f"{what} dbeta")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("m,n", ROWS)
def test_layernorm_backward(m, n, dt):
    print("layernorm_backward", m, n, dt, flush=True)
    x, gamma, _, dy = ln_data(m, n, n + 1, dt)
    xd, x64 = rounded(x, dt)
    _, mean, rstd = D.layernorm(x64)
    mean, rstd = dev(mean.astype(np.float32)), dev(rstd.astype(np.float32))
    dyd, dy64 = rounded(dy, dt)
    check_ln_bwd(dy64, x64, gamma.astype(np.float64), host(mean), host(rstd), None, R.layernorm_backward(dyd, xd, dev(gamma), mean, rstd), dt, "affine")
    xd, x64 = apart(x, dt, 5)
    dyd, dy64 = apart(dy, dt, 9)
    ad, ad64 = apart(dy[::-1].copy(), dt, 1)
    out = R.layernorm_backward(dyd, xd, None, mean, rstd, addend=ad)
    check_ln_bwd(dy64, x64, None, host(mean), host(rstd), ad64, out, dt, "plain, addend, rows apart")
    again = R.layernorm_backward(dyd, xd, None, mean, rstd, addend=ad)
    assert all(torch.equal(a, b) for a, b in zip(out, again))


# ---- dropout -------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("m,n", [(1, 1), (2, 3), (1, 4096), (5, 8), (33, 17), (300, 513), (1000, 64), (40, 20001)])
def test_dropout(m, n, dt):
    print("dropout", m, n, dt, flush=True)
    g = np.random.default_rng(n)
    x, res = g.standard_normal((m, n)).astype(np.float32), g.standard_normal((m, n)).astype(np.float32)
    for p, seed, offset in ((0.1, 5, 0), (0.5, -1, (1 << 63) - 5), (0.999, 1 << 62, -3)):
        rng = rng_tensor(seed, offset)
        xd, x64 = apart(x, dt, 3)
        rd, r64 = apart(res, dt, 6)
        want = D.dropout(x64, p, (seed, offset))
        got = R.dropout_forward(xd, p, rng)
        near(got, want, (4 * U + HALF[dt] * 1.01) * np.abs(want), f"p {p}")
        assert np.array_equal(host(got) == 0, want == 0) or dt == "bf16"
        near(R.dropout_forward(xd, p, rng, residual=rd), want + r64, 4 * U * np.abs(want) + (U + HALF[dt] * 1.01) * np.abs(want + r64), f"p {p} residual")
    xd, x64 = rounded(x, dt)
    assert torch.equal(R.dropout_forward(xd, 0.0, None), xd)


def test_dropped_elements_are_zero_whatever_they_were():
    m, n, p = 16, 65, 0.5
    keep = torch.from_numpy(D.kept((3, 4), m, n, p)).cuda()
    for bad in (float("nan"), float("inf"), -float("inf")):
        x = torch.where(keep, 1.0, bad)
        assert torch.equal(R.dropout_forward(x, p, rng_tensor(3, 4)), torch.where(keep, 2.0, 0.0))
        w = torch.eye(n, device="cuda")
        assert torch.equal(R.dropout_forward(x.bfloat16(), p, rng_tensor(3, 4)).float(), torch.where(keep, 2.0, 0.0))
        assert torch.equal(R.linear_forward(torch.ones(m, n, device="cuda"), w, p=p, rng=rng_tensor(3, 4)), torch.where(keep, 2.0, 0.0))


def slopes(z):
    return np.concatenate([z, np.array([0.0, -0.0, 1e-30, -1e-30, 15.0, -15.0, 60.0, -60.0, 3e5, -3e5, 1e19, -1e19, 3e38, -3e38])])


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("act", ACTS)
def test_gradient_through_dropout_and_activation(act, dt):
    g = np.random.default_rng(11)
    z = slopes(g.standard_normal(511 * 3 - 14) * 3).astype(np.float32).reshape(3, 511)
    dy = g.standard_normal(z.shape).astype(np.float32)
    zd, z64 = apart(z, dt, 2)
    dyd, dy64 = rounded(dy, dt)
    for p in (0.0, 0.3):
        keep = D.kept((1, 2), *z.shape, p)
        with np.errstate(over="ignore", invalid="ignore"):
            s = D.slope(z64, act)
        s = np.where(np.isfinite(s), s, (z64 > 0) * 1.0)     # where the oracle's own powers of z overflow: 0 or 1
        want = np.where(keep, dy64 / (1 - p), 0) * s
        got = R.dropout_backward(dyd, p, rng_tensor(1, 2), act=act, z=zd)
        near(got, want, np.abs(dy64) / (1 - p) * 16 * U * np.maximum(1, np.minimum(np.abs(z64), 20)) + (4 * U + HALF[dt] * 1.01) * np.abs(want), f"{act} p {p}")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("act", ACTS[1:])
def test_gradient_where_z_is_not_finite(act, dt):
    z = torch.tensor([[np.inf, -np.inf, np.nan] * 5], device="cuda").to(DT[dt])
    got = R.dropout_backward(torch.full_like(z, 3.0), 0.0, None, act=act, z=z).float().reshape(5, 3)
    assert (got[:, 0] == 3).all() and (got[:, 1] == 0).all()
    assert (got[:, 2] == 0).all() if act == "relu" else torch.isnan(got[:, 2]).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("act", ACTS)
def test_activation_of_a_dense_layer(act, dt):
    """w = 1: the product is x itself, so this is the activation over its range, and z comes back unchanged."""
    g = np.random.default_rng(12)
    x = np.concatenate([g.standard_normal(4000) * 3, np.linspace(-12, 12, 2001), [0.0, 1e-30, -1e-30, 60, -60, 3e5, -3e5, 1e30, -1e30, 3e38, -3e38]])
    xd, x64 = rounded(x.astype(np.float32)[:, None], dt)
    y, z = R.linear_forward(xd, torch.ones(1, 1, dtype=DT[dt], device="cuda"), act=act, keep_z=True)
    assert torch.equal(z, xd)
    with np.errstate(over="ignore"):
        want = D.act(x64, act)
    near(y, want, 16 * U * np.minimum(np.abs(x64), 20) + (16 * U + HALF[dt] * 1.01) * np.abs(want) + 1e-38, act)


# ---- dense layers --------------------------------------------------------------------------------------------------
SHAPES = [(1, 1, 1), (1, 64, 64), (2, 8, 16), (3, 5, 7), (1, 4096, 1000), (8, 1000, 520), (17, 100, 33), (16, 513, 64), (64, 64, 64), (130, 257, 129), (128, 2049, 40), (333, 1000, 515),
          (256, 512, 384), (70, 24, 2056), (600, 40, 72), (1030, 520, 264), (515, 1032, 776), (100, 96, 4000), (5, 3000, 6), (3, 8200, 24), (40, 4100, 70), (30, 70, 5000), (12, 65, 9001), (33, 2048, 64)]


def sums(a, b, n):
    """Bound of a product's rounding errors: |a| |b|' over n terms."""
    return (4 * np.sqrt(n) + 4) * U * (np.abs(a) @ np.abs(b))


def lin_data(m, k, n, seed):
    g = np.random.default_rng(seed)
    return (g.standard_normal((m, k)).astype(np.float32), (g.standard_normal((n, k)) / np.sqrt(k)).astype(np.float32), (0.3 * g.standard_normal(n)).astype(np.float32),
            g.standard_normal((m, n)).astype(np.float32), g.standard_normal((m, k)).astype(np.float32))


def check_linear_fwd(x, w, b, act, p, rng, res, out, z_out, dt, what):
    y, z = D.linear(x, w, b, act, p, rng, res)
    ez = sums(x, w.T, x.shape[1]) + 2 * U * np.abs(z)
    if z_out is not None:
        near(z_out, z, ez + HALF[dt] * 1.01 * np.abs(z) + 1e-38, f"{what} z")
    a = y if res is None else y - res
    ea = (1.2 * ez + (16 * U * np.minimum(np.abs(z), 20) if act != "none" else 0)) / (1 - p) * D.kept(rng, *y.shape, p) + 6 * U * np.abs(a)
    near(out, y, ea + (U + HALF[dt] * 1.01) * np.abs(y) + 1e-38, f"{what} y")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("m,k,n", SHAPES)
def test_linear_forward(m, k, n, dt):
    print("linear_forward", m, k, n, dt, flush=True)
    x, w, b, res, _ = lin_data(m, k, n, k + n)
    wd, w64 = rounded(w, dt)
    xd, x64 = rounded(x, dt)
    rd, r64 = apart(res, dt, 3)
    b64 = b.astype(np.float64)
    check_linear_fwd(x64, w64, None, "none", 0.0, None, None, R.linear_forward(xd, wd), None, dt, "plain")
    act = ACTS[1 + (m + n) % 4]
    y, z = R.linear_forward(xd, wd, dev(b), act=act, p=0.25, rng=rng_tensor(7, 9), residual=rd, keep_z=True)
    check_linear_fwd(x64, w64, b64, act, 0.25, (7, 9), r64, y, z, dt, "everything")
    xd, x64 = apart(x, dt, 5)
    rd, r64 = rounded(res, dt)
    check_linear_fwd(x64, w64, b64, "none", 0.0, None, r64, R.linear_forward(xd, wd, dev(b), residual=rd), None, dt, "rows apart")
    xd, x64 = apart(x, dt, 16)
    y = R.linear_forward(xd, wd, dev(b), act=act)
    check_linear_fwd(x64, w64, b64, act, 0.0, None, None, y, None, dt, "rows 16 apart")
    assert torch.equal(y, R.linear_forward(xd, wd, dev(b), act=act))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("m,k,n", SHAPES)
def test_linear_dgrad(m, k, n, dt):
    print("linear_dgrad", m, k, n, dt, flush=True)
    _, w, _, dz, z = lin_data(m, k, n, k + n + 1)
    wd, w64 = rounded(w, dt)
    for extra, act, p in ((0, "none", 0.0), (3, ACTS[1 + (m + n) % 4], 0.0), (8, ACTS[1 + (m + k) % 4], 0.25)):
        dzd, dz64 = apart(dz, dt, extra)
        zd, z64 = apart(z, dt, extra)
        want = D.linear_dgrad(dz64, w64, act, z64, p, (4, 4))
        got = R.linear_dgrad(dzd, wd, act=act, z=zd, p=p, rng=rng_tensor(4, 4))
        v = np.abs(D.dropout(dz64 @ w64, p, (4, 4)))
        tol = (sums(dz64, w64, n) * (1.2 if act != "none" else 1) / (1 - p)) * D.kept((4, 4), m, k, p) + v * 16 * U * np.maximum(1, np.abs(z64)) * (act != "none")
        near(got, want, tol + (4 * U + HALF[dt] * 1.01) * np.abs(want) + 1e-38, f"{act} p {p} extra {extra}")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("m,k,n", SHAPES)
def test_linear_wgrad(m, k, n, dt):
    print("linear_wgrad", m, k, n, dt, flush=True)
    x, _, _, dz, _ = lin_data(m, k, n, k + n + 2)
    for extra in (0, 3, 8):
        xd, x64 = apart(x, dt, extra)
        dzd, dz64 = apart(dz, dt, extra)
        dw, db = R.linear_wgrad(dzd, xd)
        want_w, want_b = D.linear_wgrad(dz64, x64)
        near(dw, want_w, sums(dz64.T, x64, m) + 1e-38, f"dw extra {extra}")
        near(db, want_b, (4 * np.sqrt(m) + 4) * U * np.abs(dz64).sum(0) + 1e-38, f"db extra {extra}")
    again = R.linear_wgrad(dzd, xd)
    assert torch.equal(dw, again[0]) and torch.equal(db, again[1])


# every size of tile, with ragged edges on all sides, whole and split reductions (the largest tiles: the second forward, the last in all three in bf16)
LARGE = [(4000, 264, 4104), (5000, 200, 3001), (2050, 521, 8000), (4100, 520, 4360), (1100, 2050, 2000), (300, 4090, 2100), (3990, 3000, 4090)]


def product64(a, b):
    return host(torch.from_numpy(a).cuda() @ torch.from_numpy(np.ascontiguousarray(b)).cuda())


def large_sums(a, b, n):
    return (4 * np.sqrt(n) + 4) * U * product64(np.abs(a), np.abs(b))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("m,k,n", LARGE)
def test_linear_large(m, k, n, dt):
    print("linear_large", m, k, n, dt, flush=True)
    x, w, b, res, z = lin_data(m, k, n, m)
    wd, w64 = rounded(w, dt)
    xd, x64 = apart(x, dt, 8)
    rd, r64 = apart(res, dt, 3)
    zd, z64 = rounded(z, dt)
    act = ACTS[1 + m // 10 % 4]
    want = product64(x64, w64.T) + b
    e = large_sums(x64, w64.T, k)
    near(R.linear_forward(xd, wd, dev(b)), want, e + 2 * U * np.abs(want) + HALF[dt] * 1.01 * np.abs(want), "forward")
    y, zo = R.linear_forward(xd, wd, dev(b), act=act, p=0.25, rng=rng_tensor(7, 9), residual=rd, keep_z=True)
    near(zo, want, e + 2 * U * np.abs(want) + HALF[dt] * 1.01 * np.abs(want), "z")
    a = np.where(D.kept((7, 9), m, n, 0.25), D.act(want, act) / 0.75, 0.0)
    near(y, a + r64, (1.2 * e + 16 * U * np.minimum(np.abs(want), 20)) / 0.75 + 6 * U * np.abs(a) + (U + HALF[dt] * 1.01) * np.abs(a + r64), "forward, everything")
    # gradients: of rows `res`
    want = product64(r64, w64)
    e = large_sums(r64, w64, n)
    near(R.linear_dgrad(rd, wd), want, e + HALF[dt] * 1.01 * np.abs(want), "dgrad")
    v = np.where(D.kept((4, 4), m, k, 0.25), want / 0.75, 0.0)
    s = D.slope(z64, act)
    near(R.linear_dgrad(rd, wd, act=act, z=zd, p=0.25, rng=rng_tensor(4, 4)), v * s,
         1.2 * e / 0.75 + np.abs(v) * 16 * U * np.maximum(1, np.abs(z64)) + (4 * U + HALF[dt] * 1.01) * np.abs(v * s), "dgrad through")
    dw, db = R.linear_wgrad(rd, xd)
    near(dw, product64(r64.T, x64), large_sums(r64.T, x64, m), "dw")
    near(db, r64.sum(0), (4 * np.sqrt(m) + 4) * U * np.abs(r64).sum(0), "db")
    assert all(torch.equal(p, q) for p, q in zip((dw, db), R.linear_wgrad(rd, xd)))


def test_no_rows():
    x, w = torch.empty(0, 24, device="cuda"), torch.ones(16, 24, device="cuda")
    assert R.linear_forward(x, w).shape == (0, 16) and R.linear_dgrad(torch.empty(0, 16, device="cuda"), w).shape == (0, 24)
    dw, db = R.linear_wgrad(torch.empty(0, 16, device="cuda"), x)
    assert dw.shape == (16, 24) and db.shape == (16,) and not dw.any() and not db.any()
    y, mean, rstd = R.layernorm_forward(x)
    dx, dg, dbeta = R.layernorm_backward(x, x, None, mean, rstd)
    assert y.shape == dx.shape == (0, 24) and not dg.any() and not dbeta.any() and dg.shape == dbeta.shape == (24,)
    assert R.dropout_forward(x, 0.5, rng_tensor(0, 0)).shape == (0, 24)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_operands_that_are_not_finite_stay_in_their_rows(dt):
    m, k, n = 300, 136, 264
    x, w, *_ = lin_data(m, k, n, 3)
    x[7, 5], x[40, 100], x[299, 135] = np.inf, np.nan, -np.inf
    xd, x64 = rounded(x, dt)
    wd, w64 = rounded(w, dt)
    y = host(R.linear_forward(xd, wd))
    for row, col in ((7, 5), (299, 135)):
        assert np.array_equal(y[row], np.sign(w64[:, col]) * x64[row, col])
    assert np.isnan(y[40]).all()
    fine = np.setdiff1d(np.arange(m), [7, 40, 299])
    near(y[fine], x64[fine] @ w64.T, sums(x64[fine], w64.T, k) + HALF[dt] * 1.01 * np.abs(x64[fine] @ w64.T), "the other rows")
    dw, _ = R.linear_wgrad(xd, xd)
    dw = host(dw)
    fine = np.setdiff1d(np.arange(k), [5, 100, 135])
    want = x64[:, fine].T @ x64[:, fine]
    near(dw[np.ix_(fine, fine)], want, sums(x64[:, fine].T, x64[:, fine], m), "dw of the other columns")
    assert not np.isfinite(dw[[5, 100, 135]]).any()


def test_fp32_operands_over_their_whole_range():
    """Magnitudes from the smallest to the largest normal numbers, the products in between: as exact as elsewhere."""
    m, k, n = 140, 72, 136
    x, w, *_ = lin_data(m, k, n, 5)
    for sx, sw in ((2.0 ** -100, 2.0 ** 60), (2.0 ** -120, 2.0 ** 90), (2.0 ** 120, 2.0 ** -90), (2.0 ** -60, 2.0 ** -50), (1.0, 2.0 ** 100), (2.0 ** -118, 2.0 ** 118)):
        xd, x64 = rounded((x * np.float32(sx)).astype(np.float32), "f32")
        wd, w64 = rounded((w * np.float32(sw)).astype(np.float32), "f32")
        near(R.linear_forward(xd, wd), x64 @ w64.T, sums(x64, w64.T, k), f"{sx} {sw}")
    # in tiles of every size: one value that three bf16 parts do not hold among ordinary ones
    for m, k, n in ((140, 72, 136), (1500, 320, 2600), (5000, 200, 3000)):
        x, w, *_ = lin_data(m, k, n, 6)
        x[m // 2, k // 2], w[n // 3, 5] = 2.0 ** -125, 3.4e38
        xd, x64 = rounded(x, "f32")
        wd, w64 = rounded(w * np.float32(2.0 ** -3), "f32")
        near(R.linear_forward(xd, wd), x64 @ w64.T, sums(x64, w64.T, k), f"{m} {k} {n}")
        dw, _ = R.linear_wgrad(R.linear_forward(xd, wd)[:, :n], xd)
        assert torch.isfinite(dw[: n // 3]).all()
    xd = torch.full((130, 8), 0.0, device="cuda")
    xd[:, 0] = 3.4e38                                          # a float just below the largest, kept as it is
    wd = torch.zeros(128, 8, device="cuda")
    wd[:, 0] = 1.0
    assert torch.equal(R.linear_forward(xd, wd), torch.full((130, 128), 3.4e38, device="cuda"))


# ---- as a program uses them ----------------------------------------------------------------------------------------
def mlp_forward(x, prm, act, p, rngs, stream=None):
    gamma, beta, w1, b1, w2, b2 = prm
    n, mean, rstd = R.layernorm_forward(x, gamma, beta, stream=stream)
    h, z1 = R.linear_forward(n, w1, b1, act=act, p=p, rng=rngs[0], keep_z=True, stream=stream)
    y = R.linear_forward(h, w2, b2, p=p, rng=rngs[1], residual=x, stream=stream)
    return y, (n, mean, rstd, h, z1)


def mlp_backward(dy, x, prm, saved, act, p, rngs, stream=None):
    gamma, _, w1, _, w2, _ = prm
    n, mean, rstd, h, z1 = saved
    dz2 = R.dropout_backward(dy, p, rngs[1], stream=stream)
    dw2, db2 = R.linear_wgrad(dz2, h, stream=stream)
    dz1 = R.linear_dgrad(dz2, w2, act=act, z=z1, p=p, rng=rngs[0], stream=stream)
    dw1, db1 = R.linear_wgrad(dz1, n, stream=stream)
    dx, dg, db = R.layernorm_backward(R.linear_dgrad(dz1, w1, stream=stream), x, gamma, mean, rstd, addend=dy, stream=stream)
    return dx, dg, db, dw1, db1, dw2, db2


def mlp_case(m, n, hidden, dt, seed=0):
    g = np.random.default_rng(seed)
    a = [g.standard_normal((m, n)), 1 + 0.1 * g.standard_normal(n), 0.1 * g.standard_normal(n), g.standard_normal((hidden, n)) / np.sqrt(n), 0.1 * g.standard_normal(hidden),
         g.standard_normal((n, hidden)) / np.sqrt(hidden), 0.1 * g.standard_normal(n), g.standard_normal((m, n))]
    kind = [dt, "f32", "f32", dt, "f32", dt, "f32", dt]
    return [dev(t.astype(np.float32), k) for t, k in zip(a, kind)]


@pytest.mark.parametrize("dt,m,n,hidden,act,p", [("f32", 200, 72, 260, "gelu", 0.1), ("bf16", 200, 72, 264, "gelu_tanh", 0.1), ("f32", 33, 65, 129, "silu", 0.0),
                                                 ("bf16", 513, 256, 1024, "relu", 0.2)])
def test_residual_block_and_its_gradients(dt, m, n, hidden, act, p):
    """The whole block as a training step runs it, against the oracle's from the same values.  fp32: relative 2-norm 1e-5 (six products with
    errors of a few U sqrt(n) of their terms' norm, U sqrt(1024) = 2e-6).  bf16: three to five stored intermediates on the way to any result, each off
    by 2^-8/sqrt(3) of its norm at most, added by their squares: 2^-8 sqrt(5/3), and as much again for products of two rounded factors -> 1e-2."""
    x, *prm, dy = mlp_case(m, n, hidden, dt)
    rngs = rng_tensor(5, 0), rng_tensor(5, 10 ** 6)
    y, saved = mlp_forward(x, prm, act, p, rngs)
    grads = mlp_backward(dy, x, prm, saved, act, p, rngs)
    prm64, r64 = [host(t) for t in prm], ((5, 0), (5, 10 ** 6))
    want_y, s64 = D.mlp_block(host(x), prm64, act, p, r64)
    dx, g64 = D.mlp_block_backward(host(dy), host(x), prm64, s64, act, p, r64)
    for name, got, want in zip(("y", "dx", "dgamma", "dbeta", "dw1", "db1", "dw2", "db2"), (y, *grads), (want_y, dx, *g64)):
        rel = np.linalg.norm(host(got) - want) / np.linalg.norm(want)
        # a ReLU whose input is zero to rounding may pass on one side only: a share of U sqrt(n) (fp32), 2^-9 (bf16) of the hidden units, each worth its whole gradient
        bound = (1e-5 if dt == "f32" else 1e-2) + (0.05 if act == "relu" and name != "y" else 0)
        assert rel <= bound, (name, rel)


def test_block_on_a_stream_of_its_own():
    x, *prm, dy = mlp_case(300, 128, 512, "bf16", 1)
    rngs = rng_tensor(1, 0), rng_tensor(1, 10 ** 6)
    y, saved = mlp_forward(x, prm, "gelu", 0.1, rngs)
    want = (y, *mlp_backward(dy, x, prm, saved, "gelu", 0.1, rngs))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y, saved = mlp_forward(x, prm, "gelu", 0.1, rngs, stream=side)
    got = (y, *mlp_backward(dy, x, prm, saved, "gelu", 0.1, rngs, stream=side))
    with torch.cuda.stream(side):
        y, saved = mlp_forward(x, prm, "gelu", 0.1, rngs)
        inside = (y, *mlp_backward(dy, x, prm, saved, "gelu", 0.1, rngs))
    torch.cuda.current_stream().wait_stream(side)
    for a, b, c in zip(want, got, inside):
        assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_captured_block_draws_a_new_mask_per_replay(dt):
    """Two graphs, each with a pool of its own, replayed in turn with eager work in between; the offset moves on between the replays."""
    x, *prm, dy = mlp_case(260, 96, 384, dt, 2)
    rngs = rng_tensor(9, 0), rng_tensor(9, 1 << 40)

    def block():
        y, saved = mlp_forward(x, prm, "gelu", 0.2, rngs)
        return (y, *mlp_backward(dy, x, prm, saved, "gelu", 0.2, rngs))

    block()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = block()
        graphs.append((g, out))
    last = None
    for step in range(3):
        for g, out in graphs:
            g.replay()
            want = block()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want)), step
            assert last is None or not torch.equal(last, out[0])
            last = out[0].clone()
            for r in rngs:
                r[1] += 10 ** 6
            x.mul_(1.01)


def test_outputs_in_place_and_rows_apart_through_the_c_interface():
    """What the binding never does: results over an input, results in rows apart, with everything behind and between the rows as it was."""
    L, st = R.lib(), torch.cuda.current_stream().cuda_stream
    g = np.random.default_rng(4)
    for dt, code in (("f32", 0), ("bf16", 1)):
        m, n, ld = 37, 65, 72
        a, b, z = (g.standard_normal((m, n)).astype(np.float32) for _ in range(3))

        def wide(v, rows=m + 2):
            t = torch.full((rows, ld), 123.0, dtype=DT[dt], device="cuda")
            t[:m, :n] = dev(v, dt)
            return t

        def untouched(t):
            return bool((t[m:] == 123).all() and (t[:m, n:] == 123).all())

        stat = torch.empty(2, 64, device="cuda")
        mean, rstd = stat[0, :m], stat[1, :m]
        gamma = dev(1 + 0.1 * g.standard_normal(n).astype(np.float32))
        rng = rng_tensor(2, 3)
        ptr = lambda t: t.data_ptr()
        # layer norm over x, its gradient over dy, x and the addend in turn
        x = wide(a)
        want, wmean, wrstd = R.layernorm_forward(x[:m, :n], gamma)
        assert L.resist_layernorm_forward(m, n, code, ptr(x), ld, ptr(gamma), None, 1e-5, ptr(x), ld, ptr(mean), ptr(rstd), st) == 0
        assert torch.equal(x[:m, :n], want) and untouched(x) and torch.equal(mean, wmean) and torch.equal(rstd, wrstd)
        ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
        for k in range(3):
            t = [wide(a), wide(b), wide(z)]
            want = R.layernorm_backward(t[0][:m, :n], t[1][:m, :n], gamma, wmean, wrstd, addend=t[2][:m, :n])
            assert L.resist_layernorm_backward(m, n, code, ptr(t[0]), ld, ptr(t[1]), ld, ptr(gamma), ptr(wmean), ptr(wrstd), ptr(t[2]), ld, ptr(t[k]), ld, None, None,
                                               ptr(ws), ws.numel(), st) == 0
            assert torch.equal(t[k][:m, :n], want[0]) and untouched(t[k])
        # dropout over x and over the residual, its gradient over dy and over z
        for k in range(2):
            t = [wide(a), wide(b)]
            want = R.dropout_forward(t[0][:m, :n], 0.3, rng, residual=t[1][:m, :n])
            assert L.resist_dropout_forward(m, n, code, ptr(t[0]), ld, 0.3, ptr(rng), ptr(t[1]), ld, ptr(t[k]), ld, st) == 0
            assert torch.equal(t[k][:m, :n], want) and untouched(t[k])
            t = [wide(a), wide(z)]
            want = R.dropout_backward(t[0][:m, :n], 0.3, rng, act="gelu", z=t[1][:m, :n])
            assert L.resist_dropout_backward(m, n, code, ptr(t[0]), ld, 0.3, ptr(rng), 2, ptr(t[1]), ld, ptr(t[k]), ld, st) == 0
            assert torch.equal(t[k][:m, :n], want) and untouched(t[k])
        # a dense layer over its residual, its data gradient over z: small, and large enough for the largest tiles
        for m, n, k, ld in ((37, 65, 48, 72), (1100, 1100, 64, 1104)):
            a, b = g.standard_normal((m, n)).astype(np.float32), g.standard_normal((m, k)).astype(np.float32)
            xd, w = dev(b, dt), dev(g.standard_normal((n, k)).astype(np.float32), dt)
            y, zz = wide(a, m + 2), wide(a, m + 2)
            want, wz = R.linear_forward(xd, w, act="silu", residual=y[:m, :n], p=0.3, rng=rng, keep_z=True)
            sh, size = B._LinearShape(m, k, n, k, ld, code), C.c_int64()
            assert L.resist_linear_workspace_bytes(C.byref(sh), 0, C.byref(size)) == 0
            ws = torch.empty(max(size.value, 16), dtype=torch.uint8, device="cuda")
            e = B._LinearEpilogue(None, 4, 0.3, ptr(rng), ptr(y), ld, ptr(zz), ld)
            assert L.resist_linear_forward(C.byref(sh), ptr(xd), ptr(w), C.byref(e), ptr(y), ptr(ws), size.value, st) == 0
            assert torch.equal(y[:m, :n], want) and untouched(y) and torch.equal(zz[:m, :n], wz) and untouched(zz)
            wt, zz = w.t().contiguous(), wide(a, m + 2)      # dx [m, n] = dz [m, k] . [k, n]
            want = R.linear_dgrad(xd, wt, act="gelu", z=zz[:m, :n], p=0.3, rng=rng)
            sh = B._LinearShape(m, n, k, ld, k, code)
            assert L.resist_linear_workspace_bytes(C.byref(sh), 1, C.byref(size)) == 0
            ws = torch.empty(max(size.value, 16), dtype=torch.uint8, device="cuda")
            th = B._LinearThrough(2, ptr(zz), ld, 0.3, ptr(rng))
            assert L.resist_linear_dgrad(C.byref(sh), ptr(xd), ptr(wt), C.byref(th), ptr(zz), ptr(ws), size.value, st) == 0
            assert torch.equal(zz[:m, :n], want) and untouched(zz)


def test_binding_copies_what_the_library_cannot_take():
    """Views that start off a 16-byte boundary, transposed ones, broadcast ones: the results of their copies."""
    g = torch.Generator(device="cuda").manual_seed(1)
    big = torch.randn(70, 90, device="cuda", generator=g)
    w = torch.randn(40, 33, device="cuda", generator=g)
    for v in (big[:, 1:34], big.t()[:, :33], big[:1].expand(20, 90)[:, :33], big[:, ::2][:, :33]):
        c = v.clone(memory_format=torch.contiguous_format)
        assert torch.equal(R.linear_forward(v, w), R.linear_forward(c, w))
        assert torch.equal(R.layernorm_forward(v)[0], R.layernorm_forward(c)[0])
        assert torch.equal(R.dropout_forward(v, 0.5, rng_tensor(1, 1)), R.dropout_forward(c, 0.5, rng_tensor(1, 1)))
    wt = torch.randn(33, 40, device="cuda", generator=g).t()
    assert torch.equal(R.linear_forward(big[:, :33], wt), R.linear_forward(big[:, :33], wt.contiguous()))


def test_gpu_refusals_of_the_binding():
    x, w = torch.zeros(4, 8, device="cuda"), torch.zeros(6, 8, device="cuda")
    for call in (lambda: R.linear_forward(x, w[:, :7]), lambda: R.linear_forward(x, w.bfloat16()), lambda: R.linear_forward(x, w, bias=torch.zeros(8, device="cuda")),
                 lambda: R.linear_forward(x, w, residual=x), lambda: R.linear_forward(x, w, p=0.5), lambda: R.linear_forward(x.half(), w.half()),
                 lambda: R.linear_forward(x, w, act="tanh"), lambda: R.linear_dgrad(x, w), lambda: R.linear_dgrad(x[:, :6], w, act="gelu"),
                 lambda: R.linear_wgrad(x[:3], x), lambda: R.layernorm_backward(x, x, None, None, None), lambda: R.layernorm_forward(x, eps=-1.0),
                 lambda: R.dropout_forward(x, 1.0, rng_tensor(0, 0)), lambda: R.dropout_forward(x, 0.5, torch.zeros(2, dtype=torch.int64)),
                 lambda: R.linear_forward(x[0], w), lambda: R.linear_forward(x, w.cpu())):
        with pytest.raises(R.ResistError):
            call()
