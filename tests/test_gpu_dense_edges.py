"""GPU: the dense operators where their arguments go to an end: activations far out and where z is not finite, more rows than one launch takes, rows
very far apart, layer norm in place in rows of every kind, a block's gradients from the activations it kept.

U = 2^-24 is half a step of fp32, 2^-8 of bf16; a bound that counts roundings says which."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2107_00961_amd as R
from oracle import dense as D

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": U, "bf16": 2.0 ** -8}


def host(t):
    return t.detach().double().cpu().numpy()


def near(got, want, tol, what):
    got = host(got)
    assert got.shape == want.shape and np.isfinite(got).all(), what
    over = np.abs(got - want) / np.broadcast_to(tol, want.shape)
    if (over > 1).any():
        i = np.unravel_index(np.argmax(over), over.shape)
        raise AssertionError(f"{what}: {(over > 1).sum()} of {over.size} off; worst at {i}: {got[i]:.9g} for {want[i]:.9g}, {over[i]:.3g} times the tolerance")


def function_roundings(z, act):
    """Roundings U of act(z), relative to it, before it is stored.
    GELU from Q(x)/e = t p(t), t = 1/(1 + c x), e = exp(-x^2/2): t 4 (c, the sum, a reciprocal within 2), which count 2.7 times in t p(t); p 3.1 for its
    steps and 1.8 for its coefficients, each as given; the fit 1.7; e 2 and, of an argument with three roundings, 3 x^2/2; products 3.
    SiLU and the tanh form from 1/(1 + exp(-a)): of a 2 roundings for a = z and 9 for a = 2u (and one each of exp's argument), exp and
    reciprocal 2 each, sum and product 1 each."""
    z = np.abs(z)
    if act == "gelu":
        return 24 + 1.5 * z * z
    return 6 + 2 * z if act == "silu" else 7 + 9 * 2 * np.sqrt(2 / np.pi) * z * (1 + 0.044715 * z * z)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
def test_activations_are_right_relative_to_themselves(act, dt):
    """Out to where they are no longer normal numbers; as one column (tiles) and as one row (few rows).  The product is z itself."""
    z = torch.from_numpy(np.concatenate([np.linspace(-13, -0.001, 4097), np.linspace(0.001, 13, 999)]).astype(np.float32)).cuda().to(DT[dt])
    one = torch.ones(1, 1, device="cuda", dtype=DT[dt])
    z64 = host(z)
    want = D.act(z64, act)
    tol = (HALF[dt] + U * function_roundings(z64, act)) * np.abs(want) + np.abs(z64) * 2.0 ** -125
    near(R.linear_forward(z[:, None], one, act=act)[:, 0], want, tol, "a column")
    near(R.linear_forward(one, z[:, None], act=act)[0], want, tol, "a row")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("act,want", [("relu", [np.inf, 0.0, 0.0]), ("gelu", [np.inf, 0.0, np.nan]), ("gelu_tanh", [np.inf, 0.0, np.nan]),
                                      ("silu", [np.inf, 0.0, np.nan])])
def test_activations_where_z_is_not_finite(act, want, dt):
    """The limits at both ends; a NaN stays one, but for ReLU, which passes on what is above 0 and nothing else."""
    z = torch.tensor([np.inf, -np.inf, np.nan] * 40, device="cuda").to(DT[dt])
    one = torch.ones(1, 1, device="cuda", dtype=DT[dt])
    want = torch.tensor(want * 40, device="cuda").to(DT[dt])
    for got in (R.linear_forward(z[:, None], one, act=act)[:, 0], R.linear_forward(one, z[:, None], act=act)[0]):
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(7.0), want.nan_to_num(7.0)), got[:3]


# ---- more rows than one launch takes: 2^32 threads -------------------------------------------------------------------------
def random(m, n, dt, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    torch.cuda.empty_cache()
    return torch.empty(m, n, device="cuda", dtype=DT[dt]).normal_(generator=g)


def rows_of(m):
    """The first and the last, and those on either side of multiples of 2^24 - 1 and 2^24 workgroups of 1 to 64 rows."""
    at = {0, 1, m - 2, m - 1}
    for shift in range(7):
        for e in (((1 << 24) - 1) << shift, 1 << 24 + shift, 1 << 23 + shift, ((1 << 23) - 1) << shift):
            at |= {r for r in (e - 1, e, e + 1) if r < m}
    return sorted(at)


@pytest.mark.parametrize("m,n", [((1 << 28) + 5, 8), ((1 << 26) + 3, 260), ((1 << 23) + 3, 4100)])
def test_layernorm_of_many_rows(m, n):
    """16, 64 and 512 threads a row.  Of a row: sums in a tree of 48 steps, the stored value's half step (as in test_gpu_dense.py)."""
    x = random(m, n, "bf16", 1)
    y, mean, rstd = R.layernorm_forward(x)
    at = rows_of(m)
    x64 = host(x[at])
    want, mu, r = D.layernorm(x64)
    e_mean = 48 * U * np.abs(x64).mean(1)
    rel = 56 * U + e_mean ** 2 * r ** 2
    near(mean[at], mu, e_mean + U * np.abs(mu), "mean")
    near(rstd[at], r, rel * r, "rstd")
    xhat = np.abs(x64 - mu[:, None]) * r[:, None]
    near(y[at], want, e_mean[:, None] * r[:, None] * (1 + rel[:, None]) + xhat * (rel[:, None] + 6 * U) + (4 * U + HALF["bf16"] * 1.01) * np.abs(want) + 1e-38, "y")
    # every row's mean, and y's: that of 0 but for y's own roundings, 2^-8 of at most sqrt(n) each
    step = (1 << 30) // n
    for i in range(0, m, step):
        part = x[i:i + step].float()
        assert ((mean[i:i + step] - part.mean(1)).abs() <= 100 * U * part.abs().mean(1)).all(), i
        assert (y[i:i + step].float().mean(1).abs() <= 2.0 ** -8).all(), i


def test_dense_layers_of_many_rows():
    """Rows for more workgroups of 64 than one launch takes, laid out (five and three elements a row) and multiplied."""
    m, k, n, p = (1 << 30) + 3, 5, 3, 0.25
    x, w = random(m, k, "bf16", 2), random(n, k, "bf16", 3)
    rng = torch.tensor([3, 5], dtype=torch.int64, device="cuda")
    at = rows_of(m)
    kept = np.concatenate([D.kept((3, 5 + i * 2), 1, n, p) for i in at])
    y = R.linear_forward(x, w, act="relu", p=p, rng=rng)
    z = host(x[at]) @ host(w).T
    e = (4 * np.sqrt(k) + 4) * U * (np.abs(host(x[at])) @ np.abs(host(w)).T)
    want = np.where(kept, np.maximum(z, 0) / (1 - p), 0.0)
    near(y[at], want, (1.2 * e / (1 - p) + (4 * U + HALF["bf16"] * 1.01) * np.abs(want)) + 1e-38, "forward, sampled")
    step = 1 << 26
    wf = w.float()
    y = R.linear_forward(x, w)
    for i in range(0, m, step):
        part, got = x[i:i + step].float(), y[i:i + step].float()
        for j in range(n):     # a sum of five products: 13 roundings of the sum of magnitudes, on either side
            terms = part * wf[j]
            assert ((got[:, j] - terms.sum(1)).abs() <= 26 * U * terms.abs().sum(1) + HALF["bf16"] * 1.01 * terms.sum(1).abs()).all(), (i, j)
    # y is as good a gradient as any; dx = y w
    dx = R.linear_dgrad(y, w)
    for i in range(0, m, step):
        part, got = y[i:i + step].float(), dx[i:i + step].float()
        for j in range(k):
            terms = part * wf[:, j]
            assert ((got[:, j] - terms.sum(1)).abs() <= 26 * U * terms.abs().sum(1) + HALF["bf16"] * 1.01 * terms.sum(1).abs()).all(), (i, j)
    del dx
    dw, db = R.linear_wgrad(y, x)
    sums = torch.zeros(4, n, k, dtype=torch.float64, device="cuda")
    for i in range(0, m, step):
        a, b = y[i:i + step].double(), x[i:i + step].double()
        for j in range(n):
            t = a[:, j:j + 1] * b
            sums[0, j] += t.sum(0)
            sums[1, j] += t.abs().sum(0)
            sums[2, j, 0] += a[:, j].sum()
            sums[3, j, 0] += a[:, j].abs().sum()
    bound = (4 * np.sqrt(m) + 4) * U
    near(dw, host(sums[0]), bound * host(sums[1]), "dw")
    near(db, host(sums[2, :, 0]), bound * host(sums[3, :, 0]), "db")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("m", [3, 70])
def test_dense_layers_on_rows_far_apart(m, dt):
    """The last token of every sequence of a batch is such a view: rows more than 2^20 elements apart, which the library does not take itself."""
    k, n, far = 40, 24, (1 << 20) + 16

    def apart(cols, seed):
        t = torch.full((m, far), float("nan"), device="cuda", dtype=DT[dt])
        t[:, :cols] = random(m, cols, dt, seed)
        return t[:, :cols], t[:, :cols].contiguous()

    (x, xc), (dz, dzc), (z, zc), (res, resc) = apart(k, 1), apart(n, 2), apart(k, 3), apart(n, 4)
    w = random(n, k, dt, 5)
    assert torch.equal(R.linear_forward(x, w, residual=res), R.linear_forward(xc, w, residual=resc))
    assert torch.equal(R.linear_dgrad(dz, w, act="gelu", z=z), R.linear_dgrad(dzc, w, act="gelu", z=zc))
    assert all(torch.equal(a, b) for a, b in zip(R.linear_wgrad(dz, x), R.linear_wgrad(dzc, xc)))
    # the operators on rows alone take them as they are
    assert torch.equal(R.layernorm_forward(x)[0], R.layernorm_forward(xc)[0])
    rng = torch.tensor([1, 2], dtype=torch.int64, device="cuda")
    assert torch.equal(R.dropout_forward(x, 0.5, rng, residual=z), R.dropout_forward(xc, 0.5, rng, residual=zc))


# ---- layer norm in place ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n", [7, 100, 1001, 1100, 2049, 4100, 8190, 8200])
def test_layernorm_in_place(n, dt):
    """y over x, and dx over dy, x and the addend: what results of their own hold.  Where a row is no whole number of vectors, the last one overlaps the one
    before, another thread's and beyond 1024 another wave's.  Workgroups take several rows one after the other."""
    m, code, L, st = 2500, {"f32": 0, "bf16": 1}[dt], R.lib(), torch.cuda.current_stream().cuda_stream
    x, dy, add = (random(m, n, dt, s) for s in (1, 2, 3))
    gamma = 1 + 0.1 * random(1, n, "f32", 4)[0].contiguous()
    want, mean, rstd = R.layernorm_forward(x, gamma)
    t, stat = x.clone(), torch.empty(2, m + 4, device="cuda")
    assert L.resist_layernorm_forward(m, n, code, t.data_ptr(), 0, gamma.data_ptr(), None, 1e-5, t.data_ptr(), 0, stat[0].data_ptr(), stat[1].data_ptr(), st) == 0
    assert torch.equal(t, want) and torch.equal(stat[0, :m], mean) and torch.equal(stat[1, :m], rstd)
    size = C.c_int64()
    assert L.resist_layernorm_workspace_bytes(m, n, C.byref(size)) == 0
    ws = torch.empty(size.value, dtype=torch.uint8, device="cuda")
    for addend in (None, add):
        want, dgamma, dbeta = R.layernorm_backward(dy, x, gamma, mean, rstd, addend=addend)
        for k in range(2 if addend is None else 3):
            t = [dy.clone(), x.clone(), None if addend is None else addend.clone()]
            dg, db = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
            assert L.resist_layernorm_backward(m, n, code, t[0].data_ptr(), 0, t[1].data_ptr(), 0, gamma.data_ptr(), mean.data_ptr(), rstd.data_ptr(),
                                               None if addend is None else t[2].data_ptr(), 0, t[k].data_ptr(), 0, dg.data_ptr(), db.data_ptr(), ws.data_ptr(),
                                               size.value, st) == 0
            assert torch.equal(t[k], want) and torch.equal(dg, dgamma) and torch.equal(db, dbeta), (k, addend is None)


# ---- a block's gradients ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_gradients_of_a_block_from_what_it_kept(act, dt):
    """Every operator of the backward pass against the oracle's of the very tensors it was given (what the forward pass kept, the gradients on the way as
    stored), so that no ReLU is on another side of 0 and every element has its own bound: sums of n terms 4 sqrt(n) + 4 roundings
    of the sum of magnitudes, a slope 16 max(1, |z|), a stored value half a step."""
    m, n, hidden, p = 260, 200, 520, 0.2
    x, dy, w1, w2 = random(m, n, dt, 1), random(m, n, dt, 2), random(hidden, n, dt, 3) / n ** 0.5, random(n, hidden, dt, 4) / hidden ** 0.5
    gamma, beta, b1, b2 = 1 + 0.1 * random(1, n, "f32", 5)[0], 0.1 * random(1, n, "f32", 6)[0], 0.1 * random(1, hidden, "f32", 7)[0], 0.1 * random(1, n, "f32", 8)[0]
    r1, r2 = (7, 0), (7, 1 << 33)
    rng1, rng2 = (torch.tensor(r, dtype=torch.int64, device="cuda") for r in (r1, r2))
    nx, mean, rstd = R.layernorm_forward(x, gamma, beta)
    h, z1 = R.linear_forward(nx, w1, b1, act=act, p=p, rng=rng1, keep_z=True)
    y = R.linear_forward(h, w2, b2, p=p, rng=rng2, residual=x)

    def terms(a, b, k):
        return (4 * np.sqrt(k) + 4) * U * (np.abs(a) @ np.abs(b))

    half = HALF[dt] * 1.01
    z64, _ = D.linear(host(nx), host(w1), host(b1))
    near(z1, z64, terms(host(nx), host(w1).T, n) + (2 * U + half) * np.abs(z64) + 1e-38, "z1")
    want = D.dropout(D.act(z64, act), p, r1)
    near(h, want, (1.2 * terms(host(nx), host(w1).T, n) + 16 * U * np.abs(z64)) / (1 - p) * D.kept(r1, m, hidden, p) + (6 * U + half) * np.abs(want) + 1e-38, "h")
    want, _ = D.linear(host(h), host(w2), host(b2), "none", p, r2, host(x))
    near(y, want, terms(host(h), host(w2).T, hidden) / (1 - p) + 8 * U * np.abs(want - host(x)) + (U + half) * np.abs(want) + 1e-38, "y")

    dz2 = R.dropout_backward(dy, p, rng2)
    want = D.dropout(host(dy), p, r2)
    near(dz2, want, (4 * U + half) * np.abs(want) + 1e-45, "dz2")
    dz1 = R.linear_dgrad(dz2, w2, act=act, z=z1, p=p, rng=rng1)
    v = D.dropout(host(dz2) @ host(w2), p, r1)
    want = v * D.slope(host(z1), act)
    near(dz1, want, 1.2 * terms(host(dz2), host(w2), n) / (1 - p) * D.kept(r1, m, hidden, p) * ((act != "relu") + (act == "relu") * (want != 0))
         + np.abs(v) * 16 * U * np.maximum(1, np.abs(host(z1))) * (act != "relu") + (4 * U + half) * np.abs(want) + 1e-38, "dz1")
    for name, g, a in (("2", dz2, h), ("1", dz1, nx)):
        dw, db = R.linear_wgrad(g, a)
        near(dw, host(g).T @ host(a), terms(host(g).T, host(a), m) + 1e-38, "dw" + name)
        near(db, host(g).sum(0), (4 * np.sqrt(m) + 4) * U * np.abs(host(g)).sum(0) + 1e-38, "db" + name)
    dn = R.linear_dgrad(dz1, w1)
    want = host(dz1) @ host(w1)
    near(dn, want, terms(host(dz1), host(w1), hidden) + (2 * U + half) * np.abs(want) + 1e-38, "dn")
    dx, dgamma, dbeta = R.layernorm_backward(dn, x, gamma, mean, rstd, addend=dy)
    args = host(dn), host(x), host(gamma), host(mean), host(rstd)
    want, dg, db = D.layernorm_backward(*args, host(dy))
    xhat, g = np.abs(host(x) - host(mean)[:, None]) * host(rstd)[:, None], np.abs(host(dn) * host(gamma))
    s1, s2 = g.mean(1, keepdims=True), (g * xhat).mean(1, keepdims=True)
    near(dx, want, host(rstd)[:, None] * (8 * U * (g + s1 + xhat * s2) + 54 * U * (s1 + xhat * s2)) + 2 * U * np.abs(host(dy)) + (2 * U + half) * np.abs(want) + 1e-38, "dx")
    near(dgamma, dg, (m / 128 + 12) * U * (np.abs(host(dn)) * xhat).sum(0) + 1e-38, "dgamma")
    near(dbeta, db, (m / 128 + 12) * U * np.abs(host(dn)).sum(0) + 1e-38, "dbeta")


@pytest.mark.parametrize("m", [16, 17, 32, 33])
@pytest.mark.parametrize("k,n", [(2048, 2048), (2056, 2048), (511, 1024), (511, 1030)])
def test_dense_layers_of_few_rows_and_many_weights(m, k, n):
    """bf16, on either side of where rows are too many, or weights, to go without tiles."""
    x, w, res = random(m, k, "bf16", 1), random(n, k, "bf16", 2) / k ** 0.5, random(m, n, "bf16", 3)
    y, z = R.linear_forward(x, w, act="silu", residual=res, keep_z=True)
    want = host(x) @ host(w).T
    e = (4 * np.sqrt(k) + 4) * U * (np.abs(host(x)) @ np.abs(host(w)).T)
    near(z, want, e + HALF["bf16"] * np.abs(want) + 1e-38, "z")
    out = D.act(want, "silu") + host(res)
    near(y, out, 1.2 * e + 16 * U * np.abs(want) + (U + HALF["bf16"]) * np.abs(out) + 1e-38, "y")


@pytest.mark.parametrize("dt,small", [("f32", None), ("f32", 1e-35), ("bf16", None)])
def test_weight_gradient_over_many_rows(dt, small):
    """Sums of 2^28 terms of one sign, which may not be lost against what the sum has grown to; `small`: with values that three bf16 parts do not hold.
    Ranges of 2^18 rows are summed on their own, so a sum is as exact as one of 2^18 terms, within 4 sqrt(2^18) + 4 roundings, and their joining, 2^10 more."""
    m, k, n = (1 << 28) + 5, 8, 3
    torch.cuda.empty_cache()
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(m, k, device="cuda").normal_(generator=g).to(DT[dt])
    dz = x[:, :n].relu()
    if small:
        dz[::64, 0] = small
    dw, db = R.linear_wgrad(dz, x)
    want, size = torch.zeros(2, n, k, dtype=torch.float64, device="cuda")
    sums = torch.zeros(n, dtype=torch.float64, device="cuda")
    for i in range(0, m, 1 << 25):
        a, b = dz[i:i + (1 << 25)].double(), x[i:i + (1 << 25)].double()
        sums += a.sum(0)
        for j in range(n):
            terms = a[:, j:j + 1] * b
            want[j] += terms.sum(0)
            size[j] += terms.abs().sum(0)
    bound = (4 * 2 ** 9 + 4 + 2 ** 10) * U
    near(dw, host(want), bound * host(size), "dw")
    near(db, host(sums), bound * host(sums), "db")
