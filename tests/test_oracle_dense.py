"""CPU: the float64 oracle of the dense block's operators -- generator against its published vector, gradients against central
differences, activations and their derivatives against their definitions."""
import math

import numpy as np
import pytest

from oracle import dense as D

ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def test_generator_is_splitmix64(golden_dir):
    want = [int(line, 16) for line in open(f"{golden_dir}/splitmix64_vector.txt") if not line.startswith("#") and line.strip()]
    assert [int(v) for v in D.splitmix64(0, len(want))] == want
    assert [int(v) for v in D.splitmix64(0, 1, first=1)] == want[1:2]
    # 64-bit wrap of the position
    assert int(D.splitmix64(5, 1, first=(1 << 64) - 1)[0]) == int(D.splitmix64(5 - D._STEP, 1)[0])


@pytest.mark.parametrize("n", [1, 2, 7, 64])
def test_mask_is_a_function_of_position(n):
    full = D.kept((3, 10), 50, n, 0.3)
    # later rows are those of a call whose offset was moved on by their words
    assert np.array_equal(full[20:], D.kept((3, 10 + 20 * ((n + 1) // 2)), 30, n, 0.3))
    # an odd width leaves the last word's high half unused
    if n % 2:
        assert np.array_equal(full, D.kept((3, 10), 50, n + 1, 0.3)[:, :n])
    assert not np.array_equal(D.kept((3, 10), 50, 64, 0.3), D.kept((4, 10), 50, 64, 0.3))


@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.9])
def test_mask_keeps_one_minus_p(p):
    m = D.kept((77, 0), 400, 501, p)
    sd = math.sqrt(p * (1 - p) / m.size)
    assert abs(m.mean() - (1 - p)) <= 5 * sd
    for col in (0, 1, 250, 500):   # low and high halves alike
        assert abs(m[:, col].mean() - (1 - p)) <= 5 * math.sqrt(p * (1 - p) / 400)


@pytest.mark.parametrize("name", ACTS)
def test_activations(name):
    z = np.concatenate([np.linspace(-9, 9, 181), [1e-8, 40.0, -40.0]])
    direct = {"none": lambda t: t, "relu": lambda t: max(t, 0.0), "gelu": lambda t: 0.5 * t * math.erfc(-t / math.sqrt(2)),
              "gelu_tanh": lambda t: 0.5 * t * (1 + math.tanh(math.sqrt(2 / math.pi) * (t + 0.044715 * t ** 3))),
              "silu": lambda t: t / (1 + math.exp(-t))}[name]
    np.testing.assert_allclose(D.act(z, name), [direct(t) for t in z], rtol=1e-12, atol=1e-14)
    h = 1e-5
    z = z[np.abs(z) > 1e-3]
    np.testing.assert_allclose(D.slope(z, name), (D.act(z + h, name) - D.act(z - h, name)) / (2 * h), rtol=1e-7, atol=1e-8)
    assert D.slope(np.zeros(1), "relu")[0] == 0


@pytest.mark.parametrize("name,p", [("gelu", 0.0), ("relu", 0.25), ("silu", 0.5), ("gelu_tanh", 0.1)])
def test_block_gradients_against_differences(name, p):
    rng = np.random.default_rng(1)
    M, N, H = 5, 6, 9
    x = rng.standard_normal((M, N))
    params = [1 + 0.1 * rng.standard_normal(N), 0.1 * rng.standard_normal(N), rng.standard_normal((H, N)) / 2, rng.standard_normal(H) * 0.1,
              rng.standard_normal((N, H)) / 3, rng.standard_normal(N) * 0.1]
    rngs, dy = ((9, 0), (9, 100)), rng.standard_normal((M, N))
    _, saved = D.mlp_block(x, params, name, p, rngs)
    dx, grads = D.mlp_block_backward(dy, x, params, saved, name, p, rngs)
    h = 1e-6
    for t, g in zip([x] + params, (dx,) + tuple(grads)):
        for _ in range(8):
            i = tuple(rng.integers(s) for s in t.shape)
            old = t[i]
            t[i] = old + h
            up = (D.mlp_block(x, params, name, p, rngs)[0] * dy).sum()
            t[i] = old - h
            down = (D.mlp_block(x, params, name, p, rngs)[0] * dy).sum()
            t[i] = old
            assert abs((up - down) / (2 * h) - g[i]) <= 1e-6 * max(1.0, abs(g[i]))


def test_layernorm_rows():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((4, 33)) * 3 + 100
    y, mean, rstd = D.layernorm(x, eps=0.0)
    np.testing.assert_allclose(y.mean(1), 0, atol=1e-13)
    np.testing.assert_allclose((y * y).mean(1), 1, rtol=1e-12)
    # a constant row: eps alone
    y, mean, rstd = D.layernorm(np.full((1, 7), 5.0), eps=1e-5)
    assert np.all(y == 0) and mean[0] == 5 and abs(rstd[0] - 1e5 ** 0.5) < 1e-9
