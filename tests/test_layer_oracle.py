"""Pins of the 64-bit oracle of the calls from the loss to the gradient: closed
forms, central differences of its own forward functions, and the bounds that
the checkpoint format states (CPU)."""
import math

import numpy as np
import pytest

import oracle.layer_oracle as L


def test_uniform_and_one_hot_rows():
    z = np.zeros((2, 8))
    z[1, 3] = 2000.0
    logp, lse, ent, ids, top = L.token_logprobs(z, [5, 3], 3)
    assert np.allclose([logp[0], lse[0], ent[0]], [-math.log(8), math.log(8), math.log(8)], rtol=0, atol=1e-15)
    assert (logp[1], lse[1], ent[1]) == (0.0, 2000.0, 0.0)
    assert ids.tolist() == [[0, 1, 2], [3, 0, 1]]  # ties by index
    assert np.allclose(top[0], -math.log(8)) and top[1, 0] == 0.0


def test_masked_rows():
    z = np.array([[-np.inf, 1.0, -np.inf, 1.0], [-np.inf] * 4, [0.0, np.nan, 1.0, 2.0], [np.inf, 0.0, 0.0, 0.0]])
    logp, lse, ent, ids, top = L.token_logprobs(z, [1, 0, -1, 0], 3)
    assert np.allclose([logp[0], lse[0], ent[0]], [-math.log(2), 1 + math.log(2), math.log(2)])
    assert ids[0].tolist() == [1, 3, -1] and top[0, 2] == -np.inf
    assert lse[1] == -np.inf and logp[1] == -np.inf and ent[1] == 0 and ids[1].tolist() == [-1] * 3
    assert np.isnan(lse[2]) and logp[2] == 0 and np.isnan(lse[3]) and np.isnan(logp[3]) and ids[3].tolist() == [-1] * 3


@pytest.mark.parametrize("k", [0, 3])
def test_loss_gradient_is_the_difference_quotient(k):
    r = np.random.default_rng(k)
    z = r.standard_normal((4, 11)) * 2
    z[1, ::3] = -np.inf
    t = np.array([2, 4, -1, 10])
    gl, ge, gs, gt = r.standard_normal(4), r.standard_normal(4), r.standard_normal(4), r.standard_normal((4, k))
    _, lse, ent, ids, _ = L.token_logprobs(z, t, k)

    def f(x):
        logp, s, h, _, _ = L.token_logprobs(x, t, 0)
        at = np.take_along_axis(x, np.maximum(ids, 0), 1) - s[:, None] if k else np.zeros((4, 0))
        at = np.where(ids >= 0, at, 0.0)
        return np.sum(gl * np.where(t >= 0, logp, 0)) + np.sum(ge * h) + np.sum(gs * s) + np.sum(gt * at)
    g = L.token_logprobs_grad(z, t, lse, ent, gl, gs, ge, ids, gt if k else None)
    for i in range(4):
        for j in range(11):
            if z[i, j] == -np.inf:
                continue
            h = 1e-5
            up, dn = z.copy(), z.copy()
            up[i, j] += h
            dn[i, j] -= h
            assert abs((f(up) - f(dn)) / (2 * h) - g[i, j]) <= 1e-8


@pytest.mark.parametrize("kind", [L.NONE, L.RELU, L.GELU, L.GELU_TANH, L.SILU])
def test_slope_is_the_difference_quotient(kind):
    x = np.linspace(-9, 9, 1201) + 1e-3  # 0 itself left out
    h = 1e-5
    d = (L.act(x + h, kind) - L.act(x - h, kind)) / (2 * h)
    assert np.max(np.abs(d - L.act_slope(x, kind))) <= 1e-9


def test_checkpoint_bounds_and_fixed_points():
    r = np.random.default_rng(0)
    x = (r.standard_normal((5, 70)) * np.exp(3 * r.standard_normal((5, 70)))).astype(np.float32).astype(np.float64)
    x[1, 40] = np.nan
    x[2, :32] = 0
    x[3, 64:] = 2.0 ** -140
    codes, scales = L.checkpoint(x)
    v = L.checkpoint_values(codes, scales, 70)
    assert codes.shape == (5, 96) and scales.shape == (5, 3) and not codes[:, 70:].any()
    assert np.all(np.isnan(v[1, 32:64])) and np.all(np.isfinite(np.delete(v, 1, 0)))
    for i in range(5):
        for g in range(3):
            if (i, g) == (1, 1):
                continue
            a, b = x[i, 32 * g:32 * g + 32], v[i, 32 * g:32 * g + 32]
            e = int(scales[i, g]) - 127
            assert np.all(np.abs(a - b) <= 2.0 ** (e - 1))
            top = np.abs(a).max()
            assert e >= -126 and (e == -126 or np.rint(top / 2.0 ** (e - 1)) > 127) and np.abs(codes[i]).max() <= 127
    assert L.checkpoint(np.array([[127.0, -1.0]]))[1][0, 0] == 127       # e = 0
    assert L.checkpoint(np.array([[127.49, -1.0]]))[1][0, 0] == 127
    assert L.checkpoint(np.array([[127.5, -1.0]]))[1][0, 0] == 128       # rounds to 128: e = 1
    # values that the format holds are kept exactly
    again = L.checkpoint_values(*L.checkpoint(np.nan_to_num(v)), 70)
    assert np.array_equal(again, np.nan_to_num(v))


def test_weight_grad_is_the_product():
    r = np.random.default_rng(1)
    x, dy, g = r.standard_normal((7, 3)), r.standard_normal((7, 4)), r.standard_normal((3, 4))
    ref = np.array([[sum(x[t, i] * dy[t, j] for t in range(7)) for j in range(4)] for i in range(3)])
    assert np.allclose(L.weight_grad(x, dy), ref) and np.allclose(L.weight_grad(x, dy, g, 0.5), ref + 0.5 * g)
