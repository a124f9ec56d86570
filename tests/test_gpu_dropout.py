"""Dropout on the GPU against the 64-bit oracle.  The mask is exact; a kept value is
scaled in fp32 (the scale and the product rounded: 2 u), added to the residual (u) and
rounded once to the type (half a step)."""
import pytest

from tests.gpu_util import gpu_env, say

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def env():
    torch, B, dev = gpu_env()
    h = B.shampoo_create(0)
    yield torch, B, dev, h
    B.shampoo_destroy(h)


def view(torch, dev, n, c, dtype, pad, shift, x):
    buf = torch.full((n * (c + pad) + shift,), 7.5, device=dev, dtype=dtype)
    v = buf[shift:].view(n, c + pad)[:, :c]
    v.copy_(x)
    return buf, v


def check(env, n, c, dtype, rate, seed, offset, residual, pad=0, shift=0, place="new"):
    import oracle.model_oracle as M
    torch, B, dev, h = env
    g = torch.Generator(device=dev).manual_seed(n + c)
    _, X = view(torch, dev, n, c, dtype, pad, shift, torch.randn(n, c, generator=g, device=dev))
    _, R = view(torch, dev, n, c, dtype, pad, shift, torch.randn(n, c, generator=g, device=dev))
    R = R if residual else None
    keep, cut = M.kept(n, c, rate, seed, offset)
    keep = torch.from_numpy(keep).to(dev)
    ref = M.dropout(X, keep, cut, R)
    size = M.dropout(X, keep, cut).abs() + ref.abs()
    buf, Y = view(torch, dev, n, c, dtype, pad, shift, torch.full((n, c), float("nan"), device=dev))
    Y = X if place == "x" else R if place == "r" else Y
    B.shampoo_dropout(h, X, Y, rate, seed, offset=offset, R=R)
    torch.cuda.synchronize()
    half = 2.0 ** -8 if dtype is torch.bfloat16 else U
    err = (Y.double() - ref).abs()
    assert bool((err <= half * ref.abs() * (1 + 4 * U) + 4 * U * size).all()), float(err.max())
    if not residual:
        assert bool((Y[~keep] == 0).all()) and bool((Y[keep] != 0).all())
    if place == "new":
        assert bool((buf[shift:].view(n, -1)[:, c:] == 7.5).all()) and bool((buf[:shift] == 7.5).all())


SHAPES = [(1, 1), (1, 7), (3, 8), (5, 33), (17, 100), (64, 1024), (1000, 129), (2, 40000), (4099, 61)]


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("n,c", SHAPES)
def test_dropout(env, n, c, dtype):
    dt = getattr(env[0], dtype)
    for rate, seed, offset, residual, pad, shift in ((0.1, 0, 0, False, 0, 0), (0.5, 2 ** 64 - 1, 2 ** 64 - 1, True, 8, 8),
                                                     (0.25, 0x123456789abcdef0, 5 << 32, True, 3, 1),
                                                     (0.999, 7, 9, False, 1, 5)):
        say("dropout", n, c, dtype, rate, seed, offset, residual, pad, shift)
        check(env, n, c, dt, rate, seed, offset, residual, pad, shift)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_in_place(env, dtype):
    dt = getattr(env[0], dtype)
    for place, residual in (("x", False), ("x", True), ("r", True)):
        say("dropout in place", dtype, place, residual)
        check(env, 50, 333, dt, 0.3, 5, 6, residual, 3, 1, place)


def test_rates_at_the_ends(env):
    torch, B, dev, h = env
    say("dropout rates")
    X, R = torch.randn(9, 77, device=dev), torch.randn(9, 77, device=dev)
    Y = torch.empty_like(X)
    B.shampoo_dropout(h, X, Y, 0.0, 1)
    assert torch.equal(Y, X)
    B.shampoo_dropout(h, X, Y, 1e-6, 1)  # below half of 2^-16: no element is dropped
    assert torch.equal(Y, X)
    for rate in (1.0, 1 - 1e-6):
        B.shampoo_dropout(h, X, Y, rate, 1, R=R)
        assert torch.equal(Y, R)
        B.shampoo_dropout(h, X, Y, rate, 1)
        assert bool((Y == 0).all())


def test_dropped_values_leave_no_trace(env):
    import oracle.model_oracle as M
    torch, B, dev, h = env
    say("dropout of NaN")
    X, Y = torch.ones(40, 100, device=dev), torch.empty(40, 100, device=dev)
    keep = torch.from_numpy(M.kept(40, 100, 0.5, 3, 4)[0]).to(dev)
    X[~keep] = float("nan")
    B.shampoo_dropout(h, X, Y, 0.5, 3, offset=4)
    assert torch.equal(Y, torch.where(keep, 2.0, 0.0))


def test_the_gradient_is_the_same_call(env):
    """d sum(g Y) / dX by differences: Y is linear in X, so a step of 2^-4 around whole
    numbers is exact with a scale of 2."""
    torch, B, dev, h = env
    say("dropout gradient")
    g = torch.randint(-4, 5, (6, 50), device=dev).float()
    X = torch.randint(-4, 5, (6, 50), device=dev).float()
    dX, hi, lo = (torch.empty_like(X) for _ in range(3))
    B.shampoo_dropout(h, g, dX, 0.5, 11, offset=2)
    B.shampoo_dropout(h, X + 0.0625, hi, 0.5, 11, offset=2, R=X)
    B.shampoo_dropout(h, X - 0.0625, lo, 0.5, 11, offset=2, R=X)
    assert torch.equal(dX, g * (hi - lo) * 8)


def test_masks_of_rows_and_offsets_differ(env):
    torch, B, dev, h = env
    say("dropout masks")
    X = torch.ones(64, 512, device=dev)
    ys = []
    for seed, offset in ((1, 0), (1, 1), (1, 1 << 32), (2, 0), (1 << 32, 0)):
        Y = torch.empty_like(X)
        B.shampoo_dropout(h, X, Y, 0.5, seed, offset=offset)
        ys.append(Y)
    for i in range(len(ys)):
        for j in range(i):
            # 32768 independent pairs agree in half of the places, deviation 0.003
            assert abs(float((ys[i] == ys[j]).float().mean()) - 0.5) < 0.015
    assert abs(float((ys[0][0] == ys[0][1]).float().mean()) - 0.5) < 0.11  # 512 pairs, 5 deviations


def test_far_rows(env):
    """More than 2^31 elements, and counters of rows past 2^16."""
    import oracle.model_oracle as M
    torch, B, dev, h = env
    n, c = 530000, 4096
    say("dropout far", n, c)
    X = torch.ones(n, c, device=dev, dtype=torch.bfloat16)
    B.shampoo_dropout(h, X, X, 0.5, 21, offset=22)
    torch.cuda.synchronize()
    for first in (0, 70000, n - 50):
        keep = torch.from_numpy(M.kept(50, c, 0.5, 21, 22, first)[0]).to(dev)
        assert torch.equal(X[first:first + 50] == 2, keep)
