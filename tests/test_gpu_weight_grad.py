"""Weight gradients from 8-bit checkpoints on the GPU against the 64-bit oracle.

Tolerance: products are exact (fp32 gradients: in three exact terms whose
products are), sums of K terms are rounded at each step.  For terms of random
sign the accumulated rounding of a running sum is u sqrt(K) / 4 of the result's
size (u = 2^-24), for any order no more; the bound on the relative Frobenius
error is u (16 + sqrt(K)), and 2^-8 more where G is stored in bf16."""
import numpy as np
import pytest

import oracle.layer_oracle as L
from tests.gpu_util import gpu_env, host, rel, say

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def env():
    torch, B, dev = gpu_env()
    h = B.shampoo_create(0)
    yield torch, B, dev, h
    B.shampoo_destroy(h)


def inputs(n, c, o, seed):
    r = np.random.default_rng(seed)
    x = (r.standard_normal((n, c)) * np.exp(0.7 * r.standard_normal((1, c)))).astype(np.float32)
    return x, r.standard_normal((n, o)).astype(np.float32)


def place(torch, dev, x, dtype, pad=0, shift=0):
    n, c = x.shape
    buf = torch.full((n * (c + pad) + shift,), 7.5, device=dev, dtype=dtype)
    view = buf[shift:].view(n, c + pad)[:, :c]
    view.copy_(torch.from_numpy(x).to(dtype))
    return buf, view


def checkpoint(env, x):
    torch, B, dev, h = env
    ck = torch.empty(B.shampoo_act_checkpoint_bytes(*x.shape), device=dev, dtype=torch.uint8)
    B.shampoo_act_encode(h, torch.from_numpy(x).to(dev), ckpt_x=ck)
    v = torch.empty(x.shape, device=dev)
    B.shampoo_act_decode(h, ck, v)  # exact: test_gpu_act_checkpoint
    return ck, host(v.double())


def call(env, ck, dy, G, n, beta=0.0, stream=None):
    torch, B, dev, h = env
    nws = B.shampoo_act_weight_grad_workspace_bytes(n, *G.shape)
    ws = torch.full((nws,), 0xFF, device=dev, dtype=torch.uint8) if nws else None
    B.shampoo_act_weight_grad(h, ck, dy, G, beta=beta, workspace=ws, stream=stream)


def check(env, n, c, o, dt, gt, pad=0, shift=0, beta=0.0, seed=0):
    torch, B, dev, h = env
    x, dy = inputs(n, c, o, seed + n)
    ck, held = checkpoint(env, x)
    _, d = place(torch, dev, dy, dt, pad, shift)
    g0 = np.random.default_rng(1).standard_normal((c, o)).astype(np.float32) * np.sqrt(n)
    gbuf, G = place(torch, dev, g0 if beta else np.full((c, o), np.nan, np.float32), gt, pad, shift)
    gg = host(G.double())
    call(env, ck, d, G, n, beta)
    torch.cuda.synchronize()
    ref = L.weight_grad(held, host(d.double()), gg, beta)
    tol = U * (16 + np.sqrt(n)) + (2.0 ** -8 if gt is torch.bfloat16 else 0)
    err = rel(host(G.double()), ref)
    assert err <= tol, (err, tol)
    assert bool(torch.all(gbuf[shift:].view(c, o + pad)[:, o:] == 7.5)) and bool(torch.all(gbuf[:shift] == 7.5))
    return G


SHAPES = [(1, 1, 1), (1, 32, 16), (2, 33, 17), (5, 64, 64), (31, 100, 7), (64, 128, 128), (65, 129, 130),
          (100, 300, 520), (333, 517, 96), (1000, 64, 64), (4097, 40, 33), (20000, 96, 256), (513, 1024, 1030),
          (2048, 512, 768)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("g_dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,c,o", SHAPES)
def test_product(env, n, c, o, dtype, g_dtype):
    torch = env[0]
    for pad, shift, beta in ((0, 0, 0.0), (3, 1, 0.0), (8, 0, 1.0), (0, 0, -0.5)):
        say("weight grad", n, c, o, dtype, g_dtype, pad, shift, beta)
        check(env, n, c, o, getattr(torch, dtype), getattr(torch, g_dtype), pad, shift, beta)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_elementwise(env, dtype):
    """Each element within the worst-case bound of its own sum of |terms|."""
    torch, B, dev, h = env
    n, c, o = 700, 260, 270
    say("weight grad elementwise", dtype)
    x, dy = inputs(n, c, o, 5)
    dy[:, 3] *= 1e-20
    dy[:, 4] *= 1e20
    ck, held = checkpoint(env, x)
    _, d = place(torch, dev, dy, getattr(torch, dtype))
    G = torch.empty(c, o, device=dev)
    call(env, ck, d, G, n)
    torch.cuda.synchronize()
    dd = host(d.double())
    ref = L.weight_grad(held, dd)
    bound = U * (n + 16) * (np.abs(held).T @ np.abs(dd))
    assert np.all(np.abs(host(G.double()) - ref) <= bound)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_no_tokens_and_small_integers(env, dtype):
    """No tokens: G = beta G, and zero for beta = 0 whatever G held; integers
    are summed exactly."""
    torch, B, dev, h = env
    dt = getattr(torch, dtype)
    say("weight grad no tokens", dtype)
    empty = torch.empty(0, device=dev, dtype=torch.uint8)
    G = torch.full((40, 30), float("nan"), device=dev)
    B.shampoo_act_weight_grad(h, empty, torch.empty(0, 30, device=dev, dtype=dt), G)
    H = torch.full((40, 30), 3.0, device=dev)
    B.shampoo_act_weight_grad(h, empty, torch.empty(0, 30, device=dev, dtype=dt), H, beta=0.5)
    torch.cuda.synchronize()
    assert bool(torch.all(G == 0)) and bool(torch.all(H == 1.5))
    r = np.random.default_rng(3)
    for n, c, o in ((37, 50, 60), (3000, 140, 150), (9000, 32, 64)):
        x = r.integers(-8, 9, (n, c)).astype(np.float32)
        x[:, ::32] = 100  # scale 1 in every group
        dy = r.integers(-8, 9, (n, o)).astype(np.float32)
        ck, held = checkpoint(env, x)
        assert np.array_equal(held, x)
        G = torch.empty(c, o, device=dev)
        call(env, ck, torch.from_numpy(dy).to(dev).to(dt), G, n)
        torch.cuda.synchronize()
        assert np.array_equal(host(G.double()), L.weight_grad(x, dy))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_bad_values(env, dtype):
    """A NaN group spoils its own rows of G, an infinity or NaN in dY its own
    column (infinity times zero is NaN); a tail of tokens past the last full
    stage takes part; values near the ends of the range survive."""
    torch, B, dev, h = env
    dt = getattr(torch, dtype)
    say("weight grad bad values", dtype)
    n, c, o = 77, 100, 90
    x, dy = inputs(n, c, o, 8)
    x[70, 40] = np.inf     # columns 32..63
    dy[76, 5] = np.nan
    dy[3, 6] = np.inf
    dy[:, 7] = 0
    dy[9, 7] = 3.3e38
    dy[:, 8] = 0
    dy[2, 8] = 1.5e-38
    x[9] = np.where(np.isfinite(x[9]), 0.5, x[9])
    ck, held = checkpoint(env, x)
    _, d = place(torch, dev, dy, dt)
    dd = host(d.double())
    G = torch.empty(c, o, device=dev)
    call(env, ck, d, G, n)
    torch.cuda.synchronize()
    got = host(G.double())
    rows = np.zeros(c, dtype=bool)
    rows[32:64] = True
    assert np.all(np.isnan(got[rows])) and np.all(np.isnan(got[:, 5]))
    with np.errstate(all="ignore"):
        want6 = np.where(held[3] == 0, np.nan, np.sign(held[3]) * np.inf)
    assert np.array_equal(got[~rows, 6], want6[~rows], equal_nan=True)
    cols = [j for j in range(o) if j not in (5, 6)]
    ok = np.ix_(~rows, cols)
    ref = held[:, ~rows].T @ dd[:, cols]
    bound = U * (n + 16) * (np.abs(held[:, ~rows]).T @ np.abs(dd[:, cols])) + 2.0 ** -126
    assert np.all(np.abs(got[ok] - ref) <= bound)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_subnormal_terms(env, dtype):
    """fp32 gradients around 2^-110, whose lower terms reach bf16's subnormals."""
    torch, B, dev, h = env
    say("weight grad small", dtype)
    n, c, o = 130, 64, 48
    x, dy = inputs(n, c, o, 3)
    x = x * np.float32(2.0 ** 40)
    dy = dy * np.float32(2.0 ** -110)
    ck, held = checkpoint(env, x)
    _, d = place(torch, dev, dy, getattr(torch, dtype))
    G = torch.empty(c, o, device=dev)
    call(env, ck, d, G, n)
    torch.cuda.synchronize()
    assert rel(host(G.double()), L.weight_grad(held, host(d.double()))) <= U * (16 + np.sqrt(n))


def test_deterministic_stream_and_graph(env):
    torch, B, dev, h = env
    for n, c, o, dt in ((9000, 96, 130, torch.bfloat16), (600, 300, 300, torch.float32)):
        say("weight grad deterministic", n, c, o, dt)
        x, dy = inputs(n, c, o, 2)
        ck, held = checkpoint(env, x)
        _, d = place(torch, dev, dy, dt)
        want = torch.empty(c, o, device=dev)
        call(env, ck, d, want, n)
        torch.cuda.synchronize()
        for _ in range(3):
            G = torch.empty(c, o, device=dev)
            call(env, ck, d, G, n)
            assert torch.equal(G, want)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        H = torch.zeros(c, o, device=dev)
        torch.cuda.synchronize()
        call(env, ck, d, H, n, stream=side)
        side.synchronize()
        assert torch.equal(H, want)
        nws = B.shampoo_act_weight_grad_workspace_bytes(n, c, o)
        ws = torch.zeros(nws, device=dev, dtype=torch.uint8) if nws else None
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.shampoo_act_weight_grad(h, ck, d, H, workspace=ws)
        for rep in range(4):
            H.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(H, want), rep


def test_offsets_past_32_bits(env):
    torch, B, dev, h = env
    say("weight grad large offsets")
    n, c, o, ld = 3, 64, 100, (1 << 30) + 8
    buf = torch.empty((n - 1) * ld + o, device=dev, dtype=torch.bfloat16)
    d = buf.as_strided((n, o), (ld, 1))
    x, dy = inputs(n, c, o, 6)
    d.copy_(torch.from_numpy(dy).bfloat16())
    ck, held = checkpoint(env, x)
    gbuf = torch.empty((c - 1) * (1 << 26) + o, device=dev)
    G = gbuf.as_strided((c, o), (1 << 26, 1))
    call(env, ck, d, G, n)
    torch.cuda.synchronize()
    assert rel(host(G.double()), L.weight_grad(held, host(d.double()))) <= U * 18
    n, c = 66000, 32768  # codes past 2^31 bytes
    say("weight grad large checkpoint")
    x = torch.zeros(n, c, device=dev, dtype=torch.bfloat16)
    x[-3:, -40:] = 2.0
    ck = torch.empty(B.shampoo_act_checkpoint_bytes(n, c), device=dev, dtype=torch.uint8)
    B.shampoo_act_encode(h, x, ckpt_x=ck)
    del x
    d = torch.ones(n, 5, device=dev, dtype=torch.bfloat16)
    G = torch.empty(c, 5, device=dev)
    call(env, ck, d, G, n)
    torch.cuda.synchronize()
    assert bool(torch.all(G[-40:] == 6)) and bool(torch.all(G[:-40] == 0))


# Sizes for every tile, in one part of the tokens and in several, none a multiple
# of a tile or a stage; test_layer_plans.py checks that the dispatch rules send
# them there.
LARGE = [(65, 3073, 4090), (70, 2051, 2055), (321, 2053, 4090), (1027, 1283, 3079), (8195, 1025, 515),
         (16389, 1537, 771)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,c,o", LARGE)
def test_large_tiles(env, n, c, o, dtype):
    torch = env[0]
    for g_dtype, pad, shift, beta in (("float32", 0, 0, 0.0), ("float32", 3, 1, -0.5), ("bfloat16", 6, 0, 1.0)):
        say("weight grad large", n, c, o, dtype, g_dtype, pad, shift, beta)
        check(env, n, c, o, getattr(torch, dtype), getattr(torch, g_dtype), pad, shift, beta)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,c,o", LARGE)
def test_large_tiles_contain_bad_values(env, n, c, o, dtype):
    """A NaN group spoils the rows of its columns, a NaN in dY its column; every
    other element keeps its bits."""
    torch, B, dev, h = env
    dt = getattr(torch, dtype)
    say("weight grad large bad values", n, c, o, dtype)
    g = torch.Generator(device=dev).manual_seed(n)
    x, dy = torch.randn(n, c, device=dev, generator=g), torch.randn(n, o, device=dev, generator=g).to(dt)
    ck = torch.empty(B.shampoo_act_checkpoint_bytes(n, c), device=dev, dtype=torch.uint8)
    B.shampoo_act_encode(h, x, ckpt_x=ck)
    want, G = torch.empty(c, o, device=dev), torch.empty(c, o, device=dev)
    call(env, ck, dy, want, n)
    x[n - 1, c - 1] = float("nan")   # the last, shorter group
    x[n // 2, 40] = float("inf")
    B.shampoo_act_encode(h, x, ckpt_x=ck)
    dy[0, o - 1] = float("nan")
    dy[n - 1, 130] = float("nan")
    call(env, ck, dy, G, n)
    torch.cuda.synchronize()
    rows = list(range(32, 64)) + list(range((c - 1) // 32 * 32, c))
    bad = torch.zeros(c, o, device=dev, dtype=torch.bool)
    bad[rows] = True
    bad[:, [130, o - 1]] = True
    assert bool(torch.all(torch.isnan(G[bad]))) and torch.equal(G[~bad], want[~bad])
