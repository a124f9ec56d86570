"""8-bit activation checkpoints on the GPU against the 64-bit oracle.

Codes and scale bytes are exact (powers of two scale without rounding), and so
are decoded values.  Activations and their slopes: a handful of fp32 roundings
(u = 2^-24) of terms no larger than max(1, |x|), and 2^-8 of the result where it
is stored in bf16."""
import numpy as np
import pytest

import oracle.layer_oracle as L
from tests.gpu_util import gpu_env, host, say

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
ACTS = [L.NONE, L.RELU, L.GELU, L.GELU_TANH, L.SILU]
SHAPES = [(1, 1), (1, 31), (2, 32), (3, 33), (5, 64), (1, 4096), (7, 257), (129, 96), (64, 1000), (33, 4099),
          (1031, 40)]


@pytest.fixture(scope="module")
def env():
    torch, B, dev = gpu_env()
    h = B.shampoo_create(0)
    yield torch, B, dev, h
    B.shampoo_destroy(h)


def act_input(n, c, seed):
    r = np.random.default_rng(seed)
    x = (r.standard_normal((n, c)) * np.exp(1.5 * r.standard_normal((1, c)))).astype(np.float32)
    x[r.random((n, c)) < 0.1] = 0
    return x


def place(torch, dev, x, dtype, pad=0, shift=0):
    n, c = x.shape
    buf = torch.full((n * (c + pad) + shift,), 7.5, device=dev, dtype=dtype)
    view = buf[shift:].view(n, c + pad)[:, :c]
    view.copy_(torch.from_numpy(x).to(dtype))
    return buf, view


def blank(env, n, c):
    torch, B, dev, h = env
    # filled, so that bytes the call leaves out show; 64 more bytes behind it
    return torch.full((B.shampoo_act_checkpoint_bytes(n, c) + 64,), 0x5A, device=dev, dtype=torch.uint8)


def same_checkpoint(buf, x):
    """buf holds the checkpoint of x; the bytes between its parts are free."""
    codes, scales = L.checkpoint(x)
    off = -(-codes.size // 256) * 256
    b = host(buf)
    assert np.array_equal(b[:codes.size].view(np.int8).reshape(codes.shape), codes)
    assert np.array_equal(b[off:off + scales.size].reshape(scales.shape), scales)
    assert np.all(b[-64:] == 0x5A)
    return codes, scales


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("kind", ACTS)
@pytest.mark.parametrize("n,c", SHAPES)
def test_encode_decode(env, n, c, kind, dtype):
    torch, B, dev, h = env
    dt = getattr(torch, dtype)
    for pad, shift, in_place in ((0, 0, False), (5, 1, False), (8, 0, True)):
        say("act encode", n, c, kind, dtype, pad, shift, in_place)
        xbuf, x = place(torch, dev, act_input(n, c, n + c), dt, pad, shift)
        xx = host(x.double())
        ybuf, y = (xbuf, x) if in_place else place(torch, dev, np.zeros((n, c), np.float32), dt, pad, shift)
        cx, cy = blank(env, n, c), blank(env, n, c)
        B.shampoo_act_encode(h, x, ckpt_x=cx, act=kind, Y=y, ckpt_y=cy)
        torch.cuda.synchronize()
        yy = host(y.double())
        ref = L.act(xx, kind)
        tol = 8 * U * np.abs(ref) + 4 * U * np.abs(xx) + 1e-37 + (2.0 ** -8 * np.abs(ref) if dt is torch.bfloat16 else 0)
        assert np.all(np.abs(yy - ref) <= tol), float((np.abs(yy - ref) / tol).max())
        if kind in (L.NONE, L.RELU):
            assert np.array_equal(yy, ref)
        codes, scales = same_checkpoint(cx, xx)
        codes_y, scales_y = same_checkpoint(cy, yy)  # of y as stored
        for out_t in (torch.float32, torch.bfloat16):
            vbuf, v = place(torch, dev, np.zeros((n, c), np.float32), out_t, pad, shift)
            B.shampoo_act_decode(h, cx, v)
            torch.cuda.synchronize()
            assert np.array_equal(host(v.double()), L.checkpoint_values(codes, scales, c))
            rest = vbuf[shift:].view(n, c + pad)[:, c:]
            assert bool(torch.all(rest == 7.5)) and bool(torch.all(vbuf[:shift] == 7.5))
        rest = ybuf[shift:].view(n, c + pad)[:, c:]
        assert bool(torch.all(rest == 7.5)) and bool(torch.all(ybuf[:shift] == 7.5))


def test_each_output_alone(env):
    torch, B, dev, h = env
    say("act encode outputs alone")
    n, c = 37, 200
    _, x = place(torch, dev, act_input(n, c, 3), torch.bfloat16)
    cx, cy, y = blank(env, n, c), blank(env, n, c), torch.empty_like(x)
    B.shampoo_act_encode(h, x, ckpt_x=cx, act=L.SILU, Y=y, ckpt_y=cy)
    a, b, z = blank(env, n, c), blank(env, n, c), torch.empty_like(x)
    B.shampoo_act_encode(h, x, ckpt_x=a, act=L.SILU)
    B.shampoo_act_encode(h, x, act=L.SILU, Y=z)
    B.shampoo_act_encode(h, x, act=L.SILU, ckpt_y=b)
    torch.cuda.synchronize()
    assert torch.equal(y, z)
    same_checkpoint(a, host(x.double()))
    same_checkpoint(b, host(y.double()))
    with pytest.raises(B.ShampooError):
        B.shampoo_act_encode(h, x, act=L.SILU)
    with pytest.raises(B.ShampooError):
        B.shampoo_act_encode(h, x, ckpt_x=a, act=9)
    with pytest.raises(B.ShampooError):
        B.shampoo_act_encode(h, x, ckpt_x=blank(env, n + 1, c)[1:])
    e = torch.empty(0, 8, device=dev)
    B.shampoo_act_encode(h, e, ckpt_x=torch.empty(0, device=dev, dtype=torch.uint8))
    B.shampoo_act_decode(h, torch.empty(0, device=dev, dtype=torch.uint8), e)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_extreme_values(env, dtype):
    """Zeros, subnormals, the ends of the range, rounding carries, infinities
    and NaN: one group each, in full and in short groups."""
    torch, B, dev, h = env
    dt = getattr(torch, dtype)
    low = float(torch.finfo(dt).max)
    r = np.random.default_rng(0)
    x = r.standard_normal((16, 70)).astype(np.float32)
    x[0] = 0
    x[1] = 2.0 ** -140
    x[2, ::2] = 2.0 ** -127
    x[3] *= 2.0 ** -120
    x[4, 5] = low
    x[5] = -low
    x[6, 40] = np.inf
    x[7, 69] = -np.inf
    x[8, 3] = np.nan
    x[9, 0], x[9, 32], x[9, 64] = 127.5, 127.0, 255.0
    x[10, 0], x[10, 1] = 127.0, 0.5  # a tie: rounds to even
    x[11] = 1e-38
    x[12, :32] = 126.5
    x[13] = -0.0
    x[14] = 2.0 ** 100
    say("act extremes", dtype)
    _, v = place(torch, dev, x, dt, 2)
    xx = host(v.double())
    cx = blank(env, 16, 70)
    B.shampoo_act_encode(h, v, ckpt_x=cx)
    torch.cuda.synchronize()
    codes, scales = same_checkpoint(cx, xx)
    out = torch.zeros(16, 70, device=dev, dtype=dt)
    B.shampoo_act_decode(h, cx, out)
    torch.cuda.synchronize()
    assert np.array_equal(host(out.double()), L.checkpoint_values(codes, scales, 70), equal_nan=True)
    for kind in ACTS:  # finite large values neither overflow nor turn into NaN
        y, dx = torch.zeros_like(v), torch.zeros_like(v)
        B.shampoo_act_encode(h, v, act=kind, Y=y)
        B.shampoo_act_grad(h, cx, kind, torch.ones_like(v), dx)
        torch.cuda.synchronize()
        fin = np.isfinite(xx)
        assert np.all(np.isfinite(host(y.double())[fin]))
        bad = np.isnan(host(y.double())[np.isnan(xx)])
        assert np.all(bad)
        held = L.checkpoint_values(codes, scales, 70)
        got, ref = host(dx.double()), L.act_slope(held, kind)
        if kind == L.NONE:
            assert np.all(got == 1)
        else:
            assert np.array_equal(np.isnan(got), np.isnan(held))
            ok = ~np.isnan(held)
            assert np.all(np.abs(got[ok] - ref[ok]) <= 2.0 ** -8 * np.abs(ref[ok]) + 32 * U)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("kind", ACTS)
@pytest.mark.parametrize("n,c", SHAPES)
def test_gradient(env, n, c, kind, dtype):
    torch, B, dev, h = env
    dt = getattr(torch, dtype)
    codes, scales = L.checkpoint(act_input(n, c, 2 * n + c))
    ck = torch.from_numpy(L.checkpoint_bytes(act_input(n, c, 2 * n + c))).to(dev)
    held = L.checkpoint_values(codes, scales, c)
    g = np.random.default_rng(c).standard_normal((n, c)).astype(np.float32)
    for pad, shift, in_place in ((0, 0, False), (3, 1, False), (8, 0, True)):
        say("act grad", n, c, kind, dtype, pad, shift, in_place)
        dbuf, dy = place(torch, dev, g, dt, pad, shift)
        gg = host(dy.double())
        obuf, dx = (dbuf, dy) if in_place else place(torch, dev, np.zeros((n, c), np.float32), dt, pad, shift)
        B.shampoo_act_grad(h, ck, kind, dy, dx)
        torch.cuda.synchronize()
        ref = gg * L.act_slope(held, kind)
        # the slope: a few roundings of terms up to max(1, |x| times a factor that falls as fast as exp(-x^2 / 2)
        # or exp(-|x|)): at most about 2 in size
        tol = 32 * U * np.abs(gg) + 1e-37 + (2.0 ** -8 * np.abs(ref) if dt is torch.bfloat16 else 0)
        err = np.abs(host(dx.double()) - ref)
        assert np.all(err <= tol), float((err / tol).max())
        rest = obuf[shift:].view(n, c + pad)[:, c:]
        assert bool(torch.all(rest == 7.5)) and bool(torch.all(obuf[:shift] == 7.5))


def test_offsets_past_32_bits(env):
    torch, B, dev, h = env
    say("act large offsets")
    n, c, ld = 3, 4100, (1 << 30) + 24
    buf = torch.empty((n - 1) * ld + c, device=dev, dtype=torch.bfloat16)
    x = buf.as_strided((n, c), (ld, 1))
    x.copy_(torch.from_numpy(act_input(n, c, 8)).bfloat16())
    xx = host(x.double())
    cx = blank(env, n, c)
    B.shampoo_act_encode(h, x, ckpt_x=cx, act=L.RELU, Y=x)
    torch.cuda.synchronize()
    codes, scales = same_checkpoint(cx, xx)
    assert np.array_equal(host(x.double()), np.maximum(xx, 0))
    B.shampoo_act_decode(h, cx, x)
    torch.cuda.synchronize()
    held = L.checkpoint_values(codes, scales, c)
    assert np.array_equal(host(x.double()), held)
    B.shampoo_act_grad(h, cx, L.RELU, x, x)
    torch.cuda.synchronize()
    assert np.array_equal(host(x.double()), np.maximum(held, 0))


def test_large_checkpoint(env):
    """A checkpoint of more than 2^32 codes: its last rows."""
    torch, B, dev, h = env
    n, c = 70001, 65536
    say("act large checkpoint", n, c)
    x = torch.zeros(1, c, device=dev, dtype=torch.bfloat16).expand(n, c)
    big = torch.empty(n, c, device=dev, dtype=torch.bfloat16)
    big.copy_(x)
    big[-2:] = torch.from_numpy(act_input(2, c, 12)).bfloat16().to(dev)
    cx = torch.empty(B.shampoo_act_checkpoint_bytes(n, c), device=dev, dtype=torch.uint8)
    B.shampoo_act_encode(h, big, ckpt_x=cx)
    out = torch.full_like(big, 3.0)
    B.shampoo_act_decode(h, cx, out)
    torch.cuda.synchronize()
    held = L.checkpoint_values(*L.checkpoint(host(big[-2:].double())), c)
    assert np.array_equal(host(out[-2:].double()), held)
    assert not bool(torch.any(out[:-2] != 0))


def test_more_units_than_a_launch_takes(env):
    """Beyond 2^31 units of 8 columns a pass takes several launches."""
    torch, B, dev, h = env
    n, c = 131075, 131072
    say("act several launches", n, c)
    assert n * (c // 8) > 2 ** 31
    x = torch.zeros(n, c, device=dev, dtype=torch.bfloat16)
    x[-5:] = torch.from_numpy(act_input(5, c, 17)).bfloat16().to(dev)
    last = host(x[-5:].double())
    cx = torch.empty(B.shampoo_act_checkpoint_bytes(n, c), device=dev, dtype=torch.uint8)
    B.shampoo_act_encode(h, x, ckpt_x=cx)
    x.fill_(3.0)
    B.shampoo_act_decode(h, cx, x)
    torch.cuda.synchronize()
    assert np.array_equal(host(x[-5:].double()), L.checkpoint_values(*L.checkpoint(last), c))
    assert not bool(torch.any(x[:-5] != 0))


def test_other_stream_and_graph(env):
    torch, B, dev, h = env
    say("act stream and graph")
    n, c = 130, 515
    _, x = place(torch, dev, act_input(n, c, 5), torch.bfloat16)
    want_c, want_y, want_v, want_d = blank(env, n, c), torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)

    def calls(ck, y, v, d, stream=None):
        B.shampoo_act_encode(h, x, ckpt_x=ck, act=L.GELU, Y=y, stream=stream)
        B.shampoo_act_decode(h, ck, v, stream=stream)
        B.shampoo_act_grad(h, ck, L.GELU, v, d, stream=stream)
    calls(want_c, want_y, want_v, want_d)
    torch.cuda.synchronize()
    got = [blank(env, n, c), torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    calls(*got, stream=side)
    side.synchronize()
    for a, b in zip(got, (want_c, want_y, want_v, want_d)):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(*got)
    for rep in range(4):
        for a in got[1:]:
            a.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, (want_c, want_y, want_v, want_d)):
            assert torch.equal(a, b), rep


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("kind", [L.GELU, L.GELU_TANH, L.SILU])
def test_negative_tail(env, kind, dtype):
    """Activations and slopes on [-9, -3] to a relative bound: the results fall to
    1e-28, far below any bound in the size of x.  The exponent, which grows to
    about x^2, carries a few roundings; erfc and exp are at most 16 ulp off."""
    torch, B, dev, h = env
    say("act negative tail", kind, dtype)
    dt = getattr(torch, dtype)
    x = -np.linspace(3, 9, 64 * 96).reshape(64, 96).astype(np.float32)
    _, v = place(torch, dev, x, dt)
    xx = host(v.double())
    y = torch.empty_like(v)
    ck = blank(env, 64, 96)
    B.shampoo_act_encode(h, v, ckpt_x=ck, act=kind, Y=y)
    dx = torch.empty_like(v)
    B.shampoo_act_grad(h, ck, kind, torch.ones_like(v), dx)
    torch.cuda.synchronize()
    held = L.checkpoint_values(*L.checkpoint(xx), 96)
    for got, at, ref in ((y, xx, L.act(xx, kind)), (dx, held, L.act_slope(held, kind))):
        bound = 2.0 ** -8 + 2.0 ** -15 if dt is torch.bfloat16 else U * (40 + 4 * at * at)
        err = np.abs(host(got.double()) / ref - 1)
        assert np.all(err <= bound), float((err / bound).max())


def test_overlapping_checkpoints_are_refused(env):
    """A checkpoint shares no memory with the tensors of its call or the other
    checkpoint; nothing is written then.  One buffer that holds them one after
    the other is taken."""
    torch, B, dev, h = env
    say("act overlapping buffers")
    n, c = 8, 64
    nb = B.shampoo_act_checkpoint_bytes(n, c)
    size = n * c * 2
    buf = torch.zeros(2 * size + 2 * nb, device=dev, dtype=torch.uint8)

    def tensor(at):
        return buf[at:at + size].view(torch.bfloat16).view(n, c)
    x, y, kx, ky = 0, size, 2 * size, 2 * size + nb

    def encode(x, y, kx, ky):
        B.shampoo_act_encode(h, tensor(x), ckpt_x=buf[kx:kx + nb], act=L.GELU, Y=tensor(y), ckpt_y=buf[ky:ky + nb])
    for bad in ((x, y, x + size - 16, ky), (x, y, y, ky), (x, y, kx, 16), (x, y, kx, y + 32), (x, y, kx, kx),
                (x, y, kx, ky - 16)):
        with pytest.raises(B.ShampooError, match="overlap"):
            encode(*bad)
    G = buf[:64 * 4 * 4].view(torch.float32).view(c, 4)
    with pytest.raises(B.ShampooError, match="overlap"):
        B.shampoo_act_decode(h, buf[size - 16:size - 16 + nb], tensor(0))
    with pytest.raises(B.ShampooError, match="overlap"):
        B.shampoo_act_grad(h, buf[size:size + nb], L.GELU, tensor(0), tensor(size))
    with pytest.raises(B.ShampooError, match="overlap"):
        B.shampoo_act_weight_grad(h, buf[16:16 + nb], tensor(2 * size)[:, :4], G)
    torch.cuda.synchronize()
    assert not bool(torch.any(buf))
    tensor(x).copy_(torch.from_numpy(act_input(n, c, 1)).bfloat16())
    xx = host(tensor(x).double())
    encode(x, y, kx, ky)
    torch.cuda.synchronize()
    tail = torch.full((64,), 0x5A, device=dev, dtype=torch.uint8)
    same_checkpoint(torch.cat([buf[kx:ky], tail]), xx)
    same_checkpoint(torch.cat([buf[ky:], tail]), host(tensor(y).double()))
    # halves of one wider tensor
    wide = torch.zeros(n, 2 * c, device=dev)
    wide[:, :c] = tensor(x).float()
    B.shampoo_act_encode(h, wide[:, :c], act=L.RELU, Y=wide[:, c:])
    torch.cuda.synchronize()
    assert np.array_equal(host(wide[:, c:].double()), np.maximum(xx, 0)) and np.array_equal(host(wide[:, :c].double()), xx)
