"""Token log probabilities and their gradient on the GPU against the 64-bit
oracle.

Tolerances: with u = 2^-24, a row's sums have at most `vocab` positive terms,
added in any order with random rounding, and each exponential is a few ulp
off: the relative error of the sum, which is the absolute error of lse, stays
below e = u (16 + sqrt(vocab)), plus the rounding of the value itself.  The
entropy weighs the same terms by their distance from the largest logit: its
error is at most that times e and a few ulp.  A gradient is p times a bracket
of the outputs' gradients, p off by the rounding of z - lse; a bf16 result
adds half an ulp, 2^-8."""
import numpy as np
import pytest

import oracle.layer_oracle as L
from tests.gpu_util import gpu_env, host, say

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def env():
    torch, B, dev = gpu_env()
    h = B.shampoo_create(0)
    yield torch, B, dev, h
    B.shampoo_destroy(h)


def place(torch, dev, z, dtype, pad=0, shift=0):
    """z (host) as a device view with `pad` elements between rows, `shift`
    elements into its allocation; the rest of the buffer is a sentinel."""
    n, v = z.shape
    buf = torch.full((n * (v + pad) + shift,), 7.5, device=dev, dtype=dtype)
    view = buf[shift:].view(n, v + pad)[:, :v]
    view.copy_(torch.from_numpy(z).to(dtype))
    return buf, view


def forward(env, z, t, k, stream=None):
    torch, B, dev, h = env
    n, v = z.shape
    nan = float("nan")
    tt = None if t is None else torch.from_numpy(np.ascontiguousarray(t, dtype=np.int32)).to(dev)
    logp = None if t is None else torch.full((n,), nan, device=dev)
    lse, ent = torch.full((n,), nan, device=dev), torch.full((n,), nan, device=dev)
    ids = torch.full((n, k), -7, device=dev, dtype=torch.int32) if k else None
    top = torch.full((n, k), nan, device=dev) if k else None
    nws = B.shampoo_token_logprobs_workspace_bytes(n, v, k)
    ws = torch.full((nws,), 0xA5, device=dev, dtype=torch.uint8) if nws else None
    B.shampoo_token_logprobs(h, z, tt, logp, lse, entropy=ent, top_ids=ids, top_logp=top, workspace=ws,
                             stream=stream)
    return tt, logp, lse, ent, ids, top


def close(a, ref, tol, what):
    """Equal where the reference is not finite, within tol elsewhere."""
    a, ref = np.asarray(a, dtype=np.float64), np.asarray(ref, dtype=np.float64)
    fin = np.isfinite(ref)
    assert np.array_equal(a[~fin], ref[~fin], equal_nan=True), what
    err = np.abs(a[fin] - ref[fin])
    tol = np.broadcast_to(tol, ref.shape)[fin]
    assert np.all(err <= tol), (what, float((err / tol).max()))


def check(env, z, t, k):
    torch = env[0]
    _, logp, lse, ent, ids, top = forward(env, z, t, k)
    torch.cuda.synchronize()
    zz = host(z.double())
    o_logp, o_lse, o_ent, o_ids, o_top = L.token_logprobs(zz, t, k)
    n, v = zz.shape
    e = U * (16 + np.sqrt(v))
    close(host(lse), o_lse, e + 4 * U * np.abs(np.where(np.isfinite(o_lse), o_lse, 0)), "lse")
    close(host(ent), o_ent, 40 * e + 4 * U * np.abs(np.where(np.isfinite(o_ent), o_ent, 0)), "entropy")
    if t is not None:
        close(host(logp), o_logp, e + 4 * U * np.abs(np.where(np.isfinite(o_logp), o_logp, 0)), "logp")
    if k:
        assert np.array_equal(host(ids), o_ids)
        close(host(top), o_top, e + 4 * U * np.abs(np.where(np.isfinite(o_top), o_top, 0)), "top_logp")
    return lse, ent, ids


def logits(n, v, seed, mask="none", kind="normal"):
    r = np.random.default_rng(seed)
    z = (3 * r.standard_normal((n, v))).astype(np.float32)
    if kind == "ties":
        z = np.round(z)
    elif kind == "flat":
        z[:] = 1.25
    elif kind == "up":
        z = np.broadcast_to(np.linspace(-20, 20, v, dtype=np.float32), (n, v)).copy()
    elif kind == "down":
        z = np.broadcast_to(np.linspace(20, -20, v, dtype=np.float32), (n, v)).copy()
    elif kind == "peak":
        z[np.arange(n), r.integers(0, v, n)] = 60
    t = r.integers(0, v, n)
    if mask == "some":
        z[r.random((n, v)) < 0.4] = -np.inf
    elif mask == "rows":
        z[r.random((n, v)) < 0.3] = -np.inf
        z[::2] = -np.inf
    elif mask == "one":  # a single allowed entry
        keep = z[np.arange(n), t].copy()
        z[:] = -np.inf
        z[np.arange(n), t] = keep
    elif mask == "tail":
        z[:, v // 3:] = -np.inf
    elif mask == "head":
        z[:, :v - v // 3 - 1] = -np.inf
    t[r.random(n) < 0.2] = -1
    return z, t


SHAPES = [(1, 1), (3, 2), (2, 63), (5, 64), (4, 65), (7, 511), (300, 1000), (9, 1021), (3, 2047), (2, 4097),
          (1, 32768), (6, 20011), (1, 50001), (2, 131075)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,v", SHAPES)
def test_values(env, n, v, dtype):
    torch, B, dev, h = env
    dt = getattr(torch, dtype)
    for i, (mask, kind, k, pad, shift) in enumerate([("none", "normal", 8, 0, 0), ("some", "normal", 5, 3, 1),
                                                     ("rows", "ties", 33, 8, 0), ("none", "ties", 64, 0, 3),
                                                     ("one", "normal", 2, 1, 0), ("none", "peak", 1, 0, 0)]):
        say("logprobs", n, v, dtype, mask, kind, k, pad, shift)
        z, t = logits(n, v, 100 * i + n, mask, kind)
        buf, view = place(torch, dev, z, dt, pad, shift)
        check(env, view, t, k)


@pytest.mark.parametrize("kind", ["up", "down", "flat", "ties"])
@pytest.mark.parametrize("k", [0, 1, 16, 64])
def test_orders_and_ties(env, kind, k):
    """Rows that rise or fall throughout, and rows of equal values."""
    torch, B, dev, h = env
    for n, v, mask in ((2, 9000, "none"), (3, 40000, "tail"), (1, 70001, "head"), (40, 700, "none")):
        say("logprobs order", kind, k, n, v, mask)
        z, t = logits(n, v, 5, mask, kind)
        check(env, place(torch, dev, z, torch.float32)[1], t, k)
        check(env, place(torch, dev, z, torch.bfloat16, 5)[1], t, k)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("k", [31, 32, 33, 48, 63, 64])
def test_many_alternatives(env, k, dtype):
    """Large k in rows of one block, of several waves and of several parts."""
    torch, B, dev, h = env
    for n, v in ((5, 70), (300, 1000), (9, 5000), (2, 32768), (3, 131072), (257, 9001)):
        say("logprobs many alternatives", n, v, k, dtype)
        z, t = logits(n, v, v + k)
        check(env, place(torch, dev, z, getattr(torch, dtype), 1)[1], t, k)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("v", [40, 1000, 33000])
def test_extreme_values(env, v, dtype):
    """The type's lowest value as a mask (alone it is a uniform row), values
    near the ends of the range, infinities and NaN, also in masked rows."""
    torch, B, dev, h = env
    dt = getattr(torch, dtype)
    low = float(torch.finfo(dt).min)
    r = np.random.default_rng(v)
    z = r.standard_normal((12, v)).astype(np.float32)
    z[0] = low
    z[1, : v // 2] = low
    z[2, 1:] = low
    z[3] = -low
    z[4, 3] = -low
    z[5] *= 1e30
    z[6] = -1e38
    z[6, v // 2] = -9e37
    z[7, v // 3] = np.nan
    z[8, v - 1] = np.inf
    z[9] = -np.inf
    z[9, 5] = np.nan
    z[10] = -np.inf
    z[10, :2] = low
    z[11] = 0
    z[11, ::2] = -0.0
    t = np.array([0, 1, 0, 5, 3, 2, v // 2, 1, 2, 6, 1, -1])
    say("logprobs extremes", v, dtype)
    check(env, place(torch, dev, z, dt)[1], t, 6)


def test_no_rows_and_optional_outputs(env):
    torch, B, dev, h = env
    say("logprobs optional outputs")
    B.shampoo_token_logprobs(h, torch.empty(0, 10, device=dev), torch.empty(0, device=dev, dtype=torch.int32),
                             torch.empty(0, device=dev), torch.empty(0, device=dev))
    z, t = logits(6, 3001, 1)
    _, view = place(torch, dev, z, torch.float32)
    lse = torch.zeros(6, device=dev)
    nws = B.shampoo_token_logprobs_workspace_bytes(6, 3001, 0)
    ws = torch.empty(nws, device=dev, dtype=torch.uint8) if nws else None
    B.shampoo_token_logprobs(h, view, None, None, lse, workspace=ws)
    full = forward(env, view, t, 0)
    torch.cuda.synchronize()
    assert torch.equal(lse, full[2])
    with pytest.raises(B.ShampooError):
        B.shampoo_token_logprobs(h, torch.zeros(2, 0, device=dev), None, None, torch.zeros(2, device=dev))
    with pytest.raises(B.ShampooError):
        forward(env, view, t, B.MAX_TOP + 1)


def grad_case(env, z, t, k, dtype, pad, entropy=True, g_lse=True, in_place=False):
    torch, B, dev, h = env
    n, v = z.shape
    buf, view = place(torch, dev, z, dtype, pad)
    zz = host(view.double())
    logp, lse, ent, ids, _ = L.token_logprobs(zz, t, k)
    r = np.random.default_rng(n + v)

    def dev32(x):
        return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(dev)
    gl, gs, ge, gt = (r.standard_normal(s).astype(np.float32) for s in ((n,), (n,), (n,), (n, k)))
    lse32, ent32 = lse.astype(np.float32), ent.astype(np.float32)
    tt = torch.from_numpy(np.ascontiguousarray(t, dtype=np.int32)).to(dev)
    if in_place:
        dbuf, dview = buf, view
    else:
        dbuf, dview = place(torch, dev, np.zeros_like(z), dtype, pad)
    B.shampoo_token_logprobs_grad(
        h, view, tt, dev32(lse32), dview, g_logp=dev32(gl), g_lse=dev32(gs) if g_lse else None,
        entropy=dev32(ent32) if entropy else None, g_entropy=dev32(ge) if entropy else None,
        top_ids=torch.from_numpy(ids.astype(np.int32)).to(dev) if k else None, g_top=dev32(gt) if k else None)
    torch.cuda.synchronize()
    ref = L.token_logprobs_grad(zz, t, lse32, ent32, gl, gs if g_lse else None, ge if entropy else None, ids,
                                gt if k else None)
    with np.errstate(all="ignore"):
        p = np.where(lse32[:, None] > -np.inf, np.exp(zz - lse32[:, None].astype(np.float64)), 0)
        lp = np.where(p > 0, np.abs(zz - lse32[:, None].astype(np.float64)), 0)
    size = np.abs(gl) + np.abs(gs) * g_lse + np.abs(gt).sum(1)
    bracket = size[:, None] + (np.abs(ge)[:, None] * (lp + np.abs(ent32)[:, None]) if entropy else 0)
    # p is off by u |z - lse| and a few ulp, the bracket by a few ulp of its terms
    tol = U * (8 + k + 4 * lp) * p * bracket + 4 * U * np.abs(ref) + U * size[:, None] * (ref != 0) + 1e-37
    tol = tol + (2.0 ** -8 * np.abs(ref) if dtype is torch.bfloat16 else 0)
    close(host(dview.double()), ref, tol, "dlogits")
    if pad:
        rest = dbuf.view(n, v + pad)[:, v:]
        assert bool(torch.all(rest == 7.5))
    return host(dview.double())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,v", SHAPES)
def test_gradient(env, n, v, dtype):
    torch = env[0]
    for mask, k, pad, entropy, in_place in (("none", 0, 0, False, False), ("some", 4, 3, True, False),
                                            ("rows", 17, 8, True, True), ("one", 2, 1, False, True),
                                            ("none", 64, 0, True, False)):
        say("logprobs grad", n, v, dtype, mask, k, pad, entropy, in_place)
        z, t = logits(n, v, n + 3 * k, mask)
        grad_case(env, z, t, min(k, 64), getattr(torch, dtype), pad, entropy, entropy, in_place)


def test_gradient_of_bad_rows(env):
    """NaN rows give NaN, rows without allowed entries 0; a target that is also
    an alternative takes both gradients; repeated runs agree bit for bit."""
    torch, B, dev, h = env
    say("logprobs grad bad rows")
    z, t = logits(6, 5000, 9)
    z[1, 77] = np.nan
    z[2] = -np.inf
    t[:] = [int(z[0].argmax()), 1, 2, 3, -1, 4999]
    a = grad_case(env, z, t, 5, torch.float32, 2)
    assert np.all(np.isnan(a[1])) and np.all(a[2] == 0)
    b = grad_case(env, z, t, 5, torch.float32, 2)
    assert np.array_equal(a, b, equal_nan=True)


def test_gradient_matches_differences(env):
    """Central differences of the library's own outputs along random
    directions (fp32: the quotient is good to about 1e-3)."""
    torch, B, dev, h = env
    say("logprobs grad differences")
    z, t = logits(5, 300, 21)
    t[:] = [0, 299, 17, 5, -1]
    r = np.random.default_rng(2)
    gl, ge = r.standard_normal(5), r.standard_normal(5)
    d = r.standard_normal(z.shape)

    def f(x):
        _, logp, _, ent, _, _ = forward(env, place(torch, dev, x.astype(np.float32), torch.float32)[1], t, 0)
        torch.cuda.synchronize()
        return float(host(logp).astype(np.float64) @ gl + host(ent).astype(np.float64) @ ge)
    step = 2.0 ** -6
    quotient = (f(z + step * d) - f(z - step * d)) / (2 * step)
    _, view = place(torch, dev, z, torch.float32)
    tt, _, lse, ent, _, _ = forward(env, view, t, 0)
    dz = torch.empty_like(view)
    B.shampoo_token_logprobs_grad(h, view, tt, lse, dz, g_logp=torch.from_numpy(gl).float().to(dev), entropy=ent,
                                  g_entropy=torch.from_numpy(ge).float().to(dev))
    torch.cuda.synchronize()
    got = float((host(dz).astype(np.float64) * d).sum())
    # quotient: rounding 5 outputs of size 10 at u over 2 steps, and step^2 / 6 of the third derivative
    assert abs(got - quotient) <= 1e-3 * max(1.0, abs(got))


def test_more_rows_than_a_launch_takes(env):
    """Millions of short rows: the calls split their launches; rows on both
    sides of every split against the oracle."""
    torch, B, dev, h = env
    n, v, k = (1 << 23) + 77, 9, 2
    say("logprobs many rows", n, v)
    g = torch.Generator(device=dev).manual_seed(5)
    z = torch.randn(n, v, device=dev, generator=g)
    t = torch.randint(0, v, (n,), device=dev, generator=g).to(torch.int32)
    out = [torch.full((n,), float("nan"), device=dev) for _ in range(3)]
    ids, top = torch.zeros(n, k, device=dev, dtype=torch.int32), torch.zeros(n, k, device=dev)
    B.shampoo_token_logprobs(h, z, t, out[0], out[1], entropy=out[2], top_ids=ids, top_logp=top)
    dz = torch.full_like(z, float("nan"))
    ones = torch.ones(n, device=dev)
    B.shampoo_token_logprobs_grad(h, z, t, out[1], dz, g_logp=ones)
    torch.cuda.synchronize()
    assert not any(bool(torch.isnan(x).any()) for x in out + [dz])
    some = torch.cat([torch.arange(c - 3, min(c + 3, n)) for c in (3, 1 << 20, 1 << 21, 1 << 22, 1 << 23, n - 3)])
    zz, tt = host(z[some.to(dev)].double()), host(t[some.to(dev)])
    ref = L.token_logprobs(zz, tt, k)
    for a, b in zip([x[some.to(dev)] for x in out] + [ids[some.to(dev)], top[some.to(dev)]], ref):
        close(host(a), b, 64 * U * (1 + np.abs(b)), "many rows")
    dref = L.token_logprobs_grad(zz, tt, host(out[1][some.to(dev)]), g_logp=np.ones(len(tt)))
    close(host(dz[some.to(dev)].double()), dref, 64 * U, "many rows dlogits")


def test_offsets_past_32_bits(env):
    """Rows whose offsets pass 2^31 elements."""
    torch, B, dev, h = env
    say("logprobs large offsets")
    v, ld, n = 5000, (1 << 30) + 8, 3
    buf = torch.empty((n - 1) * ld + v, device=dev, dtype=torch.bfloat16)
    view = buf.as_strided((n, v), (ld, 1))
    z, t = logits(n, v, 33)
    view.copy_(torch.from_numpy(z).bfloat16())
    t[:] = [1, 2, 3]
    lse, ent, ids = check(env, view, t, 4)
    zz = host(view.double())
    g = torch.ones(n, device=dev)
    tt = torch.tensor(t, device=dev, dtype=torch.int32)
    B.shampoo_token_logprobs_grad(h, view, tt, lse, view, g_logp=g)
    torch.cuda.synchronize()
    ref = L.token_logprobs_grad(zz, t, host(lse), g_logp=np.ones(n))
    close(host(view.double()), ref, 2.0 ** -8 * np.abs(ref) + 1e-6, "dlogits")


def test_other_stream_and_graph(env):
    """The calls run on the stream they are given, and a captured graph of them
    gives the eager results at every replay."""
    torch, B, dev, h = env
    say("logprobs stream and graph")
    for n, v, k in ((1, 60000, 8), (64, 3000, 4)):
        z, t = logits(n, v, 44)
        _, view = place(torch, dev, z, torch.bfloat16)
        eager = forward(env, view, t, k)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        other = forward(env, view, t, k, stream=side)
        side.synchronize()
        torch.cuda.synchronize()
        for a, b in zip(eager[1:], other[1:]):
            assert torch.equal(a, b)
        tt, logp, lse, ent, ids, top = (torch.zeros_like(x) for x in eager)
        tt.copy_(eager[0])
        dz = torch.zeros_like(view)
        gl = torch.ones(n, device=dev)
        nws = B.shampoo_token_logprobs_workspace_bytes(n, v, k)
        ws = torch.empty(nws, device=dev, dtype=torch.uint8) if nws else None
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.shampoo_token_logprobs(h, view, tt, logp, lse, entropy=ent, top_ids=ids, top_logp=top, workspace=ws)
            B.shampoo_token_logprobs_grad(h, view, tt, lse, dz, g_logp=gl, entropy=ent, g_entropy=gl, top_ids=ids)
        want = torch.zeros_like(view)
        B.shampoo_token_logprobs_grad(h, view, tt, eager[2], want, g_logp=gl, entropy=eager[3], g_entropy=gl,
                                      top_ids=eager[4])
        for rep in range(4):
            for x in (logp, lse, ent, ids, top, dz):
                x.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip((logp, lse, ent, ids, top, dz), eager[1:] + (want,)):
                assert torch.equal(a, b), rep


@pytest.mark.parametrize("n,v", [(40, 64), (5, 700), (2100, 2500), (9, 5000), (3, 70001)])
@pytest.mark.parametrize("centre", [1e6, -1e6, 3e5, 2e7])
def test_large_logits(env, centre, n, v):
    """fp32 logits a few units apart around large values (their spacing is 1/16
    at 1e6): mixed within lanes, and rising or falling so that lanes, blocks,
    waves and parts of a row lie on either side.  Differences of such values
    are exact, so the bounds are those of small logits."""
    torch, B, dev, h = env
    say("logprobs large logits", centre, n, v)
    r = np.random.default_rng(v)
    z = 2 * r.standard_normal((n, v))
    z[1::3] = np.linspace(-12, 12, v)
    z[2::3] = np.linspace(12, -12, v)
    t = r.integers(0, v, n)
    check(env, place(torch, dev, (centre + z).astype(np.float32), torch.float32, 1)[1], t, 7)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,v", [(3000, 64), (2100, 4100), (300, 1000), (9, 9000), (2, 131072)])
def test_outputs_stay_in_their_range(env, n, v, dtype):
    """Log probabilities are at most 0 and entropies at least 0: exactly 0 with a
    single allowed entry, whose logit is the log-sum-exp."""
    torch, B, dev, h = env
    say("logprobs range", n, v, dtype)
    for mask, lift in (("one", 0), ("none", 30), ("none", 9)):
        z, t = logits(n, v, n + v, mask)
        z += np.float32(5.3)
        if lift:
            z[np.arange(n), t] = lift + np.abs(z).max()
        _, view = place(torch, dev, z, getattr(torch, dtype))
        _, logp, lse, ent, ids, top = forward(env, view, t, 3)
        torch.cuda.synchronize()
        assert bool(torch.all(logp <= 0)) and bool(torch.all(ent >= 0)) and bool(torch.all(top <= 0))
        if mask == "one":
            assert not bool(torch.any(logp[torch.from_numpy(t).to(dev) >= 0])) and not bool(torch.any(ent))
            assert torch.equal(lse, view.float().amax(1)) and not bool(torch.any(top[:, 0]))


# Rows of several blocks to a wave for every number of waves of a workgroup (and
# parts of a row); test_layer_plans.py checks that the dispatch rules send them there.
LONG = [(2049, 9001), (1100, 20011), (600, 40001), (300, 70001), (2049, 70001), (5, 131075), (100, 131075)]
LONG_K = [0, 8, 64]
# Two blocks to a wave of the gradient: (rows, vocab, type).
LONG_GRAD = [(521, 16001, "float32"), (551, 31003, "bfloat16")]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("k", LONG_K)
@pytest.mark.parametrize("n,v", LONG)
def test_long_rows(env, n, v, k, dtype):
    """All rows against 64-bit torch operations, some of them and their
    alternatives' indices against the oracle; with and without entropy."""
    torch, B, dev, h = env
    say("logprobs long rows", n, v, k, dtype)
    g = torch.Generator(device=dev).manual_seed(n + v + k)
    z = 3 * torch.randn(n, v, device=dev, generator=g)
    z[torch.rand(n, v, device=dev, generator=g) < 0.2] = -float("inf")
    z[1] = torch.linspace(-20, 20, v, device=dev)
    z[2] = torch.linspace(20, -20, v, device=dev)
    z[3] = 1.25
    z[4] = -float("inf")
    buf = torch.full((n * (v + 5) + 1,), 7.5, device=dev, dtype=getattr(torch, dtype))
    view = buf[1:].view(n, v + 5)[:, :v]
    view.copy_(z)
    del z
    t = np.random.default_rng(v).integers(-1, v, n)
    tt, logp, lse, ent, ids, top = forward(env, view, t, k)
    lse2, ids2, top2 = (None if x is None else torch.zeros_like(x) for x in (lse, ids, top))
    nws = B.shampoo_token_logprobs_workspace_bytes(n, v, k)
    ws = torch.empty(nws, device=dev, dtype=torch.uint8) if nws else None
    B.shampoo_token_logprobs(h, view, None, None, lse2, top_ids=ids2, top_logp=top2, workspace=ws)
    torch.cuda.synchronize()
    e = U * (16 + np.sqrt(v))
    for a, b in ((lse2, lse), (top2, top)):
        if a is not None:
            close(host(a), host(b).astype(np.float64), 2 * e + 8 * U * np.abs(np.where(np.isfinite(host(b)), host(b), 0)),
                  "without entropy")
    assert k == 0 or torch.equal(ids, ids2)
    some = np.unique(np.concatenate([np.arange(min(n, 6)), np.random.default_rng(1).integers(0, n, 14), [n - 1]]))
    at = torch.from_numpy(some).to(dev)
    ref = L.token_logprobs(host(view[at].double()), t[some], k)
    for a, b, what, f in zip((logp, lse, ent, None, top), ref, ("logp", "lse", "entropy", "ids", "top"),
                             (1, 1, 40, 1, 1)):
        if a is not None:
            close(host(a[at]), b, f * e + 4 * U * np.abs(np.where(np.isfinite(b), b, 0)), what)
    if k:
        assert np.array_equal(host(ids[at]), ref[3])
    for r in range(0, n, 256):
        x = view[r:r + 256].double()
        want = torch.logsumexp(x, 1)
        tr = tt[r:r + 256].long()
        picked = torch.where(tr >= 0, x.gather(1, tr.clamp(min=0).unsqueeze(1))[:, 0] - want, torch.zeros_like(want))
        picked = torch.where((tr >= 0) & torch.isneginf(want), want, picked)
        p = torch.exp(x - want.unsqueeze(1)).nan_to_num_(0)
        lp = torch.where(p > 0, x - want.unsqueeze(1), torch.zeros_like(x))
        pairs = [(logp, picked, 1), (lse, want, 1), (ent, -(p * lp).sum(1), 40)]
        if k:
            best = torch.topk(x, k, dim=1).values - want.unsqueeze(1)
            pairs.append((top, torch.where(torch.isnan(best), torch.full_like(best, -float("inf")), best), 1))
        for a, b, f in pairs:
            b = host(b)
            close(host(a[r:r + 256]), b, f * e + 4 * U * np.abs(np.where(np.isfinite(b), b, 0)), ("all rows", r))


@pytest.mark.parametrize("n,v,dtype", LONG_GRAD)
def test_gradient_of_long_rows(env, n, v, dtype):
    torch = env[0]
    for mask, k, pad, entropy, in_place in (("none", 0, 0, False, False), ("some", 17, 3, True, True)):
        say("logprobs grad long rows", n, v, dtype, mask, k, pad, entropy, in_place)
        z, t = logits(n, v, n + k, mask)
        grad_case(env, z, t, k, getattr(torch, dtype), pad, entropy, entropy, in_place)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("k", [8, 64])
def test_time_does_not_depend_on_the_order(env, k, dtype):
    """Rows that rise with the index raise the bound on the alternatives in every
    block.  They may cost a few times what rows in random order do, not tens of
    times."""
    torch, B, dev, h = env
    n, v = 2048, 131072
    say("logprobs order and time", k, dtype)
    up = torch.linspace(-20, 20, v, device=dev)
    mixed = up[torch.randperm(v, device=dev, generator=torch.Generator(device=dev).manual_seed(1))]
    lse, top = torch.empty(n, device=dev), torch.empty(n, k, device=dev)
    ids = torch.empty(n, k, device=dev, dtype=torch.int32)
    times = []
    for row in (mixed, up):
        z = row.to(getattr(torch, dtype)).expand(n, v).contiguous()
        best = float("inf")
        for _ in range(4):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            B.shampoo_token_logprobs(h, z, None, None, lse, top_ids=ids, top_logp=top)
            b.record()
            torch.cuda.synchronize()
            best = min(best, a.elapsed_time(b))
        times.append(best)
    assert times[1] <= 10 * times[0], times


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,v", [(2050, 20011), (700, 20011), (5, 131075)])
def test_largest_in_few_lanes(env, n, v, dtype):
    """Rows that rise from block to block, with their largest entries in a few of
    the 16-byte pieces that lanes hold: fewer lanes than alternatives, at several
    distances, some with a long run of equal values at the bound."""
    torch, B, dev, h = env
    say("logprobs few lanes", n, v, dtype)
    per = 4 if dtype == "float32" else 8  # entries of a piece
    c = np.arange(v)
    lane, block = c // per % 64, c // (256 * per)
    rows = [np.where(lane < lanes, 5.0, 0.0) + 0.05 * block + fine * (c % (256 * per))
            for lanes in (1, 3, 15) for fine in (0.0, 1e-5)]
    z = np.tile(np.array(rows), (n // len(rows) + 1, 1))[:n].astype(np.float32)
    _, view = place(torch, dev, z, getattr(torch, dtype))
    t = np.random.default_rng(n).integers(0, v, n)
    for k in (5, 16, 40, 64):
        _, logp, lse, ent, ids, top = forward(env, view, t, k)
        torch.cuda.synchronize()
        some = list(range(min(n, 6))) + [n - 1]
        ref = L.token_logprobs(host(view[some].double()), t[some], k)
        e = U * (16 + np.sqrt(v))
        for a, b, f in ((logp, ref[0], 1), (lse, ref[1], 1), (ent, ref[2], 40), (top, ref[4], 1)):
            close(host(a[some]), b, f * e + 4 * U * np.abs(b), k)
        assert np.array_equal(host(ids[some]), ref[3])
        for i in range(6, n, 6):  # the same rows again
            assert torch.equal(ids[i], ids[0])
