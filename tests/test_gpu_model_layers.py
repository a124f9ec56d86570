"""The layers around the step on the GPU against the 64-bit oracle: the loss from the
last activations and the gated feed-forward block, with their gradients.

Tolerances bound every element.  Let u = 2^-24 and |A| |B| stand for the product of
the absolute values.
 * A product of K terms: terms are exact in bf16; of fp32 operands the dropped ones are
   below 2^-25 of a term, and the matrix instruction cuts a group of 8 terms at 2^-23 of
   its largest (at most 16 u of the group's size); additions in fp32 round at each
   step: error at most e = u (20 + sqrt(K)) |A| |B| (random signs: the running sum's
   roundings add up like a random walk's).
 * exp of z - lse: the difference is off by the error of z; scaling for the base-2
   exponential and the instruction add u (|z - lse| + 4) relative to it.
 * A gradient kept in one bf16 term is off by half a step, 2^-8 of it; in three by
   2^-24 (and the product by the dropped terms above).  A bf16 result adds 2^-8.
 * The activations: 2^-12 relative in bf16 (reciprocal, exponential and a fitted
   polynomial), u (16 + x^2) in fp32 (x^2 / 2 is rounded before the exponential).  The
   slope's terms reach (1 + x^2) times the slope's bound."""
import pytest

from tests.gpu_util import gpu_env, say

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = 2.0 ** -8  # half a step of bf16


@pytest.fixture(scope="module")
def env():
    torch, B, dev = gpu_env()
    h = B.shampoo_create(0)
    yield torch, B, dev, h
    B.shampoo_destroy(h)


class Sheet:
    """A rows x cols view inside a larger buffer whose other elements must stay."""

    def __init__(self, env, rows, cols, dtype, pad=0, shift=0, fill=None):
        torch, _, dev, _ = env
        self.buf = torch.full((rows * (cols + pad) + shift,), 7.5, device=dev, dtype=dtype)
        self.v = self.buf[shift:].view(rows, cols + pad)[:, :cols]
        self.v.copy_(torch.full((rows, cols), float("nan"), device=dev, dtype=dtype) if fill is None else fill.to(dtype))
        self.rows, self.cols, self.shift = rows, cols, shift

    def intact(self, torch):
        rest = self.buf[self.shift:].view(self.rows, -1)[:, self.cols:]
        return bool(torch.all(rest == 7.5)) and bool(torch.all(self.buf[:self.shift] == 7.5))


def room(env, n):
    """A workspace of exactly n bytes, its bytes NaN patterns."""
    torch, _, dev, _ = env
    return torch.full((n,), 0xFF, device=dev, dtype=torch.uint8) if n else None


def dtype_of(env, name):
    return getattr(env[0], name)


def close(got, ref, tol, what):
    """Every element within its tolerance."""
    err = (got.double() - ref).abs()
    bad = ~(err <= tol)
    assert not bool(bad.any()), (what, float(err[bad].max()), float(tol.expand_as(err)[bad].min()), int(bad.sum()))


def normal(env, seed, *shape):
    torch, _, dev, _ = env
    return torch.randn(*shape, generator=torch.Generator(device=dev).manual_seed(seed), device=dev)


# ------------------------------------------------------------------ loss
def vocab_inputs(env, n, d, v, dtype, pad, shift, seed):
    torch, _, dev, _ = env
    X = Sheet(env, n, d, dtype, pad, shift, normal(env, seed, n, d))
    W = Sheet(env, v, d, dtype, pad, shift, normal(env, seed + 1, v, d) * (2.0 / d ** 0.5))
    g = torch.Generator(device=dev).manual_seed(seed + 2)
    t = torch.randint(0, v, (n,), generator=g, device=dev, dtype=torch.int32)
    t[torch.rand(n, generator=g, device=dev) < 0.2] = -1
    return X, W, t


def z_error(X, W):
    """Bound of the error of each logit's row."""
    return U * (20 + X.shape[1] ** 0.5) * (X.double().abs() @ W.double().abs().t().contiguous()).amax(1)


def logprobs(env, X, W, t, stream=None):
    torch, B, dev, h = env
    n, d, v = X.shape[0], X.shape[1], W.shape[0]
    lse = torch.full((n,), float("nan"), device=dev)
    logp = None if t is None else torch.full((n,), float("nan"), device=dev)
    ws = room(env, B.shampoo_vocab_logprobs_workspace_bytes(n, d, v, X.dtype))
    B.shampoo_vocab_logprobs(h, X, W, t, logp, lse, workspace=ws, stream=stream)
    return logp, lse


def check_vocab(env, n, d, v, dtype, pad=0, shift=0, targets=True):
    import oracle.model_oracle as M
    torch, B, dev, h = env
    X, W, t = vocab_inputs(env, n, d, v, dtype, pad, shift, 11 + n)
    t = t if targets else None
    logp, lse = logprobs(env, X.v, W.v, t)
    torch.cuda.synchronize()
    rp, rl, z = M.vocab_logprobs(X.v, W.v, t)
    tol = z_error(X.v, W.v) + U * (32 + rl.abs())
    close(lse, rl, tol, "lse")
    if targets:
        close(logp, rp, 2 * tol + U * rp.abs() * 4, "logp")
        assert bool((logp <= 0).all())
        assert bool((logp[t < 0] == 0).all())


def check_vocab_grad(env, n, d, v, dtype, g_dtype, pad=0, shift=0, beta=0.0, with_x=True, with_w=True, penalty=True,
                     given=True):
    import oracle.model_oracle as M
    torch, B, dev, h = env
    X, W, t = vocab_inputs(env, n, d, v, dtype, pad, shift, 23 + n)
    _, _, z = M.vocab_logprobs(X.v, W.v, t)
    lse = torch.logsumexp(z, 1).float()
    g_logp = normal(env, 5, n) if given else None
    g_lse = normal(env, 6, n) if penalty else None
    old = normal(env, 7, v, d) * n ** 0.5
    dX = Sheet(env, n, d, dtype, pad, shift) if with_x else None
    dW = Sheet(env, v, d, g_dtype, pad, shift, old if beta else None) if with_w else None
    before = dW.v.double() if with_w and beta else 0.0
    ws = room(env, B.shampoo_vocab_logprobs_grad_workspace_bytes(n, d, v, dtype, g_dtype if with_w else dtype))
    B.shampoo_vocab_logprobs_grad(h, X.v, W.v, t, lse, dX=dX.v if with_x else None, dW=dW.v if with_w else None,
                                  g_logp=g_logp, g_lse=g_lse, beta=beta, workspace=ws)
    torch.cuda.synchronize()
    dz, size = M.vocab_dlogits(z, lse, t, g_logp, g_lse)
    bf = torch.bfloat16
    far = (z_error(X.v, W.v) + U * (4 + (z - lse.double().unsqueeze(1)).abs().amax(1))).unsqueeze(1)
    if with_x:
        q = HALF if dtype is bf else 2 * U
        part = (far * size + q * dz.abs() + U * (20 + v ** 0.5) * dz.abs()) @ W.v.double().abs()
        ref = dz @ W.v.double()
        close(dX.v, ref, part + (HALF if dtype is bf else U) * (ref.abs() + part), "dX")
        assert dX.intact(torch)
    if with_w:
        q = HALF if dtype is bf and g_dtype is bf else 2 * U
        part = (far * size + q * dz.abs() + U * (20 + n ** 0.5) * dz.abs()).t().contiguous() @ X.v.double().abs()
        ref = beta * before + dz.t().contiguous() @ X.v.double()
        if beta:
            part = part + 2 * U * (before * beta).abs()
        close(dW.v, ref, part + (HALF if g_dtype is bf else U) * (ref.abs() + part), "dW")
        assert dW.intact(torch)


# one row and one column up to sizes that reach every tile and cut of the contraction
VOCAB = [(1, 1, 1), (1, 8, 16), (3, 64, 128), (4, 1024, 2500), (31, 7, 33), (33, 72, 129), (128, 128, 1000),
         (257, 333, 1027), (300, 1000, 513), (513, 96, 4099), (2, 4096, 5000), (64, 2048, 700), (2048, 256, 8192),
         (1500, 1024, 5000)]
LAYOUTS = [(0, 0), (8, 8), (5, 3)]  # as it lies, padded and aligned, neither


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("n,d,v", VOCAB)
def test_vocab_logprobs(env, n, d, v, dtype):
    for pad, shift in LAYOUTS:
        say("vocab logprobs", n, d, v, dtype, pad, shift)
        check_vocab(env, n, d, v, dtype_of(env, dtype), pad, shift)
    check_vocab(env, n, d, v, dtype_of(env, dtype), targets=False)


@pytest.mark.parametrize("dtype,g_dtype", [("bfloat16", "bfloat16"), ("bfloat16", "float32"), ("float32", "float32"),
                                           ("float32", "bfloat16")])
@pytest.mark.parametrize("n,d,v", VOCAB)
def test_vocab_grad(env, n, d, v, dtype, g_dtype):
    for pad, shift in LAYOUTS:
        say("vocab grad", n, d, v, dtype, g_dtype, pad, shift)
        check_vocab_grad(env, n, d, v, dtype_of(env, dtype), dtype_of(env, g_dtype), pad, shift)


@pytest.mark.parametrize("dtype,g_dtype", [("bfloat16", "bfloat16"), ("float32", "float32")])
def test_vocab_grad_options(env, dtype, g_dtype):
    dt, gt = dtype_of(env, dtype), dtype_of(env, g_dtype)
    for n, d, v in ((70, 130, 1100), (1300, 64, 300)):
        for o in (dict(with_x=False), dict(with_w=False), dict(beta=0.5), dict(beta=1.0, penalty=False),
                  dict(given=False), dict(beta=-2.0, with_x=False)):
            say("vocab grad", n, d, v, dtype, g_dtype, o)
            check_vocab_grad(env, n, d, v, dt, gt, **o)


# sizes whose logits' gradient, or whose packed table, takes several pieces
PIECES = [(8192, 64, 20000, "bfloat16"), (8192, 64, 6000, "float32"), (70, 4096, 33000, "bfloat16"),
          (70, 4096, 11000, "float32")]


@pytest.mark.parametrize("n,d,v,dtype", PIECES)
def test_vocab_pieces(env, n, d, v, dtype):
    dt = dtype_of(env, dtype)
    say("vocab pieces", n, d, v, dtype)
    check_vocab(env, n, d, v, dt, 3, 1)
    check_vocab_grad(env, n, d, v, dt, dt, 3, 1)
    check_vocab_grad(env, n, d, v, dt, env[0].float32, beta=1.0)


# sizes that reach the remaining tiles, whole and in parts (test_stream_plans checks that all are
# reached): rows, dim, vocab, type, gradient's type, whether the matrices are copied first
VOCAB_MORE = [(6109, 3490, 72, "bfloat16", "bfloat16", True), (4951, 1163, 408, "float32", "float32", True),
              (1004, 2479, 1397, "float32", "float32", True), (474, 2138, 14, "bfloat16", "float32", True),
              (8005, 90, 114, "float32", "bfloat16", True), (524, 3188, 6586, "bfloat16", "bfloat16", True),
              (1007, 2432, 8, "float32", "bfloat16", True), (3907, 2796, 13, "bfloat16", "bfloat16", True),
              (2608, 241, 4626, "bfloat16", "float32", True), (843, 1928, 1991, "bfloat16", "float32", True),
              (922, 196, 31249, "bfloat16", "float32", True), (5525, 80, 14027, "float32", "bfloat16", True),
              (130, 3330, 23888, "bfloat16", "float32", True), (4870, 136, 17995, "bfloat16", "bfloat16", False),
              (6903, 914, 15369, "bfloat16", "float32", True), (1098, 165, 3544, "bfloat16", "bfloat16", True),
              (1, 1903, 10, "float32", "bfloat16", True), (65, 359, 9, "float32", "float32", True),
              (1445, 1406, 18, "float32", "bfloat16", True), (50, 1003, 5001, "bfloat16", "float32", True),
              (64, 100, 30001, "float32", "float32", True), (9, 439, 39541, "bfloat16", "float32", True),
              (32, 4099, 4999, "bfloat16", "bfloat16", True)]


@pytest.mark.parametrize("n,d,v,dtype,g_dtype,copied", VOCAB_MORE)
def test_vocab_tiles(env, n, d, v, dtype, g_dtype, copied):
    say("vocab tiles", n, d, v, dtype, g_dtype, copied)
    dt, gt, lay = dtype_of(env, dtype), dtype_of(env, g_dtype), (5, 3) if copied else (0, 0)
    check_vocab(env, n, d, v, dt, *lay)
    for with_x, with_w in ((True, True), (True, False), (False, True)):
        check_vocab_grad(env, n, d, v, dt, gt, *lay, with_x=with_x, with_w=with_w)


def test_vocab_rows_of_their_own(env):
    """A NaN or an infinity in one row of X stays there; targets outside the vocabulary
    are no targets; a row whose target is far above the rest has log probability 0 to
    the bit."""
    torch, B, dev, h = env
    for dt in (torch.bfloat16, torch.float32):
        for n, d, v in ((5, 64, 300), (200, 128, 3000)):
            say("vocab rows", n, d, v, dt)
            X, W, t = vocab_inputs(env, n, d, v, dt, 0, 0, 3)
            t[0], t[1], t[2] = -7, v, 2 ** 31 - 1
            want = logprobs(env, X.v, W.v, t)
            assert bool((want[0][:3] == 0).all())
            X.v[3, 5] = float("nan")
            X.v[4, 7] = float("inf")
            t[3:5] = 1
            got = logprobs(env, X.v, W.v, t)
            torch.cuda.synchronize()
            others = [r for r in range(n) if r not in (3, 4)]
            for a, b in zip(got, want):
                assert torch.equal(a[others], b[others]) and bool(torch.isnan(a[3:5]).all())
            X, W, t = vocab_inputs(env, n, d, v, dt, 0, 0, 4)
            W.v[7] = 100 * X.v[1].sign()
            t[1] = 7
            logp, lse = logprobs(env, X.v, W.v, t)
            assert float(logp[1]) == 0.0 and bool((logp <= 0).all())


def test_vocab_no_rows(env):
    torch, B, dev, h = env
    say("vocab, no rows")
    for dt in (torch.bfloat16, torch.float32):
        X, W = torch.zeros(0, 16, device=dev, dtype=dt), normal(env, 1, 40, 16).to(dt)
        none, dW = torch.zeros(0, device=dev), normal(env, 2, 40, 16)
        B.shampoo_vocab_logprobs(h, X, W, none.int(), none, none)
        want = 0.5 * dW
        B.shampoo_vocab_logprobs_grad(h, X, W, none.int(), none, dX=torch.zeros_like(X), dW=dW, g_logp=none, beta=0.5)
        assert torch.equal(dW, want)
        dW.fill_(float("nan"))
        B.shampoo_vocab_logprobs_grad(h, X, W, none.int(), none, dW=dW, g_logp=none)
        assert bool((dW == 0).all())


@pytest.mark.parametrize("d", [4096, 4095])
def test_vocab_far_offsets(env, d):
    """A table of more than 2^31 elements: rows at its end."""
    import oracle.model_oracle as M
    torch, B, dev, h = env
    n, v = 3, 524500
    say("vocab far", n, d, v)
    gen = torch.Generator(device=dev).manual_seed(1)
    W = torch.empty(v, d, device=dev, dtype=torch.bfloat16)
    for r in range(0, v, 65536):
        part = W[r:r + 65536]
        part.copy_(torch.randn(part.shape, generator=gen, device=dev) / 32)
    X = normal(env, 2, n, d).bfloat16()
    t = torch.tensor([v - 1, 5, -1], device=dev, dtype=torch.int32)
    logp, lse = logprobs(env, X, W, t)
    g = normal(env, 3, n)
    dX, dW = torch.empty_like(X), torch.empty(v, d, device=dev, dtype=torch.bfloat16)
    ws = room(env, B.shampoo_vocab_logprobs_grad_workspace_bytes(n, d, v, X.dtype, dW.dtype))
    B.shampoo_vocab_logprobs_grad(h, X, W, t, lse, dX=dX, dW=dW, g_logp=g, workspace=ws)
    torch.cuda.synchronize()
    z = torch.cat([X.double() @ W[r:r + 32768].double().t().contiguous() for r in range(0, v, 32768)], 1)
    rl = torch.logsumexp(z, 1)
    e = U * (20 + d ** 0.5) * max(float((X.double().abs() @ W[r:r + 32768].double().abs().t().contiguous()).max())
                                  for r in (0, v - 32768)) * 2
    tol = torch.full_like(rl, e) + U * (32 + rl.abs())
    close(lse, rl, tol, "lse")
    close(logp[:2], z[[0, 1], [v - 1, 5]] - rl[:2], 2 * tol[:2] + U * 100, "logp")
    dz, size = M.vocab_dlogits(z, lse, t, g)
    ref, part = torch.zeros(n, d, device=dev, dtype=torch.float64), torch.zeros(n, d, device=dev, dtype=torch.float64)
    for r in range(0, v, 32768):
        w = W[r:r + 32768].double()
        ref += dz[:, r:r + 32768] @ w
        part += ((e + 60 * U) * size + (HALF + U * 800) * dz.abs())[:, r:r + 32768] @ w.abs()
    close(dX, ref, part + HALF * (ref.abs() + part), "dX")
    tail = dz[:, -1000:].t().contiguous() @ X.double()
    far = ((e + 60 * U) * size + (HALF + 22 * U) * dz.abs())[:, -1000:].t().contiguous() @ X.double().abs()
    close(dW[-1000:], tail, far + HALF * (tail.abs() + far), "dW")


# ------------------------------------------------------------------ feed-forward block
FFN = [(1, 1, 1), (1, 8, 16), (2, 33, 17), (16, 1024, 512), (16, 64, 4096), (31, 100, 7), (65, 129, 130), (128, 128, 128),
       (200, 333, 1339), (1000, 64, 40), (520, 264, 1000), (5, 2000, 136), (2048, 512, 768), (4100, 512, 2056)]
ACTS = ["NONE", "RELU", "GELU", "GELU_TANH", "SILU"]


def ffn_inputs(env, n, d, w, dtype, pad, shift, seed):
    X = Sheet(env, n, d, dtype, pad, shift, normal(env, seed, n, d))
    Wg, Wu = (Sheet(env, d, w, dtype, pad, shift, normal(env, seed + i, d, w) / d ** 0.5) for i in (1, 2))
    return X, Wg, Wu


def act_error(x, bf):
    """Relative error of an activation at x."""
    return 2.0 ** -12 if bf else U * (16 + x * x)


def check_ffn(env, n, d, w, dtype, act, pad=0, shift=0, keep=True):
    import oracle.model_oracle as M
    torch, B, dev, h = env
    bf, kind = dtype is torch.bfloat16, getattr(B, "ACT_" + act)
    X, Wg, Wu = ffn_inputs(env, n, d, w, dtype, pad, shift, 31 + n)
    H = Sheet(env, n, w, dtype, pad, shift)
    G, Uo = (Sheet(env, n, w, dtype, pad, shift) if keep else None for _ in range(2))
    ws = room(env, B.shampoo_gated_ffn_workspace_bytes(n, d, w, dtype))
    B.shampoo_gated_ffn(h, X.v, Wg.v, Wu.v, H.v, kind, G.v if keep else None, Uo.v if keep else None, workspace=ws)
    torch.cuda.synchronize()
    rh, rg, ru = M.gated(X.v, Wg.v, Wu.v, kind)
    r = HALF if bf else U
    eg, eu = (U * (20 + d ** 0.5) * (X.v.double().abs() @ m.v.double().abs()) for m in (Wg, Wu))
    a = M.act(rg, kind).abs()
    err = ru.abs() * (1.2 * eg + act_error(rg, bf) * a) + (a + 1.2 * eg) * eu
    close(H.v, rh, err * 1.01 + r * (rh.abs() + err), "H")
    if keep:
        close(G.v, rg, eg + r * (rg.abs() + eg), "G")
        close(Uo.v, ru, eu + r * (ru.abs() + eu), "U")
    for s in (H, G, Uo):
        assert s is None or s.intact(torch)


def check_ffn_grad(env, n, d, w, dtype, g_dtype, act, keep, pad=0, shift=0, beta=0.0, with_x=True, with_w=True):
    import oracle.model_oracle as M
    torch, B, dev, h = env
    bf, gbf, kind = dtype is torch.bfloat16, g_dtype is torch.bfloat16, getattr(B, "ACT_" + act)
    X, Wg, Wu = ffn_inputs(env, n, d, w, dtype, pad, shift, 41 + n)
    dH = Sheet(env, n, w, dtype, pad, shift, normal(env, 4, n, w))
    _, rg, ru = M.gated(X.v, Wg.v, Wu.v, kind)
    eg, eu = (U * (20 + d ** 0.5) * (X.v.double().abs() @ m.v.double().abs()) for m in (Wg, Wu))
    G = Uo = None
    if keep:
        G, Uo = (Sheet(env, n, w, dtype, pad, shift, x) for x in (rg, ru))
        rg, ru, eg, eu = G.v.double(), Uo.v.double(), 0 * eg, 0 * eu
    old = [normal(env, 50 + i, d, w) * n ** 0.5 for i in range(2)]
    dX = Sheet(env, n, d, dtype, pad, shift) if with_x else None
    dW = [Sheet(env, d, w, g_dtype, pad, shift, o if beta else None) if with_w else None for o in old]
    before = [s.v.double() if s and beta else 0.0 for s in dW]
    ws = room(env, B.shampoo_gated_ffn_grad_workspace_bytes(n, d, w, dtype, g_dtype if with_w else dtype))
    B.shampoo_gated_ffn_grad(h, X.v, Wg.v, Wu.v, dH.v, kind, G.v if keep else None, Uo.v if keep else None,
                             dX.v if with_x else None, *(s.v if s else None for s in dW), beta=beta, workspace=ws)
    torch.cuda.synchronize()
    dG, dU = M.gated_grad(rg, ru, dH.v, kind)
    hh, a, s = dH.v.double().abs(), M.act(rg, kind).abs(), M.slope(rg, kind).abs()
    f = act_error(rg, bf)
    # slopes of the activation and of its slope are below 1.2
    fg = hh * (ru.abs() * (1.2 * eg + f * (1 + rg * rg)) + (s + 1.2 * eg) * eu) + 4 * U * dG.abs()
    fu = hh * (f * a + 1.2 * eg) + 4 * U * dU.abs()
    x = X.v.double()
    if with_x:
        q = (HALF if bf else 2 * U) + U * (20 + (2 * w) ** 0.5)
        ref = dG @ Wg.v.double().t().contiguous() + dU @ Wu.v.double().t().contiguous()
        err = ((fg + q * (dG.abs() + fg)) @ Wg.v.double().abs().t().contiguous() +
               (fu + q * (dU.abs() + fu)) @ Wu.v.double().abs().t().contiguous())
        close(dX.v, ref, err + (HALF if bf else U) * (ref.abs() + err), "dX")
        assert dX.intact(torch)
    if with_w:
        q = (HALF if bf and gbf else 2 * U) + U * (20 + n ** 0.5)
        for what, sheet, b, m, e in (("dWg", dW[0], before[0], dG, fg), ("dWu", dW[1], before[1], dU, fu)):
            ref = x.t().contiguous() @ m + beta * b
            err = x.abs().t().contiguous() @ (e + q * (m.abs() + e))
            if beta:
                err = err + 2 * U * (beta * b).abs()
            close(sheet.v, ref, err + (HALF if gbf else U) * (ref.abs() + err), what)
            assert sheet.intact(torch)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("n,d,w", FFN)
def test_gated_ffn(env, n, d, w, dtype):
    for i, (pad, shift) in enumerate(LAYOUTS):
        for act in (ACTS if i == 0 else ["SILU"]):
            say("ffn", n, d, w, dtype, act, pad, shift)
            check_ffn(env, n, d, w, dtype_of(env, dtype), act, pad, shift, keep=act != "GELU")


@pytest.mark.parametrize("dtype,g_dtype", [("bfloat16", "bfloat16"), ("bfloat16", "float32"), ("float32", "float32"),
                                           ("float32", "bfloat16")])
@pytest.mark.parametrize("n,d,w", FFN)
def test_gated_ffn_grad(env, n, d, w, dtype, g_dtype):
    for i, (pad, shift) in enumerate(LAYOUTS):
        for act in (ACTS if i == 0 else ["GELU"]):
            for keep in ((True, False) if act != "RELU" else (True,)):  # relu's slope jumps: see below
                say("ffn grad", n, d, w, dtype, g_dtype, act, keep, pad, shift)
                check_ffn_grad(env, n, d, w, dtype_of(env, dtype), dtype_of(env, g_dtype), act, keep, pad, shift)


# as VOCAB_MORE: rows, dim, width, type, gradient's type
FFN_MORE = [(1, 1718, 1871, "float32", "float32"), (1, 3508, 1348, "bfloat16", "bfloat16"),
            (7225, 3508, 20, "float32", "float32"), (942, 2340, 476, "bfloat16", "bfloat16"),
            (1441, 2247, 731, "float32", "bfloat16"), (4932, 884, 2504, "bfloat16", "float32"),
            (7880, 75, 269, "float32", "bfloat16"), (688, 3745, 3026, "bfloat16", "float32"),
            (5349, 2491, 844, "bfloat16", "bfloat16"), (992, 723, 2295, "bfloat16", "float32"),
            (7392, 845, 1327, "bfloat16", "float32"), (1154, 103, 436, "bfloat16", "bfloat16"),
            (76, 8, 10, "float32", "bfloat16"), (82, 8, 412, "float32", "bfloat16"), (90, 949, 8, "float32", "float32"),
            (1, 657, 1128, "bfloat16", "bfloat16"), (1, 2940, 392, "bfloat16", "bfloat16"),
            (68, 87, 2972, "float32", "float32"), (84, 1204, 330, "float32", "bfloat16"),
            (50, 1337, 1003, "bfloat16", "bfloat16"), (64, 130, 5000, "float32", "float32"),
            (11, 2243, 4039, "bfloat16", "float32"), (32, 2243, 4039, "bfloat16", "bfloat16")]


@pytest.mark.parametrize("n,d,w,dtype,g_dtype", FFN_MORE)
def test_gated_ffn_tiles(env, n, d, w, dtype, g_dtype):
    say("ffn tiles", n, d, w, dtype, g_dtype)
    dt, gt = dtype_of(env, dtype), dtype_of(env, g_dtype)
    check_ffn(env, n, d, w, dt, "SILU")
    for with_x, with_w in ((True, True), (True, False), (False, True)):
        check_ffn_grad(env, n, d, w, dt, gt, "GELU_TANH", False, with_x=with_x, with_w=with_w)


def test_weights_of_different_strides(env):
    """Wg and Wu in rows of different lengths, and one that is read as it lies beside one
    that is not: the bits of the plain call.  (Few bf16 rows have two ways through the
    weights, by whether both lie as the matrix cores take them: bits of its own each, the
    projections of both within their sums' error and a rounding.)"""
    torch, B, dev, h = env
    for n, d, w in ((3, 64, 136), (40, 72, 1000), (700, 256, 520), (3000, 512, 2056)):
        for dt in (torch.bfloat16, torch.float32):
            say("ffn strides", n, d, w, dt)
            X, g, u = normal(env, 1, n, d).to(dt), (normal(env, 2, d, w) / d).to(dt), (normal(env, 3, d, w) / d).to(dt)
            ws = room(env, B.shampoo_gated_ffn_workspace_bytes(n, d, w, dt))
            gws = room(env, B.shampoo_gated_ffn_grad_workspace_bytes(n, d, w, dt, dt))
            dH = normal(env, 4, n, w).to(dt)
            got = []
            for (pg, sg), (pu, su) in (((0, 0), (0, 0)), ((8, 0), (24, 8)), ((3, 1), (16, 0)), ((64, 8), (1, 0))):
                Wg, Wu = Sheet(env, d, w, dt, pg, sg, g).v, Sheet(env, d, w, dt, pu, su, u).v
                out = [torch.empty(n, w, device=dev, dtype=dt) for _ in range(3)]
                B.shampoo_gated_ffn(h, X, Wg, Wu, out[0], B.ACT_SILU, out[1], out[2], workspace=ws)
                out += [torch.empty_like(X), torch.empty(d, w, device=dev, dtype=dt), torch.empty(d, w, device=dev, dtype=dt)]
                B.shampoo_gated_ffn_grad(h, X, Wg, Wu, dH, B.ACT_SILU, dX=out[3], dWg=out[4], dWu=out[5], workspace=gws)
                got.append(out)
            torch.cuda.synchronize()
            two = n <= 64 and dt is torch.bfloat16
            for i, other in enumerate(got[1:], 1):
                for a, b in zip(got[2 if two and i > 2 else 0], other):
                    assert torch.equal(a, b) or (two and i == 2)
            if two:
                for a, b, m in ((got[0][1], got[2][1], g), (got[0][2], got[2][2], u)):
                    # either is the exact sum within e, rounded
                    e = U * (20 + d ** 0.5) * (X.double().abs() @ m.double().abs())
                    close(a, b.double(), 2 * e + HALF * (2 * b.double().abs() + 4 * e), "projection")


@pytest.mark.parametrize("dtype,g_dtype", [("bfloat16", "bfloat16"), ("float32", "float32")])
def test_gated_ffn_grad_options(env, dtype, g_dtype):
    dt, gt = dtype_of(env, dtype), dtype_of(env, g_dtype)
    for n, d, w in ((70, 130, 600), (1300, 64, 300)):
        for o in (dict(with_x=False), dict(with_w=False), dict(beta=0.5), dict(beta=-1.0, with_x=False)):
            for keep in (True, False):
                say("ffn grad", n, d, w, dtype, o, keep)
                check_ffn_grad(env, n, d, w, dt, gt, "SILU", keep, **o)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_whole_numbers_are_exact(env, dtype):
    """Small whole numbers: every product and sum is exact in fp32, so projections and
    fp32 gradients have to be equal, relu's recomputed slope included."""
    import oracle.model_oracle as M
    torch, B, dev, h = env
    dt = dtype_of(env, dtype)
    for n, d, w in ((1, 5, 9), (40, 72, 130), (300, 264, 520), (1030, 512, 1000), (4200, 1024, 1032)):
        g = torch.Generator(device=dev).manual_seed(n)

        def ints(*s):
            return torch.randint(-2, 3, s, generator=g, device=dev).to(dt)
        X, Wg, Wu, dH = ints(n, d), ints(d, w), ints(d, w), ints(n, w)
        say("whole numbers", n, d, w, dtype)
        G, Uo, H = (torch.empty(n, w, device=dev, dtype=dt) for _ in range(3))
        for act in (B.ACT_NONE, B.ACT_RELU):
            rh, rg, ru = M.gated(X, Wg, Wu, act)
            B.shampoo_gated_ffn(h, X, Wg, Wu, H, act, G, Uo,
                                workspace=room(env, B.shampoo_gated_ffn_workspace_bytes(n, d, w, dt)))
            assert torch.equal(G, rg.to(dt)) and torch.equal(Uo, ru.to(dt)) and torch.equal(H, rh.to(dt))
            dG, dU = M.gated_grad(rg, ru, dH, act)
            dX, dWg, dWu = (torch.empty(*s, device=dev, dtype=y) for s, y in (((n, d), dt), ((d, w), torch.float32),
                                                                              ((d, w), torch.float32)))
            B.shampoo_gated_ffn_grad(h, X, Wg, Wu, dH, act, dX=dX, dWg=dWg, dWu=dWu, workspace=room(
                env, B.shampoo_gated_ffn_grad_workspace_bytes(n, d, w, dt, torch.float32)))
            torch.cuda.synchronize()
            assert torch.equal(dWg.double(), X.double().t().contiguous() @ dG)
            assert torch.equal(dWu.double(), X.double().t().contiguous() @ dU)
            if dt is torch.float32:
                want = dG @ Wg.double().t().contiguous() + dU @ Wu.double().t().contiguous()
                big = want.abs() < 2 ** 24
                assert torch.equal(dX.double()[big], want[big])


def test_gated_ffn_no_rows(env):
    torch, B, dev, h = env
    say("ffn, no rows")
    X, Wg, Wu = torch.zeros(0, 16, device=dev), normal(env, 1, 16, 24), normal(env, 2, 16, 24)
    H, dWg, dWu = torch.zeros(0, 24, device=dev), normal(env, 3, 16, 24), normal(env, 4, 16, 24)
    B.shampoo_gated_ffn(h, X, Wg, Wu, H)
    want = (0.25 * dWg, 0.25 * dWu)
    B.shampoo_gated_ffn_grad(h, X, Wg, Wu, H, dX=torch.zeros_like(X), dWg=dWg, dWu=dWu, beta=0.25)
    assert torch.equal(dWg, want[0]) and torch.equal(dWu, want[1])


def test_gated_ffn_far_offsets(env):
    """Activations of more than 2^31 elements: the rows at their end."""
    import oracle.model_oracle as M
    torch, B, dev, h = env
    n, d, w = 525000, 4096, 24
    say("ffn far", n, d, w)
    gen = torch.Generator(device=dev).manual_seed(1)
    X = torch.empty(n, d, device=dev, dtype=torch.bfloat16)
    for r in range(0, n, 65536):
        part = X[r:r + 65536]
        part.copy_(torch.randn(part.shape, generator=gen, device=dev))
    Wg, Wu = ((normal(env, i, d, w) / 64).bfloat16() for i in (2, 3))
    H, G, Uo = (torch.empty(n, w, device=dev, dtype=torch.bfloat16) for _ in range(3))
    B.shampoo_gated_ffn(h, X, Wg, Wu, H, B.ACT_NONE, G, Uo,
                        workspace=room(env, B.shampoo_gated_ffn_workspace_bytes(n, d, w, X.dtype)))
    dX = torch.empty_like(X)
    B.shampoo_gated_ffn_grad(h, X, Wg, Wu, H, B.ACT_NONE, G, Uo, dX=dX, workspace=room(
        env, B.shampoo_gated_ffn_grad_workspace_bytes(n, d, w, X.dtype, X.dtype)))
    torch.cuda.synchronize()
    x = X[-500:].double()
    for m, got in ((Wg, G), (Wu, Uo)):
        ref = x @ m.double()
        e = U * (20 + d ** 0.5) * (x.abs() @ m.double().abs())
        close(got[-500:], ref, e + HALF * (ref.abs() + e), "projection")
    dG, dU = M.gated_grad(G[-500:].double(), Uo[-500:].double(), H[-500:], B.ACT_NONE)
    ref = dG @ Wg.double().t().contiguous() + dU @ Wu.double().t().contiguous()
    e = (HALF + 40 * U) * (dG.abs() @ Wg.double().abs().t().contiguous() + dU.abs() @ Wu.double().abs().t().contiguous())
    close(dX[-500:], ref, e + HALF * (ref.abs() + e), "dX")


# ------------------------------------------------------------------ how calls run
def test_c_entry_refusals(env):
    """What the binding lets through is refused by the library with its reason, and
    nothing is written."""
    torch, B, dev, h = env
    say("refusals")
    X, W, lse = normal(env, 1, 8, 16), normal(env, 2, 24, 16), torch.full((8,), 3.0, device=dev)
    t = torch.zeros(8, device=dev, dtype=torch.int32)
    need = B.shampoo_vocab_logprobs_workspace_bytes(8, 16, 24, X.dtype)
    ws = torch.zeros(need + 16, device=dev, dtype=torch.uint8)
    g = torch.zeros(8, device=dev)

    def refused(fn, match):
        with pytest.raises(B.ShampooError, match=match):
            fn()
    logp = g.clone()
    refused(lambda: B.shampoo_vocab_logprobs(h, X, W, t, logp, lse, workspace=ws[1:]), "aligned")
    refused(lambda: B.shampoo_vocab_logprobs(h, X, W, t, lse, lse, workspace=ws), "overlap")
    refused(lambda: B.shampoo_vocab_logprobs(h, X, W, lse.view(torch.int32), logp, lse, workspace=ws), "overlap")
    gw = torch.zeros(B.shampoo_vocab_logprobs_grad_workspace_bytes(8, 16, 24, X.dtype, X.dtype), device=dev,
                     dtype=torch.uint8)
    dX = torch.zeros_like(X)
    refused(lambda: B.shampoo_vocab_logprobs_grad(h, X, W, t, lse, dX=dX, g_logp=g, beta=float("inf"), workspace=gw),
            "finite")
    Wg, Wu, H = normal(env, 3, 16, 8), normal(env, 4, 16, 8), torch.zeros(8, 8, device=dev)
    fw = torch.zeros(B.shampoo_gated_ffn_workspace_bytes(8, 16, 8, X.dtype), device=dev, dtype=torch.uint8)
    refused(lambda: B.shampoo_gated_ffn(h, X, Wg, Wu, H, 9, workspace=fw), "activation")
    for rate in (-0.1, 1.5, float("nan")):
        refused(lambda: B.shampoo_dropout(h, X, dX, rate, 1), "rate")
    # what overlaps is refused by the library and named by the binding
    w = torch.zeros(24, 16, device=dev)
    big = torch.zeros(8 * 8 + 16 * 8 - 1, device=dev)
    for fn in (lambda: B.shampoo_vocab_logprobs_grad(h, X, w, t, lse, dW=w, g_logp=g, workspace=gw),
               lambda: B.shampoo_gated_ffn(h, X, big[:128].view(16, 8), Wu, big[127:].view(8, 8), workspace=fw),
               lambda: B.shampoo_dropout(h, big[:64].view(8, 8), big[1:65].view(8, 8), 0.5, 1)):
        with pytest.raises(ValueError, match="overlap"):
            fn()
    torch.cuda.synchronize()
    assert bool((w == 0).all()) and bool((big == 0).all())
    assert bool((dX == 0).all()) and bool((H == 0).all()) and bool((lse == 3).all())


def model_step(env, X, Wg, Wu, Wo, t, bufs, seed):
    """Block, dropout with the residual, loss and all gradients; returns the outputs."""
    torch, B, dev, h = env
    H, G, Uo, P, Y, lse, logp, gl, dY, dP, dH, dWo, dX, dWg, dWu, w = bufs
    B.shampoo_gated_ffn(h, X, Wg, Wu, H, B.ACT_SILU, G, Uo, workspace=w[0])
    torch.matmul(H, P, out=Y)
    B.shampoo_dropout(h, Y, Y, 0.1, seed, offset=3, R=X)
    B.shampoo_vocab_logprobs(h, Y, Wo, t, logp, lse, workspace=w[1])
    B.shampoo_vocab_logprobs_grad(h, Y, Wo, t, lse, dX=dY, dW=dWo, g_logp=gl, workspace=w[2])
    B.shampoo_dropout(h, dY, dP, 0.1, seed, offset=3)
    torch.matmul(dP, P.t(), out=dH)
    B.shampoo_gated_ffn_grad(h, X, Wg, Wu, dH, B.ACT_SILU, G, Uo, dX, dWg, dWu, workspace=w[3])
    return [logp, lse, dY, dWo, dX, dWg, dWu]


def model_buffers(env, n, d, w, v, dt):
    torch, B, dev, h = env

    def e(*s, dtype=dt):
        return torch.zeros(*s, device=dev, dtype=dtype)
    f4 = torch.float32
    ws = [room(env, x) for x in (B.shampoo_gated_ffn_workspace_bytes(n, d, w, dt),
                                 B.shampoo_vocab_logprobs_workspace_bytes(n, d, v, dt),
                                 B.shampoo_vocab_logprobs_grad_workspace_bytes(n, d, v, dt, f4),
                                 B.shampoo_gated_ffn_grad_workspace_bytes(n, d, w, dt, f4))]
    P = (normal(env, 9, w, d) / w ** 0.5).to(dt)
    gl = torch.full((n,), -1.0 / n, device=dev)
    return [e(n, w), e(n, w), e(n, w), P, e(n, d), e(n, dtype=f4), e(n, dtype=f4), gl, e(n, d), e(n, d), e(n, w),
            e(v, d, dtype=f4), e(n, d), e(d, w, dtype=f4), e(d, w, dtype=f4), ws]


def model_inputs(env, n, d, w, v, dt, seed):
    torch, B, dev, h = env
    t = torch.randint(-1, v, (n,), device=dev, dtype=torch.int32,
                      generator=torch.Generator(device=dev).manual_seed(seed))
    return ((normal(env, seed, n, d)).to(dt), (normal(env, 1, d, w) / d ** 0.5).to(dt),
            (normal(env, 2, d, w) / d ** 0.5).to(dt), (normal(env, 3, v, d) / d ** 0.5).to(dt), t)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_a_step_of_a_model(env, dtype):
    """All calls in a row against 64 bits (with the products between them in 64 bits
    too), then the optimizer's step on the gradients."""
    import oracle.model_oracle as M
    torch, B, dev, h = env
    dt = dtype_of(env, dtype)
    n, d, w, v = 384, 128, 264, 1000
    say("model step", dtype)
    X, Wg, Wu, Wo, t = model_inputs(env, n, d, w, v, dt, 20)
    bufs = model_buffers(env, n, d, w, v, dt)
    logp, lse, dY, dWo, dX, dWg, dWu = [x.double() for x in model_step(env, X, Wg, Wu, Wo, t, bufs, 77)]
    torch.cuda.synchronize()
    keep, cut = M.kept(n, d, 0.1, 77, 3)
    keep = torch.from_numpy(keep).to(dev)
    rh, rg, ru = M.gated(X, Wg, Wu, B.ACT_SILU)
    P = bufs[3].double()
    y = M.dropout(rh @ P, keep, cut, X)
    rp, rl, z = M.vocab_logprobs(y, Wo, t)
    dz, _ = M.vocab_dlogits(z, rl, t, bufs[7])
    ry = dz @ Wo.double()
    rdh = M.dropout(ry, keep, cut) @ P.t().contiguous()
    dG, dU = M.gated_grad(rg, ru, rdh, B.ACT_SILU)
    # Roundings of a chain, relative to the size of the results: in bf16 at most ten of
    # half a step each, root mean square 2^-9, on a path (10 2^-9 = 2%); in fp32 the sums
    # of up to 1000 terms, u sqrt(1000), each
    tol = 0.02 if dt is torch.bfloat16 else 10 * U * 32
    for what, got, ref in (("logp", logp, rp), ("lse", lse, rl), ("dY", dY, ry), ("dWo", dWo, dz.t().contiguous() @ y),
                           ("dX", dX, dG @ Wg.double().t().contiguous() + dU @ Wu.double().t().contiguous()),
                           ("dWg", dWg, X.double().t().contiguous() @ dG), ("dWu", dWu, X.double().t().contiguous() @ dU)):
        err = float((got - ref).norm() / ref.norm())
        assert err <= tol, (what, err, tol)
    # the gradients go to the optimizer as they are
    W = Wg.float()
    L, R, Lr, Rr = (torch.eye(k, device=dev) for k in (d, w, d, w))
    blk = B.Block(G=bufs[13], W=W, D=torch.zeros_like(W), P=torch.zeros_like(W), L=L, R=R, Lr=Lr, Rr=Rr)
    B.shampoo_update_stats(h, [blk], 1.0)
    B.shampoo_precondition_graft(h, [blk], 0.1)
    g = bufs[13].double()
    want = torch.eye(d, device=dev, dtype=torch.float64) + g @ g.t().contiguous()
    assert float((L.double() - want).norm() / want.norm()) <= 1e-5
    assert bool(torch.isfinite(W).all())


def test_captured_steps_share_nothing(env):
    """Two captured graphs of the step, each with its own buffers and workspaces,
    replayed in turn with eager calls between: every replay equals the eager call."""
    torch, B, dev, h = env
    n, d, w, v, dt = 200, 128, 264, 1000, torch.bfloat16
    say("captured steps")
    runs = []
    side = torch.cuda.Stream()
    for i in range(2):
        inp, bufs = model_inputs(env, n, d, w, v, dt, 30 + i), model_buffers(env, n, d, w, v, dt)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            model_step(env, *inp, bufs, 5)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = model_step(env, *inp, bufs, 5)
        runs.append((inp, bufs, graph, outs))
    eager = model_buffers(env, n, d, w, v, dt)
    for turn in range(3):
        for inp, bufs, graph, outs in runs:
            inp[0].copy_(normal(env, 100 + turn, n, d))
            for o in outs:
                o.fill_(float("nan"))
            graph.replay()
            want = model_step(env, *inp, eager, 5)
            torch.cuda.synchronize()
            for a, b in zip(outs, want):
                assert torch.equal(a, b)


def test_two_streams_and_repeats(env):
    """Calls of one handle that overlap on two streams, and repeated ones, give the
    same bits."""
    torch, B, dev, h = env
    n, d, w, v, dt = 300, 256, 520, 3001, torch.bfloat16
    say("two streams")
    inp = model_inputs(env, n, d, w, v, dt, 60)
    sets = [model_buffers(env, n, d, w, v, dt) for _ in range(3)]
    want = [x.clone() for x in model_step(env, *inp, sets[0], 9)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s, b in zip(streams, sets[1:]):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            for _ in range(3):
                model_step(env, *inp, b, 9)
    torch.cuda.synchronize()
    for b in sets[1:]:
        got = [b[6], b[5], b[8], b[11], b[12], b[13], b[14]]
        for x, y in zip(got, want):
            assert torch.equal(x, y)


def test_a_small_workspace_is_named(env):
    """The binding leaves the size to the library and says what is missing."""
    torch, B, dev, h = env
    n, d, w = 70, 24, 40
    X, g, u, dH = (normal(env, i, *s) for i, s in ((1, (n, d)), (2, (d, w)), (3, (d, w)), (4, (n, w))))
    W, t = normal(env, 5, w, d), torch.zeros(n, device=dev, dtype=torch.int32)
    lse, logp = torch.zeros(n, device=dev), torch.zeros(n, device=dev)
    H, dX, dW, dg, du = (torch.empty_like(x) for x in (dH, X, W, g, u))
    f = torch.float32
    for need, call in (
            (B.shampoo_vocab_logprobs_workspace_bytes(n, d, w, f),
             lambda ws: B.shampoo_vocab_logprobs(h, X, W, t, logp, lse, workspace=ws)),
            (B.shampoo_vocab_logprobs_grad_workspace_bytes(n, d, w, f, f),
             lambda ws: B.shampoo_vocab_logprobs_grad(h, X, W, t, lse, dX=dX, dW=dW, g_logp=logp, workspace=ws)),
            (B.shampoo_gated_ffn_workspace_bytes(n, d, w, f), lambda ws: B.shampoo_gated_ffn(h, X, g, u, H, workspace=ws)),
            (B.shampoo_gated_ffn_grad_workspace_bytes(n, d, w, f, f),
             lambda ws: B.shampoo_gated_ffn_grad(h, X, g, u, dH, dX=dX, dWg=dg, dWu=du, workspace=ws))):
        assert need > 0
        with pytest.raises(ValueError, match="at least"):
            call(torch.empty(need - 1, device=dev, dtype=torch.uint8))
        with pytest.raises(ValueError, match="needed"):
            call(None)
        with pytest.raises(ValueError, match="uint8"):
            call(torch.empty(need, device=dev))
        call(torch.empty(need, device=dev, dtype=torch.uint8))
    torch.cuda.synchronize()
