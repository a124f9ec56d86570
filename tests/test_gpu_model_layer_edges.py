"""The layers around the step at the edges of their range, on the GPU against the 64-bit
oracle: many logits, rows without gradients, the accuracy of fp32 gradients of bf16
inputs, non-finite values.  Tolerances as in test_gpu_model_layers."""
import pytest

from tests.gpu_util import say
from tests.test_gpu_model_layers import HALF, U, Sheet, close, env, logprobs, normal, room, z_error  # noqa: F401

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ many logits
@pytest.mark.parametrize("n,d,v", [(32768, 8, 262144), (4200000, 8, 2000)])
def test_many_logits(env, n, d, v):
    """Batches of 2^33 logits: taken wherever the table lies.  Rows all over the batch."""
    torch, B, dev, h = env
    X = (normal(env, 1, n, d)).bfloat16()
    t = torch.randint(-1, v, (n,), generator=torch.Generator(device=dev).manual_seed(2), device=dev, dtype=torch.int32)
    rows = torch.cat([torch.arange(0, n, max(1, n // 500), device=dev), torch.arange(n - 300, n, device=dev)])
    for pad, shift in ((0, 0), (5, 3)):
        say("many logits", n, d, v, pad, shift)
        W = Sheet(env, v, d, torch.bfloat16, pad, shift, normal(env, 3, v, d)).v
        logp, lse = logprobs(env, X, W, t)
        torch.cuda.synchronize()
        z = X[rows].double() @ W.double().t().contiguous()
        rl = torch.logsumexp(z, 1)
        on = t[rows].long()
        rp = torch.where(on >= 0, z.gather(1, on.clamp(min=0).unsqueeze(1))[:, 0] - rl, torch.zeros_like(rl))
        size = (X[rows].double().abs() @ W.double().abs().t().contiguous()).amax(1)
        tol = U * (20 + d ** 0.5) * size + U * (32 + rl.abs())
        close(lse[rows], rl, tol, "lse")
        close(logp[rows], rp, 2 * tol + U * rp.abs() * 4, "logp")
        assert bool(torch.isfinite(lse).all()) and bool((logp <= 0).all())


# ------------------------------------------------------------------ rows without gradients
TYPE_PAIRS = [("bfloat16", "bfloat16"), ("bfloat16", "float32"), ("float32", "float32"), ("float32", "bfloat16")]
# tiles of few rows, middling and large ones, a contraction in parts, tables read as they lie and copied
ROWS = [(5, 64, 300, 0), (5, 1003, 1001, 3), (40, 72, 1001, 3), (300, 128, 1500, 0), (130, 3330, 700, 5),
        (1100, 256, 4100, 0)]


@pytest.mark.parametrize("dtype,g_dtype", TYPE_PAIRS)
def test_rows_without_gradients_add_nothing(env, dtype, g_dtype):
    """Padding rows, whose gradients are 0: whatever their lse holds (zeros where it was
    never formed, though their logits lie beyond what exp holds), their dX is 0 and the
    other results are those of the call with their true lse, to the bit.  With no row
    that has a gradient, dW is 0 whatever the table holds."""
    torch, B, dev, h = env
    dt, gt = getattr(torch, dtype), getattr(torch, g_dtype)
    for n, d, v, pad in ROWS:
        say("rows without gradients", n, d, v, dtype, g_dtype, pad)
        x = normal(env, 1, n, d)
        dead = torch.arange(n, device=dev) % 3 == 0
        x[dead] *= 64
        X = Sheet(env, n, d, dt, pad, pad, x).v
        W = Sheet(env, v, d, dt, pad, pad, normal(env, 2, v, d) * (2.0 / d ** 0.5)).v
        z = X.double() @ W.double().t().contiguous()
        assert float(z[dead].amax(1).min()) > 100
        lse = torch.logsumexp(z, 1).float()
        t = torch.randint(0, v, (n,), generator=torch.Generator(device=dev).manual_seed(3), device=dev, dtype=torch.int32)
        g_logp, g_lse = normal(env, 4, n), normal(env, 5, n)
        t[::6] = -1        # dead rows without a token, whose g_logp counts for nothing
        g_logp[3::6] = 0   # and with one
        g_lse[dead] = 0
        ws = room(env, B.shampoo_vocab_logprobs_grad_workspace_bytes(n, d, v, dt, gt))

        def grads(lse, gl, gs, table=W):
            dX, dW = torch.full((n, d), 7.0, device=dev, dtype=dt), torch.full((v, d), 7.0, device=dev, dtype=gt)
            B.shampoo_vocab_logprobs_grad(h, X, table, t, lse, dX=dX, dW=dW, g_logp=gl, g_lse=gs, workspace=ws)
            torch.cuda.synchronize()
            return dX, dW
        want = grads(lse, g_logp, g_lse)
        assert bool(torch.isfinite(want[0]).all()) and bool(torch.isfinite(want[1]).all())
        for held in (0.0, -3e38, float("nan"), float("inf"), -float("inf")):
            other = lse.clone()
            other[dead] = held
            got = grads(other, g_logp, g_lse)
            assert bool((got[0][dead] == 0).all()), held
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), held
        bad = W.clone()
        bad[0, 0], bad[-1, 0] = float("nan"), float("inf")
        none = torch.zeros(n, device=dev)
        for gl, gs in ((none, none), (none, None), (None, none), (None, None)):
            assert bool((grads(lse, gl, gs, bad)[1] == 0).all())


# ------------------------------------------------------------------ fp32 gradients of bf16 inputs
def tanh_gelu(torch, x):
    """Value, slope and |w| of gelu's tanh form x p, p = 1 / (1 + e^-w), w = 2 sqrt(2 / pi) (x +
    0.044715 x^3).  1 + tanh(w / 2) = 2 p, but that sum loses all bits of p below 2^-53, where
    the library's fp32 still has 24 of them (x = -8: p = 3e-22)."""
    c = 2 * (2 / torch.pi) ** 0.5
    w = c * (x + 0.044715 * x ** 3)
    p, q = torch.sigmoid(w), torch.sigmoid(-w)
    return x * p, p + x * p * q * c * (1 + 3 * 0.044715 * x * x), w.abs()


@pytest.mark.parametrize("keep", [True, False])
@pytest.mark.parametrize("act", ["RELU", "GELU", "GELU_TANH", "SILU"])
def test_fp32_block_gradients_are_fp32(env, act, keep):
    """Rows of X that are unit vectors: G and U are rows of the weights, dWg and dWu are dG
    and dU, element by element (the other terms of their sums are zeros).  With fp32
    gradients their errors are those of fp32, of bf16 inputs too: u (16 + x^2) (1 + x^2)
    relative to 1 for an activation's slope, u (16 + x^2) of its value, and 4 u for the
    products and the terms' 2^-24.  The value of gelu's tanh form is off by u (16 + 7 |w|):
    w is two rounded constants and five rounded operations, none of which cancels, and an
    error dw of it is one of (1 - p) dw <= |dw| relative in p = 1 / (1 + e^-w).  Values below
    2^-126 and terms below 2^-133 may vanish: 2^-120 of the factors."""
    import oracle.model_oracle as M
    torch, B, dev, h = env
    kind = getattr(B, "ACT_" + act)
    for n, d, w, pad in ((1, 1, 9, 0), (5, 40, 200, 3), (30, 30, 264, 0), (200, 264, 520, 0), (1100, 1104, 1500, 5)):
        for dt in (torch.bfloat16, torch.float32):
            say("fp32 block gradients", n, d, w, dt, act, keep)
            X = Sheet(env, n, d, dt, pad, pad, torch.eye(n, d, device=dev)).v
            Wg = Sheet(env, d, w, dt, pad, pad, 2.5 * normal(env, 1, d, w)).v
            Wu = Sheet(env, d, w, dt, pad, pad, normal(env, 2, d, w)).v
            dH = Sheet(env, n, w, dt, pad, pad, normal(env, 3, n, w)).v
            dX = torch.empty(n, d, device=dev, dtype=dt)
            dWg, dWu = (torch.full((d, w), 7.0, device=dev) for _ in range(2))
            B.shampoo_gated_ffn_grad(h, X, Wg, Wu, dH, kind, Wg[:n] if keep else None, Wu[:n] if keep else None, dX, dWg,
                                     dWu, workspace=room(env, B.shampoo_gated_ffn_grad_workspace_bytes(
                                         n, d, w, dt, torch.float32)))
            torch.cuda.synchronize()
            g, u = Wg[:n].double(), Wu[:n].double()
            hh, far = dH.double().abs(), g * g
            a, s = M.act(g, kind), M.slope(g, kind)
            if act == "GELU_TANH":
                a, s, far = tanh_gelu(torch, g)
                far = 7 * far
            dG, dU = dH.double() * u * s, dH.double() * a
            least = 2.0 ** -120 * (1 + hh * (1 + u.abs()))
            close(dWg[:n], dG, hh * u.abs() * U * (16 + g * g) * (1 + g * g) + 4 * U * dG.abs() + least, "dG")
            close(dWu[:n], dU, hh * U * (16 + far) * a.abs() + 4 * U * dU.abs() + least, "dU")
            assert bool((dWg[n:] == 0).all()) and bool((dWu[n:] == 0).all())


# sizes that reach every tile of dX, whole and in parts and in pieces of the vocabulary
# (test_stream_limits checks that): rows, dim, vocabulary or width, whether matrices are copied
VOCAB_TERMS = [(1, 8, 8, 1), (66, 8, 960, 1), (739, 645, 10, 1), (746, 15, 1321, 1), (698, 1434, 175, 1),
               (7566, 387, 6018, 1), (1374, 10, 1886, 1), (6716, 8, 7080, 1), (3139, 3318, 8, 1), (7614, 1408, 5862, 0),
               (5404, 170, 4120, 1), (4175, 160, 14388, 1), (5, 3996, 4210, 1), (1, 12, 1831, 1), (2582, 8, 20755, 1),
               (1, 1441, 2188, 1), (33, 4002, 35019, 1), (2418, 1725, 8, 1), (4205, 9, 3514, 1), (5016, 9, 9385, 1),
               (6673, 131, 5552, 1)]
FFN_TERMS = [(1, 8, 8, 1), (68, 10, 481, 1), (831, 611, 8, 0), (341, 68, 936, 1), (1256, 778, 104, 0), (1502, 8, 791, 1),
             (4474, 2420, 12, 1), (2789, 129, 4045, 1), (1, 3200, 2657, 1), (30, 2243, 40, 1), (2, 8, 897, 1),
             (1, 1379, 1240, 1), (2058, 1925, 12, 1), (1390, 8, 3522, 1)]


@pytest.mark.parametrize("n,d,v,copied", VOCAB_TERMS)
def test_dx_takes_the_terms_of_dz(env, n, d, v, copied):
    """bf16 dX beside an fp32 dW: of dz in two terms, each within 2^-8 of what it stands
    for, so off by 2^-16 of dz, and rounded once, 2^-8 of the result."""
    import oracle.model_oracle as M
    torch, B, dev, h = env
    bf, pad = torch.bfloat16, 5 if copied else 0
    say("terms of dz", n, d, v, pad)
    X = Sheet(env, n, d, bf, pad, pad, normal(env, 1, n, d)).v
    W = Sheet(env, v, d, bf, pad, pad, normal(env, 2, v, d) * (2.0 / d ** 0.5)).v
    t = torch.randint(-1, v, (n,), generator=torch.Generator(device=dev).manual_seed(3), device=dev, dtype=torch.int32)
    g_logp, g_lse = normal(env, 4, n), normal(env, 5, n)
    _, lse, z = M.vocab_logprobs(X, W, t)
    lse = lse.float()
    dX, dW = Sheet(env, n, d, bf, pad, pad), torch.empty(v, d, device=dev)
    B.shampoo_vocab_logprobs_grad(h, X, W, t, lse, dX=dX.v, dW=dW, g_logp=g_logp, g_lse=g_lse, workspace=room(
        env, B.shampoo_vocab_logprobs_grad_workspace_bytes(n, d, v, bf, torch.float32)))
    torch.cuda.synchronize()
    dz, size = M.vocab_dlogits(z, lse, t, g_logp, g_lse)
    far = (z_error(X, W) + U * (4 + (z - lse.double().unsqueeze(1)).abs().amax(1))).unsqueeze(1)
    # two rounds of a sum: its roundings add up like those of twice the length
    part = (far * size + (2.0 ** -16 + U * (20 + (2 * v) ** 0.5)) * dz.abs()) @ W.double().abs()
    ref = dz @ W.double()
    close(dX.v, ref, part + HALF * (ref.abs() + part), "dX")
    assert dX.intact(torch)


# the same for dX and dW of up to 32 rows, together and each alone, and with a table read where it lies
FEW_TERMS = [(4, 8, 449, 0), (8, 68, 32989, 1), (1, 129, 45455, 1), (2, 8, 5122, 0), (1, 646, 14172, 1), (1, 270, 62204, 1),
             (1, 8, 8, 0), (3, 8, 973, 0), (32, 1024, 5000, 0), (31, 333, 1027, 1)]


@pytest.mark.parametrize("n,d,v,copied", FEW_TERMS)
def test_few_rows_take_two_terms(env, n, d, v, copied):
    """bf16 gradients of up to 32 rows of bf16: dz in two terms, off by 2^-16, and one rounding
    of each result."""
    import oracle.model_oracle as M
    torch, B, dev, h = env
    bf, pad = torch.bfloat16, 5 if copied else 0
    say("two terms of few rows", n, d, v, pad)
    X = Sheet(env, n, d, bf, pad, pad, normal(env, 1, n, d)).v
    W = Sheet(env, v, d, bf, pad, pad, normal(env, 2, v, d) * (2.0 / d ** 0.5)).v
    t = torch.randint(0, v, (n,), generator=torch.Generator(device=dev).manual_seed(3), device=dev, dtype=torch.int32)
    g_logp, g_lse = normal(env, 4, n), 0.1 * normal(env, 5, n)
    _, lse, z = M.vocab_logprobs(X, W, t)
    lse = lse.float()
    dz, size = M.vocab_dlogits(z, lse, t, g_logp, g_lse)
    far = (z_error(X, W) + U * (4 + (z - lse.double().unsqueeze(1)).abs().amax(1))).unsqueeze(1) * size
    ws = room(env, B.shampoo_vocab_logprobs_grad_workspace_bytes(n, d, v, bf, bf))
    for with_x, with_w in ((True, True), (True, False), (False, True)):
        dX, dW = Sheet(env, n, d, bf, pad, pad), Sheet(env, v, d, bf, pad, pad)
        B.shampoo_vocab_logprobs_grad(h, X, W, t, lse, dX=dX.v if with_x else None, dW=dW.v if with_w else None,
                                      g_logp=g_logp, g_lse=g_lse, workspace=ws)
        torch.cuda.synchronize()
        if with_x:
            part = (far + (2.0 ** -16 + U * (20 + (2 * v) ** 0.5)) * dz.abs()) @ W.double().abs()
            ref = dz @ W.double()
            close(dX.v, ref, part + HALF * (ref.abs() + part), "dX")
            assert dX.intact(torch)
        if with_w:
            part = (far + (2.0 ** -16 + U * (20 + (2 * n) ** 0.5)) * dz.abs()).t().contiguous() @ X.double().abs()
            ref = dz.t().contiguous() @ X.double()
            close(dW.v, ref, part + HALF * (ref.abs() + part), "dW")
            assert dW.intact(torch)


@pytest.mark.parametrize("n,d,w,copied", FFN_TERMS)
def test_dx_takes_the_terms_of_the_block(env, n, d, w, copied):
    """The same of dG and dU, of projections as kept."""
    import oracle.model_oracle as M
    torch, B, dev, h = env
    bf, pad = torch.bfloat16, 5 if copied else 0
    X = Sheet(env, n, d, bf, pad, pad, normal(env, 1, n, d)).v
    Wg, Wu = (Sheet(env, d, w, bf, pad, pad, normal(env, i, d, w) / d ** 0.5).v for i in (2, 3))
    dH, G, Uo = (Sheet(env, n, w, bf, pad, pad, normal(env, i, n, w)).v for i in (4, 5, 6))
    for act in ("NONE", "GELU", "SILU"):
        say("terms of dG and dU", n, d, w, pad, act)
        kind = getattr(B, "ACT_" + act)
        dX = Sheet(env, n, d, bf, pad, pad)
        dWg, dWu = (torch.empty(d, w, device=dev) for _ in range(2))
        B.shampoo_gated_ffn_grad(h, X, Wg, Wu, dH, kind, G, Uo, dX.v, dWg, dWu, workspace=room(
            env, B.shampoo_gated_ffn_grad_workspace_bytes(n, d, w, bf, torch.float32)))
        torch.cuda.synchronize()
        g, u, hh = G.double(), Uo.double(), dH.double().abs()
        dG, dU = M.gated_grad(g, u, dH, kind)
        f = U * (16 + g * g)
        q = 2.0 ** -16 + U * (20 + (4 * w) ** 0.5)
        fg = hh * u.abs() * f * (1 + g * g) + (4 * U + q) * dG.abs()
        fu = hh * f * M.act(g, kind).abs() + (4 * U + q) * dU.abs()
        wg, wu = Wg.double().t().contiguous(), Wu.double().t().contiguous()
        ref, err = dG @ wg + dU @ wu, fg @ wg.abs() + fu @ wu.abs()
        close(dX.v, ref, err + HALF * (ref.abs() + err), "dX")
        assert dX.intact(torch)


# ------------------------------------------------------------------ non-finite values, ends of the range
# tiles of few rows (as it lies, and through registers), small, middling and large tiles, contraction in parts
FFN_ROWS = [(3, 64, 136, 0), (5, 100, 200, 3), (40, 72, 1000, 8), (300, 128, 520, 3), (100, 3001, 64, 1), (2100, 264, 2056, 0)]


def same_but(torch, a, b, rows, cols, what):
    """a equals b to the bit outside the given rows and columns (None: none), where it is not finite."""
    on = torch.zeros(a.shape, dtype=torch.bool, device=a.device)
    if rows is not None:
        on[rows] = True
    if cols is not None:
        on[:, cols] = True
    assert not bool(torch.isfinite(a[on]).any()), what
    assert torch.equal(a[~on], b[~on]), what


@pytest.mark.parametrize("bad", ["nan", "inf", "-inf"])
@pytest.mark.parametrize("dtype,g_dtype", TYPE_PAIRS)
def test_non_finite_values_in_the_block(env, dtype, g_dtype, bad):
    """A NaN or an infinity reaches what its products reach, and nothing else: one in row r
    of X row r of the projections; one in column c of Wg column c of G and H; one in dH[r, c]
    row r of dX and column c of dWg and dWu."""
    torch, B, dev, h = env
    dt, gt, bad = getattr(torch, dtype), getattr(torch, g_dtype), float(bad)
    for n, d, w, pad in FFN_ROWS:
        say("non-finite block", n, d, w, dtype, g_dtype, bad, pad)
        r, c, k = n // 2, w // 3, d // 2
        X = Sheet(env, n, d, dt, pad, pad, normal(env, 1, n, d) + 3).v
        Wg, Wu = (Sheet(env, d, w, dt, pad, pad, normal(env, i, d, w) / d ** 0.5).v for i in (2, 3))
        dH = Sheet(env, n, w, dt, pad, pad, normal(env, 4, n, w)).v
        fw = room(env, B.shampoo_gated_ffn_workspace_bytes(n, d, w, dt))
        gw = room(env, B.shampoo_gated_ffn_grad_workspace_bytes(n, d, w, dt, gt))

        def forward():
            out = [torch.empty(n, w, device=dev, dtype=dt) for _ in range(3)]
            B.shampoo_gated_ffn(h, X, Wg, Wu, out[0], B.ACT_NONE, out[1], out[2], workspace=fw)
            torch.cuda.synchronize()
            return out

        def grads(keep):
            out = [torch.empty(n, d, device=dev, dtype=dt)] + [torch.empty(d, w, device=dev, dtype=gt) for _ in range(2)]
            B.shampoo_gated_ffn_grad(h, X, Wg, Wu, dH, B.ACT_SILU, keep and keep[1], keep and keep[2], *out, workspace=gw)
            torch.cuda.synchronize()
            return out
        want = forward()
        for keep in (want, None):
            ref, old = grads(keep), dH[r, c].clone()
            dH[r, c] = bad
            got = grads(keep)
            dH[r, c] = old
            same_but(torch, got[0], ref[0], [r], None, "dX")
            same_but(torch, got[1], ref[1], None, [c], "dWg")
            same_but(torch, got[2], ref[2], None, [c], "dWu")
        old = X[r, k].clone()
        X[r, k] = bad
        for a, b, what in zip(forward(), want, ("H", "G", "U")):
            same_but(torch, a, b, [r], None, what)
        X[r, k] = old
        Wg[k, c] = bad
        got = forward()
        same_but(torch, got[0], want[0], None, [c], "H")
        same_but(torch, got[1], want[1], None, [c], "G")
        assert torch.equal(got[2], want[2])


@pytest.mark.parametrize("dtype,g_dtype", TYPE_PAIRS)
def test_non_finite_values_in_the_gradient_of_the_loss(env, dtype, g_dtype):
    """A NaN or an infinity in g_logp[r] reaches row r of dX, and dW; one in X[r, k], of a row
    without gradients, column k of dW; the rest is as it was, to the bit."""
    torch, B, dev, h = env
    dt, gt = getattr(torch, dtype), getattr(torch, g_dtype)
    for n, d, v, pad in ROWS:
        say("non-finite loss gradient", n, d, v, dtype, g_dtype, pad)
        r, k = n // 2, d // 2
        X = Sheet(env, n, d, dt, pad, pad, normal(env, 1, n, d)).v
        W = Sheet(env, v, d, dt, pad, pad, normal(env, 2, v, d) * (2.0 / d ** 0.5)).v
        t = torch.randint(0, v, (n,), generator=torch.Generator(device=dev).manual_seed(3), device=dev, dtype=torch.int32)
        _, lse = logprobs(env, X, W, t)
        g = normal(env, 4, n)
        ws = room(env, B.shampoo_vocab_logprobs_grad_workspace_bytes(n, d, v, dt, gt))

        def grads():
            dX, dW = torch.empty(n, d, device=dev, dtype=dt), torch.empty(v, d, device=dev, dtype=gt)
            B.shampoo_vocab_logprobs_grad(h, X, W, t, lse, dX=dX, dW=dW, g_logp=g, workspace=ws)
            torch.cuda.synchronize()
            return dX, dW
        g[r] = 0
        want = grads()
        old = X[r, k].clone()
        for bad in (float("nan"), float("inf"), -float("inf")):
            X[r, k] = bad
            got = grads()
            assert torch.equal(got[0], want[0]) and bool((got[0][r] == 0).all())
            same_but(torch, got[1], want[1], None, [k], "dW")
            X[r, k] = old
            g[r] = bad
            got = grads()
            same_but(torch, got[0], want[0], [r], None, "dX")
            assert not bool(torch.isfinite(got[1]).any())
            g[r] = 0


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_ends_of_the_range(env, dtype):
    """Products of small values with large ones.  bf16 values are exact down to the smallest,
    2^-133; fp32 ones have three terms that end there, so a value x is off by 2^-134 at most,
    beside the products' own errors, and is exact from 2^-110 on.  The largest values below
    2^128 - 2^119 stay finite, those from there on become infinite in fp32."""
    torch, B, dev, h = env
    dt = getattr(torch, dtype)
    for n, d, w, pad in FFN_ROWS:
        for small in (-90, -104, -112, -120, -126, -130):
            say("ends of the range", n, d, w, dtype, small, pad)
            x = normal(env, 1, n, d) * 2.0 ** 8
            X = Sheet(env, n, d, dt, pad, pad, torch.ldexp(x, torch.tensor(small - 8, device=dev))).v
            Wg, Wu = (Sheet(env, d, w, dt, pad, pad, normal(env, i, d, w) * 2.0 ** 100).v for i in (2, 3))
            H, G, Uo = (torch.empty(n, w, device=dev, dtype=dt) for _ in range(3))
            ws = room(env, B.shampoo_gated_ffn_workspace_bytes(n, d, w, dt))
            B.shampoo_gated_ffn(h, X, Wg, Wu, H, B.ACT_NONE, G, Uo, workspace=ws)
            torch.cuda.synchronize()
            for got, m in ((G, Wg), (Uo, Wu)):
                ref, size = X.double() @ m.double(), X.double().abs() @ m.double().abs()
                cut = 0.0 if dt is torch.bfloat16 else 2.0 ** -134 * m.double().abs().sum(0, keepdim=True)
                err = U * (20 + d ** 0.5) * size + cut
                close(got, ref, err + (HALF if dt is torch.bfloat16 else U) * (ref.abs() + err), "projection")
        X = Sheet(env, n, d, dt, pad, pad, torch.zeros(n, d, device=dev)).v
        largest = torch.tensor(2.0 ** 128 - 2.0 ** 120 if dt is torch.bfloat16 else 2.0 ** 128 - 2.0 ** 119 - 2.0 ** 104,
                               dtype=torch.float64, device=dev).to(dt)
        X[0, 0], X[n - 1, d - 1] = largest, -largest
        g, u = Wg.double() * 2.0 ** -140, Wu.double() * 2.0 ** -140
        Wg.copy_(g), Wu.copy_(u)
        B.shampoo_gated_ffn(h, X, Wg, Wu, H, B.ACT_NONE, G, Uo, workspace=ws)
        torch.cuda.synchronize()
        for got, m in ((G, Wg), (Uo, Wu)):
            ref = X.double() @ m.double()
            close(got, ref, (HALF + 40 * U) * ref.abs(), "projection of the largest")
        if dt is torch.float32:
            X[0, 0] = torch.tensor(2.0 ** 128 - 2.0 ** 119, dtype=torch.float64).float()
            B.shampoo_gated_ffn(h, X, Wg, Wu, H, B.ACT_NONE, G, Uo, workspace=ws)
            torch.cuda.synchronize()
            assert not bool(torch.isfinite(G[0]).any()) and bool(torch.isfinite(G[1:]).all())


# ------------------------------------------------------------------ other calls that the header allows
@pytest.mark.parametrize("dtype,g_dtype", TYPE_PAIRS)
def test_gradient_of_lse_alone(env, dtype, g_dtype):
    """Without targets: the bits of the call whose targets are all outside the vocabulary."""
    torch, B, dev, h = env
    dt, gt = getattr(torch, dtype), getattr(torch, g_dtype)
    for n, d, v, pad in ROWS:
        say("gradient of lse", n, d, v, dtype, g_dtype, pad)
        X = Sheet(env, n, d, dt, pad, pad, normal(env, 1, n, d)).v
        W = Sheet(env, v, d, dt, pad, pad, normal(env, 2, v, d) * (2.0 / d ** 0.5)).v
        _, lse = logprobs(env, X, W, None)
        g = normal(env, 3, n)
        ws = room(env, B.shampoo_vocab_logprobs_grad_workspace_bytes(n, d, v, dt, gt))
        out = []
        for t in (None, torch.full((n,), -1, device=dev, dtype=torch.int32), torch.full((n,), v, device=dev, dtype=torch.int32)):
            dX, dW = torch.empty(n, d, device=dev, dtype=dt), torch.empty(v, d, device=dev, dtype=gt)
            B.shampoo_vocab_logprobs_grad(h, X, W, t, lse, dX=dX, dW=dW, g_lse=g, workspace=ws)
            out.append((dX, dW))
        torch.cuda.synchronize()
        for dX, dW in out[1:]:
            assert torch.equal(dX, out[0][0]) and torch.equal(dW, out[0][1])
        p = torch.softmax(X.double() @ W.double().t().contiguous(), 1) * g.double().unsqueeze(1)
        err = float((out[0][0].double() - p @ W.double()).norm() / (p @ W.double()).norm())
        # two roundings, each of at most half a step
        assert err <= (2 * HALF if dt is torch.bfloat16 else 1e-5), err


def test_rows_far_apart(env):
    """Rows 2^21 elements apart and more: the bits of the same matrices side by side (of few
    rows in bf16, whose weights lie another way then, of the copied ones)."""
    torch, B, dev, h = env
    d, w, gap = 40, 72, 2 ** 21 + 8
    for n in (3, 90):
        for dt in (torch.bfloat16, torch.float32):
            say("rows far apart", n, dt)

            def far(rows, cols, x):
                s = torch.empty(rows, gap, device=dev, dtype=dt)[:, :cols]
                s.copy_(x)
                return s

            def near(rows, cols, x):
                return Sheet(env, rows, cols, dt, 3, 1, x).v
            out = []
            for place in (near, far):
                X, W = place(n, d, normal(env, 1, n, d)), place(w, d, normal(env, 2, w, d))
                Wg, Wu, dH = (place(a, w, normal(env, i, a, w)) for i, a in ((3, d), (4, d), (5, n)))
                t = torch.arange(n, device=dev, dtype=torch.int32) % w
                logp, lse = logprobs(env, X, W, t)
                dX, dW = place(n, d, 0 * X), place(w, d, 0 * W)
                B.shampoo_vocab_logprobs_grad(h, X, W, t, lse, dX=dX, dW=dW, g_logp=normal(env, 6, n), workspace=room(
                    env, B.shampoo_vocab_logprobs_grad_workspace_bytes(n, d, w, dt, dt)))
                H, dY = place(n, w, 0 * dH), place(n, d, 0 * X)
                dg, du = place(d, w, 0 * Wg), place(d, w, 0 * Wu)
                B.shampoo_gated_ffn(h, X, Wg, Wu, H, workspace=room(
                    env, B.shampoo_gated_ffn_workspace_bytes(n, d, w, dt)))
                B.shampoo_gated_ffn_grad(h, X, Wg, Wu, dH, dX=dY, dWg=dg, dWu=du, workspace=room(
                    env, B.shampoo_gated_ffn_grad_workspace_bytes(n, d, w, dt, dt)))
                torch.cuda.synchronize()
                out.append([x.clone() for x in (logp, lse, dX, dW, H, dY, dg, du)])
            for a, b in zip(*out):
                assert torch.equal(a, b)
