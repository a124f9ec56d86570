"""The layers around the step at the edges of their range, on the GPU against the 64-bit
oracle: many logits, rows without gradients, the accuracy of fp32 gradients of bf16
inputs, non-finite values.  Tolerances as in test_gpu_model_layers."""
import pytest

from tests.gpu_util import say
from tests.test_gpu_model_layers import HALF, U, Sheet, close, env, logprobs, normal, room  # noqa: F401

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
