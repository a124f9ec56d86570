"""The training example: its gradients against 64-bit ones of the same step, and
its loss over a few steps."""
import numpy as np
import pytest

import oracle.layer_oracle as L
from tests.gpu_util import gpu_env, host, rel, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    torch, B, dev = gpu_env()
    h = B.shampoo_create(0)
    yield torch, B, dev, h
    B.shampoo_destroy(h)


def test_gradients_of_a_step(env):
    """Against 64 bits with the same weights.  The checkpoints move each kept
    value by at most 2^-7 of its group's largest (half a step: a root mean
    square of 2^-7 / sqrt 3 of it, and a group's largest of 32 normal values is
    about 2.1 times their root mean square: 1%), bf16 roundings of logits and
    activations by 2^-9 root mean square each: 5% bounds both gradients."""
    from examples.train_head import Head, data
    torch, B, dev, h = env
    say("train head gradients")
    tokens, dim, width, classes = 512, 96, 160, 301
    head = Head(h, dim, width, classes, tokens, dev, eta0=0.0)
    X, t = data(tokens, dim, classes, dev, 3)
    loss = head.step(X, t)
    torch.cuda.synchronize()
    x, w1, w2 = host(X.double()), host(head.W[0].bfloat16().double()), host(head.W[1].bfloat16().double())
    tt = host(t)
    z = x @ w1
    a = L.act(z, L.GELU)
    logp, lse, ent, _, _ = L.token_logprobs(a @ w2, tt)
    n = (tt >= 0).sum()
    assert abs(float(loss) + logp.sum() / n) <= 2e-2
    d = L.token_logprobs_grad(a @ w2, tt, lse, g_logp=np.full(tokens, -1.0 / n))
    assert rel(host(head.G[1]), a.T @ d) <= 0.05
    assert rel(host(head.G[0]), x.T @ ((d @ w2.T) * L.act_slope(z, L.GELU))) <= 0.05


def test_loss_falls(env):
    from examples.train_head import Head, data
    torch, B, dev, h = env
    say("train head steps")
    head = Head(h, 128, 256, 200, 2048, dev)
    batches = [data(2048, 128, 200, dev, s) for s in range(2)]
    losses = [float(head.step(*batches[i % 2])) for i in range(24)]
    assert all(np.isfinite(losses))
    assert losses[-1] < 0.7 * losses[0], losses
