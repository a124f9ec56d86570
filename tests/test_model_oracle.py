"""The 64-bit oracle of the layers around the step against autograd, central
differences and published values of the generator.  No GPU is used."""
import numpy as np
import pytest
import torch

import oracle.model_oracle as M


def _central(f, x, g, step=1e-6):
    """d(sum g f(x)) / dx by central differences."""
    out = torch.zeros_like(x)
    for i in np.ndindex(*x.shape):
        for s in (1, -1):
            y = x.clone()
            y[i] += s * step
            out[i] += s * float((g * f(y)).sum()) / (2 * step)
    return out


def test_vocab_gradient_is_the_difference_quotient():
    """Steps of 1e-6 leave about 1e-10 of rounding and 1e-12 of the third derivative."""
    r = torch.Generator().manual_seed(3)
    X, W = (torch.randn(*s, generator=r, dtype=torch.float64) for s in ((3, 4), (6, 4)))
    t = torch.tensor([2, -1, 6], dtype=torch.int32)  # a target, none, none
    g1, g2 = (torch.randn(3, generator=r, dtype=torch.float64) for _ in range(2))
    _, lse, z = M.vocab_logprobs(X, W, t)
    dz, size = M.vocab_dlogits(z, lse, t, g1, g2)

    def loss(x, w):
        logp, lse, _ = M.vocab_logprobs(x, w, t)
        return g1 * logp + g2 * lse
    one = torch.ones(3, dtype=torch.float64)
    assert torch.allclose(_central(lambda x: loss(x, W), X, one), dz @ W, atol=1e-8)
    assert torch.allclose(_central(lambda w: loss(X, w), W, one), dz.t() @ X, atol=1e-8)
    assert bool((size >= dz.abs() - 1e-15).all())


@pytest.mark.parametrize("kind", range(5))
def test_gated_gradient_is_the_difference_quotient(kind):
    r = torch.Generator().manual_seed(kind)
    X, Wg, Wu, dH = (torch.randn(*s, generator=r, dtype=torch.float64) for s in ((3, 4), (4, 5), (4, 5), (3, 5)))
    _, G, U = M.gated(X, Wg, Wu, kind)
    dG, dU = M.gated_grad(G, U, dH, kind)
    H = lambda x, a, b: M.gated(x, a, b, kind)[0]  # noqa: E731
    assert torch.allclose(_central(lambda x: H(x, Wg, Wu), X, dH), dG @ Wg.t() + dU @ Wu.t(), atol=1e-8)
    assert torch.allclose(_central(lambda w: H(X, w, Wu), Wg, dH), X.t() @ dG, atol=1e-8)
    assert torch.allclose(_central(lambda w: H(X, Wg, w), Wu, dH), X.t() @ dU, atol=1e-8)


def test_philox_known_answers():
    """The generator's published test vectors (10 rounds)."""
    for ctr, key, out in (
            ((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
            ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
            ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0),
             (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))):
        assert tuple(int(x) for x in M.philox(ctr, key)) == out


def test_kept_share():
    """Independent 16-bit draws: the kept share lies within 5 standard deviations."""
    for rate in (0.1, 0.5):
        keep, n = M.kept(500, 1000, rate, 12345, 1 << 40)
        assert abs(keep.mean() - (1 - n / 65536)) <= 5 * np.sqrt(rate * (1 - rate) / keep.size)
