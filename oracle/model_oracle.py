"""64-bit oracle of the layers around the step: log probabilities from the last
activations, the gated feed-forward block, dropout, and their gradients.  Plain
torch in float64 (dropout's generator: numpy, unsigned 64-bit words) from the
definitions in include/shampoo.h; no code shared with the GPU path.  Test
infrastructure."""
import math

import numpy as np
import torch

NONE, RELU, GELU, GELU_TANH, SILU = range(5)


def dense(x):
    return x.detach().to(torch.float64)


# ------------------------------------------------------------------ loss
def vocab_logprobs(X, W, targets=None):
    """(logp, lse, z)."""
    z = dense(X) @ dense(W).t().contiguous()
    lse = torch.logsumexp(z, 1)
    logp = torch.zeros_like(lse)
    if targets is not None:
        t = targets.long()
        rows = torch.nonzero((t >= 0) & (t < W.shape[0]))[:, 0]
        logp[rows] = z[rows, t[rows]] - lse[rows]
    return logp, lse, z


def vocab_dlogits(z, lse, targets=None, g_logp=None, g_lse=None):
    """dz, and the sum of the sizes of its terms."""
    n, v = z.shape
    zero = torch.zeros(n, dtype=torch.float64, device=z.device)
    gl, gs = (zero if g is None else dense(g) for g in (g_logp, g_lse))
    has = torch.zeros(n, dtype=torch.bool, device=z.device)
    if targets is not None:
        t = targets.long()
        has = (t >= 0) & (t < v)
    gl = torch.where(has, gl, zero)
    p = torch.exp(z - dense(lse).unsqueeze(1))
    dz, size = p * (gs - gl).unsqueeze(1), p * (gs - gl).abs().unsqueeze(1)
    rows = torch.nonzero(has)[:, 0]
    if len(rows):
        dz[rows, t[rows]] += gl[rows]
        size[rows, t[rows]] += gl[rows].abs()
    return dz, size


# ------------------------------------------------------------------ feed-forward block
def act(x, kind):
    if kind == RELU:
        return torch.clamp(x, min=0)
    if kind == GELU:
        return 0.5 * x * torch.erfc(-x / math.sqrt(2))
    if kind == GELU_TANH:
        return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))
    if kind == SILU:
        return x * torch.sigmoid(x)
    return x.clone()


def slope(x, kind):
    if kind == RELU:
        return (x > 0).to(x.dtype)
    if kind == GELU:
        return 0.5 * torch.erfc(-x / math.sqrt(2)) + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    if kind == GELU_TANH:
        th = torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3))
        return 0.5 * (1 + th) + 0.5 * x * (1 - th * th) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * x * x)
    if kind == SILU:
        s = torch.sigmoid(x)
        return s * (1 + x * (1 - s))
    return torch.ones_like(x)


def gated(X, Wg, Wu, kind):
    """(H, G, U)."""
    G, U = dense(X) @ dense(Wg), dense(X) @ dense(Wu)
    return act(G, kind) * U, G, U


def gated_grad(G, U, dH, kind):
    """(dG, dU)."""
    return dense(dH) * U * slope(G, kind), dense(dH) * act(G, kind)


# ------------------------------------------------------------------ dropout
def philox(counter, key):
    """Philox 4x32, 10 rounds: counter 4 and key 2 arrays (or numbers) of 32-bit values."""
    lo = np.uint64(0xffffffff)
    c = [np.asarray(x, dtype=np.uint64) for x in counter]
    k = [int(x) for x in key]
    for _ in range(10):
        p, q = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(q >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), q & lo, (p >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p & lo]
        k = [(k[0] + 0x9E3779B9) & 0xffffffff, (k[1] + 0xBB67AE85) & 0xffffffff]
    return c


def kept(rows, cols, rate, seed, offset, first_row=0):
    """Which elements stay (numpy, rows x cols), and n."""
    n = int(np.rint(rate * 65536))
    unit, row = np.meshgrid(np.arange((cols + 7) // 8), np.arange(first_row, first_row + rows))
    c = philox((unit, row, np.full_like(unit, offset & 0xffffffff), np.full_like(unit, offset >> 32)),
               (seed & 0xffffffff, seed >> 32))
    keep = np.empty((rows, unit.shape[1], 8), dtype=bool)
    for j in range(8):
        keep[:, :, j] = (c[j // 2] >> np.uint64(16 * (j % 2)) & np.uint64(0xffff)) >= n
    return keep.reshape(rows, -1)[:, :cols], n


def dropout(X, keep, n, R=None):
    """The values before they are rounded."""
    scale = 65536 / (65536 - n) if n < 65536 else 0.0
    y = torch.where(keep, dense(X) * scale, torch.zeros((), dtype=torch.float64, device=X.device))
    return y if R is None else dense(R) + y
