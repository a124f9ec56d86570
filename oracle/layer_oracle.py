"""64-bit oracle of the calls from the loss to the gradient: token log
probabilities and their gradient, 8-bit activation checkpoints, activation
gradients and weight gradients.  Plain numpy/scipy from the definitions in
include/shampoo.h; no code shared with the GPU path.  Test infrastructure."""
import math

import numpy as np
from scipy.special import erfc, expit

NONE, RELU, GELU, GELU_TANH, SILU = range(5)
GROUP = 32


# ------------------------------------------------------------------ loss
def token_logprobs(z, targets, k=0):
    """(logp, lse, entropy, top_ids, top_logp) of logits z (rows x vocab)."""
    z = np.asarray(z, dtype=np.float64)
    n, v = z.shape
    logp, lse, ent = np.zeros(n), np.zeros(n), np.zeros(n)
    ids, top = np.full((n, k), -1, dtype=np.int64), np.full((n, k), -np.inf)
    for r in range(n):
        x = z[r]
        t = None if targets is None else int(targets[r])
        t = t if t is not None and 0 <= t < v else None
        if np.any(np.isnan(x)) or np.any(x == np.inf):
            lse[r] = ent[r] = np.nan
            logp[r] = np.nan if t is not None else 0.0
            top[r] = np.nan
            continue
        allowed = x > -np.inf
        if not np.any(allowed):
            lse[r] = -np.inf
            logp[r] = -np.inf if t is not None else 0.0
            continue
        m = x[allowed].max()
        lse[r] = m + math.log(np.sum(np.exp(x[allowed] - m)))
        ls = math.log(np.sum(np.exp(x[allowed] - m)))
        lp = (x[allowed] - m) - ls
        ent[r] = -np.sum(np.exp(lp) * lp)
        if t is not None:
            logp[r] = (x[t] - m) - ls
        order = np.lexsort((np.arange(v), -x))[:k]
        order = order[x[order] > -np.inf]
        ids[r, :len(order)] = order
        top[r, :len(order)] = (x[order] - m) - ls
    return logp, lse, ent, ids, top


def token_logprobs_grad(z, targets, lse, entropy=None, g_logp=None, g_lse=None, g_entropy=None, top_ids=None,
                        g_top=None):
    """d(outputs . their gradients) / dz, with lse and entropy as given."""
    z = np.asarray(z, dtype=np.float64)
    lse = np.asarray(lse, dtype=np.float64)
    n, v = z.shape
    out = np.zeros((n, v))
    for r in range(n):
        if lse[r] == -np.inf:
            continue
        p = np.exp(z[r] - lse[r])
        if g_lse is not None:
            out[r] += float(g_lse[r]) * p
        picks = []
        if g_logp is not None:
            picks.append((int(targets[r]), float(g_logp[r])))
        if g_top is not None:
            picks += [(int(i), float(g)) for i, g in zip(top_ids[r], g_top[r])]
        for i, g in picks:
            if 0 <= i < v:
                out[r] -= g * p
                out[r, i] += g
        if g_entropy is not None:
            lp = np.where(z[r] > -np.inf, z[r] - lse[r], 0.0) if not np.isnan(lse[r]) else z[r] - lse[r]
            out[r] -= float(g_entropy[r]) * p * (lp + float(entropy[r]))
    return out


# ------------------------------------------------------------------ activations
def act(x, kind):
    x = np.asarray(x, dtype=np.float64)
    if kind == RELU:
        return np.where(x > 0, x, np.where(np.isnan(x), x, 0.0))
    if kind == GELU:
        return 0.5 * x * erfc(-x / math.sqrt(2))
    if kind == GELU_TANH:
        return x * expit(2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3))
    if kind == SILU:
        return x * expit(x)
    return x


def act_slope(x, kind):
    x = np.asarray(x, dtype=np.float64)
    if kind == RELU:
        return np.where(x > 0, 1.0, np.where(np.isnan(x), x, 0.0))
    if kind == GELU:
        return 0.5 * erfc(-x / math.sqrt(2)) + x * np.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)
    if kind == GELU_TANH:
        u = math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)
        return expit(2 * u) + 0.5 * x / np.cosh(np.clip(u, -300, 300)) ** 2 * math.sqrt(2 / math.pi) * (
            1 + 3 * 0.044715 * x * x)
    if kind == SILU:
        s = expit(x)
        return s + x * s * (1 - s)
    return np.ones_like(x)


def checkpoint(x):
    """(codes rows x ldq int8, scale bytes rows x ldq / 32 uint8) of x: for
    each group the smallest exponent whose rounded codes fit, found by trying
    exponents upwards."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    ng = -(-cols // GROUP)
    codes = np.zeros((rows, ng * GROUP), dtype=np.int8)
    scales = np.zeros((rows, ng), dtype=np.uint8)
    for r in range(rows):
        for g in range(ng):
            v = x[r, g * GROUP:(g + 1) * GROUP]
            if not np.all(np.isfinite(v)):
                scales[r, g] = 255
                continue
            top = np.abs(v).max()
            e = -126 if top == 0 else max(-126, math.frexp(top)[1] - 9)
            while e < 121 and np.rint(top / 2.0 ** e) > 127:
                e += 1
            codes[r, g * GROUP:g * GROUP + len(v)] = np.clip(np.rint(v / 2.0 ** e), -127, 127).astype(np.int8)
            scales[r, g] = e + 127
    return codes, scales


def checkpoint_bytes(x):
    """The checkpoint of x as its byte buffer."""
    codes, scales = checkpoint(x)
    off = -(-codes.size // 256) * 256
    buf = np.zeros(off + -(-scales.size // 256) * 256, dtype=np.uint8)
    buf[:codes.size] = codes.reshape(-1).view(np.uint8)
    buf[off:off + scales.size] = scales.reshape(-1)
    return buf


def checkpoint_values(codes, scales, cols):
    e = np.repeat(scales.astype(np.int64), GROUP, axis=1)[:, :cols] - 127
    out = np.ldexp(codes[:, :cols].astype(np.float64), e)
    return np.where(e == 128, np.nan, out)


def weight_grad(values, dy, G=None, beta=0.0):
    out = np.asarray(values, dtype=np.float64).T @ np.asarray(dy, dtype=np.float64)
    return out if beta == 0 else out + beta * np.asarray(G, dtype=np.float64)
