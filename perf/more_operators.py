"""Performance cases of the operators of a model's own layers around the
optimizer step: the loss straight from the last activations, a gated
feed-forward block, and dropout.

Kinds (one operator each):

* ``vocab``       log probabilities of given tokens, and log-sum-exp, of z = X W^T over a vocabulary (W vocab x dim), z not kept;
* ``vocab_grad``  dX and dW from the gradients of those outputs;
* ``ffn``         h = act(x Wg) * (x Wu), optionally with both projections kept;
* ``ffn_grad``    dx, dWg and dWu from dh, with the projections kept or formed again;
* ``dropout``     y = r + keep * x / (1 - rate), the mask from a counter-based generator.

``own`` selects the library's kernels or the plain torch form of each
operator.  ``listed()`` names the cases, ``draw()`` gives others of the same
ranges.  Sizes are those of the repository's benchmark and tests (hidden size
1024, feed-forward 4096, tables of 32768 rows, a 1000-class head) or generic.

Dropout's mask: Philox 4x32 with 10 rounds (Salmon, Moraes, Dror and Shaw,
"Parallel random numbers: as easy as 1, 2, 3", 2011), key the seed, counter
(column / 8, row, low and high word of the offset); of its four words the 16-bit
half column % 8, low halves first, decides: an element stays if that is at least
n = round(65536 rate), and is then multiplied by 65536 / (65536 - n).
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEV = "cuda"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # Scoring four tokens over a 32768-row table: the table's bytes and latency.
        dict(name="vocab_few", kind="vocab", rows=4, dim=1024, vocab=32768, pad=0, dtype="bf16"),
        # Scoring a batch over a large vocabulary: the logits would be 2 GiB.
        dict(name="vocab_large", kind="vocab", rows=8192, dim=1024, vocab=131072, pad=0, dtype="bf16"),
        # Gradients of a 1000-class head in 32 bits.
        dict(name="vocab_grad_classes", kind="vocab_grad", rows=4096, dim=1024, vocab=1000, pad=0, dtype="fp32",
             g_dtype="fp32", g_lse=False),
        # An odd vocabulary and width, rows in a padded view, 32-bit table gradient, with a log-sum-exp penalty.
        dict(name="vocab_grad_ragged", kind="vocab_grad", rows=1021, dim=333, vocab=50001, pad=3, dtype="bf16",
             g_dtype="fp32", g_lse=True),
        # A training batch over a large vocabulary.
        dict(name="vocab_grad_large", kind="vocab_grad", rows=8192, dim=1024, vocab=131072, pad=0, dtype="bf16",
             g_dtype="bf16", g_lse=False),
        # A feed-forward block on a few tokens: the weights' bytes and latency.
        dict(name="ffn_few", kind="ffn", rows=16, dim=1024, width=4096, pad=0, dtype="bf16", act="silu", kept=False),
        # A training batch through it, projections kept for the backward pass.
        dict(name="ffn_large", kind="ffn", rows=16384, dim=1024, width=4096, pad=0, dtype="bf16", act="silu",
             kept=True),
        # Its backward pass from the kept projections; and one that kept none.
        dict(name="ffn_grad_large", kind="ffn_grad", rows=16384, dim=1024, width=4096, pad=0, dtype="bf16", act="silu",
             kept=True, g_dtype="bf16"),
        dict(name="ffn_grad_ragged", kind="ffn_grad", rows=1003, dim=333, width=1339, pad=5, dtype="fp32", act="gelu",
             kept=False, g_dtype="fp32"),
        # Dropout of a few tokens: latency; of a block's output with the residual; and an odd 32-bit one.
        dict(name="dropout_few", kind="dropout", rows=8, cols=1024, pad=0, dtype="bf16", rate=0.1, residual=True),
        dict(name="dropout_large", kind="dropout", rows=16384, cols=4096, pad=0, dtype="bf16", rate=0.1,
             residual=True),
        dict(name="dropout_ragged", kind="dropout", rows=4099, cols=1339, pad=6, dtype="fp32", rate=0.25,
             residual=False),
    ]


def _size(rng, lo, hi):
    """A size spread over the logarithm of [lo, hi]: half of them 4, 5 or 7
    times a power of two, half odd."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    if rng.random() < 0.5 and v >= 8:
        two = 2 ** int(math.log2(v) - 2)
        v = max(m for m in (4, 5, 7) if m * two <= v or m == 4) * two
    else:
        v = int(v) | 1
    return max(lo, min(hi, v))


def draw(rng):
    kind = rng.choice(["vocab", "vocab_grad", "vocab_grad", "ffn", "ffn_grad", "ffn_grad", "dropout"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    pad = rng.choice([0, 0, 8, rng.randint(1, 31)])
    if kind == "dropout":
        cols = _size(rng, 32, 16384)
        size = 2 if dtype == "bf16" else 4
        rows = max(1, min(_size(rng, 1, 65536), 2 ** 27 // (size * (cols + pad))))
        return dict(kind=kind, rows=rows, cols=cols, pad=pad, dtype=dtype, rate=rng.choice([0.05, 0.1, 0.3, 0.5]),
                    residual=rng.random() < 0.5)
    dim = _size(rng, 64, 4096)
    g_dtype = "fp32" if dtype == "fp32" else rng.choice(["bf16", "fp32"])
    if kind in ("vocab", "vocab_grad"):
        vocab = _size(rng, 1000, 131072)
        rows = max(1, min(_size(rng, 1, 8192), (2 ** 39 if dtype == "bf16" else 2 ** 36) // (dim * vocab)))
        c = dict(kind=kind, rows=rows, dim=dim, vocab=vocab, pad=pad, dtype=dtype)
        if kind == "vocab_grad":
            c.update(g_dtype=g_dtype, g_lse=rng.random() < 0.5)
        return c
    width = _size(rng, 64, 16384)
    rows = max(1, min(_size(rng, 1, 65536), (2 ** 36 if dtype == "bf16" else 2 ** 34) // (dim * width)))
    c = dict(kind=kind, rows=rows, dim=dim, width=width, pad=pad, dtype=dtype,
             act=rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu", "silu"]), kept=rng.random() < 0.5)
    if kind == "ffn_grad":
        c["g_dtype"] = g_dtype
        # relu's slope jumps at 0: on which side a projection lies there may
        # hang on its last bit, so it is given
        c["kept"] = c["kept"] or c["act"] == "relu"
    return c


# ------------------------------------------------------------------ inputs
def _view(x, pad):
    """x as a view of rows that are pad elements longer."""
    if not pad:
        return x.contiguous()
    big = torch.zeros(x.shape[0], x.shape[1] + pad, device=x.device, dtype=x.dtype)
    big[:, :x.shape[1]] = x
    return big[:, :x.shape[1]]


def _empty(rows, cols, pad, dtype):
    return torch.empty(rows, cols + pad, device=DEV, dtype=dtype)[:, :cols]


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV)


_handle = None


def _lib():
    """The binding and this process's handle."""
    global _handle
    import paper_2002_09018_amd.binding as shp
    if _handle is None:
        _handle = shp.shampoo_create(torch.cuda.current_device())
    return shp, _handle


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    st = dict(case=case)
    kind, rows, pad, dt = case["kind"], case["rows"], case["pad"], TYPES[case["dtype"]]
    if kind in ("vocab", "vocab_grad"):
        # a partly trained model: logits N(0, 4), the target's a few units above
        # the rest in most rows
        dim, vocab = case["dim"], case["vocab"]
        w = _normal(gen, vocab, dim) * (2 / math.sqrt(dim))
        t = torch.randint(0, vocab, (rows,), generator=gen, device=DEV)
        wt = w[t]
        lift = (6.0 + 3.0 * _normal(gen, rows)) / (wt * wt).sum(1)
        st["x"] = _view((_normal(gen, rows, dim) + lift.unsqueeze(1) * wt).to(dt), pad)
        st["w"] = _view(w.to(dt), pad)
        t[torch.rand(rows, generator=gen, device=DEV) < 0.1] = -1  # prompt tokens: no loss
        st["t"] = t.to(torch.int32)
        st["lse"] = torch.empty(rows, device=DEV)
        if kind == "vocab":
            st["logp"] = torch.empty(rows, device=DEV)
        else:
            st["lse"].copy_(torch.logsumexp(torch.matmul(st["x"].float(), st["w"].float().t()), 1))
            st["g_logp"] = _normal(gen, rows) / rows
            st["g_lse"] = 2e-2 * st["lse"] / rows if case["g_lse"] else None
            st["dx"] = _empty(rows, dim, pad, dt)
            st["dw"] = torch.empty(vocab, dim, device=DEV, dtype=TYPES[case["g_dtype"]])
    elif kind in ("ffn", "ffn_grad"):
        # activations with a few large channels, as transformers have
        dim, width = case["dim"], case["width"]
        x = _normal(gen, rows, dim) * torch.exp(0.5 * _normal(gen, dim))
        st["x"] = _view(x.to(dt), pad)
        st["wg"], st["wu"] = (_view((_normal(gen, dim, width) / math.sqrt(dim)).to(dt), pad) for _ in range(2))
        st["g"] = st["u"] = None
        if case["kept"]:
            st["g"], st["u"] = _empty(rows, width, pad, dt), _empty(rows, width, pad, dt)
        if kind == "ffn":
            st["h"] = _empty(rows, width, pad, dt)
        else:
            if case["kept"]:
                st["g"].copy_(torch.matmul(st["x"].float(), st["wg"].float()))
                st["u"].copy_(torch.matmul(st["x"].float(), st["wu"].float()))
            st["dh"] = _view((_normal(gen, rows, width) / rows).to(dt), pad)
            st["dx"] = _empty(rows, dim, pad, dt)
            st["dwg"], st["dwu"] = (torch.empty(dim, width, device=DEV, dtype=TYPES[case["g_dtype"]]) for _ in range(2))
    else:
        cols = case["cols"]
        st["x"] = _view(_normal(gen, rows, cols).to(dt), pad)
        st["r"] = _view(_normal(gen, rows, cols).to(dt), pad) if case["residual"] else None
        st["y"] = _empty(rows, cols, pad, dt)
        st["seed"], st["offset"] = 0x9A3C5E7100000000 + seed, 5 * 2 ** 32 + 7 * seed
    if own:
        shp, _ = _lib()
        st["act"] = {"none": shp.ACT_NONE, "relu": shp.ACT_RELU, "gelu": shp.ACT_GELU, "gelu_tanh": shp.ACT_GELU_TANH,
                     "silu": shp.ACT_SILU}.get(case.get("act"))
        g = TYPES[case["g_dtype"]] if "g_dtype" in case else None
        nws = 0
        if kind == "vocab":
            nws = shp.shampoo_vocab_logprobs_workspace_bytes(rows, case["dim"], case["vocab"], dt)
        elif kind == "vocab_grad":
            nws = shp.shampoo_vocab_logprobs_grad_workspace_bytes(rows, case["dim"], case["vocab"], dt, g)
        elif kind == "ffn":
            nws = shp.shampoo_gated_ffn_workspace_bytes(rows, case["dim"], case["width"], dt)
        elif kind == "ffn_grad":
            nws = shp.shampoo_gated_ffn_grad_workspace_bytes(rows, case["dim"], case["width"], dt, g)
        st["ws"] = torch.empty(nws, device=DEV, dtype=torch.uint8) if nws else None
    return st


# ------------------------------------------------------------------ one pass
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(st):
    shp, h = _lib()
    kind = st["case"]["kind"]
    if kind == "vocab":
        shp.shampoo_vocab_logprobs(h, st["x"], st["w"], st["t"], st["logp"], st["lse"], workspace=st["ws"])
        return [st["logp"], st["lse"]]
    if kind == "vocab_grad":
        shp.shampoo_vocab_logprobs_grad(h, st["x"], st["w"], st["t"], st["lse"], dX=st["dx"], dW=st["dw"],
                                        g_logp=st["g_logp"], g_lse=st["g_lse"], workspace=st["ws"])
        return [st["dx"], st["dw"]]
    if kind == "ffn":
        shp.shampoo_gated_ffn(h, st["x"], st["wg"], st["wu"], st["h"], act=st["act"], G=st["g"], U=st["u"],
                              workspace=st["ws"])
        return [st["h"], st["g"], st["u"]] if st["g"] is not None else [st["h"]]
    if kind == "ffn_grad":
        shp.shampoo_gated_ffn_grad(h, st["x"], st["wg"], st["wu"], st["dh"], act=st["act"], G=st["g"], U=st["u"],
                                   dX=st["dx"], dWg=st["dwg"], dWu=st["dwu"], workspace=st["ws"])
        return [st["dx"], st["dwg"], st["dwu"]]
    shp.shampoo_dropout(h, st["x"], st["y"], st["case"]["rate"], st["seed"], offset=st["offset"], R=st["r"])
    return [st["y"]]


def _act32(x, act):
    if act == "relu":
        return torch.clamp(x, min=0)
    if act == "gelu":
        return 0.5 * x * (1 + torch.erf(x * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return x / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x * x * x)))
    if act == "silu":
        return x / (1 + torch.exp(-x))
    return x


def _dact32(x, act):
    if act == "relu":
        return (x > 0).float()
    if act == "gelu":
        return 0.5 * (1 + torch.erf(x * math.sqrt(0.5))) + x * torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        c = 2 * math.sqrt(2 / math.pi)
        p = 1 / (1 + torch.exp(-c * (x + 0.044715 * x * x * x)))
        return p + x * p * (1 - p) * c * (1 + 3 * 0.044715 * x * x)
    if act == "silu":
        p = 1 / (1 + torch.exp(-x))
        return p + x * p * (1 - p)
    return torch.ones_like(x)


def _low32(x):
    return x & 0xffffffff


def _philox_halves(seed, offset, rows, cols):
    """The 16-bit numbers that decide a rows x cols tensor.  Words are held in 64
    bits; a product's wrap past 2^63 leaves the bits that are taken."""
    unit = torch.arange(-(-cols // 8), device=DEV)
    row = torch.arange(rows, device=DEV).unsqueeze(1)
    c0, c1 = unit + 0 * row, row + 0 * unit
    c2, c3 = torch.full_like(c0, offset & 0xffffffff), torch.full_like(c0, offset >> 32)
    k0, k1 = seed & 0xffffffff, seed >> 32
    for _ in range(10):  # the generator's rounds
        p, q = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = _low32(q >> 32) ^ c1 ^ k0, _low32(q), _low32(p >> 32) ^ c3 ^ k1, _low32(p)
        k0, k1 = (k0 + 0x9E3779B9) & 0xffffffff, (k1 + 0xBB67AE85) & 0xffffffff
    words = torch.stack([c0, c1, c2, c3], 2)
    return torch.stack([words & 0xffff, words >> 16], 3).reshape(rows, -1)[:, :cols]


def _run_plain(st):
    case = st["case"]
    kind, dt = case["kind"], st["x"].dtype
    if kind in ("vocab", "vocab_grad"):
        x, w, t = st["x"].float(), st["w"].float(), st["t"].long()
        z = torch.matmul(x, w.t())
        has, at = t >= 0, t.clamp(min=0).unsqueeze(1)
        if kind == "vocab":
            m = z.amax(1, keepdim=True)
            ls = torch.log(torch.exp(z - m).sum(1))
            logp = (torch.gather(z, 1, at) - m)[:, 0] - ls
            return [torch.where(has, logp, torch.zeros_like(logp)), m[:, 0] + ls]
        g = torch.where(has, st["g_logp"], torch.zeros_like(st["g_logp"]))
        c = -g if st["g_lse"] is None else st["g_lse"] - g
        dz = torch.exp(z - st["lse"].unsqueeze(1)) * c.unsqueeze(1)
        dz.scatter_add_(1, at, g.unsqueeze(1))
        return [torch.matmul(dz, w).to(dt), torch.matmul(dz.t(), x).to(st["dw"].dtype)]
    if kind in ("ffn", "ffn_grad"):
        x, wg, wu, act = st["x"].float(), st["wg"].float(), st["wu"].float(), case["act"]
        if kind == "ffn":
            g, u = torch.matmul(x, wg), torch.matmul(x, wu)
            out = [(_act32(g, act) * u).to(dt)]
            return out + [g.to(dt), u.to(dt)] if case["kept"] else out
        if case["kept"]:
            g, u = st["g"].float(), st["u"].float()
        else:
            g, u = torch.matmul(x, wg), torch.matmul(x, wu)
        dh = st["dh"].float()
        dg, du = dh * u * _dact32(g, act), dh * _act32(g, act)
        gt = st["dwg"].dtype
        return [(torch.matmul(dg, wg.t()) + torch.matmul(du, wu.t())).to(dt), torch.matmul(x.t(), dg).to(gt),
                torch.matmul(x.t(), du).to(gt)]
    n = int(round(case["rate"] * 65536))
    keep = _philox_halves(st["seed"], st["offset"], case["rows"], case["cols"]) >= n
    y = torch.where(keep, st["x"].float() * (65536.0 / (65536 - n)), torch.zeros(1, device=DEV))
    return [(y if st["r"] is None else st["r"].float() + y).to(dt)]


# ------------------------------------------------------------------ work
def work(case):
    rows = case["rows"]
    b = 2 if case["dtype"] == "bf16" else 4
    gb = 2 if case.get("g_dtype") == "bf16" else 4
    if case["kind"] in ("vocab", "vocab_grad"):
        x, w = rows * case["dim"], case["vocab"] * case["dim"]
        if case["kind"] == "vocab":
            return dict(bytes=(x + w) * b + 12 * rows, flops=2 * x * case["vocab"])
        # the logits once more, since none are kept, and two products with their gradient
        return dict(bytes=(2 * x + w) * b + w * gb + 12 * rows, flops=6 * x * case["vocab"])
    if case["kind"] in ("ffn", "ffn_grad"):
        x, w, h = rows * case["dim"], 2 * case["dim"] * case["width"], rows * case["width"]
        if case["kind"] == "ffn":
            return dict(bytes=(x + w + (3 if case["kept"] else 1) * h) * b, flops=2 * rows * w)
        return dict(bytes=(2 * x + w + (3 if case["kept"] else 1) * h) * b + w * gb,
                    flops=(4 if case["kept"] else 6) * rows * w)
    n = rows * case["cols"]
    return dict(bytes=(3 if case["residual"] else 2) * n * b, flops=2 * n)


# ------------------------------------------------------------------ 64 bits
def _value64(x, act):
    if act == "relu":
        return torch.where(x > 0, x, torch.zeros_like(x))
    if act == "gelu":
        return x * 0.5 * torch.erfc(-x / math.sqrt(2.0))
    if act == "gelu_tanh":
        return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))
    return x * torch.sigmoid(x) if act == "silu" else x.clone()


def _slope64(x, act):
    if act == "relu":
        return torch.where(x > 0, torch.ones_like(x), torch.zeros_like(x))
    if act == "gelu":
        return 0.5 * torch.erfc(-x / math.sqrt(2.0)) + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        th = torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3))
        return 0.5 * (1 + th) + 0.5 * x * (1 - th * th) * math.sqrt(2 / math.pi) * (1 + 0.134145 * x * x)
    if act == "silu":
        sg = torch.sigmoid(x)
        return sg * (1 + x * (1 - sg))
    return torch.ones_like(x)


def _kept64(seed, offset, rows, cols, n):
    """Which elements stay, on the host in unsigned 64-bit words."""
    lo = np.uint64(0xffffffff)
    unit, row = np.meshgrid(np.arange((cols + 7) // 8, dtype=np.uint64), np.arange(rows, dtype=np.uint64))
    ctr = [unit, row, np.full_like(unit, offset & 0xffffffff), np.full_like(unit, offset >> 32)]
    for i in range(10):
        key = [np.uint64(((seed >> 32 * j & 0xffffffff) + i * step & 0xffffffff))
               for j, step in enumerate((0x9E3779B9, 0xBB67AE85))]
        a = np.uint64(0xD2511F53) * ctr[0]
        b = np.uint64(0xCD9E8D57) * ctr[2]
        ctr = [(b >> np.uint64(32)) ^ ctr[1] ^ key[0], b & lo, (a >> np.uint64(32)) ^ ctr[3] ^ key[1], a & lo]
    keep = np.empty((rows, unit.shape[1], 8), dtype=bool)
    for j in range(8):
        keep[:, :, j] = (ctr[j // 2] >> np.uint64(16 * (j % 2)) & np.uint64(0xffff)) >= n
    return torch.from_numpy(keep.reshape(rows, -1)[:, :cols]).to(DEV)


def exact(case, seed):
    st = prepare(case, seed)
    kind, rows = case["kind"], case["rows"]
    x = st["x"].double()
    if kind in ("vocab", "vocab_grad"):
        w = st["w"].double()
        step = max(1, 2 ** 28 // case["vocab"])
        parts, dw = [], torch.zeros_like(w) if kind == "vocab_grad" else None
        for r in range(0, rows, step):
            xs, t = x[r:r + step], st["t"][r:r + step].long()
            lp = torch.matmul(xs, w.t())
            on = torch.nonzero(t >= 0)[:, 0]
            if kind == "vocab":
                lse = torch.logsumexp(lp, 1)
                out = torch.zeros_like(lse)
                out[on] = lp[on, t[on]] - lse[on]
                parts.append((out, lse))
                continue
            # each output's own gradient, added up
            p = lp.sub_(st["lse"][r:r + step].double().unsqueeze(1)).exp_()
            gl = torch.zeros(xs.shape[0], device=DEV, dtype=torch.float64)
            gl[on] = st["g_logp"][r:r + step].double()[on]
            total = -gl
            if st["g_lse"] is not None:
                total = total + st["g_lse"][r:r + step].double()
            p.mul_(total.unsqueeze(1))
            p[on, t[on]] += gl[on]
            parts.append((torch.matmul(p, w),))
            dw += torch.matmul(p.t(), xs)
        cat = [torch.cat([p[i] for p in parts]) for i in range(len(parts[0]))]
        return cat if dw is None else cat + [dw]
    if kind in ("ffn", "ffn_grad"):
        wg, wu, act = st["wg"].double(), st["wu"].double(), case["act"]
        if kind == "ffn_grad" and case["kept"]:
            g, u = st["g"].double(), st["u"].double()
        else:
            g, u = torch.matmul(x, wg), torch.matmul(x, wu)
        if kind == "ffn":
            return [_value64(g, act) * u] + ([g, u] if case["kept"] else [])
        dh = st["dh"].double()
        dg, du = _slope64(g, act) * u * dh, _value64(g, act) * dh
        both = torch.matmul(torch.cat([dg, du], 1), torch.cat([wg, wu], 1).t())
        return [both, torch.matmul(x.t(), dg), torch.matmul(x.t(), du)]
    n = int(round(case["rate"] * 65536))
    keep = _kept64(st["seed"], st["offset"], rows, case["cols"], n)
    y = torch.where(keep, x / (1 - n / 65536), torch.zeros_like(x))
    return [y if st["r"] is None else st["r"].double() + y]
