"""Performance cases of the operators around the optimizer step: from a
layer's activations and the loss to the gradient that the optimizer takes.

Kinds (one operator each):

* ``logprobs``   log probabilities of given tokens from logits, with log-sum-exp, entropy and the k largest alternatives;
* ``loss_grad``  the gradient of those outputs with respect to the logits;
* ``store``      y = act(x) with an 8-bit checkpoint of x (with ``both``, also of y), and the values that they hold;
* ``act_grad``   dx = dy act'(x) from the checkpoint of x;
* ``weight_grad``  G = X^T dY from the checkpoint of X.

``own`` selects the library's kernels or the plain torch form of each
operator.  ``listed()`` names the cases, ``draw()`` gives others of the same
ranges.  Sizes are those of the repository's benchmark and tests (hidden size
1024, feed-forward 4096, tables of 32768 rows, a 1000-class head, 65536
lookups) or generic.

A checkpoint of a rows x cols tensor is one byte buffer: rows x ldq signed
codes, ldq = cols rounded up to 32, then at the next multiple of 256 bytes
rows x (ldq / 32) scale bytes s, one for 32 columns of a row; a code q stands
for q 2^(s - 127), s = 255 for NaN.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
GROUP = 32


def listed():
    return [
        # Scoring one token over a 32768-row table: latency counts.
        dict(name="logprobs_token", kind="logprobs", rows=1, vocab=32768, pad=0, dtype="bf16", k=8, mask="none"),
        # A 1000-class head with its five best classes, logits in 32 bits.
        dict(name="logprobs_classes", kind="logprobs", rows=4096, vocab=1000, pad=0, dtype="fp32", k=5, mask="none"),
        # Scoring a batch over a large vocabulary whose last columns are padding.
        dict(name="logprobs_large", kind="logprobs", rows=8192, vocab=131072, pad=0, dtype="bf16", k=8, mask="pad"),
        # Loss gradient over a vocabulary of odd size, rows packed without
        # padding (no row but the first is aligned), masked entries, some rows
        # fully masked.
        dict(name="loss_grad_ragged", kind="loss_grad", rows=1021, vocab=50001, pad=0, dtype="bf16", k=0, mask="rows",
             entropy=False),
        # Loss gradient of a large batch, with the entropy's and the
        # alternatives' gradients.
        dict(name="loss_grad_large", kind="loss_grad", rows=8192, vocab=131072, pad=0, dtype="bf16", k=8, mask="none",
             entropy=True),
        # Activation and checkpoint of a few tokens: latency counts.
        dict(name="store_few", kind="store", rows=8, cols=4096, pad=0, dtype="bf16", act="gelu", both=False),
        # Activation of a feed-forward layer's batch, with the checkpoints of its
        # input (for the activation's gradient) and output (for the next layer's
        # weight gradient).
        dict(name="store_ffn", kind="store", rows=16384, cols=4096, pad=0, dtype="bf16", act="relu", both=True),
        # Activation gradients: the feed-forward batch, and an odd 32-bit one in
        # a padded view.
        dict(name="act_grad_ffn", kind="act_grad", rows=16384, cols=4096, pad=0, dtype="bf16", act="gelu"),
        dict(name="act_grad_ragged", kind="act_grad", rows=4099, cols=1339, pad=6, dtype="fp32", act="silu"),
        # Weight gradients: a feed-forward layer over 65536 tokens; a small
        # square layer over many tokens (few output tiles, long sums); odd sizes
        # with 32-bit gradients.
        dict(name="weight_grad_ffn", kind="weight_grad", rows=65536, cols=1024, out=4096, pad=0, dtype="bf16",
             g_dtype="fp32"),
        dict(name="weight_grad_square", kind="weight_grad", rows=32768, cols=512, out=512, pad=0, dtype="bf16",
             g_dtype="bf16"),
        dict(name="weight_grad_ragged", kind="weight_grad", rows=4097, cols=333, out=517, pad=3, dtype="fp32",
             g_dtype="fp32"),
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
    kind = rng.choice(["logprobs", "logprobs", "loss_grad", "loss_grad", "store", "act_grad", "weight_grad",
                       "weight_grad"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    pad = rng.choice([0, 0, 8, rng.randint(1, 31)])
    size = 2 if dtype == "bf16" else 4
    if kind in ("logprobs", "loss_grad"):
        vocab = _size(rng, 1000, 131072)
        rows = max(1, min(_size(rng, 1, 8192), 2 ** 31 // (size * (vocab + pad))))
        c = dict(kind=kind, rows=rows, vocab=vocab, pad=pad, dtype=dtype, k=rng.choice([0, 1, 4, 8, 8, 16, 32]),
                 mask=rng.choice(["none", "pad", "rows"]))
        if kind == "loss_grad":
            c["entropy"] = rng.random() < 0.5
        return c
    if kind in ("store", "act_grad"):
        cols = _size(rng, 32, 16384)
        rows = max(1, min(_size(rng, 1, 65536), 2 ** 27 // (size * (cols + pad))))
        c = dict(kind=kind, rows=rows, cols=cols, pad=pad, dtype=dtype)
        if kind == "act_grad":
            c["act"] = rng.choice(["relu", "gelu", "gelu_tanh", "silu"])
        else:
            # both checkpoints where y is exact: elsewhere the codes of y follow
            # the last bit of its rounding
            c["act"] = rng.choice(["none", "relu", "relu", "gelu", "gelu_tanh", "silu"])
            c["both"] = c["act"] == "relu" and rng.random() < 0.5
        return c
    cols, out = _size(rng, 64, 4096), _size(rng, 64, 4096)
    rows = max(1, min(_size(rng, 1, 65536), 2 ** 38 // (cols * out)))
    return dict(kind=kind, rows=rows, cols=cols, out=out, pad=pad, dtype=dtype, g_dtype=rng.choice(["fp32", "bf16"]))


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


def _logits(case, gen):
    """Logits of a partly trained model: N(0, 4) with the target a few units
    above the rest in most rows, and the case's mask."""
    n, v = case["rows"], case["vocab"]
    dt = TYPES[case["dtype"]]
    z = _empty(n, v, case["pad"], dt)
    t = torch.randint(0, v, (n,), generator=gen, device=DEV)
    lift = 6.0 + 3.0 * torch.randn(n, generator=gen, device=DEV)
    step = max(1, 2 ** 28 // v)  # rows at a time
    for r in range(0, n, step):
        x = 2.0 * torch.randn(min(step, n - r), v, generator=gen, device=DEV)
        x[torch.arange(x.shape[0], device=DEV), t[r:r + step]] += lift[r:r + step]
        if case["mask"] == "rows":  # a third of the entries is not allowed
            x[torch.rand(x.shape, generator=gen, device=DEV) < 0.33] = -math.inf
        z[r:r + step] = x.to(dt)
    if case["mask"] == "pad":
        z[:, v - v // 64:] = -math.inf
    if case["mask"] == "rows":
        z[torch.rand(n, generator=gen, device=DEV) < 0.02] = -math.inf
    t[torch.rand(n, generator=gen, device=DEV) < 0.1] = -1  # prompt tokens: no loss
    return z, t.to(torch.int32)


def _activations(rows, cols, gen):
    """Activations with a few large channels, as transformers have."""
    x = torch.randn(rows, cols, generator=gen, device=DEV)
    x *= torch.exp(0.7 * torch.randn(cols, generator=gen, device=DEV))
    big = torch.randint(0, cols, (max(1, cols // 500),), generator=gen, device=DEV)
    x[:, big] *= 20.0
    return x


def _ldq(cols):
    return -(-cols // GROUP) * GROUP


def _ckpt_parts(buf, rows, cols):
    """(codes rows x ldq, scale bytes rows x ldq / 32) of a checkpoint buffer."""
    ldq = _ldq(cols)
    off = -(-rows * ldq // 256) * 256
    return (buf[:rows * ldq].view(torch.int8).view(rows, ldq),
            buf[off:off + rows * (ldq // GROUP)].view(rows, ldq // GROUP))


def _ckpt_bytes(rows, cols):
    ldq = _ldq(cols)
    return -(-rows * ldq // 256) * 256 + -(-rows * (ldq // GROUP) // 256) * 256


def _codes(x):
    """(codes, scale bytes) of x in 32 bits: the smallest power of two whose
    multiples up to 127 reach the group's largest value after rounding."""
    rows, cols = x.shape
    g = torch.zeros(rows, _ldq(cols), device=x.device)
    g[:, :cols] = x
    g = g.view(rows, -1, GROUP)
    bits = g.abs().amax(2).view(torch.int32)
    s = (((bits + 0x10000) >> 23) - 6).clamp(min=1, max=248)  # 2^121 the largest: 128 of it would overflow
    q = torch.round(g / (s << 23).view(torch.float32).unsqueeze(2)).clamp(-127, 127)
    return q.view(rows, -1), s


def _values(buf, rows, cols):
    q, s = _ckpt_parts(buf, rows, cols)
    scale = (s.int() << 23).view(torch.float32)
    return (q.view(rows, -1, GROUP).float() * scale.unsqueeze(2)).view(rows, -1)[:, :cols]


def _checkpoint(x):
    """The checkpoint buffer of x."""
    rows, cols = x.shape
    buf = torch.zeros(_ckpt_bytes(rows, cols), device=DEV, dtype=torch.uint8)
    q, s = _codes(x)
    cq, cs = _ckpt_parts(buf, rows, cols)
    cq.copy_(q.to(torch.int8))
    cs.copy_(s.to(torch.uint8))
    return buf


def _stats32(z):
    """Row statistics in 32 bits: largest logit (0 for a row without any), sum
    of exponentials, log-sum-exp and entropy."""
    m = z.amax(1, keepdim=True)
    m = torch.where(torch.isfinite(m), m, torch.zeros_like(m))
    d = z - m
    e = torch.exp(d)
    s = e.sum(1, keepdim=True)
    some = s > 0
    ls = torch.log(s)
    ent = torch.where(some, ls - (torch.where(e > 0, d, torch.zeros_like(d)) * e).sum(1, keepdim=True) / s,
                      torch.zeros_like(s))
    return m, ls, m + ls, ent


def _top32(z, k):
    """The k largest entries by value, then lowest index; -1 where fewer than k
    are allowed.  Keys hold the value's order above the index."""
    b = z.view(torch.int32).long()
    b = torch.where(b < 0, -(b & 0x7fffffff), b)  # -0 orders with 0
    key = (b << 32) - torch.arange(z.shape[1], device=z.device)
    ids = torch.topk(key, min(k, z.shape[1]), dim=1).values
    ids = (-ids) & 0xffffffff
    val = torch.gather(z, 1, ids)
    ok = val > -math.inf
    out_i = torch.full((z.shape[0], k), -1, device=z.device, dtype=torch.int32)
    out_v = torch.full((z.shape[0], k), -math.inf, device=z.device)
    out_i[:, :ids.shape[1]] = torch.where(ok, ids, torch.full_like(ids, -1)).to(torch.int32)
    out_v[:, :ids.shape[1]] = val
    return out_i, out_v


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
    dt = TYPES[case["dtype"]]
    kind, rows = case["kind"], case["rows"]
    if kind == "logprobs":
        z, t = _logits(case, gen)
        k = case["k"]
        st.update(z=z, t=t, logp=torch.empty(rows, device=DEV), lse=torch.empty(rows, device=DEV),
                  ent=torch.empty(rows, device=DEV), ids=None, top=None, ws=None)
        if k:
            st.update(ids=torch.empty(rows, k, device=DEV, dtype=torch.int32), top=torch.empty(rows, k, device=DEV))
    elif kind == "loss_grad":
        z, t = _logits(case, gen)
        k, v = case["k"], case["vocab"]
        st.update(z=z, t=t, lse=torch.empty(rows, device=DEV), ent=torch.empty(rows, device=DEV), ids=None, g_top=None)
        if k:
            st["ids"] = torch.empty(rows, k, device=DEV, dtype=torch.int32)
            st["g_top"] = torch.randn(rows, k, generator=gen, device=DEV) / rows
        step = max(1, 2 ** 27 // v)
        for r in range(0, rows, step):
            x = z[r:r + step].float()
            _, _, lse, ent = _stats32(x)
            st["lse"][r:r + step] = lse[:, 0]
            st["ent"][r:r + step] = ent[:, 0]
            if k:
                st["ids"][r:r + step] = _top32(x, k)[0]
        st["g_logp"] = torch.randn(rows, generator=gen, device=DEV) / rows
        st["g_ent"] = 0.01 * torch.ones(rows, device=DEV) / rows if case["entropy"] else None
        st["dz"] = _empty(rows, v, case["pad"], dt)
    elif kind == "store":
        cols = case["cols"]
        st["x"] = _view(_activations(rows, cols, gen).to(dt), case["pad"])
        both = case["both"]
        st["cy"] = None
        for name in ("y", "vx", "vy") if both else ("y", "vx"):
            st[name] = _empty(rows, cols, case["pad"], dt)
        for name in ("cx", "cy") if both else ("cx",):
            st[name] = torch.empty(_ckpt_bytes(rows, cols), device=DEV, dtype=torch.uint8)
    elif kind == "act_grad":
        cols = case["cols"]
        st["cx"] = _checkpoint(_activations(rows, cols, gen).to(dt).float())
        st["dy"] = _view((torch.randn(rows, cols, generator=gen, device=DEV) / rows).to(dt), case["pad"])
        st["dx"] = _empty(rows, cols, case["pad"], dt)
    else:
        cols, out = case["cols"], case["out"]
        st["cx"] = _checkpoint(_activations(rows, cols, gen).to(dt).float())
        st["dy"] = _view((torch.randn(rows, out, generator=gen, device=DEV) / rows).to(dt), case["pad"])
        st["G"] = torch.empty(cols, out, device=DEV, dtype=TYPES[case["g_dtype"]])
    if own:
        shp, _ = _lib()
        st["act"] = {"none": shp.ACT_NONE, "relu": shp.ACT_RELU, "gelu": shp.ACT_GELU, "gelu_tanh": shp.ACT_GELU_TANH,
                     "silu": shp.ACT_SILU}.get(case.get("act"))
        nws = 0
        if kind == "logprobs":
            nws = shp.shampoo_token_logprobs_workspace_bytes(rows, case["vocab"], case["k"])
        elif kind == "weight_grad":
            nws = shp.shampoo_act_weight_grad_workspace_bytes(rows, case["cols"], case["out"])
        st["ws"] = torch.empty(nws, device=DEV, dtype=torch.uint8) if nws else None
    return st


# ------------------------------------------------------------------ one pass
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(st):
    shp, h = _lib()
    kind = st["case"]["kind"]
    if kind == "logprobs":
        shp.shampoo_token_logprobs(h, st["z"], st["t"], st["logp"], st["lse"], entropy=st["ent"], top_ids=st["ids"],
                                   top_logp=st["top"], workspace=st["ws"])
        out = [st["logp"], st["lse"], st["ent"]]
        return out + [st["ids"], st["top"]] if st["ids"] is not None else out
    if kind == "loss_grad":
        shp.shampoo_token_logprobs_grad(h, st["z"], st["t"], st["lse"], st["dz"], g_logp=st["g_logp"],
                                        entropy=st["ent"], g_entropy=st["g_ent"], top_ids=st["ids"],
                                        g_top=st["g_top"])
        return [st["dz"]]
    if kind == "store":
        shp.shampoo_act_encode(h, st["x"], ckpt_x=st["cx"], act=st["act"], Y=st["y"], ckpt_y=st["cy"])
        shp.shampoo_act_decode(h, st["cx"], st["vx"])
        if st["cy"] is None:
            return [st["y"], st["vx"]]
        shp.shampoo_act_decode(h, st["cy"], st["vy"])
        return [st["y"], st["vx"], st["vy"]]
    if kind == "act_grad":
        shp.shampoo_act_grad(h, st["cx"], st["act"], st["dy"], st["dx"])
        return [st["dx"]]
    shp.shampoo_act_weight_grad(h, st["cx"], st["dy"], st["G"], workspace=st["ws"])
    return [st["G"]]


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
    p = 1 / (1 + torch.exp(-x))
    return p + x * p * (1 - p)


def _run_plain(st):
    case = st["case"]
    kind = case["kind"]
    if kind == "logprobs":
        z = st["z"].float()
        t = st["t"].long()
        m, ls, lse, ent = _stats32(z)
        at = torch.gather(z, 1, t.clamp(min=0).unsqueeze(1))
        logp = torch.where(t >= 0, ((at - m) - ls)[:, 0], torch.zeros_like(lse[:, 0]))
        # a row without any allowed entry has log probability -inf, not NaN
        logp = torch.where((t >= 0) & ~(lse[:, 0] > -math.inf), torch.full_like(logp, -math.inf), logp)
        out = [logp, lse[:, 0], ent[:, 0]]
        if case["k"]:
            ids, top = _top32(z, case["k"])
            out += [ids, torch.where(ids >= 0, (top - m) - ls, torch.full_like(top, -math.inf))]
        return out
    if kind == "loss_grad":
        z, lse = st["z"].float(), st["lse"].unsqueeze(1)
        t, v = st["t"].long(), case["vocab"]
        some = lse > -math.inf
        lp = z - torch.where(some, lse, torch.zeros_like(lse))
        p = torch.exp(lp)
        g = torch.where(t >= 0, st["g_logp"], torch.zeros_like(st["g_logp"])).unsqueeze(1) * some
        total = g
        if case["k"]:
            g_top = torch.where((st["ids"] >= 0) & some, st["g_top"], torch.zeros_like(st["g_top"]))
            total = g + g_top.sum(1, keepdim=True)
        dz = -total * p
        if case["entropy"]:
            dz = dz - st["g_ent"].unsqueeze(1) * p * torch.where(p > 0, lp + st["ent"].unsqueeze(1), torch.zeros_like(p))
        dz.scatter_add_(1, t.clamp(min=0).unsqueeze(1), g)
        if case["k"]:
            dz.scatter_add_(1, st["ids"].long().clamp(min=0), g_top)
        return [dz.to(st["z"].dtype)]
    if kind == "store":
        x = st["x"].float()
        y = _act32(x, case["act"]).to(st["x"].dtype)
        out = [y]
        for a in (x, y.float()) if case["both"] else (x,):
            q, s = _codes(a)
            rows, cols = a.shape
            val = (q.view(rows, -1, GROUP) * (s << 23).view(torch.float32).unsqueeze(2)).view(rows, -1)[:, :cols]
            out.append(val.to(st["x"].dtype))
        return out
    if kind == "act_grad":
        x = _values(st["cx"], case["rows"], case["cols"])
        return [(st["dy"].float() * _dact32(x, case["act"])).to(st["dy"].dtype)]
    x = _values(st["cx"], case["rows"], case["cols"])
    return [torch.matmul(x.t(), st["dy"].float()).to(st["G"].dtype)]


# ------------------------------------------------------------------ work
def work(case):
    rows = case["rows"]
    b = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "logprobs":
        n = rows * case["vocab"]
        return dict(bytes=n * b + rows * (16 + 8 * case["k"]), flops=6 * n)
    if case["kind"] == "loss_grad":
        n = rows * case["vocab"]
        return dict(bytes=2 * n * b + rows * (20 + 8 * case["k"]), flops=(9 if case["entropy"] else 4) * n)
    if case["kind"] == "store":
        # x read, y and the checkpoints written; then the checkpoints read and
        # their values written
        n, c = rows * case["cols"], _ckpt_bytes(rows, case["cols"])
        held = 2 if case["both"] else 1
        return dict(bytes=(2 + held) * n * b + 2 * held * c, flops=10 * n * held + 10 * n)
    if case["kind"] == "act_grad":
        n = rows * case["cols"]
        return dict(bytes=2 * n * b + _ckpt_bytes(rows, case["cols"]), flops=30 * n)
    g = 2 if case["g_dtype"] == "bf16" else 4
    return dict(bytes=_ckpt_bytes(rows, case["cols"]) + rows * case["out"] * b + case["cols"] * case["out"] * g,
                flops=2 * rows * case["cols"] * case["out"])


# ------------------------------------------------------------------ 64 bits
def _decode64(buf, rows, cols):
    width = (cols + 31) // 32 * 32
    start = (rows * width + 255) // 256 * 256
    q = buf[:rows * width].view(torch.int8).reshape(rows, width)[:, :cols].double()
    s = buf[start:start + rows * width // 32].reshape(rows, width // 32).double()
    return q * torch.exp2(s - 127).repeat_interleave(32, 1)[:, :cols]


def _nearest64(a):
    """What the checkpoint of a (rows x cols, 64 bits) holds."""
    rows, cols = a.shape
    pad = torch.nn.functional.pad(a, (0, -cols % 32)).reshape(rows, -1, 32)
    top = pad.abs().amax(2, keepdim=True)
    e = torch.floor(torch.log2(top.clamp(min=2.0 ** -149))) - 6
    e = torch.where(top >= torch.exp2(e) * 128, e + 1, e)  # the logarithm may have rounded across a power of two
    e = torch.where(top < torch.exp2(e) * 64, e - 1, e)
    e = torch.where(top >= torch.exp2(e) * 127.5, e + 1, e).clamp(min=-126, max=121)
    unit = torch.exp2(e)
    return (torch.round(pad / unit).clamp(-127, 127) * unit).reshape(rows, -1)[:, :cols]


def _act64(x, act):
    if act == "relu":
        return torch.where(x > 0, x, torch.zeros_like(x))
    if act == "gelu":
        return x * 0.5 * torch.erfc(-x / math.sqrt(2.0))
    if act == "gelu_tanh":
        return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))
    if act == "silu":
        return x * torch.sigmoid(x)
    return x


def _slope64(x, act):
    if act == "relu":
        return torch.where(x > 0, torch.ones_like(x), torch.zeros_like(x))
    if act == "gelu":
        return 0.5 * torch.erfc(-x / math.sqrt(2.0)) + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        th = torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3))
        return 0.5 * (1 + th) + 0.5 * x * (1 - th * th) * math.sqrt(2 / math.pi) * (1 + 0.134145 * x * x)
    sg = torch.sigmoid(x)
    return sg * (1 + x * (1 - sg))


def exact(case, seed):
    st = prepare(case, seed)
    kind, rows = case["kind"], case["rows"]
    if kind in ("logprobs", "loss_grad"):
        v, k = case["vocab"], case["k"]
        step = max(1, 2 ** 26 // v)
        parts = []
        for r in range(0, rows, step):
            z = st["z"][r:r + step].double()
            t = st["t"][r:r + step].long()
            n = torch.arange(z.shape[0], device=DEV)
            if kind == "logprobs":
                lse = torch.logsumexp(z, 1)
                lp = torch.where(torch.isneginf(z), torch.full_like(z, -math.inf), z - lse.unsqueeze(1))
                ent = -torch.where(torch.isneginf(lp), torch.zeros_like(lp), torch.exp(lp) * lp).sum(1)
                out = [torch.where(t >= 0, lp[n, t.clamp(min=0)], torch.zeros_like(lse)), lse, ent]
                if k:
                    top = torch.full((z.shape[0], k), -math.inf, device=DEV, dtype=torch.float64)
                    top[:, :min(k, v)] = torch.sort(torch.topk(lp, min(k, v), 1).values, 1, descending=True).values
                    out += [top]
            else:
                # the gradient as the sum of each output's own gradient
                lse = st["lse"][r:r + step].double()
                full = ~torch.isneginf(lse)
                p = torch.where(full.unsqueeze(1), torch.exp(z - lse.unsqueeze(1)), torch.zeros_like(z))
                on = (t >= 0) & full
                dz = torch.zeros_like(z)
                gl = st["g_logp"][r:r + step].double()
                dz[n[on], t[on]] += gl[on]
                dz -= torch.where(on, gl, torch.zeros_like(gl)).unsqueeze(1) * p
                if k:
                    for i in range(k):
                        idx = st["ids"][r:r + step, i].long()
                        gi = st["g_top"][r:r + step, i].double()
                        at = (idx >= 0) & full
                        dz[n[at], idx[at]] += gi[at]
                        dz -= torch.where(at, gi, torch.zeros_like(gi)).unsqueeze(1) * p
                if case["entropy"]:
                    h = st["ent"][r:r + step].double()
                    lp = torch.where(p > 0, z - lse.unsqueeze(1), torch.zeros_like(z))
                    dz -= st["g_ent"][r:r + step].double().unsqueeze(1) * p * (lp + h.unsqueeze(1))
                out = [dz]
            parts.append(out)
        cat = [torch.cat([p[i] for p in parts]) for i in range(len(parts[0]))]
        if kind == "logprobs" and k:
            cat.insert(3, None)
        return cat
    if kind == "store":
        x = st["x"].double()
        y = _act64(x, case["act"])
        return [y, _nearest64(x)] + ([_nearest64(y)] if case["both"] else [])
    x = _decode64(st["cx"], rows, case["cols"])
    if kind == "act_grad":
        return [st["dy"].double() * _slope64(x, case["act"])]
    return [torch.matmul(x.t().contiguous(), st["dy"].double())]
