"""ctypes binding of libshampoo.so (the C ABI in include/shampoo.h).

Argument marshalling only: every step of the computation runs in the HIP
kernels behind the C entry points.  Functions carry the C names.  Tensors are
torch tensors on the handle's device (torch is used for device memory and
streams); the binding passes their data pointers and the current stream.
There is no CPU fallback: if the library cannot be loaded, importing this
module raises.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional, Sequence

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("SHAMPOO_LIB", os.path.join(HERE, "libshampoo.so"))

if not os.path.exists(LIB_PATH):
    raise ImportError(f"libshampoo.so not found at {LIB_PATH}: build it with "
                      f"`python -c 'import __graft_entry__ as g; g.build()'`")
_lib = C.CDLL(LIB_PATH)

SHAMPOO_OK, SHAMPOO_EINVAL, SHAMPOO_EUNSUPPORTED, SHAMPOO_EHIP, SHAMPOO_ENOMEM = 0, -1, -2, -3, -4
SHAMPOO_F32, SHAMPOO_BF16 = 0, 1
ROOT_CONVERGED, ROOT_STAGNATED, ROOT_MAXITER, ROOT_DIVERGED, ROOT_NOT_PD = 0, 1, 2, 3, 4
PRECISION_FP32, PRECISION_AUTO, PRECISION_FP64 = 0, 1, 2
SCALING_FROBENIUS, SCALING_POWER4 = 0, 1
(KCLASS_NEWTON_F32, KCLASS_NEWTON_F64, KCLASS_STATS, KCLASS_PRECOND, KCLASS_GRAFT, KCLASS_ROOT_AUX, KCLASS_EMB,
 KCLASS_NEWTON_WARM, KCLASS_LOGPROBS, KCLASS_ACT, KCLASS_WGRAD, KCLASS_VOCAB, KCLASS_FFN,
 KCLASS_DROPOUT) = range(14)
KCLASS_NAMES = ["newton_f32", "newton_f64", "stats", "precond", "graft", "root_aux", "emb", "newton_warm", "logprobs",
                "act", "wgrad", "vocab", "ffn", "dropout"]
ACT_NONE, ACT_RELU, ACT_GELU, ACT_GELU_TANH, ACT_SILU = range(5)
MAX_TOP = 64


class shampoo_block(C.Structure):
    _fields_ = [("rows", C.c_int32), ("cols", C.c_int32), ("ld", C.c_int64),
                ("G", C.c_void_p), ("W", C.c_void_p), ("D", C.c_void_p), ("P", C.c_void_p),
                ("Mg", C.c_void_p), ("Ps", C.c_void_p), ("L", C.c_void_p), ("R", C.c_void_p),
                ("Lr", C.c_void_p), ("Rr", C.c_void_p)]


class shampoo_root_job(C.Structure):
    _fields_ = [("n", C.c_int32), ("reserved", C.c_int32), ("A", C.c_void_p), ("X", C.c_void_p)]


class shampoo_root_params(C.Structure):
    _fields_ = [("p", C.c_int32), ("eps", C.c_float), ("eps_relative", C.c_int32), ("tol", C.c_float),
                ("max_iters", C.c_int32), ("precision", C.c_int32), ("kappa32", C.c_float),
                ("maxsv_steps", C.c_int32), ("maxsv_tol", C.c_float), ("poll", C.c_int32),
                ("scaling", C.c_int32)]


class shampoo_root_info(C.Structure):
    _fields_ = [("status", C.c_int32), ("iters", C.c_int32), ("precision", C.c_int32),
                ("iters_fp32", C.c_int32), ("resid", C.c_float), ("lambda_max", C.c_float),
                ("cond_est", C.c_float), ("eps_eff", C.c_float)]


ROOT_INFO_FIELDS = [f for f, _ in shampoo_root_info._fields_]

_vp, _i, _f, _sz, _i64 = C.c_void_p, C.c_int, C.c_float, C.c_size_t, C.c_int64
_sig = {
    "shampoo_create": (_i, [C.POINTER(_vp), _i]),
    "shampoo_destroy": (_i, [_vp]),
    "shampoo_last_error": (C.c_char_p, [_vp]),
    "shampoo_version": (C.c_char_p, []),
    "shampoo_root_params_default": (None, [C.POINTER(shampoo_root_params)]),
    "shampoo_update_stats": (_i, [_vp, C.POINTER(shampoo_block), _i, _i, _f, _vp]),
    "shampoo_inv_root_workspace_bytes": (_sz, [C.POINTER(shampoo_root_job), _i, _i]),
    "shampoo_inv_root_batched": (_i, [_vp, C.POINTER(shampoo_root_job), _i, C.POINTER(shampoo_root_params),
                                      _vp, _sz, _vp, _vp]),
    "shampoo_inv_root_warm_batched": (_i, [_vp, C.POINTER(shampoo_root_job), _i, C.POINTER(shampoo_root_params),
                                           _f, _vp, _sz, _vp, _vp, _vp]),
    "shampoo_precondition": (_i, [_vp, C.POINTER(shampoo_block), _i, _i, _vp]),
    "shampoo_graft": (_i, [_vp, C.POINTER(shampoo_block), _i, _i, _f, _f, _i, _vp, _vp]),
    "shampoo_graft_lamb": (_i, [_vp, C.POINTER(shampoo_block), _i, _i, _f, _f, _i, _vp, _vp]),
    "shampoo_graft_noalloc": (_i, [_vp, C.POINTER(shampoo_block), _i, _i, _f, _f, _i, _vp, _vp]),
    "shampoo_precondition_graft": (_i, [_vp, C.POINTER(shampoo_block), _i, _i, _f, _vp, _vp]),
    "shampoo_embedding_workspace_bytes": (_sz, [_i, _i]),
    "shampoo_embedding_rows": (_i, [_vp, _vp, _vp, _vp, _i, _i64, _vp, _i, _i, _i64, _vp, _vp, _vp, _vp, _sz, _vp]),
    "shampoo_embedding_stats": (_i, [_vp, _vp, _vp, _i, _i, _vp, _f, _vp, _sz, _vp]),
    "shampoo_embedding_precondition": (_i, [_vp, _vp, _vp, _i, _i, _vp, _vp, _vp]),
    "shampoo_embedding_graft": (_i, [_vp, _vp, _vp, _i, _i, _vp, _vp, _vp, _vp, _i64, _i64, _f, _i, _vp, _vp]),
    "shampoo_token_logprobs_workspace_bytes": (_sz, [_i64, _i64, _i]),
    "shampoo_token_logprobs": (_i, [_vp, _vp, _i, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _i, _vp, _vp, _vp, _sz, _vp]),
    "shampoo_token_logprobs_grad": (_i, [_vp, _vp, _i, _i64, _i64, _i64, _vp, _vp, _vp, _i, _vp, _vp, _vp, _vp, _vp,
                                         _vp, _i64, _vp]),
    "shampoo_act_checkpoint_bytes": (_sz, [_i64, _i64]),
    "shampoo_act_encode": (_i, [_vp, _vp, _i, _i64, _i64, _i64, _i, _vp, _i64, _vp, _vp, _vp]),
    "shampoo_act_decode": (_i, [_vp, _vp, _i64, _i64, _vp, _i, _i64, _vp]),
    "shampoo_act_grad": (_i, [_vp, _vp, _i64, _i64, _i, _vp, _i, _i64, _vp, _i64, _vp]),
    "shampoo_act_weight_grad_workspace_bytes": (_sz, [_i64, _i64, _i64]),
    "shampoo_act_weight_grad": (_i, [_vp, _vp, _i64, _i64, _vp, _i, _i64, _i64, _vp, _i, _i64, _f, _vp, _sz, _vp]),
    "shampoo_vocab_logprobs_workspace_bytes": (_sz, [_i64, _i64, _i64, _i]),
    "shampoo_vocab_logprobs": (_i, [_vp, _vp, _vp, _i, _i64, _i64, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _sz, _vp]),
    "shampoo_vocab_logprobs_grad_workspace_bytes": (_sz, [_i64, _i64, _i64, _i, _i]),
    "shampoo_vocab_logprobs_grad": (_i, [_vp, _vp, _vp, _i, _i64, _i64, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _vp, _i64,
                                         _vp, _i, _i64, _f, _vp, _sz, _vp]),
    "shampoo_gated_ffn_workspace_bytes": (_sz, [_i64, _i64, _i64, _i]),
    "shampoo_gated_ffn": (_i, [_vp, _vp, _vp, _vp, _i, _i64, _i64, _i64, _i64, _i64, _i64, _i, _vp, _i64, _vp, _i64,
                               _vp, _i64, _vp, _sz, _vp]),
    "shampoo_gated_ffn_grad_workspace_bytes": (_sz, [_i64, _i64, _i64, _i, _i]),
    "shampoo_gated_ffn_grad": (_i, [_vp, _vp, _vp, _vp, _i, _i64, _i64, _i64, _i64, _i64, _i64, _i, _vp, _i64, _vp,
                                    _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _i, _f, _vp, _sz, _vp]),
    "shampoo_dropout": (_i, [_vp, _vp, _vp, _vp, _i, _i64, _i64, _i64, _i64, _i64, C.c_double, C.c_uint64, C.c_uint64,
                             _vp]),
    "shampoo_timing_enable": (_i, [_vp, _i]),
    "shampoo_timing_read": (_i, [_vp, _i, C.POINTER(C.c_double), C.POINTER(C.c_int64)]),
}
for _name, (_res, _args) in _sig.items():
    _fn = getattr(_lib, _name)
    _fn.restype = _res
    _fn.argtypes = _args

EXPORTED = tuple(_sig)


class ShampooError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"shampoo error {code}: {msg}")
        self.code = code


def _ptr(t):
    return None if t is None else t.data_ptr()


# ------------------------------------------------------------------ argument checks
# The C side cannot see shapes, strides, element types or devices: it gets
# raw pointers.  Every entry point below therefore checks its tensors against
# the layout include/shampoo.h states and raises ValueError before any C call.
# Device placement is checked last, so that a layout mistake is reported as
# such whatever the device.
_handle_device = {}


def _is_dtype(t, *names):
    return str(t.dtype).replace("torch.", "") in names


def _need(cond, msg):
    if not cond:
        raise ValueError(msg)


def _fp32(t, what):
    _need(_is_dtype(t, "float32"), f"{what}: dtype {t.dtype}, expected float32")


def _int32(t, what):
    _need(_is_dtype(t, "int32"), f"{what}: dtype {t.dtype}, expected int32")


def _contig(t, what):
    _need(t.is_contiguous(), f"{what}: must be contiguous (row-major, no gaps)")


def _square(t, n, what):
    _need(t.dim() == 2 and tuple(t.shape) == (n, n), f"{what}: shape {tuple(t.shape)}, expected ({n}, {n})")


def _min_numel(t, k, what):
    _need(t.numel() >= k, f"{what}: {t.numel()} elements, at least {k} needed")


def _devices(handle, tensors):
    """Every tensor must be a GPU tensor on the handle's device (one device
    for the call when the handle's device is not known)."""
    want = _handle_device.get(getattr(handle, "value", handle))
    for what, t in tensors:
        if t is None:
            continue
        _need(t.device.type == "cuda", f"{what}: on {t.device}, expected a GPU tensor")
        if want is None:
            want = t.device.index
        _need(t.device.index == want, f"{what}: on cuda:{t.device.index}, expected cuda:{want}")


_STATE_FIELDS = ("W", "D", "P", "Mg", "Ps")


_torch_mod = None


def _torch():
    global _torch_mod
    if _torch_mod is None:
        import torch
        _torch_mod = torch
    return _torch_mod


def _check_blocks(handle, blocks, norms=None):
    """Fast pass over the blocks (cheap accessors, no per-check calls); the
    detailed checker below runs only when something fails, to raise with the
    exact reason."""
    torch = _torch()
    f32, bf16 = torch.float32, torch.bfloat16
    want = _handle_device.get(getattr(handle, "value", handle))
    dev0 = None
    ok = True
    g_dtype = None
    for b in blocks:
        g = b.G
        if g is None or g.dim() != 2:
            ok = False
            break
        gd = g.dtype
        if g_dtype is None:
            g_dtype = gd
        if gd is not g_dtype or (gd is not f32 and gd is not bf16):
            ok = False
            break
        gs = g.size()
        m, n = gs[0], gs[1]
        gst = g.stride()
        ld = gst[0] if m > 1 else n
        dev = g.get_device()
        if dev0 is None:
            dev0 = dev
        if (n != 1 and gst[1] != 1) or dev != dev0:
            ok = False
            break
        for t in (b.W, b.D, b.P, b.Mg, b.Ps):
            if t is None:
                continue
            st = t.stride()
            if (t.dtype is not f32 or t.size() != gs or t.get_device() != dev0 or (n != 1 and st[1] != 1)
                    or (m != 1 and st[0] != ld)):
                ok = False
                break
        if not ok:
            break
        for t, k in ((b.L, m), (b.R, n), (b.Lr, m), (b.Rr, n)):
            if t is None:
                continue
            if t.dtype is not f32 or t.size() != (k, k) or not t.is_contiguous() or t.get_device() != dev0:
                ok = False
                break
        if not ok:
            break
    if ok and norms is not None:
        ok = (norms.dtype is f32 and norms.is_contiguous() and norms.numel() >= 3 * len(blocks)
              and (dev0 is None or norms.get_device() == dev0))
    if ok and (dev0 is None or (dev0 >= 0 and (want is None or dev0 == want))):
        if dev0 is None and norms is not None:
            _devices(handle, [("norms", norms)])
        return
    _check_blocks_detailed(handle, blocks, norms)
    raise ValueError("tensors of one call must all be on one GPU, the handle's")


def _check_blocks_detailed(handle, blocks, norms=None):
    tensors = []
    g_dtype = None
    for i, b in enumerate(blocks):
        g = b.G
        _need(g is not None, f"block {i}: G is required")
        _need(g.dim() == 2, f"block {i}: G has {g.dim()} dimensions, expected 2")
        _need(_is_dtype(g, "float32", "bfloat16"), f"block {i}: G dtype {g.dtype}, expected float32 or bfloat16")
        if g_dtype is None:
            g_dtype = g.dtype
        _need(g.dtype == g_dtype, f"block {i}: G dtype {g.dtype} differs from block 0's {g_dtype}: one call "
                                  f"takes one gradient type")
        m, n = int(g.shape[0]), int(g.shape[1])
        _need(n == 1 or g.stride(1) == 1, f"block {i}: G columns must be adjacent (stride(1) == 1)")
        ld = int(g.stride(0)) if m > 1 else n
        tensors.append((f"block {i}: G", g))
        for name in _STATE_FIELDS:
            t = getattr(b, name)
            if t is None:
                continue
            what = f"block {i}: {name}"
            _fp32(t, what)
            _need(tuple(t.shape) == (m, n), f"{what}: shape {tuple(t.shape)}, expected G's {(m, n)}")
            _need((n == 1 or t.stride(1) == 1) and (m == 1 or int(t.stride(0)) == ld),
                  f"{what}: strides {tuple(t.stride())}, expected G's row stride ({ld}, 1): the views of a "
                  f"block share one ld")
            tensors.append((what, t))
        for name, k in (("L", m), ("R", n), ("Lr", m), ("Rr", n)):
            t = getattr(b, name)
            if t is None:
                continue
            what = f"block {i}: {name}"
            _fp32(t, what)
            _square(t, k, what)
            _contig(t, what)
            tensors.append((what, t))
    _check_norms(handle, norms, len(blocks), tensors)


def _check_norms(handle, norms, nblocks, tensors=()):
    tensors = list(tensors)
    if norms is not None:
        _fp32(norms, "norms")
        _contig(norms, "norms")
        _min_numel(norms, 3 * nblocks, "norms")
        tensors.append(("norms", norms))
    _devices(handle, tensors)


def _check_jobs(handle, As, Xs, workspace, info, warm_out=None):
    """Fast pass (see _check_blocks); the detailed checks raise the reason."""
    torch = _torch()
    f32 = torch.float32
    want = _handle_device.get(getattr(handle, "value", handle))
    ok = len(As) == len(Xs) and workspace is not None
    dev0 = None
    if ok:
        for a, x in zip(As, Xs):
            sz = a.size()
            dev = a.get_device()
            if dev0 is None:
                dev0 = dev
            if (len(sz) != 2 or sz[0] != sz[1] or a.dtype is not f32 or x.dtype is not f32 or x.size() != sz
                    or not a.is_contiguous() or not x.is_contiguous() or dev != dev0 or x.get_device() != dev0
                    or a.data_ptr() == x.data_ptr()):
                ok = False
                break
    if ok:
        ok = (workspace.is_contiguous() and info.dtype is torch.int32 and info.is_contiguous()
              and info.numel() >= 8 * len(As) and (warm_out is None or (warm_out.dtype is torch.int32 and
                                                                        warm_out.is_contiguous() and
                                                                        warm_out.numel() >= 2 * len(As))))
        devs = [workspace.get_device(), info.get_device()] + ([] if warm_out is None else [warm_out.get_device()])
        if dev0 is None:
            dev0 = devs[0]
        ok = ok and all(d == dev0 for d in devs) and dev0 >= 0 and (want is None or dev0 == want)
    if ok:
        return
    _check_jobs_detailed(handle, As, Xs, workspace, info, warm_out)
    raise ValueError("tensors of one call must all be on one GPU, the handle's")


def _job_list_tensors(As, Xs):
    """Layout checks of the As / Xs of a root call (raise with the reason);
    returns the tensors for the device check."""
    _need(len(As) == len(Xs), f"{len(As)} statistics but {len(Xs)} outputs")
    tensors = []
    for i, (a, x) in enumerate(zip(As, Xs)):
        _need(a.dim() == 2, f"job {i}: A has {a.dim()} dimensions, expected 2")
        n = int(a.shape[0])
        for what, t in ((f"job {i}: A", a), (f"job {i}: X", x)):
            _fp32(t, what)
            _square(t, n, what)
            _contig(t, what)
            tensors.append((what, t))
        _need(a.data_ptr() != x.data_ptr() or n == 0, f"job {i}: A and X must be distinct buffers")
    return tensors


def _job_buffer_tensors(njobs, workspace, info, warm_out):
    """Layout checks of the workspace / info / warm_out of a root call of
    njobs jobs; returns the tensors for the device check."""
    _need(workspace is not None, "workspace is required")
    _contig(workspace, "workspace")
    _int32(info, "info")
    _contig(info, "info")
    _min_numel(info, 8 * njobs, "info (8 int32 per job)")
    tensors = [("workspace", workspace), ("info", info)]
    if warm_out is not None:
        _int32(warm_out, "warm_out")
        _contig(warm_out, "warm_out")
        _min_numel(warm_out, 2 * njobs, "warm_out (2 int32 per job)")
        tensors.append(("warm_out", warm_out))
    return tensors


def _check_jobs_detailed(handle, As, Xs, workspace, info, warm_out=None):
    As, Xs = list(As), list(Xs)
    tensors = _job_list_tensors(As, Xs) + _job_buffer_tensors(len(As), workspace, info, warm_out)
    _devices(handle, tensors)


def _stream(stream):
    if stream is not None:
        return stream if isinstance(stream, int) else stream.cuda_stream
    import torch
    return torch.cuda.current_stream().cuda_stream


def _check(handle, code):
    if code != SHAMPOO_OK:
        msg = _lib.shampoo_last_error(handle)
        raise ShampooError(code, msg.decode() if msg else "")


@dataclass
class Block:
    """One block view.  Tensors must share the row stride of G (``ld``)."""
    G: object
    W: Optional[object] = None
    D: Optional[object] = None
    P: Optional[object] = None
    Mg: Optional[object] = None
    Ps: Optional[object] = None
    L: Optional[object] = None
    R: Optional[object] = None
    Lr: Optional[object] = None
    Rr: Optional[object] = None


_BLOCK_PTRS = ("G", "W", "D", "P", "Mg", "Ps", "L", "R", "Lr", "Rr")


def _blocks(blocks: Sequence[Block]):
    """The shampoo_block array of a call, packed as 12 int64 words per block
    (rows | cols << 32, ld, then the ten pointers), as a ctypes pointer into a
    numpy buffer that the caller keeps alive over the C call."""
    import numpy as np
    rec = []
    for b in blocks:
        g = b.G
        m, n = g.size()
        ld = g.stride(0) if m > 1 else n   # one row: no stride used
        rec.append([m | (n << 32), ld] + [0 if t is None else t.data_ptr() for t in
                                          (b.G, b.W, b.D, b.P, b.Mg, b.Ps, b.L, b.R, b.Lr, b.Rr)])
    buf = np.array(rec if rec else [[0] * 12], dtype=np.uint64)
    assert buf.shape[1] * 8 == C.sizeof(shampoo_block)
    return _Packed(buf, buf.ctypes.data_as(C.POINTER(shampoo_block)))


class _Packed:
    """A packed host table and its ctypes pointer (the table lives as long as this object)."""
    def __init__(self, buf, ptr):
        self._buf, self._as_parameter_ = buf, ptr


def _dtype_code(blocks):
    if not blocks:
        return SHAMPOO_F32
    import torch
    dt = blocks[0].G.dtype
    return SHAMPOO_BF16 if dt == torch.bfloat16 else SHAMPOO_F32


class PackedBlocks:
    """A block list checked and packed once, for calls that repeat with the
    same views (a training loop passes the same blocks every step): every
    entry point that takes a block list accepts it in its place and skips the
    per-call checks and packing.  It records each tensor's pointer, size and
    row stride as they are when packed and keeps those tensors alive (a field
    of a Block reassigned later still leaves the packed tensor valid, if
    stale); pack again after any of them is reallocated, resized or
    replaced."""

    def __init__(self, handle, blocks):
        blocks = list(blocks)
        _check_blocks(handle, blocks)
        self.blocks = blocks
        self._tensors = [getattr(b, f) for b in blocks for f in _BLOCK_PTRS]
        self._handle = getattr(handle, "value", handle)
        self._arr = _blocks(blocks)
        self._dtype = _dtype_code(blocks)
        self._device = blocks[0].G.get_device() if blocks else None

    def __len__(self):
        return len(self.blocks)


class PackedJobs:
    """Inverse-root jobs (As, Xs) checked and packed once, as PackedBlocks:
    accepted by shampoo_inv_root_batched and shampoo_inv_root_warm_batched in
    place of As (Xs is then None).  Pack again after any tensor is
    reallocated or replaced."""

    def __init__(self, handle, As, Xs):
        As, Xs = list(As), list(Xs)
        _need(len(As) > 0, "PackedJobs: no jobs")
        _devices(handle, _job_list_tensors(As, Xs))
        self.As, self.Xs = As, Xs  # the packed tensors stay alive with this object
        self._handle = getattr(handle, "value", handle)
        self._arr = _jobs(As, Xs)
        self._device = As[0].get_device()

    def __len__(self):
        return len(self.As)


def _block_args(handle, blocks, norms=None):
    """(packed table, count, G dtype code) of a call's blocks: a PackedBlocks
    as it was packed (only norms is checked), a list checked and packed now."""
    if isinstance(blocks, PackedBlocks):
        _need(blocks._handle == getattr(handle, "value", handle), "PackedBlocks was packed for another handle")
        if norms is not None:
            _check_norms(handle, norms, len(blocks))
            _need(blocks._device is None or norms.get_device() == blocks._device,
                  "norms: not on the blocks' device")
        return blocks._arr, len(blocks), blocks._dtype
    _check_blocks(handle, blocks, norms)
    return _blocks(blocks), len(blocks), _dtype_code(blocks)


def _job_args(handle, As, Xs, workspace, info, warm_out=None):
    """(packed table, count) of a root call: a PackedJobs as it was packed (the
    workspace, info and warm_out checked now), lists checked and packed now."""
    if isinstance(As, PackedJobs):
        _need(Xs is None, "with PackedJobs, Xs must be None (the outputs are packed)")
        _need(As._handle == getattr(handle, "value", handle), "PackedJobs was packed for another handle")
        tensors = _job_buffer_tensors(len(As), workspace, info, warm_out)
        _devices(handle, tensors)
        for what, t in tensors:
            _need(t.get_device() == As._device, f"{what}: not on the jobs' device")
        return As._arr, len(As)
    _check_jobs(handle, As, Xs, workspace, info, warm_out)
    return _jobs(As, Xs), len(As)


# ------------------------------------------------------------------ entry points
def shampoo_version():
    return _lib.shampoo_version().decode()


def shampoo_root_params_default(**overrides):
    p = shampoo_root_params()
    _lib.shampoo_root_params_default(C.byref(p))
    for k, v in overrides.items():
        setattr(p, k, v)
    return p


def shampoo_create(device=0):
    h = C.c_void_p()
    code = _lib.shampoo_create(C.byref(h), int(device))
    if code != SHAMPOO_OK:
        raise ShampooError(code, f"shampoo_create(device={device}) failed")
    _handle_device[h.value] = int(device)
    return h


def shampoo_destroy(handle):
    _check(handle, _lib.shampoo_destroy(handle))
    _handle_device.pop(getattr(handle, "value", handle), None)


def shampoo_update_stats(handle, blocks, beta2=1.0, stream=None):
    """blocks: a list of Block, or a PackedBlocks."""
    arr, nb, dt = _block_args(handle, blocks)
    _check(handle, _lib.shampoo_update_stats(handle, arr, nb, dt, float(beta2), _stream(stream)))


def _jobs(As, Xs):
    """The shampoo_root_job array, packed as 3 int64 words per job (n, A, X)."""
    import numpy as np
    rec = [[a.size(0), a.data_ptr(), x.data_ptr()] for a, x in zip(As, Xs)]
    buf = np.array(rec if rec else [[0] * 3], dtype=np.uint64)
    assert buf.shape[1] * 8 == C.sizeof(shampoo_root_job)
    return _Packed(buf, buf.ctypes.data_as(C.POINTER(shampoo_root_job)))


def shampoo_inv_root_workspace_bytes(ns, precision=PRECISION_AUTO):
    arr = (shampoo_root_job * max(1, len(ns)))()
    for i, n in enumerate(ns):
        arr[i].n = int(n)
    return int(_lib.shampoo_inv_root_workspace_bytes(arr, len(ns), int(precision)))


def shampoo_inv_root_batched(handle, As, Xs, params, workspace, info, stream=None):
    """As, Xs: lists of contiguous n x n fp32 device tensors (or As a
    PackedJobs and Xs None); workspace: a uint8 device tensor; info: an int32
    device tensor of 8 * len(As)."""
    arr, nj = _job_args(handle, As, Xs, workspace, info)
    _check(handle, _lib.shampoo_inv_root_batched(handle, arr, nj, C.byref(params), _ptr(workspace),
                                                 int(workspace.numel() * workspace.element_size()),
                                                 _ptr(info), _stream(stream)))


def shampoo_inv_root_warm_batched(handle, As, Xs, params, workspace, info, warm_out=None, comm_tol=1e-3,
                                  stream=None):
    """As shampoo_inv_root_batched; Xs hold the warm starts X0 on entry.
    warm_out: None or an int32 device tensor of 2 * len(As)."""
    arr, nj = _job_args(handle, As, Xs, workspace, info, warm_out)
    _check(handle, _lib.shampoo_inv_root_warm_batched(handle, arr, nj, C.byref(params), float(comm_tol),
                                                      _ptr(workspace),
                                                      int(workspace.numel() * workspace.element_size()),
                                                      _ptr(info), _ptr(warm_out), _stream(stream)))


def shampoo_precondition(handle, blocks, stream=None):
    arr, nb, dt = _block_args(handle, blocks)
    _check(handle, _lib.shampoo_precondition(handle, arr, nb, dt, _stream(stream)))


def shampoo_graft(handle, blocks, eta0, beta1=0.0, use_shampoo=True, norms=None, stream=None):
    arr, nb, dt = _block_args(handle, blocks, norms)
    _check(handle, _lib.shampoo_graft(handle, arr, nb, dt, float(eta0), float(beta1), int(bool(use_shampoo)),
                                      _ptr(norms), _stream(stream)))


def shampoo_graft_noalloc(handle, blocks, eta0, beta1=0.0, use_shampoo=True, norms=None, stream=None):
    """shampoo_graft without any device allocation (fixed scratch; see the header for its limits)."""
    arr, nb, dt = _block_args(handle, blocks, norms)
    _check(handle, _lib.shampoo_graft_noalloc(handle, arr, nb, dt, float(eta0), float(beta1), int(bool(use_shampoo)),
                                              _ptr(norms), _stream(stream)))


def _nbytes(t):
    return 0 if t is None else int(t.numel() * t.element_size())


def shampoo_embedding_workspace_bytes(nnz, dim):
    return int(_lib.shampoo_embedding_workspace_bytes(int(nnz), int(dim)))


def _check_vec(t, k, what, kind):
    (_int32 if kind == "int32" else _fp32)(t, what)
    _contig(t, what)
    _min_numel(t, k, what)


def _check_compact(U, what="U"):
    _need(U.dim() == 2, f"{what}: {U.dim()} dimensions, expected nnz x dim")
    _fp32(U, what)
    _contig(U, what)
    return int(U.shape[0]), int(U.shape[1])


def shampoo_embedding_rows(handle, idx, feat, weight, vocab, dy, rows, U, count, workspace, stream=None):
    """idx, feat (or None): int32 [nnz]; weight: fp32 [nnz] or None; dy: m x dim
    fp32 (row-major view); rows int32 [nnz], U fp32 nnz x dim (contiguous),
    count int32 [2]; workspace: uint8 device tensor."""
    nnz = int(idx.numel())
    _check_vec(idx, nnz, "idx", "int32")
    if feat is not None:
        _need(feat.numel() == nnz, f"feat: {feat.numel()} entries, idx has {nnz}")
        _check_vec(feat, nnz, "feat", "int32")
    if weight is not None:
        _need(weight.numel() == nnz, f"weight: {weight.numel()} entries, idx has {nnz}")
        _check_vec(weight, nnz, "weight", "float32")
    _need(dy.dim() == 2, f"dy: {dy.dim()} dimensions, expected 2")
    _fp32(dy, "dy")
    _need(dy.shape[1] == 1 or dy.stride(1) == 1, "dy: columns must be adjacent (stride(1) == 1)")
    m, dim = int(dy.shape[0]), int(dy.shape[1])
    _check_vec(rows, nnz, "rows", "int32")
    u_rows, u_dim = _check_compact(U)
    _need(u_rows >= nnz and u_dim == dim, f"U: shape {tuple(U.shape)}, expected at least ({nnz}, {dim})")
    _check_vec(count, 2, "count", "int32")
    _need(workspace is not None, "workspace is required")
    _contig(workspace, "workspace")
    _devices(handle, [("idx", idx), ("feat", feat), ("weight", weight), ("dy", dy), ("rows", rows), ("U", U),
                      ("count", count), ("workspace", workspace)])
    _check(handle, _lib.shampoo_embedding_rows(handle, _ptr(idx), _ptr(feat), _ptr(weight), nnz, int(vocab),
                                               _ptr(dy), m, dim, int(dy.stride(0)), _ptr(rows), _ptr(U),
                                               _ptr(count), _ptr(workspace), _nbytes(workspace), _stream(stream)))


def shampoo_embedding_stats(handle, U, count, R, beta2=1.0, workspace=None, stream=None):
    nnz, dim = _check_compact(U)
    _check_vec(count, 2, "count", "int32")
    _fp32(R, "R")
    _square(R, dim, "R")
    _contig(R, "R")
    _need(workspace is not None, "workspace is required")
    _contig(workspace, "workspace")
    _devices(handle, [("U", U), ("count", count), ("R", R), ("workspace", workspace)])
    _check(handle, _lib.shampoo_embedding_stats(handle, _ptr(U), _ptr(count), nnz, dim, _ptr(R), float(beta2),
                                                _ptr(workspace), _nbytes(workspace), _stream(stream)))


def shampoo_embedding_precondition(handle, U, count, Rr, P, stream=None):
    nnz, dim = _check_compact(U)
    _check_vec(count, 2, "count", "int32")
    _fp32(Rr, "Rr")
    _square(Rr, dim, "Rr")
    _contig(Rr, "Rr")
    _need(_check_compact(P, "P") == (nnz, dim), f"P: shape {tuple(P.shape)}, expected U's ({nnz}, {dim})")
    _devices(handle, [("U", U), ("count", count), ("Rr", Rr), ("P", P)])
    _check(handle, _lib.shampoo_embedding_precondition(handle, _ptr(U), _ptr(count), nnz, dim, _ptr(Rr), _ptr(P),
                                                       _stream(stream)))


def shampoo_embedding_graft(handle, rows, count, U, P, W, D, eta0, use_shampoo=True, norms=None, stream=None):
    """W, D: vocab x dim fp32 tables (same row stride)."""
    nnz, dim = _check_compact(U)
    _check_vec(rows, nnz, "rows", "int32")
    _check_vec(count, 2, "count", "int32")
    _need(_check_compact(P, "P") == (nnz, dim), f"P: shape {tuple(P.shape)}, expected U's ({nnz}, {dim})")
    for what, t in (("W", W), ("D", D)):
        _fp32(t, what)
        _need(t.dim() == 2 and int(t.shape[1]) == dim, f"{what}: shape {tuple(t.shape)}, expected (vocab, {dim})")
        _need(dim == 1 or t.stride(1) == 1, f"{what}: columns must be adjacent (stride(1) == 1)")
    _need(tuple(W.shape) == tuple(D.shape) and (W.shape[0] == 1 or W.stride(0) == D.stride(0)),
          f"W {tuple(W.shape)} / {tuple(W.stride())} and D {tuple(D.shape)} / {tuple(D.stride())} must share "
          f"shape and row stride")
    _check_norms(handle, norms, 1, [("rows", rows), ("count", count), ("U", U), ("P", P), ("W", W), ("D", D)])
    _check(handle, _lib.shampoo_embedding_graft(handle, _ptr(rows), _ptr(count), nnz, dim, _ptr(U), _ptr(P),
                                                _ptr(W), _ptr(D), int(W.shape[0]), int(W.stride(0)), float(eta0),
                                                int(bool(use_shampoo)), _ptr(norms), _stream(stream)))


def shampoo_precondition_graft(handle, blocks, eta0, norms=None, stream=None):
    arr, nb, dt = _block_args(handle, blocks, norms)
    _check(handle, _lib.shampoo_precondition_graft(handle, arr, nb, dt, float(eta0), _ptr(norms), _stream(stream)))


def shampoo_graft_lamb(handle, blocks, eta0, beta1=0.0, use_shampoo=True, norms=None, stream=None):
    arr, nb, dt = _block_args(handle, blocks, norms)
    _check(handle, _lib.shampoo_graft_lamb(handle, arr, nb, dt, float(eta0), float(beta1), int(bool(use_shampoo)),
                                           _ptr(norms), _stream(stream)))


# ------------------------------------------------------------------ from the loss to the gradient
# Each call first looks its tensors over with cheap accessors; only where
# something is off does the detailed check run, to raise with the reason.
def _layout(t):
    """(rows, cols, row stride, dtype code, device, pointer) of an fp32 or bf16
    matrix of adjacent columns, or None.  One row, or none, uses no stride; rows
    that overlap (an expanded view) are no layout the library takes."""
    dt = t.dtype
    torch = _torch_mod or _torch()
    code = SHAMPOO_F32 if dt is torch.float32 else SHAMPOO_BF16 if dt is torch.bfloat16 else -1
    if code < 0 or t.dim() != 2:
        return None
    m, n = t.shape
    ld, sc = t.stride()
    if m <= 1:
        ld = n
    if ld < n or (sc != 1 and n > 1):
        return None
    return m, n, ld, code, t.get_device(), t.data_ptr()


def _plain(t, dtype, shape, dev):
    """A contiguous tensor of this type, shape and device, or None given."""
    return t is None or (t.dtype is dtype and t.shape == shape and t.is_contiguous() and t.get_device() == dev)


def _room(t, nbytes, dev):
    """A contiguous uint8 buffer of at least nbytes on dev (None where none are needed)."""
    if t is None:
        return nbytes == 0
    return (t.dtype is _torch_mod.uint8 and t.numel() >= nbytes and t.is_contiguous() and t.get_device() == dev)


def _bytes_on(t, dev):
    """A contiguous uint8 buffer on dev, or None."""
    return t is None or (t.dtype is _torch_mod.uint8 and t.is_contiguous() and t.get_device() == dev)


def _apart(a, b):
    """Whether two matrices (as from _layout) share no memory: one lies past the
    other, or the rows of each lie between those of the other (column ranges
    of one wider buffer)."""
    if a[0] == 0 or b[0] == 0 or a[1] == 0 or b[1] == 0:
        return True
    ea, eb = 4 - 2 * a[3], 4 - 2 * b[3]
    if a[5] + ((a[0] - 1) * a[2] + a[1]) * ea <= b[5] or b[5] + ((b[0] - 1) * b[2] + b[1]) * eb <= a[5]:
        return True
    row_a, row_b, pitch, other = a[1] * ea, b[1] * eb, a[2] * ea, b[2] * eb
    if a[0] == 1:
        pitch = other
    elif b[0] > 1 and other != pitch:
        return False  # rows drift past each other: taken as shared
    at = (b[5] - a[5]) % pitch
    return at >= row_a and at + row_b <= pitch


def _alike(out, src):
    """out has src's shape, type and device, and is src itself or apart from it."""
    return (out is not None and out[0] == src[0] and out[1] == src[1] and out[3] == src[3] and out[4] == src[4] and
            ((out[5] == src[5] and out[2] == src[2]) or _apart(out, src)))


def _on_handle(handle, dev):
    """dev is a GPU, the handle's where that is known."""
    return dev >= 0 and _handle_device.get(handle.value if handle is not None else None, dev) == dev


def _stream_on(stream, dev):
    """The stream of a call: the one given, else the current one of dev."""
    if stream is not None:
        return stream if isinstance(stream, int) else stream.cuda_stream
    return _torch_mod._C._cuda_getCurrentRawStream(dev)


def _refuse(handle, tensors, checks):
    """Runs the detailed checks, each of which raises with its reason, then the device check."""
    for check in checks:
        check()
    _devices(handle, tensors)
    raise ValueError("tensors of one call must all be on one GPU, the handle's")


def _check_matrix(t, what, like=None):
    torch = _torch()
    dt = t.dtype
    _need(t.dim() == 2, f"{what}: {t.dim()} dimensions, expected 2")
    _need(dt is torch.float32 or dt is torch.bfloat16, f"{what}: dtype {dt}, expected float32 or bfloat16")
    m, n = t.shape
    if like is not None:
        _need(dt is like.dtype, f"{what}: dtype {dt}, expected {like.dtype}")
        _need(t.shape == like.shape, f"{what}: shape {(m, n)}, expected {tuple(like.shape)}")
    ld, sc = t.stride()
    _need(n <= 1 or sc == 1, f"{what}: columns must be adjacent (stride(1) == 1)")
    _need(m <= 1 or ld >= n, f"{what}: row stride {ld} < {n} columns")


def _check_shape(t, shape, what, kind="float32"):
    if t is None:
        return
    (_int32 if kind == "int32" else _fp32)(t, what)
    _need(tuple(t.shape) == shape, f"{what}: shape {tuple(t.shape)}, expected {shape}")
    _contig(t, what)


def _check_bytes(t, nbytes, what):
    if t is None:
        _need(nbytes == 0, f"{what}: {nbytes} bytes needed, got None")
        return
    _need(_is_dtype(t, "uint8"), f"{what}: dtype {t.dtype}, expected uint8")
    _contig(t, what)
    _min_numel(t, nbytes, what)


def _check_apart(a, b, what, same_allowed):
    x, y = _layout(a), _layout(b)
    _need(_apart(x, y) or (same_allowed and x[5] == y[5] and x[2] == y[2]),
          f"{what} overlap" + (" without being the same view" if same_allowed else ""))


def shampoo_token_logprobs_workspace_bytes(rows, vocab, k=0):
    return int(_lib.shampoo_token_logprobs_workspace_bytes(int(rows), int(vocab), int(k)))


def shampoo_token_logprobs(handle, logits, targets, logp, lse, entropy=None, top_ids=None, top_logp=None,
                           workspace=None, stream=None):
    """logits: rows x vocab, fp32 or bf16 (row-major view); targets int32 [rows]
    and logp fp32 [rows] (both or neither); lse, entropy: fp32 [rows]; top_ids
    int32 and top_logp fp32, rows x k, for the k largest alternatives; workspace:
    uint8, shampoo_token_logprobs_workspace_bytes(rows, vocab, k)."""
    z = _layout(logits)
    ok = z is not None and lse is not None and (targets is None) == (logp is None) and (
        top_ids is None) == (top_logp is None)
    if ok:
        rows, vocab, ld, dt, dev, ptr = z
        f32, i32 = _torch_mod.float32, _torch_mod.int32
        k = top_ids.shape[-1] if top_ids is not None and top_ids.dim() == 2 else 0
        vec = (rows,)
        ok = (_plain(lse, f32, vec, dev) and _plain(targets, i32, vec, dev) and _plain(logp, f32, vec, dev) and
              _plain(entropy, f32, vec, dev) and _plain(top_ids, i32, (rows, k), dev) and
              _plain(top_logp, f32, (rows, k), dev) and _on_handle(handle, dev) and
              _room(workspace, _lib.shampoo_token_logprobs_workspace_bytes(rows, vocab, k), dev))
    if not ok:
        _refuse_logprobs(handle, logits, targets, logp, lse, entropy, top_ids, top_logp, workspace)
    _check(handle, _lib.shampoo_token_logprobs(handle, ptr, dt, rows, vocab, ld, _ptr(targets), _ptr(logp),
                                               lse.data_ptr(), _ptr(entropy), k, _ptr(top_ids), _ptr(top_logp),
                                               _ptr(workspace), 0 if workspace is None else workspace.numel(),
                                               _stream_on(stream, dev)))


def _refuse_logprobs(handle, logits, targets, logp, lse, entropy, top_ids, top_logp, workspace):
    _check_matrix(logits, "logits")
    rows, vocab = logits.shape
    _need((targets is None) == (logp is None), "targets and logp go together")
    _need((top_ids is None) == (top_logp is None), "top_ids and top_logp go together")
    _need(lse is not None, "lse is required")
    k = 0
    if top_ids is not None:
        _need(top_ids.dim() == 2, f"top_ids: {top_ids.dim()} dimensions, expected 2")
        k = int(top_ids.shape[1])
    _refuse(handle, (("logits", logits), ("targets", targets), ("logp", logp), ("lse", lse), ("entropy", entropy),
                     ("top_ids", top_ids), ("top_logp", top_logp), ("workspace", workspace)),
            (lambda: _check_shape(targets, (rows,), "targets", "int32"), lambda: _check_shape(logp, (rows,), "logp"),
             lambda: _check_shape(lse, (rows,), "lse"), lambda: _check_shape(entropy, (rows,), "entropy"),
             lambda: _check_shape(top_ids, (rows, k), "top_ids", "int32"),
             lambda: _check_shape(top_logp, (rows, k), "top_logp"),
             lambda: _check_bytes(workspace, _lib.shampoo_token_logprobs_workspace_bytes(rows, vocab, k),
                                  "workspace")))


def shampoo_token_logprobs_grad(handle, logits, targets, lse, dlogits, g_logp=None, g_lse=None, entropy=None,
                                g_entropy=None, top_ids=None, g_top=None, stream=None):
    """dlogits (logits' shape and type; may be logits) from the gradients of
    shampoo_token_logprobs' outputs: g_logp (with targets), g_lse, g_entropy
    (with entropy): fp32 [rows]; g_top (with top_ids): fp32 rows x k."""
    z, d = _layout(logits), _layout(dlogits)
    ok = (z is not None and _alike(d, z) and lse is not None and (g_logp is None or targets is not None) and
          (g_entropy is None or entropy is not None) and (g_top is None or top_ids is not None))
    if ok:
        rows, vocab, ld, dt, dev, ptr = z
        f32, i32 = _torch_mod.float32, _torch_mod.int32
        k = top_ids.shape[-1] if top_ids is not None and top_ids.dim() == 2 else 0
        vec = (rows,)
        ok = (_plain(lse, f32, vec, dev) and _plain(targets, i32, vec, dev) and _plain(g_logp, f32, vec, dev) and
              _plain(g_lse, f32, vec, dev) and _plain(entropy, f32, vec, dev) and _plain(g_entropy, f32, vec, dev) and
              _plain(top_ids, i32, (rows, k), dev) and _plain(g_top, f32, (rows, k), dev) and
              _on_handle(handle, dev))
    if not ok:
        _refuse_logprobs_grad(handle, logits, targets, lse, dlogits, g_logp, g_lse, entropy, g_entropy, top_ids, g_top)
    _check(handle, _lib.shampoo_token_logprobs_grad(handle, ptr, dt, rows, vocab, ld, _ptr(targets), lse.data_ptr(),
                                                    _ptr(entropy), k, _ptr(top_ids), _ptr(g_logp), _ptr(g_lse),
                                                    _ptr(g_entropy), _ptr(g_top), d[5], d[2],
                                                    _stream_on(stream, dev)))


def _refuse_logprobs_grad(handle, logits, targets, lse, dlogits, g_logp, g_lse, entropy, g_entropy, top_ids, g_top):
    _check_matrix(logits, "logits")
    rows = logits.shape[0]
    _check_matrix(dlogits, "dlogits", logits)
    _check_apart(dlogits, logits, "dlogits and logits", True)
    _need(g_logp is None or targets is not None, "g_logp needs targets")
    _need(g_entropy is None or entropy is not None, "g_entropy needs entropy")
    _need(g_top is None or top_ids is not None, "g_top needs top_ids")
    _need(lse is not None, "lse is required")
    k = 0
    if top_ids is not None:
        _need(top_ids.dim() == 2, f"top_ids: {top_ids.dim()} dimensions, expected 2")
        k = int(top_ids.shape[1])
    rest = (("lse", lse), ("g_logp", g_logp), ("g_lse", g_lse), ("entropy", entropy), ("g_entropy", g_entropy))
    for what, t in rest:
        _check_shape(t, (rows,), what)
    _refuse(handle, (("logits", logits), ("dlogits", dlogits), ("targets", targets), ("top_ids", top_ids),
                     ("g_top", g_top)) + rest,
            (lambda: _check_shape(targets, (rows,), "targets", "int32"),
             lambda: _check_shape(top_ids, (rows, k), "top_ids", "int32"),
             lambda: _check_shape(g_top, (rows, k), "g_top")))


def shampoo_act_checkpoint_bytes(rows, cols):
    return int(_lib.shampoo_act_checkpoint_bytes(int(rows), int(cols)))


def _check_ckpt(t, rows, cols, what):
    if t is not None:
        _check_bytes(t, _lib.shampoo_act_checkpoint_bytes(rows, cols), what)


def shampoo_act_encode(handle, X, ckpt_x=None, act=ACT_NONE, Y=None, ckpt_y=None, stream=None):
    """X: rows x cols, fp32 or bf16 (row-major view); Y = act(X): X's shape and
    type (may be X), or None; ckpt_x, ckpt_y: uint8 tensors of
    shampoo_act_checkpoint_bytes(rows, cols), or None."""
    x, y = _layout(X), None if Y is None else _layout(Y)
    ok = x is not None and (Y is None or _alike(y, x))
    if ok:
        rows, cols, ld, dt, dev, ptr = x
        need = _lib.shampoo_act_checkpoint_bytes(rows, cols)
        ok = ((ckpt_x is None or _room(ckpt_x, need, dev)) and (ckpt_y is None or _room(ckpt_y, need, dev)) and
              _on_handle(handle, dev))
    if not ok:
        _check_matrix(X, "X")
        if Y is not None:
            _check_matrix(Y, "Y", X)
            _check_apart(Y, X, "Y and X", True)
        _refuse(handle, (("X", X), ("Y", Y), ("ckpt_x", ckpt_x), ("ckpt_y", ckpt_y)),
                (lambda: _check_ckpt(ckpt_x, *X.shape, "ckpt_x"), lambda: _check_ckpt(ckpt_y, *X.shape, "ckpt_y")))
    _check(handle, _lib.shampoo_act_encode(handle, ptr, dt, rows, cols, ld, int(act), None if y is None else y[5],
                                           0 if y is None else y[2], _ptr(ckpt_x), _ptr(ckpt_y),
                                           _stream_on(stream, dev)))


def shampoo_act_decode(handle, ckpt, X, stream=None):
    """X: rows x cols, fp32 or bf16: the values that the checkpoint holds."""
    x = _layout(X)
    if x is None or ckpt is None or not _on_handle(handle, x[4]) or not _room(
            ckpt, _lib.shampoo_act_checkpoint_bytes(x[0], x[1]), x[4]):
        _check_matrix(X, "X")
        _need(ckpt is not None, "ckpt is required")
        _refuse(handle, (("ckpt", ckpt), ("X", X)), (lambda: _check_ckpt(ckpt, *X.shape, "ckpt"),))
    rows, cols, ld, dt, dev, ptr = x
    _check(handle, _lib.shampoo_act_decode(handle, ckpt.data_ptr(), rows, cols, ptr, dt, ld, _stream_on(stream, dev)))


def shampoo_act_grad(handle, ckpt, act, dY, dX, stream=None):
    """dX = dY o act'(x^), x^ the checkpoint's values; dX: dY's shape and type (may be dY)."""
    y, x = _layout(dY), _layout(dX)
    if y is None or not _alike(x, y) or ckpt is None or not _on_handle(handle, y[4]) or not _room(
            ckpt, _lib.shampoo_act_checkpoint_bytes(y[0], y[1]), y[4]):
        _check_matrix(dY, "dY")
        _check_matrix(dX, "dX", dY)
        _check_apart(dX, dY, "dX and dY", True)
        _need(ckpt is not None, "ckpt is required")
        _refuse(handle, (("ckpt", ckpt), ("dY", dY), ("dX", dX)), (lambda: _check_ckpt(ckpt, *dY.shape, "ckpt"),))
    rows, cols, ld_dy, dt, dev, ptr = y
    _check(handle, _lib.shampoo_act_grad(handle, ckpt.data_ptr(), rows, cols, int(act), ptr, dt, ld_dy, x[5], x[2],
                                         _stream_on(stream, dev)))


def shampoo_act_weight_grad_workspace_bytes(rows, cols, out):
    return int(_lib.shampoo_act_weight_grad_workspace_bytes(int(rows), int(cols), int(out)))


def shampoo_act_weight_grad(handle, ckpt, dY, G, beta=0.0, workspace=None, stream=None):
    """G (cols x out) = beta G + X^^T dY, X^ the rows x cols values of the
    checkpoint, dY rows x out; dY and G fp32 or bf16, each its own; workspace:
    uint8, shampoo_act_weight_grad_workspace_bytes(rows, cols, out)."""
    y, g = _layout(dY), _layout(G)
    ok = y is not None and g is not None and y[1] == g[1] and y[4] == g[4] and ckpt is not None and _apart(y, g)
    if ok:
        rows, out, ld_dy, dt, dev, ptr = y
        cols = g[0]
        ok = (_room(ckpt, _lib.shampoo_act_checkpoint_bytes(rows, cols), dev) and _on_handle(handle, dev) and
              _room(workspace, _lib.shampoo_act_weight_grad_workspace_bytes(rows, cols, out), dev))
    if not ok:
        _check_matrix(G, "G")
        _check_matrix(dY, "dY")
        _need(dY.shape[1] == G.shape[1], f"dY: {int(dY.shape[1])} columns, G has {int(G.shape[1])}")
        _need(ckpt is not None, "ckpt is required")
        _check_apart(G, dY, "G and dY", False)
        rows, cols, out = int(dY.shape[0]), int(G.shape[0]), int(G.shape[1])
        _refuse(handle, (("ckpt", ckpt), ("dY", dY), ("G", G), ("workspace", workspace)),
                (lambda: _check_ckpt(ckpt, rows, cols, "ckpt"),
                 lambda: _check_bytes(workspace, _lib.shampoo_act_weight_grad_workspace_bytes(rows, cols, out),
                                      "workspace")))
    _check(handle, _lib.shampoo_act_weight_grad(handle, ckpt.data_ptr(), rows, cols, ptr, dt, out, ld_dy, g[5], g[3],
                                                g[2], beta, _ptr(workspace),
                                                0 if workspace is None else workspace.numel(),
                                                _stream_on(stream, dev)))


# ------------------------------------------------------------------ the layers around the step
def _code(dtype):
    """The library's code of a torch type (its codes stand for themselves)."""
    torch = _torch_mod or _torch()
    if dtype is torch.float32:
        return SHAMPOO_F32
    if dtype is torch.bfloat16:
        return SHAMPOO_BF16
    _need(isinstance(dtype, int), f"dtype {dtype}, expected float32 or bfloat16")
    return dtype


def _fits(a, rows, cols, like):
    """a (a layout, or None) is rows x cols, of the type and device of the layout `like`."""
    return a is not None and a[0] == rows and a[1] == cols and a[3] == like[3] and a[4] == like[4]


def _opt(a):
    """Pointer and row stride of a layout that may be None."""
    return (None, 0) if a is None else (a[5], a[2])


def _failed(handle, rc, written, read, workspace, need):
    """Raises for a call's status.  The library refuses buffers that overlap and a workspace
    that is too small; which and by how much, the tensors tell."""
    if rc == SHAMPOO_EINVAL:
        _check_all_apart(written, read)
    if rc == SHAMPOO_ENOMEM:
        _check_bytes(workspace, need(), "workspace")
    _check(handle, rc)


def _check_all_apart(written, read):
    """Every written matrix (name, tensor) is apart from every other."""
    for i, (name, t) in enumerate(written):
        for other, u in written[i + 1:] + read:
            if t is not None and u is not None:
                _check_apart(t, u, f"{name} and {other}", False)


def _check_like(t, what, rows, cols, dtype=None):
    if t is None:
        return
    _check_matrix(t, what)
    _need(tuple(t.shape) == (rows, cols), f"{what}: shape {tuple(t.shape)}, expected {(rows, cols)}")
    _need(dtype is None or t.dtype is dtype, f"{what}: dtype {t.dtype}, expected {dtype}")


def shampoo_vocab_logprobs_workspace_bytes(rows, dim, vocab, dtype):
    return int(_lib.shampoo_vocab_logprobs_workspace_bytes(int(rows), int(dim), int(vocab), _code(dtype)))


def shampoo_vocab_logprobs(handle, X, W, targets, logp, lse, workspace=None, stream=None):
    """X: rows x dim, W: vocab x dim, both fp32 or both bf16 (row-major views);
    targets int32 [rows] and logp fp32 [rows] (both or neither); lse fp32 [rows];
    workspace: uint8, shampoo_vocab_logprobs_workspace_bytes(rows, dim, vocab, X.dtype)."""
    x, w = _layout(X), _layout(W)
    ok = (x is not None and w is not None and x[1] == w[1] and x[3] == w[3] and x[4] == w[4] and lse is not None and
          (targets is None) == (logp is None))
    if ok:
        rows, dim, ld, dt, dev, ptr = x
        vocab = w[0]
        f32, vec = _torch_mod.float32, (rows,)
        ok = (_plain(lse, f32, vec, dev) and _plain(logp, f32, vec, dev) and _on_handle(handle, dev) and
              _plain(targets, _torch_mod.int32, vec, dev) and
              _bytes_on(workspace, dev))
    if not ok:
        _refuse_vocab(handle, X, W, targets, lse, (("logp", logp),), workspace,
                      lambda r, d, v: _lib.shampoo_vocab_logprobs_workspace_bytes(r, d, v, _code(X.dtype)),
                      lambda: _need((targets is None) == (logp is None), "targets and logp go together"))
    rc = _lib.shampoo_vocab_logprobs(handle, ptr, w[5], dt, rows, dim, vocab, ld, w[2], _ptr(targets), _ptr(logp),
                                     lse.data_ptr(), _ptr(workspace), 0 if workspace is None else workspace.numel(),
                                     _stream_on(stream, dev))
    if rc:
        _failed(handle, rc, [], [], workspace,
                lambda: _lib.shampoo_vocab_logprobs_workspace_bytes(rows, dim, vocab, dt))


def _refuse_vocab(handle, X, W, targets, lse, vecs, workspace, room, pairs, more=()):
    _check_matrix(X, "X")
    _check_like(W, "W", int(W.shape[0]) if W.dim() else 0, int(X.shape[1]), X.dtype)
    (rows, dim), vocab = X.shape, int(W.shape[0])
    pairs()
    _need(lse is not None, "lse is required")
    for what, t in (("lse", lse),) + vecs:
        _check_shape(t, (rows,), what)
    _check_shape(targets, (rows,), "targets", "int32")
    _refuse(handle, (("X", X), ("W", W), ("targets", targets), ("lse", lse), ("workspace", workspace)) + vecs + more,
            (lambda: _check_bytes(workspace, room(rows, dim, vocab), "workspace"),))


def shampoo_vocab_logprobs_grad_workspace_bytes(rows, dim, vocab, dtype, g_dtype):
    return int(_lib.shampoo_vocab_logprobs_grad_workspace_bytes(int(rows), int(dim), int(vocab), _code(dtype),
                                                                _code(g_dtype)))


def shampoo_vocab_logprobs_grad(handle, X, W, targets, lse, dX=None, dW=None, g_logp=None, g_lse=None, beta=0.0,
                                workspace=None, stream=None):
    """dX (X's shape and type, or None) and dW = beta dW + ... (W's shape, fp32 or bf16, or
    None) from the gradients of shampoo_vocab_logprobs' outputs: g_logp (with targets),
    g_lse: fp32 [rows]; workspace: uint8, shampoo_vocab_logprobs_grad_workspace_bytes(rows,
    dim, vocab, X.dtype, dW.dtype) (without dW: X.dtype twice)."""
    x, w = _layout(X), _layout(W)
    ok = (x is not None and w is not None and x[1] == w[1] and x[3] == w[3] and x[4] == w[4] and lse is not None and
          (g_logp is None or targets is not None) and (dX is not None or dW is not None))
    if ok:
        rows, dim, ld, dt, dev, ptr = x
        vocab = w[0]
        dx = None if dX is None else _layout(dX)
        dw = None if dW is None else _layout(dW)
        gdt = dt if dw is None else dw[3]
        f32, vec = _torch_mod.float32, (rows,)
        ok = ((dX is None or _fits(dx, rows, dim, x)) and
              (dW is None or (dw is not None and dw[0] == vocab and dw[1] == dim and dw[4] == dev)) and
              _plain(lse, f32, vec, dev) and _plain(g_logp, f32, vec, dev) and _plain(g_lse, f32, vec, dev) and
              _plain(targets, _torch_mod.int32, vec, dev) and _on_handle(handle, dev) and
              _bytes_on(workspace, dev))
    if not ok:
        def pairs():
            _need(g_logp is None or targets is not None, "g_logp needs targets")
            _need(dX is not None or dW is not None, "dX or dW is required")
            _check_like(dX, "dX", *X.shape, X.dtype)
            _check_like(dW, "dW", *W.shape)
            _check_all_apart([("dX", dX), ("dW", dW)], [("X", X), ("W", W)])
        _refuse_vocab(handle, X, W, targets, lse, (("g_logp", g_logp), ("g_lse", g_lse)), workspace,
                      lambda r, d, v: _lib.shampoo_vocab_logprobs_grad_workspace_bytes(
                          r, d, v, _code(X.dtype), _code(X.dtype if dW is None else dW.dtype)), pairs,
                      (("dX", dX), ("dW", dW)))
    rc = _lib.shampoo_vocab_logprobs_grad(
        handle, ptr, w[5], dt, rows, dim, vocab, ld, w[2], _ptr(targets), lse.data_ptr(), _ptr(g_logp), _ptr(g_lse),
        *_opt(dx), _opt(dw)[0], gdt, _opt(dw)[1], beta, _ptr(workspace),
        0 if workspace is None else workspace.numel(), _stream_on(stream, dev))
    if rc:
        _failed(handle, rc, [("dX", dX), ("dW", dW)], [("X", X), ("W", W)], workspace,
                lambda: _lib.shampoo_vocab_logprobs_grad_workspace_bytes(rows, dim, vocab, dt, gdt))


def shampoo_gated_ffn_workspace_bytes(rows, dim, width, dtype):
    return int(_lib.shampoo_gated_ffn_workspace_bytes(int(rows), int(dim), int(width), _code(dtype)))


def _refuse_ffn(handle, X, Wg, Wu, wide, more, written, read, room, workspace):
    _check_matrix(X, "X")
    _check_like(Wg, "Wg", int(X.shape[1]), int(Wg.shape[-1]), X.dtype)
    _check_like(Wu, "Wu", *Wg.shape, X.dtype)
    (rows, dim), width = X.shape, int(Wg.shape[1])
    for name, t in wide:
        _check_like(t, name, rows, width, X.dtype)
    for check in more:
        check(rows, dim, width)
    base = [("X", X), ("Wg", Wg), ("Wu", Wu)]
    _check_all_apart(written, base + read)
    _refuse(handle, tuple(base + written + read) + (("workspace", workspace),),
            (lambda: _check_bytes(workspace, room(rows, dim, width), "workspace"),))


def shampoo_gated_ffn(handle, X, Wg, Wu, H, act=ACT_SILU, G=None, U=None, workspace=None, stream=None):
    """H (rows x width) = act(X Wg) o (X Wu); X: rows x dim, Wg and Wu: dim x width; G and U
    (both or neither): the projections, rows x width; all fp32 or all bf16 (row-major
    views); workspace: uint8, shampoo_gated_ffn_workspace_bytes(rows, dim, width, X.dtype)."""
    x, wg, wu, lh = _layout(X), _layout(Wg), _layout(Wu), None if H is None else _layout(H)
    lg, lu = None if G is None else _layout(G), None if U is None else _layout(U)
    ok = x is not None and wg is not None and lh is not None and (G is None) == (U is None)
    if ok:
        rows, dim, ld, dt, dev, ptr = x
        width = wg[1]
        ok = (_fits(wg, dim, width, x) and _fits(wu, dim, width, x) and _fits(lh, rows, width, x) and
              (G is None or (_fits(lg, rows, width, x) and _fits(lu, rows, width, x))) and _on_handle(handle, dev) and
              _bytes_on(workspace, dev))
    if not ok:
        _need(H is not None, "H is required")
        _need((G is None) == (U is None), "G and U go together")
        _refuse_ffn(handle, X, Wg, Wu, (("H", H), ("G", G), ("U", U)), (), [("H", H), ("G", G), ("U", U)], [],
                    lambda r, d, w: _lib.shampoo_gated_ffn_workspace_bytes(r, d, w, _code(X.dtype)), workspace)
    rc = _lib.shampoo_gated_ffn(handle, ptr, wg[5], wu[5], dt, rows, dim, width, ld, wg[2], wu[2], act, lh[5], lh[2],
                                *_opt(lg), *_opt(lu), _ptr(workspace),
                                0 if workspace is None else workspace.numel(), _stream_on(stream, dev))
    if rc:
        _failed(handle, rc, [("H", H), ("G", G), ("U", U)], [("X", X), ("Wg", Wg), ("Wu", Wu)], workspace,
                lambda: _lib.shampoo_gated_ffn_workspace_bytes(rows, dim, width, dt))


def shampoo_gated_ffn_grad_workspace_bytes(rows, dim, width, dtype, g_dtype):
    return int(_lib.shampoo_gated_ffn_grad_workspace_bytes(int(rows), int(dim), int(width), _code(dtype),
                                                           _code(g_dtype)))


def shampoo_gated_ffn_grad(handle, X, Wg, Wu, dH, act=ACT_SILU, G=None, U=None, dX=None, dWg=None, dWu=None, beta=0.0,
                           workspace=None, stream=None):
    """Gradients of shampoo_gated_ffn from dH (rows x width): dX (X's shape and type, or
    None), dWg and dWu = beta dW + ... (Wg's shape, both fp32 or both bf16; both or
    neither).  G and U: the projections as kept, or None to form them again; workspace: uint8,
    shampoo_gated_ffn_grad_workspace_bytes(rows, dim, width, X.dtype, dWg.dtype) (without
    dWg: X.dtype twice)."""
    x, wg, wu, lh = _layout(X), _layout(Wg), _layout(Wu), None if dH is None else _layout(dH)
    lg, lu = None if G is None else _layout(G), None if U is None else _layout(U)
    ok = (x is not None and wg is not None and lh is not None and (G is None) == (U is None) and
          (dWg is None) == (dWu is None) and (dX is not None or dWg is not None))
    if ok:
        rows, dim, ld, dt, dev, ptr = x
        width = wg[1]
        dx = None if dX is None else _layout(dX)
        dg = None if dWg is None else _layout(dWg)
        du = None if dWu is None else _layout(dWu)
        gdt = dt if dg is None else dg[3]
        ok = (_fits(wg, dim, width, x) and _fits(wu, dim, width, x) and _fits(lh, rows, width, x) and
              (G is None or (_fits(lg, rows, width, x) and _fits(lu, rows, width, x))) and
              (dX is None or _fits(dx, rows, dim, x)) and
              (dWg is None or (dg is not None and dg[0] == dim and dg[1] == width and dg[4] == dev and
                               _fits(du, dim, width, dg))) and _on_handle(handle, dev) and
              _bytes_on(workspace, dev))
    if not ok:
        _need(dH is not None, "dH is required")
        _need((G is None) == (U is None), "G and U go together")
        _need((dWg is None) == (dWu is None), "dWg and dWu go together")
        _need(dX is not None or dWg is not None, "dX, or dWg and dWu, are required")
        _refuse_ffn(handle, X, Wg, Wu, (("dH", dH), ("G", G), ("U", U)),
                    (lambda r, d, w: _check_like(dX, "dX", r, d, X.dtype), lambda r, d, w: _check_like(dWg, "dWg", d, w),
                     lambda r, d, w: _check_like(dWu, "dWu", d, w, None if dWg is None else dWg.dtype)),
                    [("dX", dX), ("dWg", dWg), ("dWu", dWu)], [("dH", dH), ("G", G), ("U", U)],
                    lambda r, d, w: _lib.shampoo_gated_ffn_grad_workspace_bytes(
                        r, d, w, _code(X.dtype), _code(X.dtype if dWg is None else dWg.dtype)), workspace)
    rc = _lib.shampoo_gated_ffn_grad(
        handle, ptr, wg[5], wu[5], dt, rows, dim, width, ld, wg[2], wu[2], act, *_opt(lh), *_opt(lg), *_opt(lu),
        *_opt(dx), *_opt(dg), *_opt(du), gdt, beta, _ptr(workspace), 0 if workspace is None else workspace.numel(),
        _stream_on(stream, dev))
    if rc:
        _failed(handle, rc, [("dX", dX), ("dWg", dWg), ("dWu", dWu)],
                [("X", X), ("Wg", Wg), ("Wu", Wu), ("dH", dH), ("G", G), ("U", U)], workspace,
                lambda: _lib.shampoo_gated_ffn_grad_workspace_bytes(rows, dim, width, dt, gdt))


def shampoo_dropout(handle, X, Y, rate, seed, offset=0, R=None, stream=None):
    """Y = R + kept X / (1 - rate) (R None: zero); X, Y, R: one shape and type, fp32 or bf16
    (row-major views; Y may be X or R).  seed and offset (64-bit) give the mask; the
    gradient with respect to X is the same call on dY without R."""
    x, y, r = _layout(X), _layout(Y), None if R is None else _layout(R)
    if (x is None or not _fits(y, x[0], x[1], x) or not (R is None or _fits(r, x[0], x[1], x)) or
            not _on_handle(handle, x[4]) or not (0 <= seed < 1 << 64 and 0 <= offset < 1 << 64)):
        _need(0 <= seed < 1 << 64 and 0 <= offset < 1 << 64, f"seed {seed} or offset {offset} outside [0, 2^64)")
        _check_matrix(X, "X")
        _check_matrix(Y, "Y", X)
        _check_apart(Y, X, "Y and X", True)
        if R is not None:
            _check_matrix(R, "R", X)
            _check_apart(Y, R, "Y and R", True)
        _refuse(handle, (("X", X), ("Y", Y), ("R", R)), ())
    rows, cols, ld, dt, dev, ptr = x
    rc = _lib.shampoo_dropout(handle, ptr, None if r is None else r[5], y[5], dt, rows, cols, ld, 0 if r is None else r[2],
                              y[2], rate, seed, offset, _stream_on(stream, dev))
    if rc == SHAMPOO_EINVAL:
        _check_apart(Y, X, "Y and X", True)
        if R is not None:
            _check_apart(Y, R, "Y and R", True)
    _check(handle, rc)


def shampoo_timing_enable(handle, enable=True):
    _check(handle, _lib.shampoo_timing_enable(handle, int(bool(enable))))


def shampoo_timing_read(handle, kclass):
    ms, n = C.c_double(), C.c_int64()
    _check(handle, _lib.shampoo_timing_read(handle, int(kclass), C.byref(ms), C.byref(n)))
    return ms.value, n.value


def decode_root_info(info_tensor):
    """Host view of a root-info device array: list of dicts."""
    import numpy as np
    raw = info_tensor.detach().cpu().numpy().astype(np.int32).reshape(-1, 8)
    fl = raw.view(np.float32)
    out = []
    for r, f in zip(raw, fl):
        out.append(dict(status=int(r[0]), iters=int(r[1]), precision=int(r[2]), iters_fp32=int(r[3]),
                        resid=float(f[4]), lambda_max=float(f[5]), cond_est=float(f[6]), eps_eff=float(f[7])))
    return out
