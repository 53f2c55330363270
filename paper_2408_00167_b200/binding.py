"""ctypes binding of libfinch.so: the same entry points as include/finch.h, taking torch tensors.

Argument marshalling only -- every step of the path runs in the library's CUDA kernels.  torch is used for
device memory and stream handles.  Importing this module never builds anything; loading the library fails
loudly when libfinch.so is missing (build it with ``python -m paper_2408_00167_b200.build``).
"""
from __future__ import annotations

import ctypes as C
import struct
from dataclasses import dataclass
from pathlib import Path
from typing import Optional, Sequence

import numpy as np

import os

# FINCH_LIB lets a developer load an alternative build of the library (same ABI) for experiments
_LIB_PATH = Path(os.environ.get("FINCH_LIB") or Path(__file__).resolve().parent / "libfinch.so")
_lib = None

FINCH_OK = 0
FINCH_ERR_INVALID_ARG = 1
FINCH_ERR_UNSUPPORTED = 2
FINCH_ERR_BAD_LAYOUT = 3
FINCH_ERR_WORKSPACE_TOO_SMALL = 4
FINCH_ERR_OOM = 5
FINCH_ERR_CUDA = 6
FINCH_ERR_DEVICE_STATUS = 7
FINCH_F32, FINCH_BF16 = 0, 1
FINCH_GROUP_PER_KV_HEAD, FINCH_GROUP_PER_LAYER = 0, 1
FINCH_DEV_BAD_BATCH, FINCH_DEV_TIMEOUT, FINCH_DEV_BAD_INDEX = 1, 2, 4

EXPORTS = ("finch_ctx_create", "finch_ctx_destroy", "finch_workspace_bytes", "finch_score", "finch_select",
           "finch_compact", "finch_step", "finch_device_status", "finch_launch_count", "finch_status_string", "finch_score_static", "finch_score_static_max_rows", "finch_score_static_path",
           "finch_step_host", "finch_score_plan", "finch_rope_frequencies", "finch_rope_init", "finch_rotate",
           "finch_attend_workspace_bytes", "finch_attend_plan", "finch_attend", "finch_pages_append", "finch_pages_workspace_bytes", "finch_pages_attend")


class finch_config(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("dtype", C.c_int32), ("group_mode", C.c_int32), ("scale", C.c_float),
                ("max_batch", C.c_int32), ("max_prompt", C.c_int32), ("max_candidates", C.c_int32),
                ("device", C.c_int32), ("rope_theta", C.c_float), ("rope_pairing", C.c_int32)]


class finch_tensor(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("stride_layer", C.c_int64), ("stride_head", C.c_int64),
                ("stride_tok", C.c_int64)]


class finch_batch(C.Structure):
    _fields_ = [("batch", C.c_int32), ("q_off", C.c_void_p), ("chunk_off", C.c_void_p), ("cache_off", C.c_void_p),
                ("cache_len", C.c_void_p), ("budget", C.c_void_p), ("total_q", C.c_int32),
                ("total_chunk", C.c_int32), ("total_cache", C.c_int32), ("max_q", C.c_int32),
                ("max_cache", C.c_int32), ("max_chunk", C.c_int32), ("max_budget", C.c_int32),
                ("prompt_self_lse", C.c_void_p), ("row_limit", C.c_void_p),
                ("row_norm", C.c_int32)]


FINCH_PAGE_TOKENS = 64
FINCH_ROPE_PLAIN, FINCH_ROPE_LINEAR, FINCH_ROPE_BASE, FINCH_ROPE_PARTS = 0, 1, 2, 3


class finch_rope(C.Structure):
    _fields_ = [("rotary_dim", C.c_int32), ("pairing", C.c_int32), ("magnitude", C.c_float), ("reserved", C.c_int32),
                ("inv_freq", C.c_double * 128)]


class finch_pages(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("open_k", C.c_void_p), ("open_v", C.c_void_p), ("table", C.c_void_p), ("open_slot", C.c_void_p),
                ("n_pages", C.c_int32), ("table_width", C.c_int32), ("n_open", C.c_int32)]


class finch_paged_batch(C.Structure):
    _fields_ = [("batch", C.c_int32), ("q_off", C.c_void_p), ("new_off", C.c_void_p), ("len", C.c_void_p),
                ("total_q", C.c_int32), ("total_new", C.c_int32), ("max_q", C.c_int32), ("max_new", C.c_int32),
                ("max_len", C.c_int32)]


class FinchError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {finch_status_string(status)} (status {status})")


def load() -> C.CDLL:
    """Load libfinch.so; raises if it has not been built (there is no fallback path)."""
    global _lib
    if _lib is None:
        if not _LIB_PATH.exists():
            raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2408_00167_b200.build`")
        lib = C.CDLL(str(_LIB_PATH))
        for name in EXPORTS:
            getattr(lib, name).restype = C.c_int
        lib.finch_ctx_destroy.restype = None
        lib.finch_status_string.restype = C.c_char_p
        lib.finch_score_static_max_rows.restype = C.c_size_t
        # the calls of a step take addresses and sizes: declared, plain Python integers go in without wrapper objects
        p, z = C.c_void_p, C.c_size_t
        lib.finch_score.argtypes = [p] * 8 + [z, p]
        lib.finch_select.argtypes = [p] * 6 + [z, p]
        lib.finch_compact.argtypes = [p] * 14
        lib.finch_step.argtypes = [p] * 16 + [z, p]
        lib.finch_step_host.argtypes = [p] * 21 + [z, p]
        lib.finch_score_static.argtypes = [p] * 8
        i, f, d = C.c_int32, C.c_float, C.c_double
        lib.finch_rope_frequencies.argtypes = [i, d, i, d, d, d, d, p]
        lib.finch_rope_init.argtypes = [p, i, i, f, p]
        lib.finch_rotate.argtypes = [p, p, p, i, p, p, p, p, f, p, p, p]
        lib.finch_attend_workspace_bytes.argtypes = [p] * 3
        lib.finch_attend_plan.argtypes = [p] * 5
        lib.finch_attend.argtypes = [p] * 7 + [i, p, p, p, z, p]
        lib.finch_pages_append.argtypes = [p] * 9
        lib.finch_pages_workspace_bytes.argtypes = [p] * 3
        lib.finch_pages_attend.argtypes = [p] * 7 + [z, p]
        _lib = lib
    return _lib


def finch_status_string(status: int) -> str:
    return load().finch_status_string(C.c_int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != FINCH_OK:
        raise FinchError(status, where)


# ------------------------------------------------------------------ marshalling helpers

def _view(t):
    """[L][heads][tokens][d] torch tensor (head_dim contiguous) -> the four fields of a finch_tensor; None -> null view."""
    if t is None:
        return 0, 0, 0, 0
    s = t.stride()
    if len(s) != 4 or (s[3] != 1 and t.shape[3] > 1):
        raise ValueError("expected a [layers][heads][tokens][head_dim] tensor with head_dim contiguous")
    return t.data_ptr(), s[0], s[1], s[2]     # data_ptr() of an empty tensor is 0


_VIEW_BYTES = C.sizeof(finch_tensor)
_packs = {}


def _views(*tensors):
    """The tensors as consecutive finch_tensor structs: (buffer to keep alive, address of the first)."""
    n = len(tensors)
    pack = _packs.get(n)
    if pack is None:
        pack = _packs[n] = (struct.Struct("=" + "Qqqq" * n), C.c_char * (n * _VIEW_BYTES))
    buf = pack[1]()
    fields = []
    for t in tensors:
        fields += _view(t)
    pack[0].pack_into(buf, 0, *fields)
    return buf, C.addressof(buf)


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr() or None


def _nbytes(t) -> int:
    return 0 if t is None else t.numel() * t.element_size()


_current_stream = None


def _stream(stream) -> Optional[int]:
    global _current_stream
    if stream is not None:
        return stream.cuda_stream or None
    if _current_stream is None:
        import torch
        torch.cuda.current_stream()           # initialises torch's side of CUDA
        raw, device = (getattr(torch._C, n, None) for n in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))
        if raw and device:                    # the handle itself, without a Stream object around it
            _current_stream = lambda: raw(device())
        else:
            _current_stream = lambda: torch.cuda.current_stream().cuda_stream
    return _current_stream() or None


def device_of(device):
    """The torch.device with its index: "cuda" alone is the device that is current now, and what is made later belongs beside it."""
    import torch
    device = torch.device(device)
    return torch.device("cuda", torch.cuda.current_device()) if device.type == "cuda" and device.index is None else device


@dataclass
class Batch:
    """Device-side batch metadata plus the host bounds finch_batch carries."""
    q_off: object
    chunk_off: object
    cache_off: object
    cache_len: object
    budget: object
    c: finch_batch
    prompt_self_lse: object = None   # keeps the optional device tensors alive
    row_limit: object = None

    @property
    def batch(self) -> int:
        return self.c.batch


def make_batch(q_off: Sequence[int], chunk_off: Sequence[int], cache_off: Sequence[int], cache_len: Sequence[int],
               budget: Sequence[int], device="cuda", prompt_self_lse=None, row_limit=None, row_norm=False) -> Batch:
    """Copy the offset arrays to the device and fill in the host bounds.  prompt_self_lse: optional device tensor
    [n_layers][n_q_heads][total_q] fp32; row_limit: optional device tensor [total_q] int32 (see finch_batch in the
    header)."""
    import torch
    h = [np.ascontiguousarray(a, dtype=np.int32) for a in (q_off, chunk_off, cache_off, cache_len, budget)]
    B = len(h[3])
    assert len(h[0]) == len(h[1]) == len(h[2]) == B + 1 and len(h[4]) == B
    d = [torch.from_numpy(a).to(device) for a in h]

    def diff(a):
        return (a[1:] - a[:-1]) if B else np.zeros(0, np.int32)

    def mx(a):
        return int(a.max()) if len(a) else 0
    n_cand = h[3] + diff(h[1])
    cb = finch_batch(B, *[x.data_ptr() for x in d], int(h[0][B]), int(h[1][B]), int(h[2][B]),
                     mx(diff(h[0])), mx(h[3]), mx(diff(h[1])), mx(np.minimum(h[4], n_cand)) if B else 0,
                     prompt_self_lse.data_ptr() if prompt_self_lse is not None else None,
                     row_limit.data_ptr() if row_limit is not None else None, int(bool(row_norm)))
    return Batch(*d, cb, prompt_self_lse, row_limit)


# ------------------------------------------------------------------ the entry points

def finch_ctx_create(n_layers, n_q_heads, n_kv_heads, head_dim, dtype, group_mode=FINCH_GROUP_PER_KV_HEAD, scale=0.0,
                     max_batch=1, max_prompt=256, max_candidates=8192, device=0, rope_theta=0.0,
                     rope_pairing=0) -> C.c_void_p:
    cfg = finch_config(n_layers, n_q_heads, n_kv_heads, head_dim, dtype, group_mode, scale, max_batch, max_prompt,
                       max_candidates, device, rope_theta, rope_pairing)
    ctx = C.c_void_p()
    _check(load().finch_ctx_create(C.byref(cfg), C.byref(ctx)), "finch_ctx_create")
    # what the operators' tensors have to be: a call takes addresses and strides, the sizes are the context's
    ctx.model = n_layers, n_q_heads, n_kv_heads, head_dim, int(dtype), int(device)
    ctx.pages = n_layers, n_kv_heads, head_dim, int(dtype), int(device)
    return ctx


def finch_ctx_destroy(ctx) -> None:
    if ctx:
        load().finch_ctx_destroy(ctx)


def finch_workspace_bytes(ctx, batch: Batch) -> int:
    out = C.c_size_t()
    _check(load().finch_workspace_bytes(ctx, C.byref(batch.c), C.byref(out)), "finch_workspace_bytes")
    return int(out.value)


def finch_score(ctx, prompt_q, cache_k, chunk_k, batch: Batch, scores, row_lse=None, ws=None, stream=None) -> None:
    keep, v = _views(prompt_q, cache_k, chunk_k)
    _check(load().finch_score(ctx, v, v + _VIEW_BYTES, v + 2 * _VIEW_BYTES, C.addressof(batch.c), _ptr(scores), _ptr(row_lse),
                              _ptr(ws), _nbytes(ws), _stream(stream)), "finch_score")


def finch_select(ctx, scores, batch: Batch, kept_idx, out_len, ws=None, stream=None) -> None:
    _check(load().finch_select(ctx, _ptr(scores), C.addressof(batch.c), _ptr(kept_idx), _ptr(out_len), _ptr(ws),
                               _nbytes(ws), _stream(stream)), "finch_select")


def finch_compact(ctx, kept_idx, out_len, cache_k, cache_v, cache_pos, chunk_k, chunk_v, chunk_pos, batch: Batch,
                  out_k, out_v, out_pos, stream=None) -> None:
    keep, v = _views(cache_k, cache_v, chunk_k, chunk_v, out_k, out_v)
    z = _VIEW_BYTES
    _check(load().finch_compact(ctx, _ptr(kept_idx), _ptr(out_len), v, v + z, _ptr(cache_pos), v + 2 * z, v + 3 * z,
                                _ptr(chunk_pos), C.addressof(batch.c), v + 4 * z, v + 5 * z, _ptr(out_pos),
                                _stream(stream)), "finch_compact")


def finch_step(ctx, prompt_q, cache_k, cache_v, cache_pos, chunk_k, chunk_v, chunk_pos, batch: Batch, out_k, out_v,
               out_pos, kept_idx, out_len, scores=None, ws=None, stream=None) -> None:
    keep, v = _views(prompt_q, cache_k, cache_v, chunk_k, chunk_v, out_k, out_v)
    z = _VIEW_BYTES
    _check(load().finch_step(ctx, v, v + z, v + 2 * z, _ptr(cache_pos), v + 3 * z, v + 4 * z, _ptr(chunk_pos),
                             C.addressof(batch.c), v + 5 * z, v + 6 * z, _ptr(out_pos), _ptr(kept_idx), _ptr(out_len),
                             _ptr(scores), _ptr(ws), _nbytes(ws), _stream(stream)), "finch_step")


def finch_device_status(ctx, stream=None) -> int:
    """Synchronises the stream and returns the status word (0 = clean); the word is cleared."""
    out = C.c_int32()
    st = load().finch_device_status(ctx, C.c_void_p(_stream(stream)), C.byref(out))
    if st not in (FINCH_OK, FINCH_ERR_DEVICE_STATUS):
        raise FinchError(st, "finch_device_status")
    return int(out.value)


def finch_launch_count(ctx) -> int:
    """Kernels enqueued through this context since it was created."""
    out = C.c_uint64()
    _check(load().finch_launch_count(ctx, C.byref(out)), "finch_launch_count")
    return int(out.value)


def finch_score_static(ctx, prompt_q, cache_k, chunk_k, batch: Batch, scores, row_lse=None, stream=None) -> None:
    """finch_score without a workspace: the scratch is a fixed array inside the library (see finch.h for the
    row limit and the sharing rules).  For callers that may not allocate device memory."""
    keep, v = _views(prompt_q, cache_k, chunk_k)
    _check(load().finch_score_static(ctx, v, v + _VIEW_BYTES, v + 2 * _VIEW_BYTES, C.addressof(batch.c), _ptr(scores),
                                     _ptr(row_lse), _stream(stream)), "finch_score_static")


def finch_score_static_max_rows() -> int:
    return int(load().finch_score_static_max_rows())


FINCH_SCORE_WARP_LEVEL, FINCH_SCORE_TWO_LAUNCH, FINCH_SCORE_ONE_KERNEL = 0, 1, 2


def finch_score_plan(ctx, batch: Batch):
    """(path, window): which kernels finch_score / finch_step run for this batch and, on the one-kernel path, the
    window length in key tiles."""
    path, window = C.c_int32(), C.c_int32()
    _check(load().finch_score_plan(ctx, C.byref(batch.c), C.byref(path), C.byref(window)), "finch_score_plan")
    return path.value, window.value


def finch_score_static_path(ctx, batch: Batch) -> bool:
    """True when finch_score_static would run this batch on the tensor-core kernels, False: warp-level kernels."""
    out = C.c_int32()
    _check(load().finch_score_static_path(ctx, C.byref(batch.c), C.byref(out)), "finch_score_static_path")
    return bool(out.value)


def finch_step_host(ctx, host_prompt_q, host_chunk_k, host_chunk_v, host_chunk_pos, stage_q, stage_chunk_k,
                    stage_chunk_v, stage_chunk_pos, cache_k, cache_v, cache_pos, batch: Batch, out_k, out_v, out_pos,
                    kept_idx, out_len, host_kept_idx, host_out_len, ws, stream=None) -> None:
    """finch_step with this step's inputs in host memory (torch CPU tensors, ideally pinned) and the kept indices
    and lengths returned to host tensors; the call returns after the stream has finished."""
    keep, v = _views(stage_q, stage_chunk_k, stage_chunk_v, cache_k, cache_v, out_k, out_v)
    z = _VIEW_BYTES
    _check(load().finch_step_host(
        ctx, _ptr(host_prompt_q), _ptr(host_chunk_k), _ptr(host_chunk_v), _ptr(host_chunk_pos), v, v + z, v + 2 * z,
        _ptr(stage_chunk_pos), v + 3 * z, v + 4 * z, _ptr(cache_pos), C.addressof(batch.c), v + 5 * z, v + 6 * z,
        _ptr(out_pos), _ptr(kept_idx), _ptr(out_len), _ptr(host_kept_idx), _ptr(host_out_len), _ptr(ws), _nbytes(ws),
        _stream(stream)), "finch_step_host")


# ------------------------------------------------------------------ rotation, attention, the paged 8-bit cache

def _model(what: str, ctx, like, q, kv):
    """(n_layers, n_q_heads, n_kv_heads, head_dim) of a context, which `like` has to fit in type and device.  Of a handle that
    finch_ctx_create of this module has not made, the tensors' own sizes have to do."""
    m = getattr(ctx, "model", None)
    if m is None:
        shapes = [t.shape for t in (q, kv) if t is not None]
        if not shapes or any(len(s) != 4 for s in shapes):
            raise ValueError(f"{what}: expected [layers][heads][tokens][head_dim] tensors")
        return shapes[0][0], shapes[0][1], shapes[-1][1], shapes[0][3]
    L, Hq, Hkv, d, code, device = m
    dtype = (_dtypes or _dtypes_of())[2 + code]
    if like.dtype != dtype or (device >= 0 and like.get_device() != device):
        raise ValueError(f"{what}: the context is for {dtype} on device {device}, got {like.dtype} on {like.device}")
    return L, Hq, Hkv, d


def _views_like(what: str, like, *tensors):
    """_views of tensors that have to be on `like`'s device and of its dtype: a kernel would read the bits of another one all the
    same.  The checks of a call are most of what it takes on the host, hence one pass over the tensors."""
    n = len(tensors)
    pack = _packs.get(n)
    if pack is None:
        pack = _packs[n] = (struct.Struct("=" + "Qqqq" * n), C.c_char * (n * _VIEW_BYTES))
    buf = pack[1]()
    dtype, device = like.dtype, like.get_device()
    fields = []
    for t in tensors:
        if t is None:
            fields += (0, 0, 0, 0)
            continue
        if t.dtype != dtype or t.get_device() != device:
            raise ValueError(f"{what}: expected {dtype} on {like.device}, got {t.dtype} on {t.device}")
        st = t.stride()
        if len(st) != 4 or (st[3] != 1 and t.shape[3] > 1):
            raise ValueError(f"{what}: expected a [layers][heads][tokens][head_dim] tensor with head_dim contiguous")
        fields += (t.data_ptr(), st[0], st[1], st[2])
    pack[0].pack_into(buf, 0, *fields)
    return buf, C.addressof(buf)


def _holds(what: str, shape, want) -> None:
    """A tensor of four axes has `want`'s sizes, and rows at least: a kernel reads and writes behind the end of one that has fewer."""
    if want[2] and (len(shape) != 4 or shape[2] < want[2] or (shape[0], shape[1], shape[3]) != (want[0], want[1], want[3])):
        raise ValueError(f"{what}: expected {want} or more rows, got {tuple(shape)}")


def _space(what: str, ws, like):
    """Address and bytes of a workspace on `like`'s device."""
    if ws is None:
        return None, 0
    if ws.get_device() != like.get_device() or not ws.is_contiguous():
        raise ValueError(f"{what}: expected a contiguous workspace on {like.device}, got one on {ws.device}")
    return ws.data_ptr() or None, ws.numel() * ws.element_size()


def _array(what: str, t, dtype, like, shape):
    """Address of a contiguous tensor of the given dtype and shape on `like`'s device; None: none."""
    if t is None:
        return None
    if t.dtype != dtype or t.get_device() != like.get_device() or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what}: expected a contiguous {dtype} tensor of shape {tuple(shape)} on {like.device}, got {t.dtype} of "
                         f"{tuple(t.shape)} on {t.device}")
    return t.data_ptr() or None


def _rows_of(what: str, t, dtype, like, n: int) -> None:
    """An array of the batch description: n entries, or at least so many where it has one axis (more axes of other sizes would be read
    with the wrong pitch)."""
    if t.dtype != dtype or t.get_device() != like.get_device() or not t.is_contiguous() or t.numel() < n or (t.dim() > 1 and t.numel() != n):
        raise ValueError(f"{what}: expected {n} contiguous {dtype} on {like.device}, got {t.dtype} of {tuple(t.shape)} on {t.device}")


def _same_shape(what: str, t, shape) -> None:
    if t.shape != shape:
        raise ValueError(f"{what}: expected shape {tuple(shape)}, got {tuple(t.shape)}")


_dtypes = None


def _dtypes_of():
    """int32, float32, and the types of FINCH_F32 and FINCH_BF16."""
    global _dtypes
    if _dtypes is None:
        import torch
        _dtypes = torch.int32, torch.float32, torch.float32, torch.bfloat16
    return _dtypes


def finch_rope_frequencies(rotary_dim: int, theta: float = 10000.0, scaling: int = FINCH_ROPE_PLAIN, factor: float = 1.0,
                           original: float = 8192.0, low: float = 1.0, high: float = 4.0):
    """Angle per position of every pair, float64 [rotary_dim / 2] (see the header for the scalings)."""
    out = np.zeros(max(rotary_dim // 2, 1), dtype=np.float64)
    _check(load().finch_rope_frequencies(rotary_dim, theta, scaling, factor, original, low, high, out.ctypes.data),
           "finch_rope_frequencies")
    return out


def finch_rope_init(rotary_dim: int, inv_freq, pairing: int = 0, magnitude: float = 1.0) -> finch_rope:
    freq = np.ascontiguousarray(inv_freq, dtype=np.float64)
    if freq.shape != (rotary_dim // 2,):
        raise ValueError(f"expected {rotary_dim // 2} frequencies, got shape {freq.shape}")
    rope = finch_rope()
    _check(load().finch_rope_init(C.addressof(rope), rotary_dim, pairing, magnitude, freq.ctypes.data), "finch_rope_init")
    return rope


def _rope(rope) -> Optional[int]:
    return None if rope is None else C.addressof(rope)


def finch_rotate(ctx, q, k, pos, out_q, out_k, rope: Optional[finch_rope] = None, q_weight=None, k_weight=None, eps: float = 1e-6,
                 stream=None) -> None:
    """Norm (with weights) and rotation (with rope and positions) of q and k, [n_layers][heads][tokens][head_dim]; either may be
    None, together with its output."""
    like = q if q is not None else k
    if like is None or (q is None) != (out_q is None) or (k is None) != (out_k is None):
        raise ValueError("finch_rotate: q, k or both, each with its output")
    keep, v = _views_like("finch_rotate", like, q, k, out_q, out_k)
    L, Hq, Hkv, d = _model("finch_rotate", ctx, like, q, k)
    shape = like.shape
    tokens = shape[2]
    if q is not None:
        if shape != (L, Hq, tokens, d) or out_q.shape != shape:
            raise ValueError(f"finch_rotate: expected q and out_q of {(L, Hq, tokens, d)}, got {tuple(shape)}, {tuple(out_q.shape)}")
    if k is not None:
        shape = k.shape
        if shape != (L, Hkv, tokens, d) or out_k.shape != shape:
            raise ValueError(f"finch_rotate: expected k and out_k of {(L, Hkv, tokens, d)}, got {tuple(shape)}, {tuple(out_k.shape)}")
    z, dtype = _VIEW_BYTES, like.dtype
    _check(load().finch_rotate(ctx, v, v + z, tokens, _array("finch_rotate: pos", pos, _dtypes_of()[0], like, (tokens,)), _rope(rope),
                               _array("finch_rotate: q_weight", q_weight, dtype, like, (L, d)),
                               _array("finch_rotate: k_weight", k_weight, dtype, like, (L, d)), eps, v + 2 * z, v + 3 * z,
                               _stream(stream)), "finch_rotate")


def finch_attend_workspace_bytes(ctx, batch: Batch) -> int:
    out = C.c_size_t()
    _check(load().finch_attend_workspace_bytes(ctx, C.addressof(batch.c), C.addressof(out)), "finch_attend_workspace_bytes")
    return int(out.value)


FINCH_ATTEND_MULTIPLY_ADD, FINCH_ATTEND_ONE_STREAM, FINCH_ATTEND_ROW_PAIRS, FINCH_ATTEND_KEY_PAIRS = 0, 1, 2, 3


def finch_attend_plan(ctx, batch: Batch):
    """(path, cluster, splits): how finch_attend shares out this batch (see the header)."""
    out = [C.c_int32() for _ in range(3)]
    _check(load().finch_attend_plan(ctx, C.addressof(batch.c), *map(C.addressof, out)), "finch_attend_plan")
    return tuple(x.value for x in out)


def finch_attend(ctx, q, cache_k, cache_v, chunk_k, chunk_v, batch: Batch, out, row_lse=None, causal: bool = True, ws=None,
                 stream=None) -> None:
    """Attention of the packed query rows over [cache ; chunk] (see the header).  Tensors hold the batch's rows (total_q, total_cache,
    total_chunk) or more; `out` has q's shape, row_lse is [n_layers][n_q_heads][total_q]."""
    keep, v = _views_like("finch_attend", q, q, cache_k, cache_v, chunk_k, chunk_v, out)
    L, Hq, Hkv, d = _model("finch_attend", ctx, q, q, chunk_k if chunk_k is not None else cache_k)
    c, shape = batch.c, q.shape
    rows = c.total_q
    if shape != (L, Hq, rows, d):
        _holds("finch_attend: q", shape, (L, Hq, rows, d))
    if out.shape != shape:
        _same_shape("finch_attend: out", out, shape)
    for n, k, value in ((c.total_cache, cache_k, cache_v), (c.total_chunk, chunk_k, chunk_v)):
        if n and k is not None and value is not None:       # the library refuses what is missing
            want = L, Hkv, n, d
            if k.shape != want:
                _holds("finch_attend: keys", k.shape, want)
            if value.shape != want:
                _holds("finch_attend: values", value.shape, want)
    f32 = _dtypes_of()[1]
    if batch.q_off.get_device() != q.get_device():
        raise ValueError(f"finch_attend: the batch description is on {batch.q_off.device}, the tensors on {q.device}")
    if batch.prompt_self_lse is not None:
        _rows_of("finch_attend: prompt_self_lse", batch.prompt_self_lse, f32, q, L * Hq * rows)
    if batch.row_limit is not None:
        _rows_of("finch_attend: row_limit", batch.row_limit, _dtypes_of()[0], q, rows)
    z = _VIEW_BYTES
    ws, ws_bytes = _space("finch_attend", ws, q)
    _check(load().finch_attend(ctx, v, v + z, v + 2 * z, v + 3 * z, v + 4 * z, C.addressof(c), 1 if causal else 0, v + 5 * z,
                               _array("finch_attend: row_lse", row_lse, f32, q, (L, Hq, rows)), ws, ws_bytes,
                               _stream(stream)), "finch_attend")


@dataclass
class Pages:
    """The tensors of a paged cache and the finch_pages that describes them."""
    tensors: tuple
    c: finch_pages
    kind: tuple = ()     # n_layers, n_kv_heads, head_dim, dtype, device index: those of a context
    requests: int = 0    # rows of the page table


def make_pages(k, v, k_scale, v_scale, open_k, open_v, table, open_slot=None) -> Pages:
    """k, v: uint8 [n_layers][n_pages][n_kv_heads][64][head_dim]; scales: float32 [n_layers][n_pages][n_kv_heads]; open_k, open_v:
    [n_layers][n_open][n_kv_heads][64][head_dim] in the context's dtype; table: int32 [batch][table_width]; open_slot: int32 [batch]."""
    import torch
    L, n_pages, Hkv, page, d = k.shape
    n_open = open_k.shape[1]
    for name, t, dtype, shape in (("k", k, torch.uint8, k.shape), ("v", v, torch.uint8, k.shape),
                                  ("k_scale", k_scale, torch.float32, (L, n_pages, Hkv)),
                                  ("v_scale", v_scale, torch.float32, (L, n_pages, Hkv)),
                                  ("open_k", open_k, open_k.dtype, (L, n_open, Hkv, page, d)),
                                  ("open_v", open_v, open_k.dtype, (L, n_open, Hkv, page, d)),
                                  ("table", table, torch.int32, (table.shape[0], table.shape[-1])),
                                  ("open_slot", open_slot, torch.int32, (table.shape[0],))):
        if t is None and name == "open_slot":
            continue
        if t.dtype != dtype or t.device != k.device or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
            raise ValueError(f"make_pages: {name} is to be contiguous {dtype} {tuple(shape)} on {k.device}, got {t.dtype} {tuple(t.shape)}")
    if open_k.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError(f"make_pages: open rows are float32 or bfloat16, got {open_k.dtype}")
    if page != FINCH_PAGE_TOKENS:
        raise ValueError(f"make_pages: a page has {FINCH_PAGE_TOKENS} tokens, got {page}")
    tensors = (k, v, k_scale, v_scale, open_k, open_v, table, open_slot)
    kind = L, Hkv, d, FINCH_F32 if open_k.dtype == torch.float32 else FINCH_BF16, k.get_device()
    return Pages(tensors, finch_pages(*map(_ptr, tensors), n_pages, table.shape[1], n_open), kind, table.shape[0])


def _check_paged(what: str, ctx, pages: Pages, batch: "PagedBatch") -> None:
    """The pages are of the context's model and device, and their table has the batch's requests."""
    kind = getattr(ctx, "pages", None)
    if kind is not None and pages.kind != kind and (pages.kind[:4] != kind[:4] or kind[4] >= 0):
        raise ValueError(f"{what}: layers, KV heads, head_dim, dtype and device of the pages are {pages.kind}, of the context {kind}")
    if batch.c.batch > pages.requests or batch.device != pages.kind[4]:
        raise ValueError(f"{what}: {batch.c.batch} requests on device {batch.device}, a page table of {pages.requests} on {pages.kind[4]}")


@dataclass
class PagedBatch:
    """Device-side metadata of a call on a paged cache plus the host bounds finch_paged_batch carries."""
    q_off: object
    new_off: object
    len: object
    c: finch_paged_batch
    device: int = -1     # index

    @property
    def batch(self) -> int:
        return self.c.batch


def make_paged_batch(lengths: Sequence[int], q_off: Optional[Sequence[int]] = None, new_off: Optional[Sequence[int]] = None,
                     device="cuda", len_tensor=None, max_len: Optional[int] = None) -> PagedBatch:
    """lengths: tokens of each request in the cache (for an append, before it).  len_tensor: a device tensor that holds them
    instead (a length that an earlier append wrote), with max_len as the bound on them."""
    import torch
    h = np.ascontiguousarray(lengths, dtype=np.int32)
    B = len(h)
    d_len = torch.from_numpy(h).to(device) if len_tensor is None else len_tensor
    if d_len.dtype != torch.int32 or not d_len.is_contiguous() or d_len.numel() < B:
        raise ValueError("make_paged_batch: lengths are contiguous int32, one for each request")
    offs = []
    for off in (q_off, new_off):
        if off is None:
            offs.append((None, 0, 0))
            continue
        o = np.ascontiguousarray(off, dtype=np.int32)
        assert len(o) == B + 1
        offs.append((torch.from_numpy(o).to(device), int(o[B]), int(np.diff(o).max()) if B else 0))
    if any(t is not None and t.get_device() != d_len.get_device() for t, _, _ in offs):
        raise ValueError(f"make_paged_batch: lengths on {d_len.device}, offsets on {device}")
    longest = (int(h.max()) if B else 0) if max_len is None else int(max_len)
    c = finch_paged_batch(B, _ptr(offs[0][0]), _ptr(offs[1][0]), _ptr(d_len), offs[0][1], offs[1][1], offs[0][2], offs[1][2], longest)
    return PagedBatch(offs[0][0], offs[1][0], d_len, c, d_len.get_device())


def finch_pages_append(ctx, pages: Pages, batch: PagedBatch, new_k, new_v, out_len=None, rope: Optional[finch_rope] = None, pos=None,
                       stream=None) -> None:
    """Rows of new_k (turned to their positions with rope) and new_v, total_new or more, behind each request's tokens (see the header)."""
    c, kind = batch.c, pages.kind
    if getattr(ctx, "pages", None) != kind or c.batch > pages.requests or batch.device != kind[4]:
        _check_paged("finch_pages_append", ctx, pages, batch)
    like, rows = pages.tensors[4], c.total_new
    keep, v = _views_like("finch_pages_append", like, new_k, new_v)
    if rows and new_k is not None and new_v is not None:        # the library refuses what is missing
        want = kind[0], kind[1], rows, kind[2]
        if new_k.shape != want:
            _holds("finch_pages_append: new_k", new_k.shape, want)
        if new_v.shape != want:
            _holds("finch_pages_append: new_v", new_v.shape, want)
    i32 = _dtypes_of()[0]
    _check(load().finch_pages_append(ctx, C.addressof(pages.c), C.addressof(c), v, v + _VIEW_BYTES, _rope(rope),
                                     None if pos is None else _array("finch_pages_append: pos", pos, i32, like, new_k.shape[2:3]),
                                     _array("finch_pages_append: out_len", out_len, i32, like, (c.batch,)), _stream(stream)),
           "finch_pages_append")


def finch_pages_workspace_bytes(ctx, batch: PagedBatch) -> int:
    out = C.c_size_t()
    _check(load().finch_pages_workspace_bytes(ctx, C.addressof(batch.c), C.addressof(out)), "finch_pages_workspace_bytes")
    return int(out.value)


def finch_pages_attend(ctx, pages: Pages, batch: PagedBatch, q, out, row_lse=None, ws=None, stream=None) -> None:
    """Attention of each request's newest tokens over its paged cache (see the header).  q holds the batch's total_q rows or more;
    `out` has q's shape, row_lse is [n_layers][n_q_heads][total_q]."""
    c, kind = batch.c, pages.kind
    if getattr(ctx, "pages", None) != kind or c.batch > pages.requests or batch.device != kind[4]:
        _check_paged("finch_pages_attend", ctx, pages, batch)
    keep, v = _views_like("finch_pages_attend", pages.tensors[4], q, out)
    rows, shape, m = c.total_q, q.shape, getattr(ctx, "model", None)
    L, Hq = kind[0], m[1] if m is not None else shape[1]
    if shape != (L, Hq, rows, kind[2]):
        _holds("finch_pages_attend: q", shape, (L, Hq, rows, kind[2]))
    if out.shape != shape:
        _same_shape("finch_pages_attend: out", out, shape)
    ws, ws_bytes = _space("finch_pages_attend", ws, q)
    _check(load().finch_pages_attend(ctx, C.addressof(pages.c), C.addressof(c), v, v + _VIEW_BYTES,
                                     _array("finch_pages_attend: row_lse", row_lse, _dtypes_of()[1], q, (L, Hq, rows)), ws, ws_bytes,
                                     _stream(stream)), "finch_pages_attend")
