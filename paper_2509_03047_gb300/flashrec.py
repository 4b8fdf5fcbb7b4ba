"""Thin ctypes binding of libflashrec (include/flashrec.h), same names as the C ABI.

Argument marshalling only: every step of the sweep runs in the library's CUDA
kernels.  PyTorch supplies device memory and streams.  If the compiled library
is missing or cannot be loaded, importing this module raises -- there is no
fallback of any kind.
"""
from __future__ import annotations

import array
import contextlib
import ctypes
import os
from typing import List, Optional, Sequence

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libflashrec.so")

FR_OK = 0
FR_ERR_INVALID_ARG = 1
FR_ERR_ALIGNMENT = 2
FR_ERR_BUFFER_TOO_SMALL = 3
FR_ERR_CAPACITY = 4
FR_ERR_PLAN_MISMATCH = 5
FR_ERR_DEVICE_TIMEOUT = 6
FR_ERR_CUDA = 7

FR_DT_BYTES, FR_DT_BF16, FR_DT_F32 = 0, 1, 2
FP_ENTRY_BYTES = 16
FR_OPT_BLOCK = 256
FR_ROUND_NEAREST, FR_ROUND_RANDOM = 0, 1
FR_MUON_MOST, FR_MUON_MOST_SIDE = 10, 1 << 20
FR_MUON_BY_TYPE, FR_MUON_ONE = 0, 1
FR_MUON_BOTH_HALVES = 2
CLIP_BYTES = 16

_TORCH_TO_FR = {torch.bfloat16: FR_DT_BF16, torch.float32: FR_DT_F32, torch.uint8: FR_DT_BYTES,
                torch.int8: FR_DT_BYTES}


class fr_tensor(ctypes.Structure):
    _fields_ = [("ptr", ctypes.c_void_p), ("nbytes", ctypes.c_uint64), ("dtype", ctypes.c_uint32),
                ("flags", ctypes.c_uint32)]


class fr_piece(ctypes.Structure):
    _fields_ = [("source", ctypes.c_uint32), ("reserved", ctypes.c_uint32), ("src_off", ctypes.c_uint64),
                ("dst_off", ctypes.c_uint64), ("nbytes", ctypes.c_uint64)]


class fr_opt_tensor(ctypes.Structure):
    _fields_ = [("weight", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("master", ctypes.c_void_p),
                ("m", ctypes.c_void_p), ("v", ctypes.c_void_p), ("m_exp", ctypes.c_void_p), ("v_exp", ctypes.c_void_p),
                ("n", ctypes.c_uint64), ("weight_dtype", ctypes.c_uint32), ("grad_dtype", ctypes.c_uint32),
                ("state_dtype", ctypes.c_uint32), ("flags", ctypes.c_uint32), ("lr_scale", ctypes.c_float),
                ("decay_scale", ctypes.c_float)]


class fr_adamw(ctypes.Structure):
    """One step's numbers; a training loop keeps one and counts `step` up."""
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
                ("weight_decay", ctypes.c_double), ("step", ctypes.c_uint64), ("seed", ctypes.c_uint64),
                ("rounding", ctypes.c_uint32), ("reserved", ctypes.c_uint32)]


class fr_muon_tensor(ctypes.Structure):
    _fields_ = [("weight", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("master", ctypes.c_void_p),
                ("momentum", ctypes.c_void_p), ("update", ctypes.c_void_p), ("rows", ctypes.c_uint64),
                ("cols", ctypes.c_uint64), ("weight_dtype", ctypes.c_uint32), ("grad_dtype", ctypes.c_uint32),
                ("update_dtype", ctypes.c_uint32), ("flags", ctypes.c_uint32), ("lr_scale", ctypes.c_float),
                ("decay_scale", ctypes.c_float), ("update_scale", ctypes.c_float), ("reserved", ctypes.c_uint32)]


class fr_muon(ctypes.Structure):
    """One step's numbers (see muon()); a training loop keeps one and counts `step` up."""
    _fields_ = [("lr", ctypes.c_double), ("beta", ctypes.c_double), ("weight_decay", ctypes.c_double),
                ("coef", ctypes.c_double * 3 * FR_MUON_MOST), ("step", ctypes.c_uint64), ("seed", ctypes.c_uint64),
                ("iterations", ctypes.c_uint32), ("nesterov", ctypes.c_uint32), ("rounding", ctypes.c_uint32),
                ("products", ctypes.c_uint32)]


class FlashrecError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s: %s (%s)" % (where, fr_status_str(status), fr_last_error()))


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError("libflashrec.so is not built (%s); run __graft_entry__.build()" % LIB_PATH)
    L = ctypes.CDLL(LIB_PATH)
    vp, u64, u32 = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_uint32
    u64p = ctypes.POINTER(ctypes.c_uint64)
    L.fr_plan_create.argtypes = [ctypes.POINTER(fr_tensor), u64, u64, ctypes.POINTER(vp)]
    L.fr_plan_info.argtypes = [vp, u64p, u64p, u64p]
    L.fr_plan_chunk.argtypes = [vp, u64, ctypes.POINTER(u32), u64p, u64p, u64p]
    L.fr_plan_destroy.argtypes = [vp]
    L.fr_plan_destroy.restype = None
    L.fr_fingerprint.argtypes = [vp, vp, vp]
    L.fr_pack.argtypes = [vp, vp, u64, vp]
    L.fr_unpack_verify.argtypes = [vp, vp, u64, vp, u64, vp, vp]
    L.fr_diff.argtypes = [vp, vp, u64, vp, u64, vp, vp]
    L.fr_sync_status.argtypes = [vp, vp]
    L.fr_fingerprint_static.argtypes = [ctypes.POINTER(fr_tensor), u64, u64, vp, vp]
    L.fr_plan_create_batched.argtypes = [ctypes.POINTER(fr_tensor), u64, u64, u32, ctypes.POINTER(vp)]
    L.fr_plan_batch.argtypes = [vp, u32, ctypes.POINTER(u32), u64p, u64p]
    L.fr_pack_batch.argtypes = [vp, u32, vp, u64, vp]
    L.fr_unpack_verify_batch.argtypes = [vp, u32, vp, u64, vp]
    L.fr_unpack_collect.argtypes = [vp, vp, u64, vp, vp]
    L.fr_resend.argtypes = [vp, vp, vp, u64, u64p, vp, vp]
    L.fr_restore.argtypes = [vp, vp, vp, u64, u32, vp, u64, vp, vp, vp]
    L.fr_shard_pieces.argtypes = [u64, u32, u32, u32, u32, ctypes.POINTER(fr_piece), u64, u64p]
    L.fr_pack_fp.argtypes = [vp, vp, u64, vp, vp]
    L.fr_unpack_verify_fp.argtypes = [vp, vp, u64, vp, u64, vp, vp, vp]
    L.fr_restore_fp.argtypes = [vp, vp, vp, u64, u32, vp, u64, vp, vp, vp, vp, vp]
    L.fr_resend_fp.argtypes = [vp, vp, vp, u64, u64p, vp, vp, vp, vp]
    L.fr_restore_multi.argtypes = [ctypes.POINTER(vp), u32, vp, vp, u64, u32, vp, u64, vp, vp,
                                   ctypes.POINTER(vp), vp]
    L.fr_opt_create.argtypes = [ctypes.POINTER(fr_opt_tensor), u64, ctypes.POINTER(vp)]
    L.fr_opt_info.argtypes = [vp, u64p, u64p, u64p]
    L.fr_opt_destroy.argtypes = [vp]
    L.fr_opt_destroy.restype = None
    L.fr_grad_clip.argtypes = [vp, ctypes.c_float, ctypes.c_float, vp, vp]
    L.fr_adamw_step.argtypes = [vp, ctypes.POINTER(fr_adamw), vp, vp]
    L.fr_opt_convert.argtypes = [vp, vp, u32, u64, vp]
    L.fr_muon_create.argtypes = [ctypes.POINTER(fr_muon_tensor), u64, ctypes.POINTER(vp)]
    L.fr_muon_info.argtypes = [vp, u64p, u64p, u64p]
    L.fr_muon_destroy.argtypes = [vp]
    L.fr_muon_destroy.restype = None
    L.fr_muon_step.argtypes = [vp, ctypes.POINTER(fr_muon), vp, vp]
    L.fr_muon_sync_status.argtypes = [vp, vp]
    L.fr_orthogonalize.argtypes = [vp, ctypes.POINTER(fr_muon), vp]
    L.fr_embed_create.argtypes = [u64, u64, u64, u64, ctypes.POINTER(vp)]
    L.fr_embed_info.argtypes = [vp, u64p, u64p, u64p, u64p]
    L.fr_embed_destroy.argtypes = [vp]
    L.fr_embed_destroy.restype = None
    L.fr_embed_lookup.argtypes = [vp, vp, u32, vp, u32, u64, ctypes.c_float, vp, u32, vp]
    L.fr_embed_grad.argtypes = [vp, vp, u32, vp, u32, u64, ctypes.c_float, vp, u32, u32, vp]
    L.fr_status_str.argtypes = [ctypes.c_int]
    L.fr_status_str.restype = ctypes.c_char_p
    L.fr_last_error.argtypes = []
    L.fr_last_error.restype = ctypes.c_char_p
    L.fr_version.argtypes = []
    for name in ["fr_plan_create", "fr_plan_info", "fr_plan_chunk", "fr_fingerprint", "fr_pack",
                 "fr_unpack_verify", "fr_diff", "fr_sync_status", "fr_version", "fr_fingerprint_static",
                 "fr_plan_create_batched", "fr_plan_batch", "fr_pack_batch", "fr_unpack_verify_batch",
                 "fr_unpack_collect", "fr_resend", "fr_restore", "fr_shard_pieces", "fr_pack_fp", "fr_unpack_verify_fp",
                 "fr_restore_fp", "fr_resend_fp", "fr_restore_multi", "fr_opt_create", "fr_opt_info", "fr_grad_clip",
                 "fr_adamw_step", "fr_opt_convert", "fr_muon_create", "fr_muon_info", "fr_muon_step", "fr_muon_sync_status", "fr_orthogonalize",
                 "fr_embed_create", "fr_embed_info", "fr_embed_lookup", "fr_embed_grad"]:
        getattr(L, name).restype = ctypes.c_int
    return L


lib = _load()


def fr_status_str(status: int) -> str:
    return lib.fr_status_str(status).decode()


def fr_last_error() -> str:
    return lib.fr_last_error().decode()


def fr_version() -> int:
    return lib.fr_version()


def _check(status: int, where: str) -> None:
    if status != FR_OK:
        raise FlashrecError(status, where)


def _stream(stream) -> int:
    if stream is None:  # the current stream's handle (3 us less than through a torch.cuda.Stream)
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _allocating_on(stream, device: torch.device):
    """A context in which a tensor that a call on `stream` writes is allocated and filled in that stream's order."""
    if stream is None:
        return contextlib.nullcontext()
    if not isinstance(stream, torch.cuda.Stream):
        # 0 and 1 are the legacy default stream's handles; torch makes a stream of its own of a 0, and takes no 1
        stream = torch.cuda.default_stream(device) if int(stream) in (0, 1) else torch.cuda.ExternalStream(int(stream), device=device)
    return torch.cuda.stream(stream)


def fr_dtype_of(t: torch.Tensor) -> int:
    try:
        return _TORCH_TO_FR[t.dtype]
    except KeyError:
        raise ValueError("unsupported dtype %s (bf16, fp32 or bytes)" % t.dtype)


# ---------------------------------------------------------------- C names

def _tensor_array(tensors, dtypes=None, on_device=True):
    """fr_tensor array of `tensors`.  Filled as one flat buffer of words: ctypes
    field assignments took 0.8 us per tensor, which a call that plans every
    time (fr_fingerprint_static) spends more on than on its sweep."""
    words = array.array("Q")
    push, codes = words.extend, _TORCH_TO_FR
    for i, t in enumerate(tensors):
        nbytes = t.nbytes
        if nbytes and on_device and not t.is_cuda:
            raise ValueError("tensor %d is not on a CUDA device" % i)
        if not t.is_contiguous():
            raise ValueError("tensor %d is not contiguous" % i)
        if dtypes is not None:
            code = dtypes[i] & 0xFFFFFFFF  # the high word is flags, 0
        else:
            code = codes.get(t.dtype)
            if code is None:
                code = fr_dtype_of(t)
        push((t.data_ptr() if nbytes else 0, nbytes, code))
    if not words:
        words.extend((0, 0, 0))
    return (fr_tensor * (len(words) // 3)).from_buffer(words)


def fr_plan_create(tensors: Sequence[torch.Tensor], chunk_bytes: int, dtypes: Optional[Sequence[int]] = None):
    """Plan over contiguous CUDA tensors.  Returns the opaque handle (int)."""
    h = ctypes.c_void_p()
    _check(lib.fr_plan_create(_tensor_array(tensors, dtypes), len(tensors), chunk_bytes, ctypes.byref(h)),
           "fr_plan_create")
    return h.value


def fr_plan_create_batched(tensors: Sequence[torch.Tensor], chunk_bytes: int, n_batches: int,
                           dtypes: Optional[Sequence[int]] = None):
    h = ctypes.c_void_p()
    _check(lib.fr_plan_create_batched(_tensor_array(tensors, dtypes), len(tensors), chunk_bytes, n_batches,
                                      ctypes.byref(h)), "fr_plan_create_batched")
    return h.value


def fr_plan_batch(plan, batch: int):
    nb, first, n = ctypes.c_uint32(), ctypes.c_uint64(), ctypes.c_uint64()
    _check(lib.fr_plan_batch(plan, batch, ctypes.byref(nb), ctypes.byref(first), ctypes.byref(n)), "fr_plan_batch")
    return nb.value, first.value, n.value


def fr_pack_batch(plan, batch: int, dst: torch.Tensor, stream=None) -> None:
    _check(lib.fr_pack_batch(plan, batch, dst.data_ptr() if dst.numel() else None, dst.numel(), _stream(stream)),
           "fr_pack_batch")


def fr_unpack_verify_batch(plan, batch: int, src: torch.Tensor, stream=None) -> None:
    _check(lib.fr_unpack_verify_batch(plan, batch, src.data_ptr() if src.numel() else None, src.numel(),
                                      _stream(stream)), "fr_unpack_verify_batch")


def fr_unpack_collect(plan, mismatch: Optional[torch.Tensor], count: torch.Tensor, stream=None) -> None:
    cap = 0 if mismatch is None else mismatch.numel()
    _check(lib.fr_unpack_collect(plan, mismatch.data_ptr() if cap else None, cap, count.data_ptr(), _stream(stream)),
           "fr_unpack_collect")


def fr_resend(src_plan, dst_plan, staging: torch.Tensor, stream_src=None, stream_dst=None) -> int:
    n = ctypes.c_uint64()
    _check(lib.fr_resend(src_plan, dst_plan, staging.data_ptr() if staging.numel() else None, staging.numel(),
                         ctypes.byref(n), _stream(stream_src), _stream(stream_dst)), "fr_resend")
    return n.value


def fr_restore(src_plan, dst_plan, staging: torch.Tensor, max_retries: int, mismatch: Optional[torch.Tensor],
               count: torch.Tensor, stream_src=None, stream_dst=None) -> None:
    cap = 0 if mismatch is None else mismatch.numel()
    _check(lib.fr_restore(src_plan, dst_plan, staging.data_ptr() if staging.numel() else None, staging.numel(),
                          max_retries, mismatch.data_ptr() if cap else None, cap, count.data_ptr(),
                          _stream(stream_src), _stream(stream_dst)), "fr_restore")


def _table_ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def fr_pack_fp(plan, dst: torch.Tensor, fp: Optional[torch.Tensor], stream=None) -> None:
    """fr_pack that also writes the fingerprint table `fp` (uint8, 16 B per chunk)."""
    _check(lib.fr_pack_fp(plan, dst.data_ptr() if dst.numel() else None, dst.numel() * dst.element_size(),
                          _table_ptr(fp), _stream(stream)), "fr_pack_fp")


def fr_unpack_verify_fp(plan, src: torch.Tensor, mismatch: Optional[torch.Tensor], count: torch.Tensor,
                        fp: Optional[torch.Tensor], stream=None) -> None:
    """fr_unpack_verify that also writes the restored tensors' fingerprint table."""
    cap = 0 if mismatch is None else mismatch.numel()
    _check(lib.fr_unpack_verify_fp(plan, src.data_ptr() if src.numel() else None, src.numel() * src.element_size(),
                                   mismatch.data_ptr() if cap else None, cap, count.data_ptr(), _table_ptr(fp),
                                   _stream(stream)), "fr_unpack_verify_fp")


def fr_restore_fp(src_plan, dst_plan, staging: torch.Tensor, max_retries: int, mismatch: Optional[torch.Tensor],
                  count: torch.Tensor, fp_src: Optional[torch.Tensor], fp_dst: Optional[torch.Tensor],
                  stream_src=None, stream_dst=None) -> None:
    """fr_restore that also writes both fingerprint tables."""
    cap = 0 if mismatch is None else mismatch.numel()
    _check(lib.fr_restore_fp(src_plan, dst_plan, staging.data_ptr() if staging.numel() else None, staging.numel(),
                             max_retries, mismatch.data_ptr() if cap else None, cap, count.data_ptr(),
                             _table_ptr(fp_src), _table_ptr(fp_dst), _stream(stream_src), _stream(stream_dst)),
           "fr_restore_fp")


def fr_resend_fp(src_plan, dst_plan, staging: torch.Tensor, fp_src: Optional[torch.Tensor],
                 fp_dst: Optional[torch.Tensor], stream_src=None, stream_dst=None) -> int:
    """fr_resend that also rewrites the re-sent chunks' fingerprint entries."""
    n = ctypes.c_uint64()
    _check(lib.fr_resend_fp(src_plan, dst_plan, staging.data_ptr() if staging.numel() else None, staging.numel(),
                            ctypes.byref(n), _table_ptr(fp_src), _table_ptr(fp_dst), _stream(stream_src),
                            _stream(stream_dst)), "fr_resend_fp")
    return n.value


def fr_restore_multi(src_plans, dst_plan, staging: torch.Tensor, max_retries: int, mismatch: Optional[torch.Tensor],
                     count: torch.Tensor, fp_dst: Optional[torch.Tensor] = None, streams_src=None,
                     stream_dst=None) -> None:
    """Restore `dst_plan` from several replicas, batch b packed by replica b % len(src_plans)."""
    n = len(src_plans)
    plans = (ctypes.c_void_p * n)(*[p for p in src_plans])
    streams = None
    if streams_src is not None:
        streams = (ctypes.c_void_p * n)(*[_stream(x) for x in streams_src])
    cap = 0 if mismatch is None else mismatch.numel()
    _check(lib.fr_restore_multi(plans, n, dst_plan, staging.data_ptr() if staging.numel() else None, staging.numel(),
                                max_retries, mismatch.data_ptr() if cap else None, cap, count.data_ptr(),
                                _table_ptr(fp_dst), streams, _stream(stream_dst)), "fr_restore_multi")


def fr_plan_info(plan):
    n, packed, state = ctypes.c_uint64(), ctypes.c_uint64(), ctypes.c_uint64()
    _check(lib.fr_plan_info(plan, ctypes.byref(n), ctypes.byref(packed), ctypes.byref(state)), "fr_plan_info")
    return n.value, packed.value, state.value


def fr_plan_chunk(plan, chunk_id: int):
    t, off, ln, poff = ctypes.c_uint32(), ctypes.c_uint64(), ctypes.c_uint64(), ctypes.c_uint64()
    _check(lib.fr_plan_chunk(plan, chunk_id, ctypes.byref(t), ctypes.byref(off), ctypes.byref(ln),
                             ctypes.byref(poff)), "fr_plan_chunk")
    return t.value, off.value, ln.value, poff.value


def fr_plan_destroy(plan) -> None:
    if plan:
        lib.fr_plan_destroy(plan)


def fr_fingerprint(plan, out: torch.Tensor, stream=None) -> None:
    """`out`: CUDA uint8 tensor of n_chunks * 16 bytes (fr_fp entries)."""
    _check(lib.fr_fingerprint(plan, out.data_ptr() if out.numel() else None, _stream(stream)), "fr_fingerprint")


def fr_pack(plan, dst: torch.Tensor, stream=None) -> None:
    """`dst`: uint8 tensor (CUDA, or pinned CPU memory) of >= packed_bytes."""
    _check(lib.fr_pack(plan, dst.data_ptr() if dst.numel() else None, dst.numel() * dst.element_size(),
                       _stream(stream)), "fr_pack")


def fr_unpack_verify(plan, src: torch.Tensor, mismatch: Optional[torch.Tensor], count: torch.Tensor,
                     stream=None, src_bytes: Optional[int] = None) -> None:
    """`mismatch`: CUDA int32/uint32 tensor (capacity = numel); `count`: CUDA int64 tensor of 1."""
    cap = 0 if mismatch is None else mismatch.numel()
    nbytes = src.numel() * src.element_size() if src_bytes is None else src_bytes
    _check(lib.fr_unpack_verify(plan, src.data_ptr() if src.numel() else None, nbytes,
                                mismatch.data_ptr() if cap else None, cap, count.data_ptr(), _stream(stream)),
           "fr_unpack_verify")


def fr_diff(a: torch.Tensor, b: torch.Tensor, n_chunks: int, diverged: Optional[torch.Tensor],
            count: torch.Tensor, stream=None) -> None:
    cap = 0 if diverged is None else diverged.numel()
    _check(lib.fr_diff(a.data_ptr() if n_chunks else None, b.data_ptr() if n_chunks else None, n_chunks,
                       diverged.data_ptr() if cap else None, cap, count.data_ptr(), _stream(stream)), "fr_diff")


def fr_sync_status(plan, stream=None) -> int:
    return lib.fr_sync_status(plan, _stream(stream))


FR_STATIC_MAX_CHUNKS = 16384


def fr_fingerprint_static(tensors: Sequence[torch.Tensor], chunk_bytes: int, out: torch.Tensor,
                          stream=None) -> None:
    """The fingerprint without a plan and without any device allocation, for
    callers that cannot allocate (see include/flashrec.h); `out` holds
    n_chunks * 16 bytes."""
    arr = _tensor_array(tensors, on_device=False)
    _check(lib.fr_fingerprint_static(arr, len(tensors), chunk_bytes, out.data_ptr() if out.numel() else None,
                                     _stream(stream)), "fr_fingerprint_static")


# ---------------------------------------------------------------- optimizer step

_FLOATS = {torch.bfloat16: FR_DT_BF16, torch.float32: FR_DT_F32}
_MOMENTS = {torch.float32: FR_DT_F32, torch.uint8: FR_DT_BYTES}
_F32 = {torch.float32: FR_DT_F32}
_U8 = {torch.uint8: FR_DT_BYTES}


def _opt_array(weights, grads, m, v, masters, m_exp, v_exp, lr_scale, decay_scale):
    """(fr_opt_tensor array, its length): 11 words per tensor, filled column by column."""
    lists = [("weights", weights, _FLOATS, 1), ("grads", grads, _FLOATS, 1), ("masters", masters, _F32, 1),
             ("m", m, _MOMENTS, 1), ("v", v, _MOMENTS, 1), ("m_exp", m_exp, _U8, FR_OPT_BLOCK),
             ("v_exp", v_exp, _U8, FR_OPT_BLOCK)]
    given = [x for _, x, _, _ in lists if x is not None]
    if not given:
        raise ValueError("a plan needs weights, gradients or moments")
    count = len(given[0])
    sizes = [None] * count
    columns, codes = [], {}
    device = None  # of every tensor that has elements
    for name, tensors, allowed, per in lists:
        if tensors is None:
            columns.append([0] * count)
            codes[name] = [0] * count
            continue
        if len(tensors) != count:
            raise ValueError("%s holds %d tensors, not %d" % (name, len(tensors), count))
        column, code = [], []
        for i, t in enumerate(tensors):
            if t is None:
                column.append(0)
                code.append(0)
                continue
            n = t.numel()
            if n and t.get_device() != device:
                if not t.is_cuda:
                    raise ValueError("%s[%d] is not on a CUDA device" % (name, i))
                if device is not None:
                    raise ValueError("%s[%d] is on CUDA device %d, the tensors before it on %d" % (name, i, t.get_device(), device))
                device = t.get_device()
            if not t.is_contiguous():
                raise ValueError("%s[%d] is not contiguous" % (name, i))
            c = allowed.get(t.dtype)
            if c is None:
                raise ValueError("%s[%d]: unsupported dtype %s" % (name, i, t.dtype))
            if per == 1:
                if sizes[i] is None:
                    sizes[i] = n
                elif sizes[i] != n:
                    raise ValueError("%s[%d] holds %d elements, not %d" % (name, i, n, sizes[i]))
            elif n != -(-(sizes[i] or 0) // per):
                raise ValueError("%s[%d] holds %d bytes, one per block of %d is needed" % (name, i, n, per))
            column.append(t.data_ptr() if n else 0)
            code.append(c)
        columns.append(column)
        codes[name] = code
    if any(a != b for a, b in zip(codes["m"], codes["v"])):
        raise ValueError("m and v differ in type")
    if device is not None and device != torch.cuda.current_device():  # the one that the plan is bound to
        raise ValueError("the tensors are on CUDA device %d, the current one is %d" % (device, torch.cuda.current_device()))

    def factors(x):
        x = array.array("f", [1.0] * count if x is None else x)
        if len(x) != count:
            raise ValueError("%d factors for %d tensors" % (len(x), count))
        return array.array("I", x.tobytes())

    words = array.array("Q", bytes(8 * 11 * max(count, 1)))
    for k, column in enumerate(columns):
        words[k:11 * count:11] = array.array("Q", column)
    words[7:11 * count:11] = array.array("Q", [n or 0 for n in sizes])
    words[8:11 * count:11] = array.array("Q", [w | g << 32 for w, g in zip(codes["weights"], codes["grads"])])
    words[9:11 * count:11] = array.array("Q", codes["m"])
    words[10:11 * count:11] = array.array("Q", [a | b << 32 for a, b in zip(factors(lr_scale), factors(decay_scale))])
    return (fr_opt_tensor * max(count, 1)).from_buffer(words), count


def fr_opt_create(weights=None, grads=None, m=None, v=None, masters=None, m_exp=None, v_exp=None, lr_scale=None,
                  decay_scale=None):
    """Plan over lists of contiguous CUDA tensors on the current device (a list, or an entry, may be None; factors default
    to 1).  Moments are fp32, or uint8 codes with one uint8 exponent per FR_OPT_BLOCK elements.  Returns the opaque handle
    (int)."""
    arr, count = _opt_array(weights, grads, m, v, masters, m_exp, v_exp, lr_scale, decay_scale)
    h = ctypes.c_void_p()
    _check(lib.fr_opt_create(arr, count, ctypes.byref(h)), "fr_opt_create")
    return h.value


def fr_opt_info(plan):
    """(tensors, elements, blocks)"""
    t, n, b = ctypes.c_uint64(), ctypes.c_uint64(), ctypes.c_uint64()
    _check(lib.fr_opt_info(plan, ctypes.byref(t), ctypes.byref(n), ctypes.byref(b)), "fr_opt_info")
    return t.value, n.value, b.value


def fr_opt_destroy(plan) -> None:
    if plan:
        lib.fr_opt_destroy(plan)


def _record(t: torch.Tensor) -> int:
    if not t.is_cuda or not t.is_contiguous() or t.nbytes < CLIP_BYTES:
        raise ValueError("a clip record is %d bytes of CUDA memory" % CLIP_BYTES)
    return t.data_ptr()


def fr_grad_clip(plan, max_norm: float, grad_scale: float, out: torch.Tensor, stream=None) -> None:
    """`out`: CUDA tensor of 16 bytes, the fr_clip record (see clip_view)."""
    _check(lib.fr_grad_clip(plan, max_norm, grad_scale, _record(out), _stream(stream)), "fr_grad_clip")


def fr_adamw_step(plan, hyper: fr_adamw, clip: Optional[torch.Tensor] = None, stream=None) -> None:
    _check(lib.fr_adamw_step(plan, hyper, None if clip is None else _record(clip), _stream(stream)), "fr_adamw_step")


def fr_opt_convert(src, dst, rounding: int = FR_ROUND_NEAREST, seed: int = 0, stream=None) -> None:
    """The moments of plan `dst` from those of plan `src`, 32 bits to 8 or back."""
    _check(lib.fr_opt_convert(src, dst, rounding, seed, _stream(stream)), "fr_opt_convert")


# ---------------------------------------------------------------- orthogonalised updates

MUON_COEFFICIENTS = ((3.4445, -4.7750, 2.0315),) * 5


def muon(lr: float = 0.0, beta: float = 0.95, weight_decay: float = 0.0, nesterov: bool = True,
         coefficients=MUON_COEFFICIENTS, step: int = 1, seed: int = 0, rounding: int = FR_ROUND_NEAREST,
         products: int = FR_MUON_BY_TYPE) -> fr_muon:
    """The numbers of a step: one (a, b, c) per iteration."""
    if not 1 <= len(coefficients) <= FR_MUON_MOST:
        raise ValueError("1 to %d iterations, not %d" % (FR_MUON_MOST, len(coefficients)))
    h = fr_muon(lr, beta, weight_decay, step=step, seed=seed, iterations=len(coefficients), nesterov=bool(nesterov), rounding=rounding,
                products=products)
    for i, abc in enumerate(coefficients):
        h.coef[i][:] = abc
    return h


def _muon_array(weights, grads, momenta, masters, updates, lr_scale, decay_scale, update_scale, both_halves=False):
    """(fr_muon_tensor array, its length)"""
    lists = [("weights", "weight", weights, _FLOATS), ("grads", "grad", grads, _FLOATS), ("masters", "master", masters, _F32),
             ("momenta", "momentum", momenta, _F32), ("updates", "update", updates, _FLOATS)]
    given = [x for _, _, x, _ in lists if x is not None]
    if not given:
        raise ValueError("a plan needs weights, gradients or momenta")
    count = len(given[0])
    arr = (fr_muon_tensor * max(count, 1))()
    shapes = [None] * count
    device = None  # of every matrix that has elements
    for name, field, tensors, allowed in lists:
        if tensors is None:
            continue
        if len(tensors) != count:
            raise ValueError("%s holds %d matrices, not %d" % (name, len(tensors), count))
        typed = field in ("weight", "grad", "update")
        for i, t in enumerate(tensors):
            if t is None:
                continue
            if t.dim() != 2:
                raise ValueError("%s[%d] has %d dimensions, a matrix has two" % (name, i, t.dim()))
            if t.numel() and t.get_device() != device:
                if not t.is_cuda:
                    raise ValueError("%s[%d] is not on a CUDA device" % (name, i))
                if device is not None:
                    raise ValueError("%s[%d] is on CUDA device %d, the matrices before it on %d" % (name, i, t.get_device(), device))
                device = t.get_device()
            if not t.is_contiguous():
                raise ValueError("%s[%d] is not contiguous" % (name, i))
            code = allowed.get(t.dtype)
            if code is None:
                raise ValueError("%s[%d]: unsupported dtype %s" % (name, i, t.dtype))
            if shapes[i] is None:
                shapes[i] = t.shape
                arr[i].rows, arr[i].cols = t.shape
            elif shapes[i] != t.shape:
                raise ValueError("%s[%d] is %d x %d, not %d x %d" % (name, i, *t.shape, *shapes[i]))
            if t.numel():
                setattr(arr[i], field, t.data_ptr())
            if typed:
                setattr(arr[i], field + "_dtype", code)
    if device is not None and device != torch.cuda.current_device():  # the one that the plan is bound to
        raise ValueError("the matrices are on CUDA device %d, the current one is %d" % (device, torch.cuda.current_device()))
    for field, x in (("lr_scale", lr_scale), ("decay_scale", decay_scale), ("update_scale", update_scale)):
        x = [1.0] * count if x is None else list(x)
        if len(x) != count:
            raise ValueError("%d factors for %d matrices" % (len(x), count))
        for i, v in enumerate(x):
            setattr(arr[i], field, v)
    for i in range(count):
        arr[i].flags = FR_MUON_BOTH_HALVES if both_halves else 0
    return arr, count


def fr_muon_create(weights=None, grads=None, momenta=None, masters=None, updates=None, lr_scale=None, decay_scale=None,
                   update_scale=None, both_halves=False):
    """Plan over lists of contiguous two-dimensional CUDA tensors on the current device (a list, or an entry, may be None;
    factors default to 1).  Momenta and masters are fp32, the others bf16 or fp32.  `both_halves`: matrices with bf16 outputs get
    the products that those with fp32 ones have, in 2.5 times the time (see include/flashrec.h).  Returns the opaque handle
    (int)."""
    arr, count = _muon_array(weights, grads, momenta, masters, updates, lr_scale, decay_scale, update_scale, both_halves)
    h = ctypes.c_void_p()
    _check(lib.fr_muon_create(arr, count, ctypes.byref(h)), "fr_muon_create")
    return h.value


def fr_muon_info(plan):
    """(matrices, elements, bytes of device memory)"""
    t, n, b = ctypes.c_uint64(), ctypes.c_uint64(), ctypes.c_uint64()
    _check(lib.fr_muon_info(plan, ctypes.byref(t), ctypes.byref(n), ctypes.byref(b)), "fr_muon_info")
    return t.value, n.value, b.value


def fr_muon_destroy(plan) -> None:
    if plan:
        lib.fr_muon_destroy(plan)


def fr_muon_step(plan, hyper: fr_muon, clip: Optional[torch.Tensor] = None, stream=None) -> None:
    _check(lib.fr_muon_step(plan, hyper, None if clip is None else _record(clip), _stream(stream)), "fr_muon_step")


def fr_muon_sync_status(plan, stream=None) -> int:
    return lib.fr_muon_sync_status(plan, _stream(stream))


def fr_orthogonalize(plan, hyper: fr_muon, stream=None) -> None:
    _check(lib.fr_orthogonalize(plan, hyper, _stream(stream)), "fr_orthogonalize")


# ---------------------------------------------------------------- embeddings

_TOKENS = {torch.int32: 4, torch.int64: 8}


def _buffer(name: str, t: torch.Tensor, allowed):
    """(address, code of the type) of a contiguous CUDA tensor"""
    code = allowed.get(t.dtype)
    if code is None:
        raise ValueError("%s: unsupported dtype %s" % (name, t.dtype))
    if not t.is_cuda and t.numel():
        raise ValueError("%s is not on a CUDA device" % name)
    if not t.is_contiguous():
        raise ValueError("%s is not contiguous" % name)
    return t.data_ptr(), code  # (of an empty tensor 0, NULL)


def fr_embed_create(rows: int, dim: int, max_tokens: int, first: int = 0):
    """Plan of an embedding's slice [first, first + rows) on the current device.  Returns the opaque handle (int)."""
    if min(rows, dim, max_tokens, first) < 0:
        raise ValueError("rows, dim, max_tokens and first are not negative")
    h = ctypes.c_void_p()
    _check(lib.fr_embed_create(rows, dim, max_tokens, first, ctypes.byref(h)), "fr_embed_create")
    return h.value


def fr_embed_info(plan):
    """(rows, dim, max_tokens, bytes of device memory)"""
    x = [ctypes.c_uint64() for _ in range(4)]
    _check(lib.fr_embed_info(plan, *(ctypes.byref(v) for v in x)), "fr_embed_info")
    return tuple(v.value for v in x)


def fr_embed_destroy(plan) -> None:
    if plan:
        lib.fr_embed_destroy(plan)


def _embed_sizes(plan, name: str, table: torch.Tensor, tokens: torch.Tensor, out: torch.Tensor) -> None:
    """The library takes addresses alone: a table of another size than the plan's, or another number of rows than tokens, would
    be read and written beyond its end."""
    rows, dim, _, _ = fr_embed_info(plan)
    if table.numel() != rows * dim:
        raise ValueError("%s holds %d elements, not %d rows of %d" % (name, table.numel(), rows, dim))
    if out.numel() != tokens.numel() * dim:
        raise ValueError("out holds %d elements, not %d rows of %d" % (out.numel(), tokens.numel(), dim))
    devices = {t.get_device() for t in (table, tokens, out) if t.numel()}
    if len(devices) > 1:
        raise ValueError("%s, tokens and out are on several devices" % name)


def _embed_lookup(plan, table, tokens, scale, out, stream) -> None:
    w, wt = _buffer("table", table, _FLOATS)
    t, tb = _buffer("tokens", tokens, _TOKENS)
    o, ot = _buffer("out", out, _FLOATS)
    _check(lib.fr_embed_lookup(plan, w, wt, t, tb, tokens.numel(), scale, o, ot, _stream(stream)), "fr_embed_lookup")


def _embed_grad(plan, out, tokens, grad, scale, accumulate, stream) -> None:
    o, ot = _buffer("out", out, _FLOATS)
    t, tb = _buffer("tokens", tokens, _TOKENS)
    g, gt = _buffer("grad", grad, _FLOATS)
    _check(lib.fr_embed_grad(plan, o, ot, t, tb, tokens.numel(), scale, g, gt, int(bool(accumulate)), _stream(stream)), "fr_embed_grad")


def fr_embed_lookup(plan, table: torch.Tensor, tokens: torch.Tensor, scale: float, out: torch.Tensor, stream=None) -> None:
    """`out`: as many rows as `tokens` (int32 or int64) has elements."""
    _embed_sizes(plan, "table", table, tokens, out)
    _embed_lookup(plan, table, tokens, scale, out, stream)


def fr_embed_grad(plan, out: torch.Tensor, tokens: torch.Tensor, grad: torch.Tensor, scale: float = 1.0, accumulate: bool = False,
                  stream=None) -> None:
    """The table's gradient `grad` from the rows' gradients `out`."""
    _embed_sizes(plan, "grad", grad, tokens, out)
    _embed_grad(plan, out, tokens, grad, scale, accumulate, stream)


# ---------------------------------------------------------------- convenience

def fr_shard_pieces(n_elems: int, elem_bytes: int, n_dst: int, rank: int, n_src: int):
    """Pieces of shard `rank` (of `n_dst`) among `n_src` shards of one flat
    group: a list of (source, src_off, dst_off, nbytes), ascending.  Host only."""
    n = ctypes.c_uint64(0)
    cap = max(int(n_src), 1)
    arr = (fr_piece * cap)()
    _check(lib.fr_shard_pieces(n_elems, elem_bytes, n_dst, rank, n_src, arr, cap, ctypes.byref(n)),
           "fr_shard_pieces")
    return [(arr[i].source, arr[i].src_off, arr[i].dst_off, arr[i].nbytes) for i in range(n.value)]


def fp_view(table: torch.Tensor):
    """(crc32c as int64, nonfinite as int64, sumsq as float64) views of a
    fingerprint table held as uint8 [n * 16]."""
    t = table.view(-1, FP_ENTRY_BYTES)
    w = t.view(torch.int32)
    crc = w[:, 0].to(torch.int64) & 0xFFFFFFFF
    nf = w[:, 1].to(torch.int64) & 0xFFFFFFFF
    sumsq = t[:, 8:16].contiguous().view(torch.float64).view(-1)
    return crc, nf, sumsq


class Plan:
    """A plan over a list of CUDA tensors, with allocation helpers."""

    def __init__(self, tensors: Sequence[torch.Tensor], chunk_bytes: int, n_batches: int = 1):
        self.tensors: List[torch.Tensor] = list(tensors)
        self.chunk_bytes = chunk_bytes
        self.device = self.tensors[0].device if self.tensors else torch.device("cuda", torch.cuda.current_device())
        if n_batches > 1:
            self.handle = fr_plan_create_batched(self.tensors, chunk_bytes, n_batches)
        else:
            self.handle = fr_plan_create(self.tensors, chunk_bytes)
        self.n_batches = fr_plan_batch(self.handle, 0)[0] if n_batches > 1 else 1
        self.n_chunks, self.packed_bytes, self.state_bytes = fr_plan_info(self.handle)

    def close(self) -> None:
        if self.handle:
            fr_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def new_table(self) -> torch.Tensor:
        return torch.empty(self.n_chunks * FP_ENTRY_BYTES, dtype=torch.uint8, device=self.device)

    def new_packed(self, pinned: bool = False) -> torch.Tensor:
        if pinned:
            return torch.empty(self.packed_bytes, dtype=torch.uint8, pin_memory=True)
        return torch.empty(self.packed_bytes, dtype=torch.uint8, device=self.device)

    def fingerprint(self, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        out = self.new_table() if out is None else out
        fr_fingerprint(self.handle, out, stream)
        return out

    def pack(self, dst: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        dst = self.new_packed() if dst is None else dst
        fr_pack(self.handle, dst, stream)
        return dst

    def unpack_verify(self, src: torch.Tensor, cap: Optional[int] = None, stream=None,
                      mismatch: Optional[torch.Tensor] = None, count: Optional[torch.Tensor] = None):
        """Returns (mismatch id tensor (first min(cap, count)), count) after a sync."""
        if mismatch is None:
            cap = self.n_chunks if cap is None else cap
            mismatch = torch.empty(max(cap, 1), dtype=torch.int32, device=self.device)[:cap]
        if count is None:
            count = torch.empty(1, dtype=torch.int64, device=self.device)
        fr_unpack_verify(self.handle, src, mismatch, count, stream)
        n = int(count.item())
        return mismatch[: min(n, mismatch.numel())], n

    def pack_fp(self, dst: Optional[torch.Tensor] = None, table: Optional[torch.Tensor] = None, stream=None):
        """fr_pack_fp: returns (packed buffer, this state's fingerprint table)."""
        dst = self.new_packed() if dst is None else dst
        table = self.new_table() if table is None else table
        fr_pack_fp(self.handle, dst, table, stream)
        return dst, table

    def unpack_verify_fp(self, src: torch.Tensor, table: Optional[torch.Tensor] = None, cap: Optional[int] = None,
                         stream=None):
        """fr_unpack_verify_fp: returns (mismatch ids, count, the restored state's
        fingerprint table) after a sync."""
        cap = self.n_chunks if cap is None else cap
        mismatch = torch.empty(max(cap, 1), dtype=torch.int32, device=self.device)[:cap]
        count = torch.empty(1, dtype=torch.int64, device=self.device)
        table = self.new_table() if table is None else table
        fr_unpack_verify_fp(self.handle, src, mismatch, count, table, stream)
        n = int(count.item())
        return mismatch[: min(n, mismatch.numel())], n, table

    def sync_status(self, stream=None) -> int:
        return fr_sync_status(self.handle, stream)


def diff(a: torch.Tensor, b: torch.Tensor, cap: Optional[int] = None, stream=None):
    n = a.numel() // FP_ENTRY_BYTES
    cap = n if cap is None else cap
    out = torch.empty(max(cap, 1), dtype=torch.int32, device=a.device)[:cap]
    count = torch.empty(1, dtype=torch.int64, device=a.device)
    fr_diff(a, b, n, out, count, stream)
    k = int(count.item())
    return out[: min(k, cap)], k


def clip_view(record: torch.Tensor):
    """(norm, scale, nonfinite) of an fr_clip record, as views of one element each."""
    b = record.view(torch.uint8).view(-1)
    return b[0:4].view(torch.float32), b[4:8].view(torch.float32), b[8:16].view(torch.int64)


class OptPlan:
    """A plan of the optimizer step over lists of CUDA tensors (arguments as fr_opt_create)."""

    def __init__(self, weights=None, grads=None, m=None, v=None, masters=None, m_exp=None, v_exp=None, lr_scale=None,
                 decay_scale=None):
        lists = [weights, grads, m, v, masters, m_exp, v_exp]
        self.buffers = [None if x is None else list(x) for x in lists]  # the plan holds their addresses
        # (a tensor without elements may lie anywhere)
        first = next((t for x in self.buffers if x for t in x if t is not None and t.numel()), None)
        self.device = first.device if first is not None else torch.device("cuda", torch.cuda.current_device())
        self.handle = None
        self.handle = fr_opt_create(*self.buffers, lr_scale=lr_scale, decay_scale=decay_scale)
        self.n_tensors, self.n_elems, self.n_blocks = fr_opt_info(self.handle)

    def close(self) -> None:
        if self.handle:
            fr_opt_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def new_clip(self) -> torch.Tensor:
        return torch.zeros(CLIP_BYTES, dtype=torch.uint8, device=self.device)

    def _here(self, record: torch.Tensor) -> None:
        if record.device != self.device:
            raise ValueError("the clip record is on %s, the plan on %s" % (record.device, self.device))

    def clip(self, max_norm: float = float("inf"), grad_scale: float = 1.0, out: Optional[torch.Tensor] = None,
             stream=None) -> torch.Tensor:
        """fr_grad_clip: returns the record, for step()."""
        if out is None:
            with _allocating_on(stream, self.device):
                out = self.new_clip()
        self._here(out)
        fr_grad_clip(self.handle, max_norm, grad_scale, out, stream)
        return out

    def step(self, hyper: fr_adamw, clip: Optional[torch.Tensor] = None, stream=None) -> None:
        if clip is not None:
            self._here(clip)
        fr_adamw_step(self.handle, hyper, clip, stream)

    def convert_to(self, dst: "OptPlan", rounding: int = FR_ROUND_NEAREST, seed: int = 0, stream=None) -> None:
        fr_opt_convert(self.handle, dst.handle, rounding, seed, stream)


class MuonPlan:
    """A plan of the orthogonalised update over lists of two-dimensional CUDA tensors (arguments as fr_muon_create).  The
    clip record comes from an OptPlan over all gradients."""

    def __init__(self, weights=None, grads=None, momenta=None, masters=None, updates=None, lr_scale=None, decay_scale=None,
                 update_scale=None, both_halves=False):
        lists = [weights, grads, momenta, masters, updates]
        self.buffers = [None if x is None else list(x) for x in lists]  # the plan holds their addresses
        first = next((t for x in self.buffers if x for t in x if t is not None and t.numel()), None)
        self.device = first.device if first is not None else torch.device("cuda", torch.cuda.current_device())
        self.handle = None
        self.handle = fr_muon_create(*self.buffers, lr_scale=lr_scale, decay_scale=decay_scale, update_scale=update_scale,
                                     both_halves=both_halves)
        self.n_tensors, self.n_elems, self.device_bytes = fr_muon_info(self.handle)

    def close(self) -> None:
        if self.handle:
            fr_muon_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def step(self, hyper: fr_muon, clip: Optional[torch.Tensor] = None, stream=None) -> None:
        if clip is not None and clip.device != self.device:
            raise ValueError("the clip record is on %s, the plan on %s" % (clip.device, self.device))
        fr_muon_step(self.handle, hyper, clip, stream)

    def sync_status(self, stream=None) -> int:
        """FR_OK, or FR_ERR_DEVICE_TIMEOUT once: a step was left half done, and nothing has been written since."""
        return fr_muon_sync_status(self.handle, stream)

    def orthogonalize(self, hyper: Optional[fr_muon] = None, stream=None) -> None:
        """Writes the plan's updates from its gradients."""
        fr_orthogonalize(self.handle, muon() if hyper is None else hyper, stream)


class EmbedPlan:
    """A plan of an embedding's slice on the current device (arguments as fr_embed_create)."""

    def __init__(self, rows: int, dim: int, max_tokens: int, first: int = 0):
        self.device = torch.device("cuda", torch.cuda.current_device())
        self.handle = None
        self.handle = fr_embed_create(rows, dim, max_tokens, first)
        self.rows, self.dim, self.max_tokens, self.device_bytes = fr_embed_info(self.handle)
        self.first = first

    def close(self) -> None:
        if self.handle:
            fr_embed_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _here(self, name: str, t: torch.Tensor, shape) -> None:
        if t.get_device() != self.device.index and t.numel():
            raise ValueError("%s is on %s, the plan on %s" % (name, t.device, self.device))
        if shape is not None and t.shape != shape:
            raise ValueError("%s has the shape %s, not %s" % (name, tuple(t.shape), tuple(shape)))

    def lookup(self, table: torch.Tensor, tokens: torch.Tensor, scale: float = 1.0, out: Optional[torch.Tensor] = None,
               stream=None) -> torch.Tensor:
        """scale * table[tokens - first], of the shape of `tokens` and dim; by default in the table's type."""
        self._here("table", table, (self.rows, self.dim))
        self._here("tokens", tokens, None)
        if out is None:
            with _allocating_on(stream, self.device):
                out = torch.empty(*tokens.shape, self.dim, dtype=table.dtype, device=self.device)
        self._here("out", out, (*tokens.shape, self.dim))
        _embed_lookup(self.handle, table, tokens, scale, out, stream)  # (sizes and devices are looked at above)
        return out

    def grad(self, out: torch.Tensor, tokens: torch.Tensor, grad: Optional[torch.Tensor] = None, scale: float = 1.0,
             accumulate: bool = False, stream=None) -> torch.Tensor:
        """The table's gradient from the gradient `out` of what lookup() gave, in `grad` (by default a new one, in fp32), or
        added to what is there."""
        self._here("out", out, (*tokens.shape, self.dim))
        self._here("tokens", tokens, None)
        if grad is None:
            if accumulate:
                raise ValueError("accumulate needs a gradient to add to")
            with _allocating_on(stream, self.device):
                grad = torch.empty(self.rows, self.dim, dtype=torch.float32, device=self.device)
        self._here("grad", grad, (self.rows, self.dim))
        _embed_grad(self.handle, out, tokens, grad, scale, accumulate, stream)
        return grad
