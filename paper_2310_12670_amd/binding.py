"""ctypes binding of ``include/reft.h``: the same entry points, arguments marshalled from Python.

Pointers may be given as ``torch.Tensor`` (its ``data_ptr()`` is used), as ``int`` addresses or as
``None``; pointer arrays as sequences of those or as a ctypes array made with :func:`ptr_array`
(worth it when the same list is passed many times).  The operators of a training step take tensors
only, as they read sizes, row lengths and types off them.  Streams may be ``torch.cuda.Stream``,
``int`` (a ``hipStream_t``) or ``None`` (the default stream).  Every failing call raises
:class:`ReftError` carrying the library's code and message.
"""
from __future__ import annotations

import ctypes
import importlib
import operator
import os
from typing import Optional, Sequence

__all__ = [
    "ReftError", "REFT_OK", "REFT_EINVAL", "REFT_ESIZE", "REFT_EHIP", "REFT_EUNRECOVERABLE",
    "REFT_MAX_K", "lib_path", "ptr_array",
    "reft_plan_create", "reft_plan_destroy", "reft_plan_stream_bytes", "reft_plan_num_spans",
    "reft_plan_num_buckets", "reft_plan_max_bucket_bytes", "reft_plan_staging_slot_bytes",
    "reft_plan_bucket_range", "reft_plan_split", "reft_plan_span_offset", "reft_plan_tile_info",
    "reft_plan_tile_first_span",
    "reft_snapshot_pack", "reft_snapshot_pack_range", "reft_plan_bucket_of", "reft_snapshot_wait",
    "reft_snapshot_query", "reft_ckpt_create", "reft_ckpt_destroy", "reft_ckpt_begin",
    "reft_ckpt_commit", "reft_ckpt_latest", "reft_ckpt_wait", "REFT_EBUSY",
    "reft_plan_staged_work", "reft_plan_burst_stats", "reft_recovery_plan",
    "REFT_RECOVER_COPY", "REFT_RECOVER_DECODE",
    "reft_pack_device", "reft_unpack_device", "reft_parity_encode", "reft_parity_encode_noalloc",
    "reft_parity_encode_pack", "reft_reconstruct",
    "reft_reconstruct_spans", "reft_segment_bytes", "reft_parity_encode_rotated",
    "reft_reconstruct_rotated", "reft_restore", "reft_restore_wait",
    "reft_set_tunable", "reft_get_tunable", "reft_last_error", "reft_version",
    "REFT_F32", "REFT_BF16", "REFT_F16", "REFT_E4M3", "REFT_E5M2", "reft_dropout", "reft_norm_forward",
    "reft_norm_backward", "reft_norm_backward_workspace", "reft_quantize", "reft_product",
    "reft_product_workspace",
]

REFT_OK, REFT_EINVAL, REFT_ESIZE, REFT_EHIP, REFT_EUNRECOVERABLE, REFT_EBUSY = 0, -1, -2, -3, -4, -5
REFT_MAX_K = 32
REFT_RECOVER_COPY, REFT_RECOVER_DECODE = 1, 2
REFT_F32, REFT_BF16, REFT_F16, REFT_E4M3, REFT_E5M2 = 0, 1, 2, 3, 4

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libreft.so")
_lib = None
_marshal = None


class ReftError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"libreft error {code}: {message}")
        self.code = code
        self.message = message


def lib_path() -> str:
    return _LIB_PATH


def _load():
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise ImportError(
            f"{_LIB_PATH} is not built; run `python -c 'import __graft_entry__ as g; g.build()'` "
            "(there is no fallback path)")
    lib = ctypes.CDLL(_LIB_PATH)
    u64, u32, vp, i, f64 = ctypes.c_uint64, ctypes.c_uint32, ctypes.c_void_p, ctypes.c_int, ctypes.c_double
    pu64 = ctypes.POINTER(ctypes.c_uint64)
    sig = {
        "reft_plan_create": (i, [vp, u64, vp, u64, u64, ctypes.POINTER(vp)]),
        "reft_plan_destroy": (None, [vp]),
        "reft_plan_stream_bytes": (u64, [vp]),
        "reft_plan_num_spans": (u64, [vp]),
        "reft_plan_num_buckets": (u64, [vp]),
        "reft_plan_max_bucket_bytes": (u64, [vp]),
        "reft_plan_staging_slot_bytes": (u64, [vp]),
        "reft_plan_bucket_range": (i, [vp, u64, pu64, pu64]),
        "reft_plan_span_offset": (i, [vp, u64, pu64]),
        "reft_plan_tile_info": (i, [vp, pu64, pu64]),
        "reft_plan_tile_first_span": (i, [vp, u64, pu64]),
        "reft_plan_split": (i, [vp, ctypes.c_double, ctypes.c_double, pu64]),
        "reft_snapshot_pack": (i, [vp, vp, vp, u64, vp, u64, vp, vp]),
        "reft_snapshot_pack_range": (i, [vp, vp, vp, u64, vp, u64, u64, u64, vp, vp]),
        "reft_plan_bucket_of": (i, [vp, u64, pu64]),
        "reft_ckpt_create": (i, [vp, vp, vp, u64, ctypes.POINTER(vp)]),
        "reft_ckpt_destroy": (None, [vp]),
        "reft_ckpt_begin": (i, [vp, ctypes.POINTER(vp), pu64]),
        "reft_ckpt_commit": (i, [vp, vp]),
        "reft_ckpt_latest": (i, [vp, ctypes.POINTER(vp), pu64]),
        "reft_snapshot_wait": (i, [vp]),
        "reft_snapshot_query": (i, [vp]),
        "reft_pack_device": (i, [vp, vp, vp, u64, vp]),
        "reft_unpack_device": (i, [vp, vp, u64, vp, vp]),
        "reft_parity_encode": (i, [vp, vp, u32, vp, vp]),
        "reft_parity_encode_noalloc": (i, [vp, vp, u32, vp, vp]),
        "reft_parity_encode_pack": (i, [vp, vp, u32, u32, vp, vp, u64, vp]),
        "reft_plan_staged_work": (i, [vp, pu64, pu64]),
        "reft_plan_burst_stats": (i, [vp, pu64]),
        "reft_ckpt_wait": (i, [vp]),
        "reft_recovery_plan": (i, [u32, vp, u32, i, vp, vp, ctypes.POINTER(u32)]),
        "reft_reconstruct": (i, [vp, u32, vp, u64, vp, ctypes.POINTER(u32), vp]),
        "reft_reconstruct_spans": (i, [vp, vp, u32, u32, vp, vp, vp]),
        "reft_segment_bytes": (u64, [vp, u32]),
        "reft_parity_encode_rotated": (i, [vp, vp, u32, u32, vp, vp]),
        "reft_reconstruct_rotated": (i, [vp, vp, vp, u32, u32, vp, vp]),
        "reft_restore": (i, [vp, vp, u64, vp, u64, vp, vp, vp]),
        "reft_restore_wait": (i, [vp]),
        "reft_set_tunable": (i, [ctypes.c_char_p, u64]),
        "reft_get_tunable": (i, [ctypes.c_char_p, pu64]),
        "reft_dropout": (i, [vp, u64, vp, u64, u64, u64, i, f64, u64, u64, vp]),
        "reft_norm_forward": (i, [vp, u64, vp, u64, vp, u64, u64, i, i, i, f64, f64, u64, u64, vp, u64, vp, vp, u64,
                                  vp, u64, i, vp, u64, vp]),
        "reft_norm_backward_workspace": (u64, [u64, u64]),
        "reft_norm_backward": (i, [vp, u64, vp, u64, vp, u64, vp, vp, u64, u64, i, i, i, f64, u64, u64, vp, u64, vp,
                                   u64, vp, vp, u64, vp]),
        "reft_quantize": (i, [vp, u64, u64, u64, i, i, i, vp, u64, vp, u64, vp, u64, vp, u64, vp]),
        "reft_product_workspace": (u64, [u64, u64, u64]),
        "reft_product": (i, [vp, u64, i, vp, u64, vp, u64, i, vp, u64, i, u64, u64, u64, vp, u64, i, vp, u64, vp]),
        "reft_last_error": (ctypes.c_char_p, []),
        "reft_version": (ctypes.c_char_p, []),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


class _NoMarshal:
    """In place of the binding's C part where it could not be built: no call is the usual case."""

    def __getattr__(self, name):
        return lambda *args: None


def _load_marshal():
    global _marshal
    if _marshal is None:
        _load()
        try:
            _marshal = importlib.import_module("._marshal", __package__)
        except ModuleNotFoundError:
            _marshal = _NoMarshal()
    return _marshal


# ------------------------------------------------------------------------------------------------
# marshalling
# ------------------------------------------------------------------------------------------------
def _addr(x) -> Optional[int]:
    if x is None:
        return None
    if isinstance(x, int):
        return x or None
    if hasattr(x, "data_ptr"):
        return x.data_ptr() or None
    if hasattr(x, "ctypes"):          # numpy array (host memory)
        return x.ctypes.data or None
    raise TypeError(f"cannot take the address of {type(x).__name__}")


def _nbytes(x) -> int:
    if hasattr(x, "element_size"):
        return x.numel() * x.element_size()
    return x.nbytes


def ptr_array(items: Sequence):
    """ctypes ``void*[]`` holding the addresses of ``items`` (tensors, ints or None)."""
    if isinstance(items, ctypes.Array):
        return items
    return (ctypes.c_void_p * max(1, len(items)))(*[_addr(x) for x in items])


def _u64s(vals: Optional[Sequence[int]]):
    if vals is None:
        return None, 0
    return (ctypes.c_uint64 * max(1, len(vals)))(*[int(v) for v in vals]), len(vals)


def _stream(s) -> Optional[int]:
    if s is None:
        return None
    if isinstance(s, int):
        return s or None
    return s.cuda_stream or None


def _done(rc: int) -> None:
    if rc < 0:
        _check(rc)


def _check(rc: int) -> int:
    if rc < 0:
        raise ReftError(rc, (_load().reft_last_error() or b"").decode())
    return rc


# ------------------------------------------------------------------------------------------------
# entry points (same names and argument order as include/reft.h)
# ------------------------------------------------------------------------------------------------
def reft_plan_create(span_nbytes: Sequence[int], bucket_nbytes: Optional[Sequence[int]] = None,
                     uniform_bucket: int = 0) -> int:
    """Returns the plan handle (an opaque address).  Destroy with :func:`reft_plan_destroy`."""
    lib = _load()
    spans, T = _u64s(span_nbytes)
    buckets, NB = _u64s(bucket_nbytes)
    out = ctypes.c_void_p()
    _check(lib.reft_plan_create(spans, T, buckets, NB, int(uniform_bucket), ctypes.byref(out)))
    return out.value


def reft_plan_destroy(plan) -> None:
    _load().reft_plan_destroy(plan)


def reft_plan_stream_bytes(plan) -> int:
    return int(_load().reft_plan_stream_bytes(plan))


def reft_plan_num_spans(plan) -> int:
    return int(_load().reft_plan_num_spans(plan))


def reft_plan_num_buckets(plan) -> int:
    return int(_load().reft_plan_num_buckets(plan))


def reft_plan_max_bucket_bytes(plan) -> int:
    return int(_load().reft_plan_max_bucket_bytes(plan))


def reft_plan_staging_slot_bytes(plan) -> int:
    return int(_load().reft_plan_staging_slot_bytes(plan))


def reft_plan_bucket_range(plan, b: int):
    lo, hi = ctypes.c_uint64(), ctypes.c_uint64()
    _check(_load().reft_plan_bucket_range(plan, int(b), ctypes.byref(lo), ctypes.byref(hi)))
    return lo.value, hi.value


def reft_plan_span_offset(plan, t: int) -> int:
    v = ctypes.c_uint64()
    _check(_load().reft_plan_span_offset(plan, int(t), ctypes.byref(v)))
    return v.value


def reft_plan_tile_info(plan):
    """(tile_bytes, ntiles)"""
    a, b = ctypes.c_uint64(), ctypes.c_uint64()
    _check(_load().reft_plan_tile_info(plan, ctypes.byref(a), ctypes.byref(b)))
    return a.value, b.value


def reft_plan_tile_first_span(plan, t: int) -> int:
    v = ctypes.c_uint64()
    _check(_load().reft_plan_tile_first_span(plan, int(t), ctypes.byref(v)))
    return v.value


def reft_plan_split(plan, t_bubble: float, t_ss: float) -> int:
    cut = ctypes.c_uint64()
    _check(_load().reft_plan_split(plan, float(t_bubble), float(t_ss), ctypes.byref(cut)))
    return cut.value


def reft_snapshot_pack(plan, span_ptrs, staging, host_dst, pack_stream=None, copy_stream=None,
                       staging_bytes: Optional[int] = None, host_cap: Optional[int] = None) -> None:
    _check(_load().reft_snapshot_pack(
        plan, ptr_array(span_ptrs), _addr(staging),
        (0 if staging is None else _nbytes(staging)) if staging_bytes is None else int(staging_bytes),
        _addr(host_dst), _nbytes(host_dst) if host_cap is None else int(host_cap),
        _stream(pack_stream), _stream(copy_stream)))


def reft_snapshot_pack_range(plan, span_ptrs, staging, host_dst, bucket_begin: int, bucket_end: int,
                             pack_stream=None, copy_stream=None,
                             staging_bytes: Optional[int] = None,
                             host_cap: Optional[int] = None) -> None:
    _check(_load().reft_snapshot_pack_range(
        plan, ptr_array(span_ptrs), _addr(staging),
        (0 if staging is None else _nbytes(staging)) if staging_bytes is None else int(staging_bytes),
        _addr(host_dst), _nbytes(host_dst) if host_cap is None else int(host_cap),
        int(bucket_begin), int(bucket_end), _stream(pack_stream), _stream(copy_stream)))


def reft_plan_bucket_of(plan, offset: int) -> int:
    b = ctypes.c_uint64()
    _check(_load().reft_plan_bucket_of(plan, int(offset), ctypes.byref(b)))
    return b.value


def reft_ckpt_create(plan, host_buf0, host_buf1, cap: Optional[int] = None) -> int:
    out = ctypes.c_void_p()
    _check(_load().reft_ckpt_create(plan, _addr(host_buf0), _addr(host_buf1),
                                    min(_nbytes(host_buf0), _nbytes(host_buf1)) if cap is None
                                    else int(cap), ctypes.byref(out)))
    return out.value


def reft_ckpt_destroy(ckpt) -> None:
    _load().reft_ckpt_destroy(ckpt)


def reft_ckpt_begin(ckpt):
    """(address of the ongoing host buffer, generation)"""
    dst, gen = ctypes.c_void_p(), ctypes.c_uint64()
    _check(_load().reft_ckpt_begin(ckpt, ctypes.byref(dst), ctypes.byref(gen)))
    return dst.value, gen.value


def reft_ckpt_commit(ckpt, stream=None) -> None:
    _check(_load().reft_ckpt_commit(ckpt, _stream(stream)))


def reft_ckpt_latest(ckpt):
    """(address of the newest complete host snapshot or None, its generation or 0)"""
    src, gen = ctypes.c_void_p(), ctypes.c_uint64()
    _check(_load().reft_ckpt_latest(ckpt, ctypes.byref(src), ctypes.byref(gen)))
    return src.value, gen.value


def reft_ckpt_wait(ckpt) -> None:
    _check(_load().reft_ckpt_wait(ckpt))


def reft_plan_staged_work(plan):
    """(gather kernel launches, copies) of a staged snapshot of the whole stream"""
    a, b = ctypes.c_uint64(), ctypes.c_uint64()
    _check(_load().reft_plan_staged_work(plan, ctypes.byref(a), ctypes.byref(b)))
    return a.value, b.value


def reft_plan_burst_stats(plan):
    """(rounds met, rounds timed out, rounds not waited, group completions) of the last burst launch"""
    v = (ctypes.c_uint64 * 4)()
    _check(_load().reft_plan_burst_stats(plan, v))
    return tuple(int(x) for x in v)


def reft_recovery_plan(k: int, copy_offsets: Sequence[int], parity_units: bool, lost: Sequence[int]):
    """``lost``: the lost members' indices.  Returns (steps, recoverable) with steps a list of
    (member, how, source, which); ``recoverable`` is False where the library answers
    REFT_EUNRECOVERABLE (the steps of the members that can be recovered still come back)."""
    lib = _load()
    flags = (ctypes.c_uint8 * max(1, k))(*[1 if x in set(lost) else 0 for x in range(k)])
    offs = (ctypes.c_uint32 * max(1, len(copy_offsets)))(*[int(d) for d in copy_offsets])
    steps = (ctypes.c_uint32 * (4 * max(1, k)))()
    n = ctypes.c_uint32()
    rc = lib.reft_recovery_plan(int(k), offs, len(copy_offsets), 1 if parity_units else 0, flags,
                                steps, ctypes.byref(n))
    if rc not in (REFT_OK, REFT_EUNRECOVERABLE):
        _check(rc)
    out = [tuple(steps[4 * j:4 * j + 4]) for j in range(n.value)]
    return out, rc == REFT_OK


def reft_snapshot_wait(plan) -> None:
    _check(_load().reft_snapshot_wait(plan))


def reft_snapshot_query(plan) -> bool:
    return bool(_check(_load().reft_snapshot_query(plan)))


def reft_pack_device(plan, span_ptrs, dst_dev, stream=None, dst_cap: Optional[int] = None) -> None:
    _check(_load().reft_pack_device(plan, ptr_array(span_ptrs), _addr(dst_dev),
                                    _nbytes(dst_dev) if dst_cap is None else int(dst_cap),
                                    _stream(stream)))


def reft_unpack_device(plan, src_dev, span_ptrs, stream=None,
                       src_bytes: Optional[int] = None) -> None:
    _check(_load().reft_unpack_device(plan, _addr(src_dev),
                                      _nbytes(src_dev) if src_bytes is None else int(src_bytes),
                                      ptr_array(span_ptrs), _stream(stream)))


def reft_parity_encode(plan, shard_span_ptrs, k: int, parity_dev, stream=None) -> None:
    """``shard_span_ptrs``: k*T entries, row-major (entry s*T + t = span t of shard s)."""
    _check(_load().reft_parity_encode(plan, ptr_array(shard_span_ptrs), int(k), _addr(parity_dev),
                                      _stream(stream)))


def reft_parity_encode_pack(plan, shard_span_ptrs, k: int, own: int, parity_dev, packed_dev,
                            stream=None, packed_cap: Optional[int] = None) -> None:
    _check(_load().reft_parity_encode_pack(plan, ptr_array(shard_span_ptrs), int(k), int(own),
                                           _addr(parity_dev), _addr(packed_dev),
                                           _nbytes(packed_dev) if packed_cap is None else int(packed_cap),
                                           _stream(stream)))


def reft_parity_encode_noalloc(plan, shard_span_ptrs, k: int, parity_dev, stream=None) -> None:
    _check(_load().reft_parity_encode_noalloc(plan, ptr_array(shard_span_ptrs), int(k),
                                              _addr(parity_dev), _stream(stream)))


def reft_reconstruct(shards, parity, L: int, out_dev, stream=None) -> int:
    """``shards``: the k packed streams with ``None`` for the lost one.  Returns the lost index."""
    lost = ctypes.c_uint32(0xFFFFFFFF)
    _check(_load().reft_reconstruct(ptr_array(shards), len(shards), _addr(parity), int(L),
                                    _addr(out_dev), ctypes.byref(lost), _stream(stream)))
    return lost.value


def reft_reconstruct_spans(plan, shard_span_ptrs, k: int, lost: int, parity_dev, out_span_ptrs,
                           stream=None) -> None:
    _check(_load().reft_reconstruct_spans(plan, ptr_array(shard_span_ptrs), int(k), int(lost),
                                          _addr(parity_dev), ptr_array(out_span_ptrs),
                                          _stream(stream)))


def reft_segment_bytes(plan, k: int) -> int:
    return int(_load().reft_segment_bytes(plan, int(k)))


def reft_parity_encode_rotated(plan, shard_span_ptrs, k: int, member: int, parity_dev,
                               stream=None) -> None:
    _check(_load().reft_parity_encode_rotated(plan, ptr_array(shard_span_ptrs), int(k), int(member),
                                              _addr(parity_dev), _stream(stream)))


def reft_reconstruct_rotated(plan, shard_span_ptrs, parity_ptrs, k: int, lost: int, out_span_ptrs,
                             stream=None) -> None:
    _check(_load().reft_reconstruct_rotated(plan, ptr_array(shard_span_ptrs), ptr_array(parity_ptrs),
                                            int(k), int(lost), ptr_array(out_span_ptrs),
                                            _stream(stream)))


def reft_restore(plan, host_src, staging, span_ptrs, copy_stream=None, unpack_stream=None,
                 host_bytes: Optional[int] = None, staging_bytes: Optional[int] = None) -> None:
    _check(_load().reft_restore(
        plan, _addr(host_src), _nbytes(host_src) if host_bytes is None else int(host_bytes),
        _addr(staging),
        (0 if staging is None else _nbytes(staging)) if staging_bytes is None else int(staging_bytes),
        ptr_array(span_ptrs), _stream(copy_stream), _stream(unpack_stream)))


def reft_restore_wait(plan) -> None:
    _check(_load().reft_restore_wait(plan))


# ------------------------------------------------------------------------------------------------
# operators of a training step: sizes, row lengths and types are those of the tensors given, which are written without a word to
# autograd; kernels run on `stream`, or the default stream (not torch's current one) where it is None
# ------------------------------------------------------------------------------------------------
_TYPES = {"torch.float32": REFT_F32, "torch.bfloat16": REFT_BF16, "torch.float16": REFT_F16,
          "torch.float8_e4m3fn": REFT_E4M3, "torch.float8_e5m2": REFT_E5M2}
_TYPE_OF: dict = {}                       # the same by torch.dtype, filled as they are met (and told to _marshal)
_FLOATS, _EIGHTS = (REFT_F32, REFT_BF16, REFT_F16), (REFT_E4M3, REFT_E5M2)
_OR_F32 = {REFT_F32: (REFT_F32,), REFT_BF16: (REFT_BF16, REFT_F32), REFT_F16: (REFT_F16, REFT_F32)}
_ONLY = {c: (c,) for c in _FLOATS + _EIGHTS}
_JUST_F32 = (REFT_F32,)
_NONE = (None, 0, 0)


def _refuse(who: str, what: str):
    raise ReftError(REFT_EINVAL, f"{who}: {what}")


def _type(t):
    """The number of a tensor's type; None if no operator takes it."""
    code = _TYPE_OF.get(t.dtype)
    if code is None and str(t.dtype) in _TYPES:
        code = _TYPE_OF[t.dtype] = _TYPES[str(t.dtype)]
        _load_marshal().know(t.dtype, code)
    return code


# Each operator's call goes through _marshal first (reft_marshal.c), which makes it where every operand is as expected.  What
# follows takes what is unusual but right (a type met for the first time, one row of any stride, no weight, pinned host memory), and
# says what is wrong.
def _tensors(who: str, operands: dict, needed: str) -> None:
    """Sizes, row lengths and types are read off the operands: an address alone will not do."""
    for name, t in operands.items():
        if t is None:
            if name in needed.split():
                _refuse(who, f"{name} is left out")
        elif not (hasattr(t, "data_ptr") and hasattr(t, "stride")):
            _refuse(who, f"{name} is no tensor but {type(t).__name__}")


def _counter(who: str, name: str, v) -> int:
    """A seed or an offset: 64 bits, where -1 stands for 2^64 - 1 and so on."""
    v = operator.index(v)
    if not -2 ** 63 <= v < 2 ** 64:
        _refuse(who, f"{name} has more than 64 bits")
    return v


def _matrix(who: str, name: str, t, shape, types):
    """(address, row length, type) of a 2-D tensor of that shape whose rows are contiguous."""
    if len(shape) != 2 or tuple(t.shape) != tuple(shape):
        _refuse(who, f"{name} has the shape {tuple(t.shape)}" + (f", not {tuple(shape)}" if len(shape) == 2 else ""))
    code = _type(t)
    if code not in types:
        _refuse(who, f"{name} is {t.dtype}")
    down, along = t.stride()
    if along != 1 and shape[1] > 1:
        _refuse(who, f"{name}'s rows are not contiguous")
    return t.data_ptr(), down if shape[0] > 1 else shape[1], code


def _vector(who: str, name: str, t, n: int, types):
    """(address, type) of a contiguous vector of n values."""
    code = _type(t)
    if code not in types or t.shape != (n,) or not t.is_contiguous():
        _refuse(who, f"{name} is no contiguous vector of {n} values of a type that it may have")
    return t.data_ptr(), code


def _scales(who: str, name: str, t, rows: int, cols: int):
    """(address, words from one word of a row to its next) of bytes [ceil(cols / 512)][rows][4]."""
    words = (cols + 511) >> 9
    if t.shape != (words, rows, 4) or t.element_size() != 1:
        _refuse(who, f"{name} are not bytes [{words}][{rows}][4]")
    wide, row, one = t.stride()
    if (one != 1 or (rows > 1 and row != 4) or (words > 1 and wide % 4)) and t.numel():
        _refuse(who, f"{name}: the words of a row's scales are not contiguous")
    return t.data_ptr(), wide // 4 if words > 1 else rows


def _scratch(who: str, t):
    """(address, bytes) of memory without gaps: what lies in them is not the call's to write."""
    if t is None:
        return None, 0
    if not t.is_contiguous():
        _refuse(who, "the workspace is not contiguous")
    return t.data_ptr(), t.numel() * t.element_size()


_CHECK_ONLY = 2 ** 64 - 1                 # in place of a stream: the library checks its arguments and enqueues nothing


def _seen(t) -> bool:
    """Whether kernels on the current GPU may read and write the tensor: its own memory, or pinned host memory."""
    if t is None or t.numel() == 0:
        return True
    if t.get_device() < 0:
        return t.is_pinned()
    device = ctypes.c_int()
    return _load().hipGetDevice(ctypes.byref(device)) == 0 and t.get_device() == device.value


def _call(who: str, fn, operands: dict, stream, *args) -> None:
    """A library call where every operand is seen; else what is wrong with it, beginning with what the library says."""
    unseen = [name for name, t in operands.items() if not _seen(t)]
    _check(fn(*args, _CHECK_ONLY if unseen else _stream(stream)))
    if unseen:
        _refuse(who, f"{unseen[0]} is on {operands[unseen[0]].device}, and not in memory that the current GPU sees")


def reft_dropout(x, y, p: float, seed: int, offset: int = 0, stream=None) -> None:
    """``y`` (may be ``x``) gets ``x`` with elements dropped by the counter (seed, offset)."""
    rc = (_marshal or _load_marshal()).dropout(x, y, p, seed, offset, stream)
    if rc is not None:
        return _done(rc)
    who, operands = "reft_dropout", dict(x=x, y=y)
    _tensors(who, operands, "x y")
    ax, ld_x, code = _matrix(who, "x", x, x.shape, _FLOATS)
    rows, cols = shape = x.shape
    ay, ld_y, _ = _matrix(who, "y", y, shape, _ONLY[code])
    _call(who, _load().reft_dropout, operands, stream, ax, ld_x, ay, ld_y, rows, cols, code, p, _counter(who, "seed", seed),
          _counter(who, "offset", offset))


def reft_norm_forward(x, residual, weight, eps: float, p: float = 0.0, seed: int = 0, offset: int = 0, *, h=None,
                      rstd=None, y=None, q=None, scales=None, stream=None) -> None:
    rc = (_marshal or _load_marshal()).norm_forward(x, residual, weight, eps, p, seed, offset, h, rstd, y, q, scales, stream)
    if rc is not None:
        return _done(rc)
    who, operands = "reft_norm_forward", dict(x=x, residual=residual, weight=weight, h=h, rstd=rstd, y=y, q=q, scales=scales)
    _tensors(who, operands, "x")
    ax, ld_x, code = _matrix(who, "x", x, x.shape, _FLOATS)
    rows, cols = shape = x.shape
    wide = _OR_F32[code]
    ar, ld_r, r_code = (None, 0, None) if residual is None else _matrix(who, "residual", residual, shape, wide)
    ah, ld_h, h_code = (None, 0, code) if h is None else _matrix(who, "h", h, shape, wide if r_code is None else _ONLY[r_code])
    aw, w_code = (None, code) if weight is None else _vector(who, "weight", weight, cols, wide)
    arstd = None if rstd is None else _vector(who, "rstd", rstd, rows, _JUST_F32)[0]
    ay, ld_y, _ = _NONE if y is None else _matrix(who, "y", y, shape, _ONLY[code])
    aq, ld_q, fmt = _NONE if q is None else _matrix(who, "q", q, shape, _EIGHTS)
    asc, ld_s = (None, 0) if scales is None else _scales(who, "scales", scales, rows, cols)
    _call(who, _load().reft_norm_forward, operands, stream, ax, ld_x, ar, ld_r, aw, rows, cols, code,
          h_code if r_code is None else r_code, w_code, eps, p, _counter(who, "seed", seed), _counter(who, "offset", offset), ah, ld_h,
          arstd, ay, ld_y, aq, ld_q, fmt, asc, ld_s)


def reft_norm_backward(dy, dh, h, rstd, weight, p: float = 0.0, seed: int = 0, offset: int = 0, *, dres=None, dx=None,
                       dweight=None, workspace=None, stream=None) -> None:
    rc = (_marshal or _load_marshal()).norm_backward(dy, dh, h, rstd, weight, p, seed, offset, dres, dx, dweight, workspace, stream)
    if rc is not None:
        return _done(rc)
    who = "reft_norm_backward"
    operands = dict(dy=dy, dh=dh, h=h, rstd=rstd, weight=weight, dres=dres, dx=dx, dweight=dweight, workspace=workspace)
    _tensors(who, operands, "dy h")
    ady, ld_dy, code = _matrix(who, "dy", dy, dy.shape, _FLOATS)
    rows, cols = shape = dy.shape
    wide = _OR_F32[code]
    ah, ld_h, r_code = _matrix(who, "h", h, shape, wide)
    adh, ld_dh, _ = _NONE if dh is None else _matrix(who, "dh", dh, shape, _ONLY[r_code])
    arstd = None if rstd is None else _vector(who, "rstd", rstd, rows, _JUST_F32)[0]
    aw, w_code = (None, code) if weight is None else _vector(who, "weight", weight, cols, wide)
    adres, ld_dres, _ = _NONE if dres is None else _matrix(who, "dres", dres, shape, _ONLY[r_code])
    adx, ld_dx, _ = _NONE if dx is None else _matrix(who, "dx", dx, shape, _ONLY[code])
    adw = None if dweight is None else _vector(who, "dweight", dweight, cols, _JUST_F32)[0]
    ws, ws_bytes = _scratch(who, workspace)
    _call(who, _load().reft_norm_backward, operands, stream, ady, ld_dy, adh, ld_dh, ah, ld_h, arstd, aw, rows, cols, code, r_code,
          w_code, p, _counter(who, "seed", seed), _counter(who, "offset", offset), adres, ld_dres, adx, ld_dx, adw, ws, ws_bytes)


def reft_norm_backward_workspace(rows: int, cols: int) -> int:
    return int(_load().reft_norm_backward_workspace(int(rows), int(cols)))


def reft_quantize(x, q=None, scales=None, q_t=None, scales_t=None, *, blocks: bool = False, stream=None) -> None:
    """``q`` and ``q_t`` are float8 tensors of the shape of ``x`` and of its transpose."""
    rc = (_marshal or _load_marshal()).quantize(x, q, scales, q_t, scales_t, blocks, stream)
    if rc is not None:
        return _done(rc)
    who, operands = "reft_quantize", dict(x=x, q=q, scales=scales, q_t=q_t, scales_t=scales_t)
    _tensors(who, operands, "x")
    ax, ld_x, code = _matrix(who, "x", x, x.shape, _FLOATS)
    rows, cols = shape = x.shape
    aq, ld_q, fmt = (None, 0, None) if q is None else _matrix(who, "q", q, shape, _EIGHTS)
    at, ld_t, fmt_t = _NONE if q_t is None else _matrix(who, "q_t", q_t, (cols, rows), _EIGHTS if fmt is None else _ONLY[fmt])
    tall, wide = ((rows + 127) >> 7, (cols + 127) >> 7) if blocks else (rows, cols)
    asc, ld_s = (None, 0) if scales is None else _scales(who, "scales", scales, tall, cols)
    ast, ld_st = (None, 0) if scales_t is None else _scales(who, "scales_t", scales_t, wide, rows)
    _call(who, _load().reft_quantize, operands, stream, ax, ld_x, rows, cols, code, fmt_t if fmt is None else fmt, 1 if blocks else 0,
          aq, ld_q, asc, ld_s, at, ld_t, ast, ld_st)


def reft_product(a, a_scales, b, b_scales, c, workspace=None, *, b_blocks: bool = False, stream=None) -> None:
    """``c`` [M, N] = ``a`` [M, K] times the transpose of ``b`` [N, K], both float8 with their scales."""
    rc = (_marshal or _load_marshal()).product(a, a_scales, b, b_scales, c, workspace, b_blocks, stream)
    if rc is not None:
        return _done(rc)
    who, operands = "reft_product", dict(a=a, a_scales=a_scales, b=b, b_scales=b_scales, c=c, workspace=workspace)
    _tensors(who, operands, "a b c")
    aa, ld_a, fa = _matrix(who, "a", a, a.shape, _EIGHTS)
    ab, ld_b, fb = _matrix(who, "b", b, b.shape, _EIGHTS)
    M, K = a.shape
    N, K2 = b.shape
    if K != K2:
        _refuse(who, f"a has {K} columns and b {K2}")
    asa, ld_as = (None, 0) if a_scales is None else _scales(who, "a_scales", a_scales, M, K)
    asb, ld_bs = (None, 0) if b_scales is None else _scales(who, "b_scales", b_scales, (N + 127) >> 7 if b_blocks else N, K)
    ac, ld_c, fc = _matrix(who, "c", c, (M, N), _FLOATS)
    ws, ws_bytes = _scratch(who, workspace)
    _call(who, _load().reft_product, operands, stream, aa, ld_a, fa, asa, ld_as, ab, ld_b, fb, asb, ld_bs, 1 if b_blocks else 0, M, N, K,
          ac, ld_c, fc, ws, ws_bytes)


def reft_product_workspace(M: int, N: int, K: int) -> int:
    return int(_load().reft_product_workspace(int(M), int(N), int(K)))


def reft_set_tunable(name: str, value: int) -> None:
    _check(_load().reft_set_tunable(name.encode(), int(value)))


def reft_get_tunable(name: str) -> int:
    v = ctypes.c_uint64()
    _check(_load().reft_get_tunable(name.encode(), ctypes.byref(v)))
    return v.value


def reft_last_error() -> str:
    return (_load().reft_last_error() or b"").decode()


def reft_version() -> str:
    return _load().reft_version().decode()
