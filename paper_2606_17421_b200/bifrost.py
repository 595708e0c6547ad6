"""ctypes binding of libbifrost's C ABI (include/bifrost.h): argument marshalling only.

Every function has the name and the argument order of its C counterpart.  Device buffers are
passed as torch CUDA tensors (or raw integer addresses); PyTorch is used for nothing but device
memory and streams.  There is no fallback: if the CUDA library has not been built, load() raises.
"""
from __future__ import annotations

import ctypes
import functools
import os
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libbifrost.so")

BF_OK = 0
BF_ERR_INVALID_ARG = -1
BF_ERR_BAD_PRIME = -2
BF_ERR_SHAPE = -3
BF_ERR_LEVEL = -4
BF_ERR_MISSING_KEY = -5
BF_ERR_OOM = -6
BF_ERR_CUDA = -7
BF_ERR_RANGE = -8
BF_ERR_TOO_LARGE = -9
BF_ERR_TIMEOUT = -10


BF_PLAN_COMPLEX_PACK = 1
BF_PLAN_MODDOWN_PER_OUTPUT = 2
BF_PLAN_DOUBLE_HOIST = 4


class bf_plan(ctypes.Structure):
    """bf_plan(tile_D, tau, bsgs_b, bsgs_g[, flags]); flags = BF_PLAN_* bits, 0 by default."""
    _fields_ = [("tile_D", ctypes.c_uint32), ("tau", ctypes.c_uint32),
                ("bsgs_b", ctypes.c_uint32), ("bsgs_g", ctypes.c_uint32), ("flags", ctypes.c_uint32)]


BF_F32 = 0
BF_F16 = 1
BF_BF16 = 2


_ROW_TYPES = {"torch.float32": BF_F32, "torch.float16": BF_F16, "torch.bfloat16": BF_BF16}
_KINDS = {}                       # torch dtype -> its name, which is slow to make, and its type of rows or None


def _kind(dtype):
    name = str(dtype)
    _KINDS[dtype] = kind = name, _ROW_TYPES.get(name)
    return kind


def _dense(tensor, dtype: str, what: str):
    if (_KINDS.get(tensor.dtype) or _kind(tensor.dtype))[0] != dtype or not tensor.is_contiguous():
        raise ValueError(f"{what}: a contiguous {dtype} tensor is wanted")
    return tensor.data_ptr()


def _where(tensor):
    """The number of the device that a tensor is on, -1 on the host, None where any device reaches it (pinned memory)."""
    device = tensor.get_device()
    return device if device >= 0 or not tensor.is_pinned() else None


def _common(*tensors):
    """The device of all of them; -1 where they are not on one."""
    devices = {_where(x) for x in tensors} - {None}
    return devices.pop() if len(devices) == 1 else -1 if devices else None


# Descriptors made of tensors (`of`) keep what calls compare with what they read and write: `device`, and of rows `extent`.  Those made of
# addresses have neither, and are taken at their word.

class bf_rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("row_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("type", ctypes.c_int32)]
    __slots__ = ("device", "extent", "__dict__")

    @classmethod
    def of(cls, tensor):
        """Rows [n][channels] or [n][heads][channels] of a tensor, which must live as long; any strides but the channels'."""
        shape, strides, kind = tensor.shape, tensor.stride(), (_KINDS.get(tensor.dtype) or _kind(tensor.dtype))[1]
        dims = len(strides)
        if (dims != 3 and dims != 2) or (strides[-1] != 1 and shape[-1] != 1):
            raise ValueError("rows are [n][channels] or [n][heads][channels] with the channels side by side")
        if kind is None:
            raise ValueError(f"rows are float32, float16 or bfloat16, not {tensor.dtype}")
        rows = cls(tensor.data_ptr(), strides[0], strides[1] if dims == 3 else 0, kind)
        rows.extent, device = shape, tensor.get_device()
        rows.device = device if device >= 0 else _where(tensor)
        return rows


class bf_q4_matrix(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("offsets", ctypes.c_void_p), ("row_bytes", ctypes.c_uint64),
                ("group_stride", ctypes.c_uint32), ("d_out", ctypes.c_uint32), ("d_in", ctypes.c_uint32), ("group", ctypes.c_uint32)]
    __slots__ = ("device", "__dict__")

    @classmethod
    def of(cls, codes, scales, offsets, d_in: int, group: int):
        """codes uint8 [d_out][row_bytes], scales (and offsets, or None) float16 [d_out][group_stride]; they must live as long."""
        c, s = codes.shape, scales.shape
        if offsets is not None and offsets.shape != s:
            raise ValueError("offsets have the shape of the scales")
        if len(c) != 2 or len(s) != 2 or c[0] != s[0]:
            raise ValueError("codes and scales have a row for each output")
        matrix = cls(_dense(codes, "torch.uint8", "codes"), _dense(scales, "torch.float16", "scales"),
                     None if offsets is None else _dense(offsets, "torch.float16", "offsets"), c[1], s[1], c[0], d_in, group)
        device = codes.get_device()
        if device < 0 or scales.get_device() != device or (offsets is not None and offsets.get_device() != device):
            device = _common(codes, scales) if offsets is None else _common(codes, scales, offsets)
        matrix.device = device
        return matrix


class bf_kv4_cache(ctypes.Structure):
    _fields_ = [("pool", ctypes.c_void_p), ("tables", ctypes.c_void_p), ("lengths", ctypes.c_void_p), ("refs", ctypes.c_void_p)] + \
               [(name, ctypes.c_uint32) for name in ("n_layers", "n_pages", "n_kv_heads", "head_dim", "group", "page_tokens", "n_seqs", "max_pages")]
    __slots__ = ("device", "__dict__")

    @classmethod
    def of(cls, pool, tables, lengths, refs, head_dim: int, group: int, page_tokens: int):
        """pool uint8 [layers][pages][kv heads][block bytes], tables int32 [seqs][max_pages], lengths int32 [seqs], refs int32 [pages];
        they must live as long."""
        layers, pages, heads, block = pool.shape
        if block != bf_kv4_block_bytes(head_dim, group, page_tokens):
            raise BifrostError(BF_ERR_SHAPE, "bf_kv4_cache", f"a block of {block} bytes")
        seqs, n_seqs, n_refs = tables.shape, lengths.shape, refs.shape
        if len(seqs) != 2 or len(n_seqs) != 1 or len(n_refs) != 1 or n_seqs[0] != seqs[0] or n_refs[0] != pages:
            raise BifrostError(BF_ERR_SHAPE, "bf_kv4_cache", "tables, lengths and refs do not fit together")
        cache = cls(_dense(pool, "torch.uint8", "pool"), _dense(tables, "torch.int32", "tables"), _dense(lengths, "torch.int32", "lengths"),
                    _dense(refs, "torch.int32", "refs"), layers, pages, heads, head_dim, group, page_tokens, seqs[0], seqs[1])
        device = pool.get_device()
        if device < 0 or tables.get_device() != device or lengths.get_device() != device or refs.get_device() != device:
            device = _common(pool, tables, lengths, refs)
        cache.device = device
        return cache


class BifrostError(RuntimeError):
    def __init__(self, code: int, where: str, detail: str = ""):
        self.code = code
        super().__init__(f"{where}: {bf_strerror(code)} ({code}) {detail}".strip())


_vp = ctypes.c_void_p
_u32 = ctypes.c_uint32
_u64 = ctypes.c_uint64
_lib = None

_SIGNATURES = {
    "bf_ctx_create": (ctypes.c_int, [ctypes.POINTER(_vp), _u32, ctypes.POINTER(_u64), _u32, ctypes.c_double,
                                     ctypes.POINTER(bf_plan), _vp]),
    "bf_ctx_destroy": (None, [_vp]),
    "bf_load_eval_keys": (ctypes.c_int, [_vp, ctypes.POINTER(_u32), _u32, _vp]),
    "bf_set_cache_budget": (ctypes.c_int, [_vp, _u64]),
    "bf_cache_bytes_used": (_u64, [_vp]),
    "bf_weights_bytes": (_u64, [_vp, _u32, _u32]),
    "bf_encode_weights": (ctypes.c_int, [_vp, _vp, _u32, _u32, ctypes.POINTER(_vp)]),
    "bf_encode_weights_split": (ctypes.c_int, [_vp, _vp, _u32, _u32, _u32, _u32, ctypes.POINTER(_vp)]),
    "bf_weights_free": (None, [_vp, _vp]),
    "bf_linear": (ctypes.c_int, [_vp, _vp, _u32, _vp, _vp, _u32, _u32, _vp, _u32]),
    "bf_linear_rescaled": (ctypes.c_int, [_vp, _vp, _u32, _vp, _vp, _u32, _u32, _vp, _u32, ctypes.POINTER(ctypes.c_double)]),
    "bf_device_status": (ctypes.c_int, [_vp]),
    "bf_set_graph_replay": (ctypes.c_int, [_vp, ctypes.c_int]),
    "bf_set_dependent_launch": (ctypes.c_int, [_vp, ctypes.c_int]),
    "bf_set_lanes": (ctypes.c_int, [_vp, ctypes.c_int]),
    "bf_set_compact_cache": (ctypes.c_int, [_vp, ctypes.c_int]),
    "bf_set_coefficient_cache": (ctypes.c_int, [_vp, ctypes.c_int]),
    "bf_set_encode_scratch": (ctypes.c_int, [_vp, _u64]),
    "bf_rescale": (ctypes.c_int, [_vp, _vp, _vp, _u32, _u32, ctypes.POINTER(ctypes.c_double)]),
    "bf_fold": (ctypes.c_int, [_vp, _vp, _u32]),
    "bf_linear_host": (ctypes.c_int, [_vp, _vp, _u32, _vp, _vp, _u32, _u32, _vp, _u32]),
    "bf_rotate": (ctypes.c_int, [_vp, _vp, _u32, _vp]),
    "bf_negacyclic_mul": (ctypes.c_int, [_vp, _vp, _vp, _vp, _u32]),
    "bf_negacyclic_mul_noalloc": (ctypes.c_int, [_vp, _vp, _vp, _vp, _u32]),
    "bf_noalloc_max_words": (_u64, []),
    "bf_weights_export": (ctypes.c_int, [_vp, _vp, _u32, _u32, _u32, _u32, _vp]),
    "bf_set_stage_timing": (ctypes.c_int, [_vp, ctypes.c_int]),
    "bf_get_stage_ms": (ctypes.c_int, [_vp, ctypes.POINTER(ctypes.c_float)]),
    "bf_set_kernel_timing": (ctypes.c_int, [_vp, ctypes.c_int]),
    "bf_kernel_categories": (ctypes.c_int, []),
    "bf_kernel_category_name": (ctypes.c_char_p, [ctypes.c_int]),
    "bf_get_kernel_stats": (ctypes.c_int, [_vp, ctypes.POINTER(_u64), ctypes.POINTER(ctypes.c_float)]),
    "bf_measure_imad_rate": (ctypes.c_int, [_vp, ctypes.POINTER(ctypes.c_double)]),
    "bf_measure_fma64_rate": (ctypes.c_int, [_vp, ctypes.POINTER(ctypes.c_double)]),
    "bf_get_key_stream_bytes": (ctypes.c_int, [_vp, ctypes.POINTER(_u64), ctypes.POINTER(_u64)]),
    "bf_get_mac_key_bytes": (ctypes.c_int, [_vp, ctypes.POINTER(_u64)]),
    "bf_trusted_create": (ctypes.c_int, [ctypes.POINTER(_vp), _u64, _vp]),
    "bf_trusted_destroy": (None, [_vp]),
    "bf_trusted_status": (ctypes.c_int, [_vp]),
    "bf_trusted_last_cuda_error": (ctypes.c_char_p, [_vp]),
    "bf_q4_linear": (ctypes.c_int, [_vp, _vp, _vp, _u32, _vp]),
    "bf_encode_weights_q4": (ctypes.c_int, [_vp, _vp, _u32, _u32, ctypes.POINTER(_vp)]),
    "bf_linear_q4": (ctypes.c_int, [_vp, _vp, _u32, _vp, _vp, _u32]),
    "bf_kv4_block_bytes": (_u64, [_u32, _u32, _u32]),
    "bf_kv4_grow": (ctypes.c_int, [_vp, _vp, _vp, _vp, _u32]),
    "bf_kv4_append": (ctypes.c_int, [_vp, _vp, _u32, _vp, _vp, _u32, _u32, _vp, _vp]),
    "bf_kv4_read": (ctypes.c_int, [_vp, _vp, _u32, _vp, _vp, _vp, _u32, _u32, _vp, _vp]),
    "bf_kv4_attention": (ctypes.c_int, [_vp, _vp, _u32, _vp, _vp, _u32, _u32, _u32, _vp, _u32, _vp, ctypes.c_float, _u32, _vp]),
    "bf_kv4_fork": (ctypes.c_int, [_vp, _vp, _vp, _vp, _u32]),
    "bf_kv4_free": (ctypes.c_int, [_vp, _vp, _vp, _u32]),
    "bf_kv4_compact": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp]),
    "bf_strerror": (ctypes.c_char_p, [ctypes.c_int]),
    "bf_last_cuda_error": (ctypes.c_char_p, [_vp]),
}


def exported_symbols() -> list[str]:
    return sorted(_SIGNATURES)


def load():
    """Load libbifrost.so.  Raises if it is missing: there is no other implementation to fall back to."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} not found: build it with `python -m paper_2606_17421_b200.build` "
                               "(there is no CPU fallback)")
        lib = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib


def _ptr(x):
    """Device or host address of a torch tensor / numpy array / int / None."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if hasattr(x, "data_ptr"):
        return x.data_ptr()
    if hasattr(x, "ctypes"):
        return x.ctypes.data
    raise TypeError(type(x))


def _check(code: int, where: str, ctx=None):
    if code != BF_OK:
        detail = ""
        if code == BF_ERR_CUDA and ctx:
            detail = (load().bf_last_cuda_error(ctx) or b"").decode()
        raise BifrostError(code, where, detail)


def bf_strerror(code: int) -> str:
    return load().bf_strerror(code).decode()


def bf_ctx_create(N: int, primes, n_ct_primes: int, scale: float, plan: bf_plan, cuda_stream: int = 0):
    arr = (_u64 * len(primes))(*primes)
    out = _vp()
    _check(load().bf_ctx_create(ctypes.byref(out), N, arr, n_ct_primes, scale, ctypes.byref(plan), cuda_stream),
           "bf_ctx_create")
    return out


def bf_ctx_destroy(ctx):
    load().bf_ctx_destroy(ctx)


def bf_load_eval_keys(ctx, rot_steps, n_keys: int, keys):
    arr = (_u32 * max(1, len(rot_steps)))(*rot_steps)
    _check(load().bf_load_eval_keys(ctx, arr, n_keys, _ptr(keys)), "bf_load_eval_keys", ctx)


def bf_set_cache_budget(ctx, nbytes: int):
    _check(load().bf_set_cache_budget(ctx, nbytes), "bf_set_cache_budget", ctx)


def bf_cache_bytes_used(ctx) -> int:
    return load().bf_cache_bytes_used(ctx)


def bf_weights_bytes(ctx, d_out: int, d_in: int) -> int:
    return load().bf_weights_bytes(ctx, d_out, d_in)


def bf_encode_weights(ctx, W, d_out: int, d_in: int):
    out = _vp()
    _check(load().bf_encode_weights(ctx, _ptr(W), d_out, d_in, ctypes.byref(out)), "bf_encode_weights", ctx)
    return out


def bf_encode_weights_split(ctx, W, d_out: int, d_in: int, bsgs_b: int, bsgs_g: int):
    out = _vp()
    _check(load().bf_encode_weights_split(ctx, _ptr(W), d_out, d_in, bsgs_b, bsgs_g, ctypes.byref(out)),
           "bf_encode_weights_split", ctx)
    return out


def bf_weights_free(ctx, w):
    load().bf_weights_free(ctx, w)


def bf_linear(ctx, ct_in, n_in: int, pt_weights, W_raw, d_out: int, d_in: int, ct_out, n_out: int):
    _check(load().bf_linear(ctx, _ptr(ct_in), n_in, pt_weights, _ptr(W_raw), d_out, d_in, _ptr(ct_out), n_out),
           "bf_linear", ctx)


def bf_device_status(ctx):
    """Synchronises; raises if a device-side wait gave up or the on-the-fly encoder overflowed."""
    _check(load().bf_device_status(ctx), "bf_device_status", ctx)


def bf_set_graph_replay(ctx, on: bool):
    _check(load().bf_set_graph_replay(ctx, 1 if on else 0), "bf_set_graph_replay", ctx)


def bf_set_compact_cache(ctx, on: bool):
    _check(load().bf_set_compact_cache(ctx, 1 if on else 0), "bf_set_compact_cache", ctx)


def bf_set_coefficient_cache(ctx, bits: int):
    _check(load().bf_set_coefficient_cache(ctx, bits), "bf_set_coefficient_cache", ctx)


def bf_set_encode_scratch(ctx, n_bytes: int):
    _check(load().bf_set_encode_scratch(ctx, n_bytes), "bf_set_encode_scratch", ctx)


def bf_set_lanes(ctx, n_lanes: int):
    _check(load().bf_set_lanes(ctx, n_lanes), "bf_set_lanes", ctx)


def bf_set_dependent_launch(ctx, on: bool):
    _check(load().bf_set_dependent_launch(ctx, 1 if on else 0), "bf_set_dependent_launch", ctx)


def bf_rescale(ctx, ct_in, ct_out, n_ct: int, level: int, scale: float | None = None):
    """Returns the new scale when `scale` is given."""
    s = ctypes.c_double(scale if scale is not None else 0.0)
    _check(load().bf_rescale(ctx, _ptr(ct_in), _ptr(ct_out), n_ct, level,
                             ctypes.byref(s) if scale is not None else None), "bf_rescale", ctx)
    return s.value if scale is not None else None


def bf_linear_rescaled(ctx, ct_in, n_in: int, pt_weights, W_raw, d_out: int, d_in: int, ct_low, n_out: int,
                       scale: float | None = None):
    """Returns the new scale when `scale` is given."""
    s = ctypes.c_double(scale if scale is not None else 0.0)
    _check(load().bf_linear_rescaled(ctx, _ptr(ct_in), n_in, pt_weights, _ptr(W_raw), d_out, d_in, _ptr(ct_low), n_out,
                                     ctypes.byref(s) if scale is not None else None), "bf_linear_rescaled", ctx)
    return s.value if scale is not None else None


def bf_linear_host(ctx, host_ct_in, n_in: int, pt_weights, W_raw, d_out: int, d_in: int, host_ct_out, n_out: int):
    _check(load().bf_linear_host(ctx, _ptr(host_ct_in), n_in, pt_weights, _ptr(W_raw), d_out, d_in,
                                 _ptr(host_ct_out), n_out), "bf_linear_host", ctx)


def bf_rotate(ctx, ct_in, steps: int, ct_out):
    _check(load().bf_rotate(ctx, _ptr(ct_in), steps, _ptr(ct_out)), "bf_rotate", ctx)


def bf_fold(ctx, ct, n_ct: int):
    """Sums the tau partial results inside n_ct full-level ciphertexts, in place."""
    _check(load().bf_fold(ctx, _ptr(ct), n_ct), "bf_fold", ctx)


def bf_negacyclic_mul(ctx, a, b, out, n_polys: int):
    _check(load().bf_negacyclic_mul(ctx, _ptr(a), _ptr(b), _ptr(out), n_polys), "bf_negacyclic_mul", ctx)


def bf_negacyclic_mul_noalloc(ctx, a, b, out, n_polys: int):
    """bf_negacyclic_mul without any device allocation: scratch is a fixed array in the library image."""
    _check(load().bf_negacyclic_mul_noalloc(ctx, _ptr(a), _ptr(b), _ptr(out), n_polys), "bf_negacyclic_mul_noalloc", ctx)


def bf_noalloc_max_words() -> int:
    return load().bf_noalloc_max_words()


def bf_weights_export(ctx, w, p: int, q: int, j: int, k: int, out):
    _check(load().bf_weights_export(ctx, w, p, q, j, k, _ptr(out)), "bf_weights_export", ctx)


def bf_set_stage_timing(ctx, on: bool):
    _check(load().bf_set_stage_timing(ctx, 1 if on else 0), "bf_set_stage_timing", ctx)


def bf_get_stage_ms(ctx) -> list[float]:
    arr = (ctypes.c_float * 4)()
    _check(load().bf_get_stage_ms(ctx, arr), "bf_get_stage_ms", ctx)
    return list(arr)


def bf_set_kernel_timing(ctx, on: bool):
    _check(load().bf_set_kernel_timing(ctx, 1 if on else 0), "bf_set_kernel_timing", ctx)


def bf_kernel_categories() -> int:
    return load().bf_kernel_categories()


def bf_kernel_category_name(cat: int) -> str:
    return load().bf_kernel_category_name(cat).decode()


def bf_get_kernel_stats(ctx) -> dict:
    """{category name: (launches, summed event ms)} since the previous call."""
    n = bf_kernel_categories()
    launches = (_u64 * n)()
    ms = (ctypes.c_float * n)()
    _check(load().bf_get_kernel_stats(ctx, launches, ms), "bf_get_kernel_stats", ctx)
    return {bf_kernel_category_name(c): (int(launches[c]), float(ms[c])) for c in range(n)}


def bf_measure_imad_rate(ctx) -> float:
    out = ctypes.c_double(0.0)
    _check(load().bf_measure_imad_rate(ctx, ctypes.byref(out)), "bf_measure_imad_rate", ctx)
    return out.value


def bf_measure_fma64_rate(ctx) -> float:
    out = ctypes.c_double(0.0)
    _check(load().bf_measure_fma64_rate(ctx, ctypes.byref(out)), "bf_measure_fma64_rate", ctx)
    return out.value


def bf_get_key_stream_bytes(ctx) -> tuple[int, int]:
    """(bytes counted once per distinct key of each launch, bytes counted once per rotation) since the previous call."""
    a, b = _u64(0), _u64(0)
    _check(load().bf_get_key_stream_bytes(ctx, ctypes.byref(a), ctypes.byref(b)), "bf_get_key_stream_bytes", ctx)
    return int(a.value), int(b.value)


def bf_get_mac_key_bytes(ctx) -> int:
    """Bytes of rotation keys that multiply-accumulates read since the previous call, once per key and launch."""
    a = _u64(0)
    _check(load().bf_get_mac_key_bytes(ctx, ctypes.byref(a)), "bf_get_mac_key_bytes", ctx)
    return int(a.value)


# ---- the trusted half: descriptors (bf_rows, bf_q4_matrix, bf_kv4_cache) are passed by reference, lists as int32 tensors or None

def _check_trusted(code: int, where: str, t):
    if code != BF_OK:
        detail = (load().bf_trusted_last_cuda_error(t) or b"").decode() if code == BF_ERR_CUDA and t else ""
        raise BifrostError(code, where, detail)


# A context made beside torch knows its device (`own` below, else None), a descriptor made of tensors theirs (None: any).

def _elsewhere(device, own, where: str, what: str):
    if device is not None and device != own and (device < 0 or own is not None):
        raise BifrostError(BF_ERR_INVALID_ARG, where, f"{what}: not on the context's device")


def _ref(struct, own, where: str):
    if struct is None:
        return None
    device = getattr(struct, "device", None)
    if device != own:
        _elsewhere(device, own, where, "a descriptor")
    return ctypes.addressof(struct)


def _plain_rows(rows, own, where: str, n: int, width: int):
    """Looks at n rows without heads, `width` channels side by side."""
    extent = getattr(rows, "extent", None)
    if extent is not None:
        _elsewhere(rows.device, own, where, "rows")
        if extent[0] < n or (extent[-1] if len(extent) == 2 else (extent[1] - 1) * rows.head_stride + extent[2]) < width:
            raise BifrostError(BF_ERR_SHAPE, where, f"rows {tuple(extent)} where {n} of {width} channels are wanted")


def _head_rows(rows, own, where: str, n: int, heads: int, width: int):
    """The address of n rows of heads."""
    if rows is None:
        return None
    extent = getattr(rows, "extent", None)
    if extent is not None:
        if rows.device != own:
            _elsewhere(rows.device, own, where, "rows")
        if extent[0] < n or extent[-1] < width or (extent[1] < heads if len(extent) == 3 else heads > 1):
            raise BifrostError(BF_ERR_SHAPE, where, f"rows {tuple(extent)} where {n} of {heads} heads of {width} channels are wanted")
    return ctypes.addressof(rows)


def _list(x, own, where: str, n: int, dtype: str = "torch.int32"):
    if x is None or isinstance(x, int):
        return x
    at = _dense(x, dtype, "a list")
    if x.get_device() != own:
        _elsewhere(_where(x), own, where, "a list")
    if x.numel() < n:
        raise BifrostError(BF_ERR_SHAPE, where, f"a list of {x.numel()} where {n} are wanted")
    return at


def bf_trusted_create(workspace_bytes: int = 0, cuda_stream: int = 0):
    out = _vp()
    _check_trusted(load().bf_trusted_create(ctypes.byref(out), workspace_bytes, cuda_stream), "bf_trusted_create", None)
    torch = sys.modules.get("torch")
    out.device = torch.cuda.current_device() if torch and torch.cuda.is_available() else None
    return out


def bf_trusted_destroy(t):
    load().bf_trusted_destroy(t)


def bf_trusted_status(t):
    """Synchronises; raises what the kernels found wrong in device memory since the last call."""
    _check_trusted(load().bf_trusted_status(t), "bf_trusted_status", t)


def bf_q4_linear(t, W: bf_q4_matrix, x: bf_rows, n: int, y: bf_rows):
    own = getattr(t, "device", None)
    try:                         # (in one go: the smallest products take as long as their arguments)
        xs, ys = x.extent, y.extent
        fits = W.device == own and x.device == own and y.device == own and xs[0] >= n and ys[0] >= n and xs[-1] >= W.d_in and ys[-1] >= W.d_out
    except AttributeError:
        fits = False
    if not fits:
        _ref(W, own, "bf_q4_linear")
        _plain_rows(x, own, "bf_q4_linear", n, W.d_in if W else 0)
        _plain_rows(y, own, "bf_q4_linear", n, W.d_out if W else 0)
    address = ctypes.addressof
    code = load().bf_q4_linear(t, W and address(W), x and address(x), n, y and address(y))
    if code:
        _check_trusted(code, "bf_q4_linear", t)


def bf_encode_weights_q4(ctx, W: bf_q4_matrix, bsgs_b: int = 0, bsgs_g: int = 0):
    out, where = _vp(), "bf_encode_weights_q4"
    _check(load().bf_encode_weights_q4(ctx, _ref(W, None, where), bsgs_b, bsgs_g, ctypes.byref(out)), where, ctx)
    return out


def bf_linear_q4(ctx, ct_in, n_in: int, W: bf_q4_matrix, ct_out, n_out: int):
    where = "bf_linear_q4"
    _check(load().bf_linear_q4(ctx, _ptr(ct_in), n_in, _ref(W, None, where), _ptr(ct_out), n_out), where, ctx)


@functools.lru_cache(None)
def bf_kv4_block_bytes(head_dim: int, group: int, page_tokens: int) -> int:
    return load().bf_kv4_block_bytes(head_dim, group, page_tokens)


# (rows that a call reads or writes are known here where each sequence has one: without `starts`)

def bf_kv4_grow(t, cache: bf_kv4_cache, seqs, counts, n: int):
    where, own = "bf_kv4_grow", getattr(t, "device", None)
    code = load().bf_kv4_grow(t, _ref(cache, own, where), _list(seqs, own, where, n), _list(counts, own, where, n), n)
    if code:
        _check_trusted(code, where, t)


def bf_kv4_append(t, cache: bf_kv4_cache, layer: int, seqs, starts, n: int, max_new: int, k: bf_rows, v: bf_rows):
    where, own = "bf_kv4_append", getattr(t, "device", None)
    at, known = _ref(cache, own, where), n if starts is None else 0
    heads, width = (cache.n_kv_heads, cache.head_dim) if at else (0, 0)
    code = load().bf_kv4_append(t, at, layer, _list(seqs, own, where, n), _list(starts, own, where, n + 1), n, max_new,
                                _head_rows(k, own, where, known, heads, width), _head_rows(v, own, where, known, heads, width))
    if code:
        _check_trusted(code, where, t)


def bf_kv4_read(t, cache: bf_kv4_cache, layer: int, seqs, starts, first, n: int, max_tokens: int, k: bf_rows, v: bf_rows):
    where, own = "bf_kv4_read", getattr(t, "device", None)
    at, known = _ref(cache, own, where), n if starts is None else 0
    heads, width = (cache.n_kv_heads, cache.head_dim) if at else (0, 0)
    code = load().bf_kv4_read(t, at, layer, _list(seqs, own, where, n), _list(starts, own, where, n + 1), _list(first, own, where, n), n, max_tokens,
                              _head_rows(k, own, where, known, heads, width), _head_rows(v, own, where, known, heads, width))
    if code:
        _check_trusted(code, where, t)


def bf_kv4_attention(t, cache: bf_kv4_cache, layer: int, seqs, starts, n: int, max_q: int, max_len: int, q: bf_rows, n_q_heads: int,
                     out: bf_rows, scale: float, window: int = 0, lse=None):
    where, own = "bf_kv4_attention", getattr(t, "device", None)
    at, known = _ref(cache, own, where), n if starts is None else 0
    width = cache.head_dim if at else 0
    code = load().bf_kv4_attention(t, at, layer, _list(seqs, own, where, n), _list(starts, own, where, n + 1), n, max_q, max_len,
                                   _head_rows(q, own, where, known, n_q_heads, width), n_q_heads, _head_rows(out, own, where, known, n_q_heads, width),
                                   scale, window, _list(lse, own, where, known * n_q_heads, "torch.float32"))
    if code:
        _check_trusted(code, where, t)


def bf_kv4_fork(t, cache: bf_kv4_cache, src, dst, n: int):
    where, own = "bf_kv4_fork", getattr(t, "device", None)
    code = load().bf_kv4_fork(t, _ref(cache, own, where), _list(src, own, where, n), _list(dst, own, where, n), n)
    if code:
        _check_trusted(code, where, t)


def bf_kv4_free(t, cache: bf_kv4_cache, seqs, n: int):
    where, own = "bf_kv4_free", getattr(t, "device", None)
    code = load().bf_kv4_free(t, _ref(cache, own, where), _list(seqs, own, where, n), n)
    if code:
        _check_trusted(code, where, t)


def bf_kv4_compact(t, cache: bf_kv4_cache, tables_out=None, refs_out=None, n_live=None):
    where, own = "bf_kv4_compact", getattr(t, "device", None)
    at = _ref(cache, own, where)
    entries, pages = (cache.n_seqs * cache.max_pages, cache.n_pages) if at else (0, 0)
    code = load().bf_kv4_compact(t, at, _list(tables_out, own, where, entries), _list(refs_out, own, where, pages), _list(n_live, own, where, 1))
    if code:
        _check_trusted(code, where, t)
