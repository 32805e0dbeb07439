"""Thin ctypes binding of libcomet (include/comet.h): same entry-point names,
argument marshalling only.  Every step of the codec runs in the HIP kernels of
``libcomet.so``; PyTorch supplies device tensors and streams, nothing else.

The library must have been built (``python -m paper_2111_09562_amd.build``);
there is no fallback: a missing library raises at first use.
"""
from __future__ import annotations

import ctypes as C
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcomet.so")

OK, ERR_INVALID, ERR_CAPACITY, ERR_FORMAT, ERR_HIP, ERR_NOMEM, ERR_INTERNAL, ERR_CODEBOOK = 0, -1, -2, -3, -4, -5, -6, -7
HEADER_BYTES = 128
DEFAULT_CHUNK_SYMS = 64

EXPORTS = (
    "comet_create", "comet_destroy", "comet_set_chunk_syms", "comet_set_zero_chunks", "comet_compress_bound", "comet_compress", "comet_compress_with_codebook",
    "comet_decompress", "comet_decompress_static", "comet_compress_16", "comet_decompress_16", "comet_sync", "comet_peek", "comet_adapt_defaults", "comet_adapt_eb", "comet_abs_mean",
    "comet_controller_init", "comet_controller_tick", "comet_controller_update",
    "comet_rope_steps", "comet_rope", "comet_cache_bytes", "comet_cache_append", "comet_cache_fetch", "comet_cache_attend_work", "comet_cache_attend",
    "comet_stage_quantize", "comet_stage_codebook", "comet_stage_encode", "comet_stage_decode",
    "comet_stage_reconstruct", "comet_profile_enable", "comet_profile_reset", "comet_profile_read", "comet_strerror",
)
KERNEL_NAMES = ("k_quantize_rows", "k_codebook", "k_encode_pack", "k_decode_tables", "k_scan_store", "k_decode_chunks",
                "k_gather_records", "k_encode_count", "k_decode_scan")


class Shape(C.Structure):
    _fields_ = [("n", C.c_uint32), ("c", C.c_uint32), ("h", C.c_uint32), ("w", C.c_uint32)]


class Info(C.Structure):
    _fields_ = [("shape", Shape), ("nbins", C.c_uint32), ("chunk_syms", C.c_uint32), ("n_chunks", C.c_uint32),
                ("n_active", C.c_uint32), ("max_len", C.c_uint32), ("n_outlier_records", C.c_uint32),
                ("n_value_records", C.c_uint32), ("eb", C.c_float), ("nnz", C.c_uint64),
                ("payload_words", C.c_uint64), ("total_bytes", C.c_uint64)]


class LayerStats(C.Structure):
    _fields_ = [("momentum_abs_mean", C.c_double), ("loss_grad_mean", C.c_double), ("nonzero_ratio", C.c_double),
                ("batch", C.c_uint32)]


class AdaptCfg(C.Structure):
    _fields_ = [("a", C.c_double), ("sigma_frac", C.c_double), ("eb_min", C.c_float), ("eb_max", C.c_float)]


class CacheShape(C.Structure):
    _fields_ = [("n_pages", C.c_uint32), ("page_tokens", C.c_uint32), ("n_slots", C.c_uint32), ("heads", C.c_uint32), ("dim", C.c_uint32)]


class CacheBatch(C.Structure):
    _fields_ = [("n_seqs", C.c_uint32), ("table_width", C.c_uint32), ("dev_starts", C.c_void_p), ("dev_lens", C.c_void_p),
                ("dev_table", C.c_void_p), ("dev_slots", C.c_void_p)]


class CacheRows(C.Structure):
    _fields_ = [("dev", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class RopePlan(C.Structure):
    _fields_ = [("rot", C.c_uint32), ("layout", C.c_uint32), ("amp", C.c_float), ("dev_steps", C.c_void_p)]


class RopeCfg(C.Structure):
    _fields_ = [("rot", C.c_uint32), ("scaling", C.c_uint32), ("base", C.c_double), ("factor", C.c_double), ("original_len", C.c_double),
                ("beta_fast", C.c_double), ("beta_slow", C.c_double)]


class CometError(RuntimeError):
    def __init__(self, code: int, where: str):
        super().__init__(f"{where}: {strerror(code)} ({code})")
        self.code = code


_lib = None


def lib():
    """Load libcomet.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2111_09562_amd.build`")
        L = C.CDLL(LIB_PATH)
        vp, u64 = C.c_void_p, C.c_uint64
        L.comet_create.argtypes = [C.POINTER(vp), u64, C.c_uint32]
        L.comet_destroy.argtypes = [vp]
        L.comet_destroy.restype = None
        L.comet_set_chunk_syms.argtypes = [vp, C.c_uint32]
        L.comet_set_zero_chunks.argtypes = [vp, C.c_int]
        L.comet_compress_bound.argtypes = [Shape, C.c_uint32, C.c_uint32]
        L.comet_compress_bound.restype = u64
        L.comet_compress.argtypes = [vp, vp, Shape, C.c_float, C.c_uint32, vp, vp, u64, C.POINTER(u64)]
        L.comet_compress_with_codebook.argtypes = [vp, vp, Shape, C.c_float, C.c_uint32, vp, vp, vp, u64, C.POINTER(u64)]
        L.comet_decompress.argtypes = [vp, vp, u64, Shape, vp, vp]
        L.comet_decompress_static.argtypes = [vp, u64, Shape, vp, vp, vp]
        L.comet_compress_16.argtypes = [vp, vp, C.c_int, Shape, C.c_float, C.c_uint32, vp, vp, u64, C.POINTER(u64)]
        L.comet_decompress_16.argtypes = [vp, vp, u64, Shape, C.c_int, vp, vp]
        L.comet_sync.argtypes = [vp, vp]
        L.comet_abs_mean.argtypes = [vp, vp, u64, vp, C.POINTER(C.c_double)]
        L.comet_controller_init.argtypes = [vp, C.c_uint32]
        L.comet_controller_tick.argtypes = [vp, C.POINTER(C.c_int)]
        L.comet_controller_update.argtypes = [vp, vp, vp, C.c_uint32]
        L.comet_peek.argtypes = [vp, vp, u64, vp, C.POINTER(Info)]
        L.comet_adapt_defaults.argtypes = [C.POINTER(AdaptCfg)]
        L.comet_adapt_defaults.restype = None
        L.comet_adapt_eb.argtypes = [C.POINTER(LayerStats), C.POINTER(AdaptCfg), C.POINTER(C.c_float)]
        u32, i32 = C.c_uint32, C.c_int
        batch, plan = C.POINTER(CacheBatch), C.POINTER(RopePlan)
        L.comet_rope_steps.argtypes = [C.POINTER(RopeCfg), vp, C.POINTER(C.c_float)]
        L.comet_rope.argtypes = [plan, CacheRows, CacheRows, u32, u32, u32, i32, vp, i32, vp]
        L.comet_cache_bytes.argtypes = [CacheShape]
        L.comet_cache_append.argtypes = [vp, CacheShape, batch, u32, CacheRows, CacheRows, CacheRows, CacheRows, u32, i32, plan, vp, vp, vp]
        L.comet_cache_fetch.argtypes = [vp, CacheShape, batch, u32, CacheRows, CacheRows, i32, vp, vp]
        L.comet_cache_attend_work.argtypes = [CacheShape, u32, u32, u32]
        L.comet_cache_attend.argtypes = [vp, CacheShape, batch, u32, CacheRows, u32, i32, C.c_float, i32, CacheRows, vp, vp, u64, vp, vp]
        L.comet_cache_bytes.restype = L.comet_cache_attend_work.restype = u64
        L.comet_stage_quantize.argtypes = [vp, vp, Shape, C.c_float, C.c_uint32, vp, vp, vp, vp, u64, vp]
        L.comet_stage_codebook.argtypes = [vp, vp, C.c_uint32, vp, vp, vp]
        L.comet_stage_encode.argtypes = [vp, vp, u64, C.c_uint32, C.c_uint32, vp, vp, vp, u64, vp]
        L.comet_stage_decode.argtypes = [vp, vp, C.c_uint32, vp, vp, u64, u64, C.c_uint32, vp, vp]
        L.comet_stage_reconstruct.argtypes = [vp, vp, vp, u64, Shape, C.c_uint32, C.c_float, vp, vp]
        L.comet_profile_enable.argtypes = [vp, C.c_int]
        L.comet_profile_reset.argtypes = [vp]
        L.comet_profile_read.argtypes = [vp, C.c_uint32, C.POINTER(C.c_uint32), C.POINTER(C.c_double)]
        L.comet_strerror.argtypes = [C.c_int]
        L.comet_strerror.restype = C.c_char_p
        for name in EXPORTS:
            if name not in ("comet_destroy", "comet_compress_bound", "comet_adapt_defaults", "comet_strerror", "comet_cache_bytes",
                            "comet_cache_attend_work"):
                getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


def strerror(code: int) -> str:
    return lib().comet_strerror(code).decode()


def _chk(rc: int, where: str) -> None:
    if rc != OK:
        raise CometError(rc, where)


F16, BF16 = 1, 2


def _dtype16(t) -> int:
    name = str(t.dtype)
    if name == "torch.float16":
        return F16
    if name == "torch.bfloat16":
        return BF16
    raise TypeError(f"float16 or bfloat16 tensor expected, got {name}")


def _ptr(t):
    """Device pointer of a torch tensor (or None)."""
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device, contiguous tensors only"
    return C.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is None:
        import torch
        return C.c_void_p(torch.cuda.current_stream().cuda_stream)
    return C.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def _shape(shape) -> Shape:
    n, c, h, w = (int(v) for v in shape)
    return Shape(n, c, h, w)


def comet_compress_bound(shape, nbins: int, chunk_syms: int = DEFAULT_CHUNK_SYMS) -> int:
    return int(lib().comet_compress_bound(_shape(shape), nbins, chunk_syms))


def comet_adapt_eb(momentum_abs_mean: float, loss_grad_mean: float, nonzero_ratio: float, batch: int,
                   a: float | None = None, sigma_frac: float | None = None,
                   eb_min: float | None = None, eb_max: float | None = None) -> float:
    st = LayerStats(momentum_abs_mean, loss_grad_mean, nonzero_ratio, batch)
    cfg = AdaptCfg()
    lib().comet_adapt_defaults(C.byref(cfg))
    if a is not None:
        cfg.a = a
    if sigma_frac is not None:
        cfg.sigma_frac = sigma_frac
    if eb_min is not None:
        cfg.eb_min = eb_min
    if eb_max is not None:
        cfg.eb_max = eb_max
    out = C.c_float()
    _chk(lib().comet_adapt_eb(C.byref(st), C.byref(cfg), C.byref(out)), "comet_adapt_eb")
    return out.value


STATIC_MAX_ELEMS = 4 << 20


def comet_decompress_static(container, nbytes: int, shape, out, status=None, stream=None) -> None:
    """comet_decompress without a context (the library's static scratch array; allocates nothing).
    status: optional int32 device tensor of one element that receives 0 or ERR_FORMAT."""
    _chk(lib().comet_decompress_static(_ptr(container), int(nbytes), _shape(shape), _stream(stream), _ptr(out), _ptr(status)),
         "comet_decompress_static")


class ControllerState(C.Structure):
    _fields_ = [("w_default", C.c_uint32), ("w", C.c_uint32), ("since", C.c_uint32)]


class Controller:
    """The active factor W of the controller (host-side counter)."""

    def __init__(self, w_default: int = 0):
        self._s = ControllerState()
        _chk(lib().comet_controller_init(C.byref(self._s), int(w_default)), "comet_controller_init")

    @property
    def w(self) -> int:
        return int(self._s.w)

    def comet_controller_tick(self) -> bool:
        c = C.c_int()
        _chk(lib().comet_controller_tick(C.byref(self._s), C.byref(c)), "comet_controller_tick")
        return bool(c.value)

    def comet_controller_update(self, eb_old, eb_new) -> int:
        n = len(eb_old)
        assert n == len(eb_new)
        a = (C.c_float * n)(*[float(v) for v in eb_old])
        b = (C.c_float * n)(*[float(v) for v in eb_new])
        _chk(lib().comet_controller_update(C.byref(self._s), a, b, n), "comet_controller_update")
        return self.w


class Context:
    """Owns one comet_ctx (device workspace).  One per stream."""

    def __init__(self, max_elems: int, max_nbins: int = 65536):
        self._h = C.c_void_p()
        _chk(lib().comet_create(C.byref(self._h), int(max_elems), int(max_nbins)), "comet_create")

    def close(self):
        if getattr(self, "_h", None) is not None and self._h:
            lib().comet_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def comet_set_zero_chunks(self, enable: bool) -> None:
        """Containers of version 2: chunks that hold the centre code only take no payload words."""
        _chk(lib().comet_set_zero_chunks(self._h, 1 if enable else 0), "comet_set_zero_chunks")

    def comet_set_chunk_syms(self, chunk_syms: int) -> None:
        _chk(lib().comet_set_chunk_syms(self._h, chunk_syms), "comet_set_chunk_syms")

    def comet_compress(self, x, eb: float, nbins: int, out, stream=None, sync: bool = True):
        """x: fp32 NCHW device tensor; out: uint8 device tensor (the container buffer).
        Returns the container size in bytes when sync, else None."""
        assert x.dim() == 4 and str(x.dtype) == "torch.float32"
        used = C.c_uint64()
        rc = lib().comet_compress(self._h, _ptr(x), _shape(x.shape), C.c_float(eb), nbins, _stream(stream), _ptr(out),
                                  out.numel() * out.element_size(), C.byref(used) if sync else None)
        _chk(rc, "comet_compress")
        return int(used.value) if sync else None

    def comet_compress_with_codebook(self, x, eb: float, nbins: int, dev_len, out, stream=None, sync: bool = True):
        """As comet_compress, with the code lengths of an earlier compression: dev_len is a uint8 device tensor of
        nbins entries (e.g. ``earlier_container[HEADER_BYTES:HEADER_BYTES + nbins]``)."""
        assert x.dim() == 4 and str(x.dtype) == "torch.float32"
        assert str(dev_len.dtype) == "torch.uint8" and dev_len.numel() == nbins and dev_len.is_contiguous()
        used = C.c_uint64()
        rc = lib().comet_compress_with_codebook(self._h, _ptr(x), _shape(x.shape), C.c_float(eb), nbins, _ptr(dev_len),
                                                _stream(stream), _ptr(out), out.numel() * out.element_size(),
                                                C.byref(used) if sync else None)
        _chk(rc, "comet_compress_with_codebook")
        return int(used.value) if sync else None

    def comet_decompress(self, container, nbytes: int, shape, out, stream=None) -> None:
        _chk(lib().comet_decompress(self._h, _ptr(container), int(nbytes), _shape(shape), _stream(stream), _ptr(out)),
             "comet_decompress")

    def comet_compress_16(self, x, eb: float, nbins: int, out, stream=None, sync: bool = True):
        """As comet_compress for a float16 or bfloat16 NCHW device tensor."""
        assert x.dim() == 4
        used = C.c_uint64()
        rc = lib().comet_compress_16(self._h, _ptr(x), _dtype16(x), _shape(x.shape), C.c_float(eb), nbins, _stream(stream),
                                     _ptr(out), out.numel() * out.element_size(), C.byref(used) if sync else None)
        _chk(rc, "comet_compress_16")
        return int(used.value) if sync else None

    def comet_decompress_16(self, container, nbytes: int, shape, out, stream=None) -> None:
        """As comet_decompress into a float16 or bfloat16 device tensor."""
        _chk(lib().comet_decompress_16(self._h, _ptr(container), int(nbytes), _shape(shape), _dtype16(out), _stream(stream),
                                       _ptr(out)), "comet_decompress_16")

    def comet_abs_mean(self, x, stream=None) -> float:
        """Mean of |x| over a contiguous fp32 device tensor (synchronises the stream)."""
        assert str(x.dtype) == "torch.float32" and x.is_contiguous()
        out = C.c_double()
        _chk(lib().comet_abs_mean(self._h, _ptr(x), x.numel(), _stream(stream), C.byref(out)), "comet_abs_mean")
        return out.value

    def comet_sync(self, stream=None) -> None:
        _chk(lib().comet_sync(self._h, _stream(stream)), "comet_sync")

    def comet_peek(self, container, nbytes: int, stream=None) -> Info:
        info = Info()
        _chk(lib().comet_peek(self._h, _ptr(container), int(nbytes), _stream(stream), C.byref(info)), "comet_peek")
        return info

    def comet_profile_enable(self, enable: bool) -> None:
        _chk(lib().comet_profile_enable(self._h, 1 if enable else 0), "comet_profile_enable")

    def comet_profile_reset(self) -> None:
        _chk(lib().comet_profile_reset(self._h), "comet_profile_reset")

    def comet_profile_read(self, kernel_id: int):
        """(launches, total milliseconds) of one kernel since the last reset."""
        n, ms = C.c_uint32(), C.c_double()
        _chk(lib().comet_profile_read(self._h, kernel_id, C.byref(n), C.byref(ms)), "comet_profile_read")
        return int(n.value), float(ms.value)

    # ---- stage-level entry points -------------------------------------------------
    def comet_stage_quantize(self, x, eb: float, nbins: int, codes, hist, records, counts, stream=None) -> None:
        cap = 0 if records is None else records.numel() // 2
        _chk(lib().comet_stage_quantize(self._h, _ptr(x), _shape(x.shape), C.c_float(eb), nbins, _stream(stream), _ptr(codes),
                                        _ptr(hist), _ptr(records), cap, _ptr(counts)), "comet_stage_quantize")

    def comet_stage_codebook(self, hist, nbins: int, lens, codes=None, stream=None) -> None:
        _chk(lib().comet_stage_codebook(self._h, _ptr(hist), nbins, _stream(stream), _ptr(lens), _ptr(codes)),
             "comet_stage_codebook")

    def comet_stage_encode(self, codes, n: int, nbins: int, chunk_syms: int, chunk_off, payload, payload_words, stream=None) -> None:
        _chk(lib().comet_stage_encode(self._h, _ptr(codes), n, nbins, chunk_syms, _stream(stream), _ptr(chunk_off), _ptr(payload),
                                      payload.numel(), _ptr(payload_words)), "comet_stage_encode")

    def comet_stage_decode(self, lens, nbins: int, chunk_off, payload, payload_words: int, n: int, chunk_syms: int, codes_out,
                           stream=None) -> None:
        _chk(lib().comet_stage_decode(self._h, _ptr(lens), nbins, _ptr(chunk_off), _ptr(payload), payload_words, n, chunk_syms,
                                      _stream(stream), _ptr(codes_out)), "comet_stage_decode")

    def comet_stage_reconstruct(self, codes, records, n_records: int, shape, nbins: int, eb: float, out, stream=None) -> None:
        _chk(lib().comet_stage_reconstruct(self._h, _ptr(codes), _ptr(records), n_records, _shape(shape), nbins, C.c_float(eb),
                                           _stream(stream), _ptr(out)), "comet_stage_reconstruct")


# ---- keys and values of attention layers ----------------------------------------------------------------------------
F32 = 0
CACHE_BLOCK = 32
ROPE_SCALING = {"none": 0, "linear": 1, "base": 2, "parts": 3}


def _elsewhere(dev: int, stream):
    """Contexts that make the tensors' device current and, where a stream is given, that stream: memory for results then comes from the
    allocator's pool of the stream that uses it.  None where the call can go ahead as it is."""
    import torch
    if dev < 0:
        raise ValueError("device tensors only")
    if stream is None:
        return None if torch._C._cuda_getDevice() == dev else torch.cuda.device(dev)
    if not hasattr(stream, "cuda_stream"):
        stream = torch.cuda.ExternalStream(int(stream), device=torch.device("cuda", dev)) if int(stream) else torch.cuda.default_stream(dev)
    if stream.device.index != dev:
        raise ValueError(f"a stream of device {stream.device.index} for tensors on device {dev}")
    return torch.cuda.stream(stream)                 # (makes the stream's device current, too)


def _no_gradient(where: str, *tensors) -> None:
    """These calls have no gradient: where one is asked for they would lose it without a word."""
    for t in tensors:
        if t is not None and t is not True and t.requires_grad:
            import torch
            if torch.is_grad_enabled():
                raise RuntimeError(f"{where}: a tensor asks for a gradient, which this call does not have (a rotation has one in autograd.rotate; "
                                   "detach the tensor, or call under torch.no_grad())")


def _written(*tensors) -> None:
    """Tells autograd that tensors of the caller were written: a graph that saved one refuses its backward pass."""
    import torch
    tensors = [t for t in tensors if t is not None and not t.is_inference()]
    if tensors:
        torch.autograd.graph.increment_version(tensors)


def _raw_stream(dev: int) -> int:
    import torch
    return torch._C._cuda_getCurrentRawStream(dev)


def _int32(t, where: str, dev: int, *shape):
    """Device pointer of a contiguous int32 tensor of that shape (None: any) on that device."""
    if str(t.dtype) != "torch.int32" or not t.is_contiguous() or t.dim() != len(shape) or any(n is not None and n != m for n, m in zip(shape, t.shape)):
        raise ValueError(f"{where}: contiguous int32 tensor of shape {shape} expected, got {t.dtype} {tuple(t.shape)}")
    if t.get_device() != dev:
        raise ValueError(f"{where}: on another device than the other tensors")
    return t.data_ptr()


def _rows3(t, where: str, dev: int, tokens, heads, dim, dtype) -> CacheRows:
    """A [tokens, heads, dim] tensor (None: any) of a type on a device, its heads' values contiguous."""
    if t.dim() != 3:
        raise ValueError(f"{where}: tensor of three dimensions expected, got {tuple(t.shape)}")
    s = t.shape
    if s[0] != tokens or (heads is not None and s[1] != heads) or s[2] != dim:
        raise ValueError(f"{where}: tensor of [tokens={tokens}, heads={heads}, dim={dim}] expected, got {tuple(s)}")
    if t.dtype is not dtype:
        raise TypeError(f"{where}: {dtype} expected, got {t.dtype}")
    if t.get_device() != dev:
        raise ValueError(f"{where}: on another device than the other tensors")
    a, b, c = t.stride()
    if c != 1 and dim > 1:
        raise ValueError(f"{where}: the values of a head must be contiguous")
    return CacheRows(t.data_ptr(), a, b)


def _row_dtype(t) -> int:
    return F32 if str(t.dtype) == "torch.float32" else _dtype16(t)


def _status_ptr(status, dev: int):
    if status is None:
        return None
    if str(status.dtype) != "torch.int32" or status.numel() != 1 or status.get_device() != dev:
        raise ValueError("status: int32 tensor of one element on the device of the others expected")
    return status.data_ptr()


def comet_rope_steps(rot: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, original_len: float = 4096,
                     beta_fast: float = 32.0, beta_slow: float = 1.0):
    """(steps, amp) of a rotation: turns per position of every pair in units of 2^-64, the factor on the turned values."""
    if scaling not in ROPE_SCALING:
        raise ValueError(f"scaling: one of {sorted(ROPE_SCALING)} expected, got {scaling!r}")
    cfg = RopeCfg(int(rot), ROPE_SCALING[scaling], base, factor, original_len, beta_fast, beta_slow)
    steps, amp = (C.c_uint64 * max(1, int(rot) // 2))(), C.c_float()
    _chk(lib().comet_rope_steps(C.byref(cfg), steps, C.byref(amp)), "comet_rope_steps")
    return list(steps), amp.value


class Rope:
    """A rotation by positions, its steps in device memory: the first `rot` values of a head in pairs (i, i + rot/2), or (2i, 2i + 1)
    if interleaved; scaling "none", "linear", "base" or "parts" for contexts `factor` times as long as original_len.  amp: the factor on the
    turned values, if it is not to be the scaling's own (1 but for "parts")."""

    def __init__(self, rot: int, base: float = 10000.0, interleaved: bool = False, scaling: str = "none", factor: float = 1.0,
                 original_len: float = 4096, beta_fast: float = 32.0, beta_slow: float = 1.0, device=None, amp: float | None = None):
        import torch
        steps, self.amp = comet_rope_steps(rot, base, scaling, factor, original_len, beta_fast, beta_slow)
        if amp is not None:
            self.amp = C.c_float(amp).value
            if not abs(self.amp) < float("inf"):
                raise ValueError(f"amp: a number of float32 expected, got {amp}")
        self.rot, self.interleaved = int(rot), bool(interleaved)
        self.steps = torch.tensor(steps, dtype=torch.int64).to(torch.device("cuda", torch.cuda.current_device()) if device is None else device)
        self.device_index = self.steps.get_device()
        self._plan = RopePlan(self.rot, 1 if interleaved else 0, self.amp, self.steps.data_ptr())


def comet_rope(x, rope: Rope, positions=None, out=None, backward: bool = False, stream=None):
    """x [tokens, heads, dim] (fp32, fp16 or bf16, any strides with contiguous heads) turned by its tokens' positions (int32, or None for
    0, 1, ..); backward: the other way.  out: the result's tensor, x itself is fine.  Has no gradient (``autograd.rotate`` has)."""
    _no_gradient("comet_rope", x, out)
    dev = x.get_device()
    on = _elsewhere(dev, stream)
    if on is not None:
        with on:
            return comet_rope(x, rope, positions, out, backward)
    if x.dim() != 3:
        raise ValueError(f"comet_rope: x [tokens, heads, dim] expected, got {tuple(x.shape)}")
    tokens, heads, dim = x.shape
    rx = _rows3(x, "comet_rope: x", dev, tokens, heads, dim, x.dtype)
    given = out
    if out is None:
        out = x.new_empty((tokens, heads, dim))
    ry = _rows3(out, "comet_rope: out", dev, tokens, heads, dim, x.dtype)
    if rope.device_index != dev:
        raise ValueError("comet_rope: the rotation's steps are on another device")
    pos = None if positions is None else _int32(positions, "comet_rope: positions", dev, tokens)
    _chk(lib().comet_rope(rope._plan, rx, ry, tokens, heads, dim, _row_dtype(x), pos, 1 if backward else 0, _raw_stream(dev)), "comet_rope")
    if given is not None:
        _written(given)
    return out


class Batch:
    """Which tokens of which sequences a call on a cache is about (int32 device tensors, read when the call runs): starts [n + 1], lens [n]
    (tokens held once the batch's are in), table [n, pages], slots [n] or None.  A length may be set back between calls, never to less than
    CACHE_BLOCK tokens below the greatest it has been, nor into a block of a page that another sequence shares."""

    def __init__(self, starts, lens, table, slots=None):
        dev = self.device_index = lens.get_device()
        if dev < 0:
            raise ValueError("Batch: device tensors only")
        n = self.n_seqs = lens.shape[0]
        self.tensors = (starts, lens, table, slots)
        self._c = CacheBatch(n, table.shape[1], _int32(starts, "Batch: starts", dev, n + 1), _int32(lens, "Batch: lens", dev, n),
                             _int32(table, "Batch: table", dev, n, None), None if slots is None else _int32(slots, "Batch: slots", dev, n))


class Cache:
    """Keys and values in blocks of 32 tokens, 8 bits a value; one device buffer (`buf`: uint8, allocated if None)."""

    def __init__(self, n_pages: int, page_tokens: int, n_slots: int, heads: int, dim: int, buf=None, device=None):
        import torch
        self.shape = CacheShape(int(n_pages), int(page_tokens), int(n_slots), int(heads), int(dim))
        self.heads, self.dim = int(heads), int(dim)
        self.nbytes = comet_cache_bytes(n_pages, page_tokens, n_slots, heads, dim)
        if not self.nbytes:
            raise CometError(ERR_INVALID, "comet_cache_bytes")
        if buf is None:
            buf = torch.empty(self.nbytes, dtype=torch.uint8, device=torch.device("cuda", torch.cuda.current_device()) if device is None else device)
        if str(buf.dtype) != "torch.uint8" or not buf.is_contiguous() or buf.numel() < self.nbytes or not buf.is_cuda:
            raise ValueError(f"buf: contiguous uint8 device tensor of {self.nbytes} bytes expected")
        self.buf, self.device_index = buf, buf.get_device()
        self._p = buf.data_ptr()

    def _same(self, where: str, batch: Batch, rope=None) -> int:
        dev = self.device_index
        if batch.device_index != dev or (rope is not None and rope.device_index != dev):
            raise ValueError(f"{where}: cache, batch and rotation on different devices")
        return dev

    def comet_cache_append(self, batch: Batch, k, v, rope: Rope | None = None, q=None, q_out=None, positions=None, status=None, stream=None):
        """Put the batch's keys and values [tokens, heads, dim] (fp16 or bf16) into the cache, the keys turned by `rope` on the way.
        q [tokens, query heads, dim]: turned as well, into q_out (a new tensor if None; q itself is fine), which is returned.  Has no gradient."""
        _no_gradient("comet_cache_append", k, v, q, q_out)
        dev = self._same("comet_cache_append", batch, rope)
        on = _elsewhere(dev, stream)
        if on is not None:
            with on:
                return self.comet_cache_append(batch, k, v, rope, q, q_out, positions, status)
        tokens, dt, dim, given = k.shape[0], k.dtype, self.dim, q_out
        rk = _rows3(k, "comet_cache_append: k", dev, tokens, self.heads, dim, dt)
        rv = _rows3(v, "comet_cache_append: v", dev, tokens, self.heads, dim, dt)
        if q is not None:
            rq = _rows3(q, "comet_cache_append: q", dev, tokens, None, dim, dt)
            q_heads = q.shape[1]
            if q_out is None:
                q_out = q.new_empty((tokens, q_heads, dim))
            ro = _rows3(q_out, "comet_cache_append: q_out", dev, tokens, q_heads, dim, dt)
        elif q_out is None:
            q_heads, rq = 0, CacheRows()
            ro = rq
        else:
            raise ValueError("comet_cache_append: q_out without q")
        pos = None if positions is None else _int32(positions, "comet_cache_append: positions", dev, tokens)
        _chk(lib().comet_cache_append(self._p, self.shape, batch._c, tokens, rk, rv, rq, ro, q_heads, _dtype16(k), None if rope is None else rope._plan,
                                      pos, _raw_stream(dev), _status_ptr(status, dev)), "comet_cache_append")
        if given is not None:
            _written(given)
        return q_out

    def comet_cache_fetch(self, batch: Batch, k=None, v=None, dtype=None, tokens: int | None = None, status=None, stream=None):
        """The batch's keys and values as the cache holds them, (k, v): into the tensors given, or new ones of `dtype` with `tokens` rows (those
        that belong to no sequence stay as the allocator left them)."""
        import torch
        _no_gradient("comet_cache_fetch", k, v)
        dev = self._same("comet_cache_fetch", batch)
        on = _elsewhere(dev, stream)
        if on is not None:
            with on:
                return self.comet_cache_fetch(batch, k, v, dtype, tokens, status)
        given = v if k is None else k
        if given is not None:
            tokens = given.shape[0] if tokens is None else tokens
            dtype = given.dtype if dtype is None else dtype
        written = (k, v)
        if tokens is None or dtype is None:
            raise ValueError("comet_cache_fetch: tokens and dtype, or tensors for the result, expected")
        if k is None:
            k = torch.empty((tokens, self.heads, self.dim), dtype=dtype, device=self.buf.device)
        if v is None:
            v = torch.empty((tokens, self.heads, self.dim), dtype=dtype, device=self.buf.device)
        rk = _rows3(k, "comet_cache_fetch: k", dev, tokens, self.heads, self.dim, dtype)
        rv = _rows3(v, "comet_cache_fetch: v", dev, tokens, self.heads, self.dim, dtype)
        _chk(lib().comet_cache_fetch(self._p, self.shape, batch._c, tokens, rk, rv, _dtype16(k), _raw_stream(dev), _status_ptr(status, dev)),
             "comet_cache_fetch")
        if given is not None:
            _written(*written)
        return k, v

    def comet_cache_attend(self, batch: Batch, q, out=None, lse=None, scale: float | None = None, causal: bool = True, work=None, status=None,
                           stream=None):
        """Attention of the batch's queries [tokens, query heads, dim] over the cache; scale: 1 / sqrt(dim) if None.  lse: a float32 tensor
        [tokens, query heads] for the log-sum-exp of every row, or True for a new one; then (out, lse) is returned, else out.  work: uint8 tensor
        of comet_cache_attend_work bytes, allocated if None.  Has no gradient."""
        import torch
        _no_gradient("comet_cache_attend", q, out, lse)
        dev = self._same("comet_cache_attend", batch)
        on = _elsewhere(dev, stream)
        if on is not None:
            with on:
                return self.comet_cache_attend(batch, q, out, lse, scale, causal, work, status)
        tokens, dt, dim = q.shape[0], q.dtype, self.dim
        rq = _rows3(q, "comet_cache_attend: q", dev, tokens, None, dim, dt)
        q_heads = q.shape[1]
        given = (out, None if lse is True else lse)
        if out is None:
            out = q.new_empty((tokens, q_heads, dim))
        ro = _rows3(out, "comet_cache_attend: out", dev, tokens, q_heads, dim, dt)
        if lse is True:
            lse = q.new_empty((tokens, q_heads), dtype=torch.float32)
        elif lse is not None and (lse.dtype is not torch.float32 or not lse.is_contiguous() or tuple(lse.shape) != (tokens, q_heads) or lse.get_device() != dev):
            raise ValueError("comet_cache_attend: lse: contiguous float32 tensor [tokens, query heads] on the device of the others expected")
        L = lib()
        if work is None:
            need = L.comet_cache_attend_work(self.shape, batch.n_seqs, tokens, q_heads)
            if not need:
                raise CometError(ERR_INVALID, "comet_cache_attend_work")
            work = torch.empty(need, dtype=torch.uint8, device=q.device)
        elif not work.is_contiguous() or work.get_device() != dev:
            raise ValueError("comet_cache_attend: work: contiguous tensor on the device of the others expected")
        _chk(L.comet_cache_attend(self._p, self.shape, batch._c, tokens, rq, q_heads, _dtype16(q), dim ** -0.5 if scale is None else scale,
                                  1 if causal else 0, ro, None if lse is None else lse.data_ptr(), work.data_ptr(),
                                  work.numel() * work.element_size(), _raw_stream(dev), _status_ptr(status, dev)), "comet_cache_attend")
        if given[0] is not None or given[1] is not None:
            _written(*given)
        return out if lse is None else (out, lse)


def comet_cache_bytes(n_pages: int, page_tokens: int, n_slots: int, heads: int, dim: int) -> int:
    return int(lib().comet_cache_bytes(CacheShape(int(n_pages), int(page_tokens), int(n_slots), int(heads), int(dim))))


def comet_cache_attend_work(cache: Cache, n_seqs: int, n_tokens: int, q_heads: int) -> int:
    return int(lib().comet_cache_attend_work(cache.shape, int(n_seqs), int(n_tokens), int(q_heads)))
