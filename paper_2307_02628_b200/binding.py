"""Thin ctypes binding of include/skipdecode.h: argument marshalling only.

Every step of the path runs in the CUDA library; torch is used here for device
memory, streams and nothing else.  Opening the library fails loudly when it has
not been built (`python -m paper_2307_02628_b200.build`); there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import os
import threading

import torch

from .shapes import ModelShape, storage_dtype

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libskipdecode.so")
_lib = None

SD_OK, SD_ERR_ARG, SD_ERR_STATE, SD_ERR_POSITION, SD_ERR_CAPACITY, SD_ERR_CUDA, SD_ERR_DEVICE = 0, -1, -2, -3, -4, -5, -6
SD_OPT_GRAPHS, SD_OPT_ATTN_CHUNK, SD_OPT_GEMM, SD_OPT_TIMING, SD_OPT_PDL, SD_OPT_PREFILL_ATTN, SD_OPT_GEMM_PERSISTENT, SD_OPT_GEMM_SPLITK, SD_OPT_DETERMINISTIC, SD_OPT_TEST_WAIT_EXPIRY, SD_OPT_ATTN_STAGED = 1, 2, 3, 4, 5, 8, 10, 11, 12, 13, 14
KERNEL_CLASSES = ("embed", "layernorm", "gemm_qkv", "kv_append", "attention", "lm_head", "gemm_out", "gemm_fc1", "gemm_fc2")

EXPORTS = ("sd_arena_bytes", "sd_create", "sd_schedule", "sd_schedule_compute", "sd_schedule_power_compute",
           "sd_schedule_custom", "sd_layer_capacity",
           "sd_prefill", "sd_decode_step", "sd_decode_step_static", "sd_rewind", "sd_launch_count", "sd_decode_step_host", "sd_greedy", "sd_sample_top_p", "sd_set_padding", "sd_set_rows", "sd_status", "sd_stats",
           "sd_set_option", "sd_kernel_time", "sd_kernel_time_reset", "sd_strerror", "sd_destroy",
           "sd_sample", "sd_cache_bytes", "sd_cache_create", "sd_cache_layer", "sd_cache_append", "sd_cache_read", "sd_cache_attention",
           "sd_cache_status", "sd_cache_set_option", "sd_cache_destroy", "sd_extend")


class SdConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "d_model", "n_heads", "d_ffn", "vocab", "max_pos",
                                          "max_batch", "max_prompt", "max_gen", "dtype")] + [("ln_eps", C.c_float)]


_PP = C.POINTER(C.c_void_p)
_LAYER_FIELDS = ("ln1_g", "ln1_b", "w_qkv", "b_qkv", "w_o", "b_o", "ln2_g", "ln2_b", "w_fc1", "b_fc1", "w_fc2", "b_fc2")


class SdWeights(C.Structure):
    _fields_ = [("tok_emb", C.c_void_p), ("pos_emb", C.c_void_p)] + [(n, _PP) for n in _LAYER_FIELDS] + \
               [("lnf_g", C.c_void_p), ("lnf_b", C.c_void_p), ("lm_head", C.c_void_p)]


class SdPlan(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("max_layers", "min_layers", "warmup", "gen_len", "full_capacity")]


class SdSampling(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("temperature", "top_k", "top_p", "min_p")]


class SdCacheConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "n_heads", "n_kv_heads", "head_dim", "page_len", "n_pages",
                                          "max_seqs", "max_tokens", "dtype")]


class SdBatch(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("pages", "first", "len")] + \
               [(n, C.c_int32) for n in ("n_seqs", "pages_per_seq", "n_tokens", "max_new", "max_len")]


class SdHeads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("row_stride", C.c_int64), ("head_stride", C.c_int64), ("dtype", C.c_int32)]


# element types of a paged cache and of the rows handed to its calls
SD_DTYPE_FP32, SD_DTYPE_BF16, SD_DTYPE_FP16, SD_DTYPE_INT8, SD_DTYPE_E4M3 = 0, 1, 2, 3, 4
_CACHE_TYPES = {"fp32": (SD_DTYPE_FP32, torch.float32), "bf16": (SD_DTYPE_BF16, torch.bfloat16),
                "int8": (SD_DTYPE_INT8, torch.int8), "e4m3": (SD_DTYPE_E4M3, torch.float8_e4m3fn)}
_ROW_TYPES = {torch.float32: SD_DTYPE_FP32, torch.bfloat16: SD_DTYPE_BF16, torch.float16: SD_DTYPE_FP16}
SD_CACHE_OPT_TEST_WAIT_EXPIRY = 1
# bits of the status words
STATUS_BAD_TOKEN, STATUS_WAIT_EXPIRED, STATUS_BAD_BATCH, STATUS_BAD_SETTING, STATUS_NOT_FINITE = 1, 2, 16, 32, 64


class SdError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        msg = lib().sd_strerror(code).decode() if _lib is not None else str(code)
        super().__init__(f"{where}: {msg} ({code})")


def lib() -> C.CDLL:
    """Opens libskipdecode.so (built in-tree) and declares the prototypes."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(f"{_LIB_PATH} is missing: build it with `python -m paper_2307_02628_b200.build`; "
                           "there is no fallback path")
    L = C.CDLL(_LIB_PATH)
    vp, i32p = C.c_void_p, C.POINTER(C.c_int32)
    L.sd_arena_bytes.argtypes = [C.POINTER(SdConfig), C.POINTER(SdPlan), C.POINTER(C.c_size_t)]
    L.sd_create.argtypes = [C.POINTER(SdConfig), C.POINTER(SdWeights), C.POINTER(SdPlan), vp, C.c_size_t, vp, C.POINTER(vp)]
    L.sd_schedule.argtypes = [vp, C.c_int, C.c_int, C.c_int, C.c_int, i32p, i32p]
    L.sd_schedule_compute.argtypes = [C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, i32p, i32p]
    L.sd_schedule_power_compute.argtypes = [C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, i32p, i32p]
    L.sd_schedule_custom.argtypes = [vp, i32p, C.c_int, C.c_int, i32p]
    L.sd_layer_capacity.argtypes = [C.POINTER(SdConfig), C.POINTER(SdPlan), i32p]
    L.sd_prefill.argtypes = [vp, vp, C.c_int, C.c_int, vp]
    L.sd_decode_step.argtypes = [vp, vp, C.c_int, vp]
    L.sd_decode_step_static.argtypes = [vp, vp, C.c_int, vp]
    L.sd_rewind.argtypes = [vp]
    L.sd_launch_count.argtypes = [vp, C.POINTER(C.c_int64)]
    L.sd_decode_step_host.argtypes = [vp, vp, C.c_int, vp]
    L.sd_greedy.argtypes = [vp, vp, C.c_int, vp]
    L.sd_set_padding.argtypes = [vp, vp, C.c_int]
    L.sd_set_rows.argtypes = [vp, vp, C.c_int]
    L.sd_sample_top_p.argtypes = [vp, vp, C.c_int, C.c_float, C.c_float, vp, vp]
    L.sd_status.argtypes = [vp, i32p]
    L.sd_stats.argtypes = [vp, C.POINTER(C.c_int64), C.POINTER(C.c_int64)]
    L.sd_set_option.argtypes = [vp, C.c_int, C.c_int]
    L.sd_kernel_time.argtypes = [vp, C.c_int, C.POINTER(C.c_double), C.POINTER(C.c_int64)]
    L.sd_kernel_time_reset.argtypes = [vp]
    L.sd_sample.argtypes = [vp, vp, C.c_int, C.POINTER(SdSampling), vp, vp]
    L.sd_cache_bytes.argtypes = [C.POINTER(SdCacheConfig), C.POINTER(C.c_size_t)]
    L.sd_cache_create.argtypes = [C.POINTER(SdCacheConfig), vp, C.c_size_t, vp, C.POINTER(vp)]
    L.sd_cache_layer.argtypes = [vp, C.c_int, C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), C.POINTER(vp)]
    L.sd_cache_append.argtypes = [vp, C.c_int, vp, vp, vp]          # structures by address
    L.sd_cache_read.argtypes = L.sd_cache_append.argtypes
    L.sd_cache_attention.argtypes = [vp, C.c_int, vp, vp, C.c_float, vp]
    L.sd_cache_status.argtypes = [vp, i32p]
    L.sd_cache_set_option.argtypes = [vp, C.c_int, C.c_int]
    L.sd_cache_destroy.argtypes = [vp]
    L.sd_cache_destroy.restype = None
    L.sd_extend.argtypes = [vp, vp, C.POINTER(SdBatch), vp, C.c_int, C.c_int, vp]
    L.sd_strerror.argtypes = [C.c_int]
    L.sd_strerror.restype = C.c_char_p
    L.sd_destroy.argtypes = [vp]
    L.sd_destroy.restype = None
    for name in EXPORTS:
        if name not in ("sd_strerror", "sd_destroy", "sd_cache_destroy"):
            getattr(L, name).restype = C.c_int
    _lib = L
    return L


def _check(code: int, where: str):
    if code != SD_OK:
        raise SdError(code, where)


def make_config(shape: ModelShape, max_batch: int, max_prompt: int, max_gen: int) -> SdConfig:
    return SdConfig(shape.n_layers, shape.d_model, shape.n_heads, shape.d_ffn, shape.vocab, shape.max_pos,
                    max_batch, max_prompt, max_gen, 0 if shape.dtype == "fp32" else 1, 1e-5)


def schedule_compute(n_layers: int, max_layers: int, min_layers: int, warmup: int, gen_len: int):
    """The library's integer schedule, host only: (n_active, top_begin) as lists."""
    n = (C.c_int32 * max(gen_len, 1))()
    t = (C.c_int32 * max(gen_len, 1))()
    _check(lib().sd_schedule_compute(n_layers, max_layers, min_layers, warmup, gen_len, n, t), "sd_schedule_compute")
    return list(n)[:gen_len], list(t)[:gen_len]


def schedule_power_compute(n_layers: int, max_layers: int, min_layers: int, warmup: int, gen_len: int, alpha: int):
    """Power-law budget table, host only: (n_active, top_begin) as lists."""
    n = (C.c_int32 * max(gen_len, 1))()
    t = (C.c_int32 * max(gen_len, 1))()
    _check(lib().sd_schedule_power_compute(n_layers, max_layers, min_layers, warmup, gen_len, alpha, n, t),
           "sd_schedule_power_compute")
    return list(n)[:gen_len], list(t)[:gen_len]


def layer_capacity(cfg: SdConfig, plan: SdPlan):
    cap = (C.c_int32 * cfg.n_layers)()
    _check(lib().sd_layer_capacity(C.byref(cfg), C.byref(plan), cap), "sd_layer_capacity")
    return list(cap)


def arena_bytes(cfg: SdConfig, plan: SdPlan) -> int:
    need = C.c_size_t(0)
    _check(lib().sd_arena_bytes(C.byref(cfg), C.byref(plan), C.byref(need)), "sd_arena_bytes")
    return need.value


def cache_bytes(cfg: SdCacheConfig) -> int:
    need = C.c_size_t(0)
    _check(lib().sd_cache_bytes(C.byref(cfg), C.byref(need)), "sd_cache_bytes")
    return need.value


def _raw_stream(index: int) -> int:
    """The handle of torch's current stream on a device (a plain integer; building a Stream object takes ten times as long)."""
    return torch._C._cuda_getCurrentRawStream(index)


class CacheBatch:
    """The sequences of a call and their new tokens (sd_batch).

    pages [n_seqs, pages_per_seq], first [n_seqs + 1], length [n_seqs]: int32 CUDA tensors, read by the device at the call (their
    contents may change between calls).  Rows first[s] .. first[s + 1] of the token tensors are the last positions of the
    length[s] of sequence s.  n_tokens, max_new, max_len: the host's bounds on the rows, on a sequence's new tokens and on its
    length (0: as far as the table reaches).
    """

    def __init__(self, pages: torch.Tensor, first: torch.Tensor, length: torch.Tensor, n_tokens: int, max_new: int, max_len: int = 0):
        for name, t in (("pages", pages), ("first", first), ("length", length)):
            if t.dtype != torch.int32 or not t.is_cuda or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous int32 CUDA tensor")
        if pages.dim() != 2 or first.shape != (pages.shape[0] + 1,) or length.shape != (pages.shape[0],):
            raise ValueError("shapes must be pages [n, pages_per_seq], first [n + 1], length [n]")
        if not pages.device == first.device == length.device:
            raise ValueError("pages, first and length must be on one device")
        self.pages, self.first, self.length, self.n_tokens = pages, first, length, int(n_tokens)
        self.device, self.index = pages.device, pages.device.index
        self.c = SdBatch(pages.data_ptr(), first.data_ptr(), length.data_ptr(), pages.shape[0], pages.shape[1], int(n_tokens), int(max_new), int(max_len))
        self.ref = C.addressof(self.c)


class _Described(threading.local):
    """The two tensors of a call as the library takes them: a pair for each thread, since other threads run between the filling and
    the call (new structures for every call take 0.5 us longer)."""

    def __init__(self):
        self.pair = (SdHeads(), SdHeads())
        self.refs = tuple(C.addressof(t) for t in self.pair)


class PagedCache:
    """A paged KV cache (sd_cache) in an arena of its own.

    dtype: "fp32", "bf16", "int8" or "e4m3".  Calls are enqueued on `stream` (default: a stream of its own).  When torch's current
    stream is another one, the two are ordered around every call, so tensors can be used as if the call ran on the current one.
    Several threads may call one cache; each call's work is enqueued as a whole.
    """

    def __init__(self, n_layers: int, n_heads: int, n_kv_heads: int, head_dim: int, page_len: int, n_pages: int,
                 max_seqs: int, max_tokens: int, dtype: str = "int8", device: str = "cuda:0", stream=None):
        if dtype not in _CACHE_TYPES:
            raise ValueError(f"dtype must be one of {sorted(_CACHE_TYPES)}")
        self.cfg = SdCacheConfig(n_layers, n_heads, n_kv_heads, head_dim, page_len, n_pages, max_seqs, max_tokens, _CACHE_TYPES[dtype][0])
        self.arena_bytes = cache_bytes(self.cfg)
        if not torch.cuda.is_available():
            raise RuntimeError("no CUDA device: the cache has no CPU fallback")
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.stream = stream if stream is not None else torch.cuda.Stream(device=self.device)
        self._index, self._raw = self.device.index, self.stream.cuda_stream
        self.arena = torch.empty(self.arena_bytes + 256, dtype=torch.uint8, device=self.device)
        self._base = (self.arena.data_ptr() + 255) // 256 * 256 - self.arena.data_ptr()
        self.h = C.c_void_p()
        self._fork()
        _check(lib().sd_cache_create(C.byref(self.cfg), self.arena.data_ptr() + self._base, self.arena_bytes,
                                     self.stream.cuda_stream, C.byref(self.h)), "sd_cache_create")
        self._join()
        L = lib()
        self._append, self._read, self._attention = L.sd_cache_append, L.sd_cache_read, L.sd_cache_attention
        self._heads, self._kv_heads, self._head_dim = n_heads, n_kv_heads, head_dim
        self._described = _Described()

    def layer(self, layer: int) -> dict:
        """Views of one layer's pools: k, v [n_pages, n_kv_heads, page_len, head_dim], in 8 bits also k_scale, v_scale."""
        p = [C.c_void_p() for _ in range(4)]
        _check(lib().sd_cache_layer(self.h, layer, *[C.byref(x) for x in p]), "sd_cache_layer")
        c = self.cfg
        shape = (c.n_pages, c.n_kv_heads, c.page_len)
        dt = next(t for code, t in _CACHE_TYPES.values() if code == c.dtype)
        out = {}
        for name, ptr, dtype, shp in (("k", p[0], dt, shape + (c.head_dim,)), ("v", p[1], dt, shape + (c.head_dim,)),
                                      ("k_scale", p[2], torch.float32, shape), ("v_scale", p[3], torch.float32, shape)):
            if ptr.value:
                at = ptr.value - self.arena.data_ptr()
                n = dtype.itemsize
                for s in shp:
                    n *= s
                out[name] = self.arena[at:at + n].view(dtype).view(shp)
        return out

    def append(self, layer: int, k: torch.Tensor, v: torch.Tensor, batch: CacheBatch):
        """k, v: the new tokens' keys and values [n_tokens, n_kv_heads, head_dim], fp32, bf16 or fp16, elements of a head adjacent."""
        n = self._kv_heads
        self._rows(0, "k", k, n, batch)
        self._rows(1, "v", v, n, batch)
        self._call(self._append, "sd_cache_append", layer, batch)

    def read(self, layer: int, batch: CacheBatch, dtype: torch.dtype = torch.float32, k: torch.Tensor | None = None,
             v: torch.Tensor | None = None):
        """The keys and values at the new tokens' places, as (k, v) [n_tokens, n_kv_heads, head_dim] of `dtype`."""
        n = self._kv_heads
        if k is None:
            k = torch.empty(batch.n_tokens, n, self._head_dim, dtype=dtype, device=self.device)
        if v is None:
            v = torch.empty(batch.n_tokens, n, self._head_dim, dtype=dtype, device=self.device)
        self._rows(0, "k", k, n, batch)
        self._rows(1, "v", v, n, batch)
        self._call(self._read, "sd_cache_read", layer, batch)
        return k, v

    def attention(self, layer: int, q: torch.Tensor, batch: CacheBatch, scale: float | None = None, out: torch.Tensor | None = None):
        """Causal attention of the new tokens' queries [n_tokens, n_heads, head_dim] over their sequences; out: like q unless given."""
        if scale is None:
            scale = 0.0                                        # the library's default, head_dim^-1/2
        elif not 0 < abs(C.c_float(scale).value) < float("inf"):   # as the library gets it: 0 would stand for the default
            raise ValueError("scale must be a number other than 0 within the range of fp32")
        n = self._heads
        if out is None:
            out = torch.empty(batch.n_tokens, n, self._head_dim, dtype=q.dtype, device=self.device)
        self._rows(0, "q", q, n, batch)
        self._rows(1, "out", out, n, batch)
        self._call(self._attention, "sd_cache_attention", layer, batch, scale)
        return out

    def status(self) -> int:
        v = C.c_int32(0)
        code = lib().sd_cache_status(self.h, C.byref(v))
        if code not in (SD_OK, SD_ERR_DEVICE):
            raise SdError(code, "sd_cache_status")
        return v.value

    def set_option(self, option: int, value: int):
        _check(lib().sd_cache_set_option(self.h, option, value), "sd_cache_set_option")

    def close(self):
        if getattr(self, "h", None) is not None and self.h.value:
            self.stream.synchronize()
            lib().sd_cache_destroy(self.h)
            self.h = C.c_void_p()
        self.arena = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # describes a tensor in one of this thread's two structures that a call passes on (they are read during the call only)
    def _rows(self, which: int, name: str, t: torch.Tensor, heads: int, batch: CacheBatch):
        code = _ROW_TYPES.get(t.dtype)
        if code is None or t.get_device() != self._index or batch.index != self._index:
            raise ValueError(f"{name} must be an fp32, bf16 or fp16 tensor on {self.device}, and so must the batch be there")
        if t.shape != (batch.n_tokens, heads, self._head_dim):
            raise ValueError(f"{name} must be [{batch.n_tokens}, {heads}, {self._head_dim}], got {tuple(t.shape)}")
        r = self._described.pair[which]
        r.row_stride, r.head_stride, step = t.stride()
        if step != 1 and t.numel():
            raise ValueError(f"{name}'s elements of a head must be adjacent, got strides {t.stride()}")
        r.data = t.data_ptr()
        r.dtype = code

    def _call(self, fn, name: str, layer: int, batch: CacheBatch, *scale):
        other = _raw_stream(self._index) != self._raw
        if other:
            self._fork()
        first, second = self._described.refs
        code = fn(self.h, layer, batch.ref, first, *scale, second)
        if code != SD_OK:
            raise SdError(code, name)
        if other:
            self._join()

    # work before the call on the current stream is seen by it, and work after the call sees its results (and reuses its memory)
    def _fork(self):
        cur = torch.cuda.current_stream(self.device)
        if cur != self.stream:
            self.stream.wait_stream(cur)

    def _join(self):
        cur = torch.cuda.current_stream(self.device)
        if cur != self.stream:
            cur.wait_stream(self.stream)


class Decoder:
    """A handle of the CUDA library plus the device buffers it was given.

    weights: a dict {tok_emb, pos_emb, lnf_g, lnf_b, [lm_head], layers: [{ln1_g, ..., b_fc2}]} (CPU or CUDA tensors in the
    configuration's storage type); they are moved to `device` and kept alive here.
    plan: (max_layers, min_layers, warmup, gen_len) the KV caches are sized for.
    """

    def __init__(self, shape: ModelShape, weights: dict, max_batch: int, max_prompt: int, max_gen: int,
                 plan=None, full_capacity: bool = False, device: str = "cuda:0", stream=None):
        L = lib()
        if not torch.cuda.is_available():
            raise RuntimeError("no CUDA device: the decode path has no CPU fallback")
        self.shape, self.device = shape, torch.device(device)
        self.cfg = make_config(shape, max_batch, max_prompt, max_gen)
        mx, mn, w, G = plan if plan is not None else (shape.n_layers, shape.n_layers, 0, max_gen)
        self.plan = SdPlan(mx, mn, w, G, 1 if full_capacity else 0)
        self.arena_bytes = arena_bytes(self.cfg, self.plan)
        torch.cuda.set_device(self.device)
        self.stream = stream if stream is not None else torch.cuda.Stream(device=self.device)
        dt = storage_dtype(shape)
        self._keep = []

        def dev(t):
            t = t.to(device=self.device, dtype=dt).contiguous()
            self._keep.append(t)
            return t.data_ptr()

        n = shape.n_layers
        self._arrs = {nm: (C.c_void_p * n)(*[dev(weights["layers"][l][nm]) for l in range(n)]) for nm in _LAYER_FIELDS}
        head = weights.get("lm_head")
        self.w = SdWeights(dev(weights["tok_emb"]), dev(weights["pos_emb"]),
                           *[C.cast(self._arrs[nm], _PP) for nm in _LAYER_FIELDS],
                           dev(weights["lnf_g"]), dev(weights["lnf_b"]), dev(head) if head is not None else None)
        self.arena = torch.empty(self.arena_bytes + 256, dtype=torch.uint8, device=self.device)
        base = (self.arena.data_ptr() + 255) // 256 * 256
        self.h = C.c_void_p()
        torch.cuda.synchronize(self.device)
        _check(L.sd_create(C.byref(self.cfg), C.byref(self.w), C.byref(self.plan), base, self.arena_bytes,
                           self.stream.cuda_stream, C.byref(self.h)), "sd_create")
        self.B = self.P = None
        self._keep_io = None

    # -- the four calls ---------------------------------------------------------------
    def schedule(self, max_layers: int, min_layers: int, warmup: int, gen_len: int):
        n = (C.c_int32 * max(gen_len, 1))()
        t = (C.c_int32 * max(gen_len, 1))()
        _check(lib().sd_schedule(self.h, max_layers, min_layers, warmup, gen_len, n, t), "sd_schedule")
        return list(n)[:gen_len], list(t)[:gen_len]

    def schedule_custom(self, n_active, warmup: int):
        G = len(n_active)
        n = (C.c_int32 * G)(*n_active)
        t = (C.c_int32 * G)()
        _check(lib().sd_schedule_custom(self.h, n, warmup, G, t), "sd_schedule_custom")
        return list(t)

    def prefill(self, tokens: torch.Tensor, logits: torch.Tensor | None = None) -> torch.Tensor:
        B, P = tokens.shape
        tokens = self._dev_i32(tokens)
        if logits is None:
            logits = torch.empty(B, self.shape.vocab, dtype=torch.float32, device=self.device)
        self._order()
        _check(lib().sd_prefill(self.h, tokens.data_ptr(), B, P, logits.data_ptr()), "sd_prefill")
        self._keep_io = (tokens, logits)
        self.B, self.P = B, P
        self._n_rows = None
        return logits

    def decode_step(self, ids: torch.Tensor, position: int, logits: torch.Tensor | None = None) -> torch.Tensor:
        ids = self._dev_i32(ids)
        n = getattr(self, "_n_rows", None) or self.B
        if n is not None:              # before a prefill the library itself reports the state error
            assert ids.numel() == n, f"{ids.numel()} token ids for {n} generating rows"
        if logits is None:
            logits = torch.empty(ids.shape[0], self.shape.vocab, dtype=torch.float32, device=self.device)
        self._order()
        _check(lib().sd_decode_step(self.h, ids.data_ptr(), position, logits.data_ptr()), "sd_decode_step")
        self._keep_io = (ids, logits)
        return logits

    def decode_step_static(self, ids: torch.Tensor, position: int, logits: torch.Tensor | None = None) -> torch.Tensor:
        """sd_decode_step_static: the same step with the attention partials in the library's
        own static device array, for callers that may not allocate (the tensors passed here
        must already exist: this wrapper allocates `logits` only when it is not given)."""
        ids = self._dev_i32(ids)
        if logits is None:
            logits = torch.empty(ids.shape[0], self.shape.vocab, dtype=torch.float32, device=self.device)
        self._order()
        _check(lib().sd_decode_step_static(self.h, ids.data_ptr(), position, logits.data_ptr()), "sd_decode_step_static")
        self._keep_io = (ids, logits)
        return logits

    def decode_step_host(self, ids: torch.Tensor, position: int, logits: torch.Tensor) -> torch.Tensor:
        """ids, logits: CPU tensors (int32 [B], fp32 [B, vocab]); returns after the copy back."""
        assert ids.device.type == "cpu" and logits.device.type == "cpu" and ids.dtype == torch.int32
        assert logits.dtype == torch.float32 and logits.is_contiguous() and ids.is_contiguous()
        _check(lib().sd_decode_step_host(self.h, ids.data_ptr(), position, logits.data_ptr()), "sd_decode_step_host")
        return logits

    def rewind(self):
        _check(lib().sd_rewind(self.h), "sd_rewind")

    def launch_count(self) -> int:
        v = C.c_int64(0)
        _check(lib().sd_launch_count(self.h, C.byref(v)), "sd_launch_count")
        return v.value

    # -- helpers ----------------------------------------------------------------------
    def greedy(self, logits: torch.Tensor, out: torch.Tensor | None = None) -> torch.Tensor:
        B = logits.shape[0]
        if out is None:
            out = torch.empty(B, dtype=torch.int32, device=self.device)
        _check(lib().sd_greedy(self.h, logits.data_ptr(), B, out.data_ptr()), "sd_greedy")
        return out

    def set_padding(self, pad=None):
        """Left-padding slots per row (host list), or None to remove; call before prefill."""
        if pad is None:
            _check(lib().sd_set_padding(self.h, None, 0), "sd_set_padding")
            return
        arr = (C.c_int32 * len(pad))(*[int(p) for p in pad])
        _check(lib().sd_set_padding(self.h, arr, len(pad)), "sd_set_padding")

    def set_rows(self, rows=None):
        """Rows that still generate (host list, increasing), or None for all; call after prefill."""
        if rows is None:
            _check(lib().sd_set_rows(self.h, None, 0), "sd_set_rows")
            self._n_rows = None
            return
        arr = (C.c_int32 * len(rows))(*[int(r) for r in rows])
        _check(lib().sd_set_rows(self.h, arr, len(rows)), "sd_set_rows")
        self._n_rows = len(rows)

    def sample_top_p(self, logits: torch.Tensor, uniforms: torch.Tensor, temperature: float = 0.3,
                     top_p: float = 0.7, out: torch.Tensor | None = None) -> torch.Tensor:
        B = logits.shape[0]
        if out is None:
            out = torch.empty(B, dtype=torch.int32, device=self.device)
        assert uniforms.dtype == torch.float32 and uniforms.is_cuda and uniforms.numel() == B
        self._order()
        _check(lib().sd_sample_top_p(self.h, logits.data_ptr(), B, temperature, top_p, uniforms.data_ptr(),
                                     out.data_ptr()), "sd_sample_top_p")
        return out

    def sample(self, logits: torch.Tensor, uniforms: torch.Tensor, temperature: torch.Tensor | None = None,
               top_k: torch.Tensor | None = None, top_p: torch.Tensor | None = None, min_p: torch.Tensor | None = None,
               out: torch.Tensor | None = None) -> torch.Tensor:
        """One token per row with the row's own settings (CUDA tensors [B], fp32, top_k int32; None: off)."""
        B = logits.shape[0]
        index = self.arena.get_device()
        if logits.dtype != torch.float32 or logits.shape != (B, self.shape.vocab) or not logits.is_contiguous() or logits.get_device() != index:
            raise ValueError(f"logits must be a contiguous fp32 [{B}, {self.shape.vocab}] on {self.device}")
        if out is None:
            out = torch.empty(B, dtype=torch.int32, device=self.device)
        ptr = []
        for name, t, dt in (("temperature", temperature, torch.float32), ("top_k", top_k, torch.int32), ("top_p", top_p, torch.float32),
                            ("min_p", min_p, torch.float32), ("uniforms", uniforms, torch.float32), ("out", out, torch.int32)):
            if t is None and name not in ("uniforms", "out"):
                ptr.append(None)
            elif t.dtype != dt or t.shape != (B,) or not t.is_contiguous() or t.get_device() != index:
                raise ValueError(f"{name} must be a contiguous {dt} [{B}] on {self.device}")
            else:
                ptr.append(t.data_ptr())
        other = _raw_stream(index) != self.stream.cuda_stream
        if other:
            self._order()
        _check(lib().sd_sample(self.h, logits.data_ptr(), B, SdSampling(*ptr[:4]), ptr[4], ptr[5]), "sd_sample")
        if other:
            self._after()
        return out

    def extend(self, cache: PagedCache, batch: CacheBatch, tokens: torch.Tensor, n_active: int | None = None, warmup: int = 0,
               logits: torch.Tensor | None = None) -> torch.Tensor:
        """The batch's new tokens [n_tokens] through the model over a paged cache made with this decoder's stream; n_active layers
        (default all).  Returns the logits [n_seqs, vocab] of each sequence's last new token."""
        tokens = self._dev_i32(tokens)
        if tokens.shape != (batch.n_tokens,):
            raise ValueError(f"tokens must be [{batch.n_tokens}]")
        if logits is None:
            logits = torch.empty(batch.c.n_seqs, self.shape.vocab, dtype=torch.float32, device=self.device)
        elif logits.shape != (batch.c.n_seqs, self.shape.vocab) or logits.dtype != torch.float32 or not logits.is_contiguous() or \
                logits.get_device() != self.arena.get_device():
            raise ValueError(f"logits must be a contiguous fp32 [{batch.c.n_seqs}, {self.shape.vocab}] on {self.device}")
        if batch.index != self.arena.get_device():
            raise ValueError(f"the batch must be on {self.device}")
        self._order()
        _check(lib().sd_extend(self.h, cache.h, C.byref(batch.c), tokens.data_ptr(), self.shape.n_layers if n_active is None else n_active, warmup,
                               logits.data_ptr()), "sd_extend")
        self._after()
        return logits

    def status(self) -> int:
        v = C.c_int32(0)
        code = lib().sd_status(self.h, C.byref(v))
        if code not in (SD_OK, SD_ERR_DEVICE):
            raise SdError(code, "sd_status")
        return v.value

    def stats(self):
        a, b = C.c_int64(0), C.c_int64(0)
        _check(lib().sd_stats(self.h, C.byref(a), C.byref(b)), "sd_stats")
        return a.value, b.value

    def set_option(self, option: int, value: int):
        _check(lib().sd_set_option(self.h, option, value), "sd_set_option")

    def kernel_times(self) -> dict:
        out = {}
        for i, name in enumerate(KERNEL_CLASSES):
            ms, n = C.c_double(0), C.c_int64(0)
            _check(lib().sd_kernel_time(self.h, i, C.byref(ms), C.byref(n)), "sd_kernel_time")
            out[name] = (ms.value, n.value)
        return out

    def kernel_times_reset(self):
        _check(lib().sd_kernel_time_reset(self.h), "sd_kernel_time_reset")

    def synchronize(self):
        self.stream.synchronize()

    def close(self):
        if getattr(self, "h", None) is not None and self.h.value:
            self.stream.synchronize()
            lib().sd_destroy(self.h)
            self.h = C.c_void_p()
        self.arena = None
        self._keep = []

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _dev_i32(self, t: torch.Tensor) -> torch.Tensor:
        return t.to(device=self.device, dtype=torch.int32).contiguous()

    def _order(self):
        # buffers produced on torch's current stream must be complete before the library's stream reads them
        cur = torch.cuda.current_stream(self.device)
        if cur != self.stream:
            self.stream.wait_stream(cur)

    def _after(self):
        # and what the library's stream wrote is seen, and its inputs' memory reused, only after it
        cur = torch.cuda.current_stream(self.device)
        if cur != self.stream:
            cur.wait_stream(self.stream)
