"""Thin binding of librdkv (include/rdkv.h): ctypes, and for the calls of decode
loops native code (_rdkv_call, csrc/rdkv_call.cpp), which makes the same calls
for less host time; where it does not load, ctypes makes them and a warning says so.

Argument marshalling only: every step of the path runs in the HIP kernels of the
shared library.  PyTorch supplies device memory and streams.  There is no CPU
fallback: if the library is missing or fails to load, importing this module
raises.
"""
import ctypes
import os
import warnings

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "librdkv.so")

RDKV_OK = 0
RDKV_K_TOKENWISE, RDKV_K_CHANNELWISE = 0, 1
(RDKV_EXPORT_COUNTS, RDKV_EXPORT_TIER_IDX, RDKV_EXPORT_SEG_OFF, RDKV_EXPORT_ARENA,
 RDKV_EXPORT_BITS_TOK, RDKV_EXPORT_BITS_CH, RDKV_EXPORT_LAMBDA, RDKV_EXPORT_ITERATIONS) = range(8)
STATUS_NAMES = {0: "RDKV_OK", 1: "RDKV_ERR_INVALID_ARG", 2: "RDKV_ERR_SHAPE", 3: "RDKV_ERR_UNSUPPORTED",
                4: "RDKV_ERR_ALLOC", 5: "RDKV_ERR_HIP", 6: "RDKV_ERR_INTERNAL"}

EXPORTED_SYMBOLS = [
    "rdkv_version", "rdkv_last_error", "rdkv_config_default", "rdkv_weights", "rdkv_allocate", "rdkv_allocate_info", "rdkv_pack", "rdkv_cache_max_bytes", "rdkv_cache_max_table_bytes",
    "rdkv_compress", "rdkv_decode_attn", "rdkv_decode_bf16_workspace_bytes", "rdkv_decode_attn_bf16",
    "rdkv_decode_bf16_noalloc_max_bytes", "rdkv_decode_attn_bf16_noalloc",
    "rdkv_cache_reserve_tail", "rdkv_cache_append", "rdkv_cache_tail_len", "rdkv_cache_tail_len_sync", "rdkv_calibrate_eps",
    "rdkv_cache_rebudget_tail", "rdkv_cache_generations", "rdkv_cache_generation",
    "rdkv_cache_stats", "rdkv_cache_export_bytes", "rdkv_cache_export", "rdkv_cache_free",
    "rdkv_kernel_timing_enable", "rdkv_kernel_timing_read", "rdkv_k_row_words", "rdkv_k_row_words_max",
    "rdkv_prompt_default", "rdkv_prompt_attn_bf16",
    "rdkv_slots_tree_workspace_bytes", "rdkv_slots_tree_attn", "rdkv_slots_accept_workspace_bytes", "rdkv_slots_accept",
    "rdkv_slots_default", "rdkv_slots_side_bytes", "rdkv_slots_fill_workspace_bytes", "rdkv_slots_fill", "rdkv_slots_append",
    "rdkv_slots_decode_workspace_bytes", "rdkv_slots_decode_attn", "rdkv_slots_read",
]
(RDKV_TIME_DECODE_TIERED, RDKV_TIME_DECODE_BF16, RDKV_TIME_WEIGHTS, RDKV_TIME_ALLOCATE, RDKV_TIME_PACK,
 RDKV_TIME_CALIBRATE) = range(6)

_ALLOC_FN = ctypes.CFUNCTYPE(ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p)
_FREE_FN = ctypes.CFUNCTYPE(None, ctypes.c_void_p, ctypes.c_void_p)


class rdkv_config(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("hq", ctypes.c_int32), ("hkv", ctypes.c_int32), ("head_dim", ctypes.c_int32),
        ("seq_lens", ctypes.POINTER(ctypes.c_int32)),
        ("s_obs", ctypes.c_int32), ("pool_kernel", ctypes.c_int32), ("causal", ctypes.c_int32),
        ("k_mode", ctypes.c_int32), ("group_size", ctypes.c_int32),
        ("budget_bits", ctypes.POINTER(ctypes.c_float)),
        ("kv_split_rk", ctypes.c_float), ("k_scale_per_channel", ctypes.c_int32),
        ("n_tiers", ctypes.c_int32), ("tiers", ctypes.c_int32 * 5),
        ("eps_v", ctypes.c_float * 5), ("eps_k", ctypes.c_float * 5),
        ("rel_tol", ctypes.c_float), ("max_iters", ctypes.c_int32),
        ("alloc", _ALLOC_FN), ("free_", _FREE_FN), ("alloc_user", ctypes.c_void_p),
    ]


class rdkv_slots(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("hq", ctypes.c_int32), ("hkv", ctypes.c_int32), ("head_dim", ctypes.c_int32),
        ("capacity", ctypes.c_int32), ("bits", ctypes.c_int32), ("sinks", ctypes.c_int32), ("recent", ctypes.c_int32),
        ("window", ctypes.c_int32), ("score_cap", ctypes.c_float), ("decay", ctypes.c_float), ("slopes", ctypes.c_void_p),
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("pos", ctypes.c_void_p), ("weight", ctypes.c_void_p),
        ("len", ctypes.c_void_p), ("next", ctypes.c_void_p),
    ]


class rdkv_prompt(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("hq", ctypes.c_int32), ("hkv", ctypes.c_int32), ("head_dim", ctypes.c_int32),
        ("seq_lens", ctypes.POINTER(ctypes.c_int32)), ("window", ctypes.c_int32), ("sinks", ctypes.c_int32),
        ("score_cap", ctypes.c_float), ("slopes", ctypes.c_void_p),
        ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64), ("out_stride", ctypes.c_int64),
    ]


class rdkv_stats(ctypes.Structure):
    _fields_ = [
        ("n_items", ctypes.c_int64), ("rows", ctypes.c_int64 * 4), ("evicted", ctypes.c_int64),
        ("stored_bytes", ctypes.c_int64), ("arena_bytes", ctypes.c_int64), ("index_bytes", ctypes.c_int64),
        ("n_chunks", ctypes.c_int64), ("dense_bytes", ctypes.c_int64),
        ("alloc_info", ctypes.c_int64), ("iterations_max", ctypes.c_int64),
        ("lambda_min", ctypes.c_double), ("lambda_max", ctypes.c_double),
    ]


class RdkvError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run `python -c 'import __graft_entry__ as g; g.build()'`")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    cfgp = ctypes.POINTER(rdkv_config)
    lib.rdkv_version.restype = ctypes.c_char_p
    lib.rdkv_last_error.restype = ctypes.c_char_p
    lib.rdkv_config_default.argtypes = [cfgp]
    lib.rdkv_weights.argtypes = [cfgp, vp, vp, vp, vp, vp]
    lib.rdkv_allocate.argtypes = [cfgp, vp, vp, vp, vp, vp]
    lib.rdkv_allocate_info.argtypes = [cfgp, vp, vp, vp, vp, vp, vp, vp]
    lib.rdkv_cache_max_bytes.argtypes = [cfgp]
    lib.rdkv_cache_max_bytes.restype = sz
    lib.rdkv_cache_max_table_bytes.argtypes = [cfgp]
    lib.rdkv_cache_max_table_bytes.restype = sz
    lib.rdkv_pack.argtypes = [cfgp, vp, vp, vp, vp, vp, ctypes.POINTER(vp)]
    lib.rdkv_compress.argtypes = [cfgp, vp, vp, vp, vp, ctypes.POINTER(vp)]
    lib.rdkv_decode_attn.argtypes = [vp, vp, vp, vp, vp]
    lib.rdkv_decode_bf16_workspace_bytes.argtypes = [ctypes.POINTER(i32), i32, i32, i32, i32]
    lib.rdkv_decode_bf16_workspace_bytes.restype = sz
    lib.rdkv_decode_attn_bf16.argtypes = [vp, vp, ctypes.POINTER(i32), i32, i32, i32, i32, vp, vp, vp, vp, sz, vp]
    lib.rdkv_decode_bf16_noalloc_max_bytes.argtypes = []
    lib.rdkv_decode_bf16_noalloc_max_bytes.restype = sz
    lib.rdkv_decode_attn_bf16_noalloc.argtypes = [vp, vp, ctypes.POINTER(i32), i32, i32, i32, i32, vp, vp, vp, vp]
    lib.rdkv_cache_reserve_tail.argtypes = [vp, i32, vp]
    lib.rdkv_cache_append.argtypes = [vp, vp, vp, vp]
    lib.rdkv_cache_tail_len.argtypes = [vp]
    lib.rdkv_cache_tail_len.restype = i32
    lib.rdkv_cache_tail_len_sync.argtypes = [vp, vp, ctypes.POINTER(i32)]
    lib.rdkv_calibrate_eps.argtypes = [cfgp, vp, vp, vp, vp, vp]
    lib.rdkv_cache_rebudget_tail.argtypes = [vp, cfgp, vp, vp]
    lib.rdkv_cache_generations.argtypes = [vp]
    lib.rdkv_cache_generations.restype = i32
    lib.rdkv_cache_generation.argtypes = [vp, i32]
    lib.rdkv_cache_generation.restype = vp
    lib.rdkv_cache_stats.argtypes = [vp, ctypes.POINTER(rdkv_stats)]
    lib.rdkv_cache_export_bytes.argtypes = [vp, i32]
    lib.rdkv_cache_export_bytes.restype = sz
    lib.rdkv_cache_export.argtypes = [vp, i32, vp, sz]
    lib.rdkv_cache_free.argtypes = [vp]
    lib.rdkv_cache_free.restype = None
    lib.rdkv_k_row_words.argtypes = [vp]
    lib.rdkv_k_row_words.restype = i32
    lib.rdkv_k_row_words_max.argtypes = []
    lib.rdkv_k_row_words_max.restype = i32
    lib.rdkv_prompt_default.argtypes = [ctypes.POINTER(rdkv_prompt)]
    lib.rdkv_prompt_attn_bf16.argtypes = [ctypes.POINTER(rdkv_prompt), vp, vp, vp, vp, vp, vp]
    slp = ctypes.POINTER(rdkv_slots)
    lib.rdkv_slots_default.argtypes = [slp]
    lib.rdkv_slots_side_bytes.argtypes = [slp]
    lib.rdkv_slots_side_bytes.restype = sz
    lib.rdkv_slots_fill_workspace_bytes.argtypes = [slp, i32, ctypes.POINTER(i32)]
    lib.rdkv_slots_fill_workspace_bytes.restype = sz
    lib.rdkv_slots_fill.argtypes = [slp, i32, i32, ctypes.POINTER(i32), vp, vp, vp, vp, sz, vp]
    lib.rdkv_slots_append.argtypes = [slp, vp, vp, vp, vp]
    lib.rdkv_slots_decode_workspace_bytes.argtypes = [slp]
    lib.rdkv_slots_decode_workspace_bytes.restype = sz
    lib.rdkv_slots_decode_attn.argtypes = [slp, vp, vp, vp, vp, sz, vp]
    lib.rdkv_slots_tree_workspace_bytes.argtypes = [slp, i32]
    lib.rdkv_slots_tree_workspace_bytes.restype = sz
    lib.rdkv_slots_tree_attn.argtypes = [slp, i32, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.rdkv_slots_accept_workspace_bytes.argtypes = [slp]
    lib.rdkv_slots_accept_workspace_bytes.restype = sz
    lib.rdkv_slots_accept.argtypes = [slp, i32, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.rdkv_slots_read.argtypes = [slp, vp, i32, vp, vp, vp]
    lib.rdkv_kernel_timing_enable.argtypes = [i32]
    lib.rdkv_kernel_timing_read.argtypes = [i32, ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_double)]
    return lib


lib = _load()
try:
    from . import _rdkv_call as _call
    _call.bind(*(ctypes.cast(f, ctypes.c_void_p).value for f in (lib.rdkv_decode_attn, lib.rdkv_cache_append)))
    _call.bind_slots(*(ctypes.cast(f, ctypes.c_void_p).value for f in (
        lib.rdkv_slots_append, lib.rdkv_slots_decode_attn, lib.rdkv_slots_read, lib.rdkv_slots_fill, lib.rdkv_slots_fill_workspace_bytes)))
    _call.bind_tree(*(ctypes.cast(f, ctypes.c_void_p).value for f in (
        lib.rdkv_slots_tree_attn, lib.rdkv_slots_tree_workspace_bytes, lib.rdkv_slots_accept, lib.rdkv_slots_accept_workspace_bytes,
        lib.rdkv_prompt_attn_bf16)))
except ImportError as e:
    _call = None
    warnings.warn(f"_rdkv_call.so is not built or does not fit this PyTorch ({e}): a decode step takes the host 2 us more; "
                  "run `python -c 'import __graft_entry__ as g; g.build()'`")


def _check(status):
    if status != RDKV_OK:
        raise RdkvError(status, lib.rdkv_last_error().decode())


def _ptr(t):
    if t is None:
        return None
    assert t.is_contiguous()
    return t.data_ptr()


# A decode step is one launch of 3 us on the host: what surrounds it must not cost more.  The raw handle of the current
# stream comes from the bindings below torch.cuda.current_stream(), which builds a Stream object around it (2.9 us, 0.2 so).
_current_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else None
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)

if _current_device is not None and _raw_stream is not None:
    def _stream():
        if not torch.cuda.is_initialized():
            torch.cuda.init()
        return _raw_stream(_current_device())
else:
    def _stream():
        return torch.cuda.current_stream().cuda_stream


def _empty_f32(shape, strides, device):
    return torch.empty_strided(shape, strides, dtype=torch.float32, device=device)      # 1.3 us; torch.empty 1.7


def rdkv_version():
    return lib.rdkv_version().decode()


class Config:
    """Owns an rdkv_config and the host arrays it points to."""

    def __init__(self, seq_lens, hq, hkv, head_dim=128, budget_bits=None, **overrides):
        self.c = rdkv_config()
        _check(lib.rdkv_config_default(ctypes.byref(self.c)))
        self._seq = (ctypes.c_int32 * len(seq_lens))(*[int(x) for x in seq_lens])
        self.c.batch, self.c.hq, self.c.hkv, self.c.head_dim = len(seq_lens), hq, hkv, head_dim
        self.c.seq_lens = ctypes.cast(self._seq, ctypes.POINTER(ctypes.c_int32))
        if budget_bits is not None:
            self._bud = (ctypes.c_float * len(seq_lens))(*[float(x) for x in budget_bits])
            self.c.budget_bits = ctypes.cast(self._bud, ctypes.POINTER(ctypes.c_float))
        for k, v in overrides.items():
            if k in ("tiers", "eps_v", "eps_k"):
                arr = getattr(self.c, k)
                for i, x in enumerate(v):
                    arr[i] = x
                if k == "tiers":
                    self.c.n_tiers = len(v)
            else:
                setattr(self.c, k, v)
        self.seq_lens = [int(x) for x in seq_lens]
        self.hq, self.hkv, self.d = hq, hkv, head_dim

    @property
    def total_tokens(self):
        return sum(self.seq_lens) * self.hkv

    def ref(self):
        return ctypes.byref(self.c)


class Cache:
    """Handle of a packed cache (library-owned device memory)."""

    def __init__(self, handle, cfg):
        self.h = handle
        self.cfg = cfg

    def stats(self):
        st = rdkv_stats()
        _check(lib.rdkv_cache_stats(self.h, ctypes.byref(st)))
        return {"n_items": st.n_items, "rows": list(st.rows), "evicted": st.evicted,
                "stored_bytes": st.stored_bytes, "arena_bytes": st.arena_bytes, "index_bytes": st.index_bytes,
                "n_chunks": st.n_chunks, "dense_bytes": st.dense_bytes, "alloc_info": st.alloc_info,
                "iterations_max": st.iterations_max, "lambda_min": st.lambda_min, "lambda_max": st.lambda_max}

    def export(self, what, dtype):
        n = lib.rdkv_cache_export_bytes(self.h, what)
        buf = np.zeros(n, dtype=np.uint8)
        if n:
            _check(lib.rdkv_cache_export(self.h, what, buf.ctypes.data_as(ctypes.c_void_p), n))
        return buf.view(dtype)

    def free(self):
        if self.h:
            lib.rdkv_cache_free(self.h)
            self.h = None

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass


def rdkv_weights(cfg, K, Q_obs, want_channel=False):
    w_tok = torch.empty(cfg.total_tokens, dtype=torch.float32, device=K.device)
    w_ch = torch.empty(len(cfg.seq_lens) * cfg.hkv * cfg.d, dtype=torch.float32, device=K.device) if want_channel else None
    _check(lib.rdkv_weights(cfg.ref(), _ptr(K), _ptr(Q_obs), _ptr(w_tok), _ptr(w_ch), _stream()))
    return w_tok, w_ch


def rdkv_allocate(cfg, w_tok, w_ch=None):
    bits_tok = torch.empty(cfg.total_tokens, dtype=torch.uint8, device=w_tok.device)
    bits_ch = None
    if cfg.c.k_mode == RDKV_K_CHANNELWISE:
        bits_ch = torch.empty(len(cfg.seq_lens) * cfg.hkv * cfg.d, dtype=torch.uint8, device=w_tok.device)
    _check(lib.rdkv_allocate(cfg.ref(), _ptr(w_tok), _ptr(w_ch), _ptr(bits_tok), _ptr(bits_ch), _stream()))
    return bits_tok, bits_ch


def rdkv_allocate_info(cfg, w_tok, w_ch=None):
    """(bits_tok, bits_ch, lambda, iterations): the last two as device tensors [maps, items]."""
    n = len(cfg.seq_lens) * cfg.hkv
    mixed = cfg.c.k_mode == RDKV_K_CHANNELWISE
    bits_tok = torch.empty(cfg.total_tokens, dtype=torch.uint8, device=w_tok.device)
    bits_ch = torch.empty(n * cfg.d, dtype=torch.uint8, device=w_tok.device) if mixed else None
    lam = torch.empty((2 if mixed else 1, n), dtype=torch.float64, device=w_tok.device)
    iters = torch.empty((2 if mixed else 1, n), dtype=torch.int32, device=w_tok.device)
    _check(lib.rdkv_allocate_info(cfg.ref(), _ptr(w_tok), _ptr(w_ch), _ptr(bits_tok), _ptr(bits_ch), _ptr(lam),
                                  _ptr(iters), _stream()))
    return bits_tok, bits_ch, lam, iters


def rdkv_cache_max_bytes(cfg):
    return int(lib.rdkv_cache_max_bytes(cfg.ref()))


def rdkv_cache_max_table_bytes(cfg):
    return int(lib.rdkv_cache_max_table_bytes(cfg.ref()))


def rdkv_pack(cfg, K, V, bits_tok, bits_ch=None):
    h = ctypes.c_void_p()
    _check(lib.rdkv_pack(cfg.ref(), _ptr(K), _ptr(V), _ptr(bits_tok), _ptr(bits_ch), _stream(), ctypes.byref(h)))
    return Cache(h, cfg)


def rdkv_compress(cfg, K, V, Q_obs):
    h = ctypes.c_void_p()
    _check(lib.rdkv_compress(cfg.ref(), _ptr(K), _ptr(V), _ptr(Q_obs), _stream(), ctypes.byref(h)))
    return Cache(h, cfg)


def rdkv_decode_attn(cache, q, out=None, lse=None):
    cfg = cache.cfg
    done = _call and _call.decode(cache.h, _stream(), len(cfg.seq_lens), cfg.hq, cfg.d, q, out, lse)
    if done is not None:
        if done[0] != RDKV_OK:
            _check(done[0])
        return done[1:]
    if out is None:
        out = _empty_f32((len(cfg.seq_lens), cfg.hq, cfg.d), (cfg.hq * cfg.d, cfg.d, 1), q.device)
    if lse is None:
        lse = _empty_f32((len(cfg.seq_lens), cfg.hq), (cfg.hq, 1), q.device)
    _check(lib.rdkv_decode_attn(cache.h, _ptr(q), _ptr(out), _ptr(lse), _stream()))
    return out, lse


def rdkv_cache_reserve_tail(cache, max_new_tokens):
    _check(lib.rdkv_cache_reserve_tail(cache.h, int(max_new_tokens), _stream()))


def rdkv_cache_append(cache, k_new, v_new):
    status = _call and _call.append(cache.h, _stream(), k_new, v_new)
    if status is not None:
        return _check(status)
    _check(lib.rdkv_cache_append(cache.h, _ptr(k_new), _ptr(v_new), _stream()))


def rdkv_cache_tail_len(cache):
    return int(lib.rdkv_cache_tail_len(cache.h))


def rdkv_cache_tail_len_sync(cache):
    n = ctypes.c_int32()
    _check(lib.rdkv_cache_tail_len_sync(cache.h, _stream(), ctypes.byref(n)))
    return n.value


# what torch.cuda.caching_allocator_alloc / _delete call, without their device guard and Stream object
_raw_alloc = getattr(torch._C, "_cuda_cudaCachingAllocator_raw_alloc", None) or \
    (lambda nbytes, stream: torch.cuda.caching_allocator_alloc(nbytes))
_raw_delete = getattr(torch._C, "_cuda_cudaCachingAllocator_raw_delete", None) or torch.cuda.caching_allocator_delete


@_ALLOC_FN
def _torch_alloc(nbytes, user):
    return _raw_alloc(nbytes, _stream())


@_FREE_FN
def _torch_free(ptr, user):
    _raw_delete(ptr)


def torch_allocator_hooks():
    """Config overrides that route the library's device allocations through PyTorch's caching allocator
    (`Config(..., **torch_allocator_hooks())`): hipMalloc / hipFree of the large scratch and arena buffers cost more
    than the kernels of a compression pass over one 128K-token layer."""
    return {"alloc": _torch_alloc, "free_": _torch_free}


class _Borrowed(Cache):
    """A generation of another cache: never freed from here."""

    def __init__(self, handle, cfg, owner):
        super().__init__(handle, cfg)
        self._owner = owner

    def free(self):
        self.h = None


def rdkv_cache_rebudget_tail(cache, cfg, Q_obs):
    _check(lib.rdkv_cache_rebudget_tail(cache.h, cfg.ref(), _ptr(Q_obs), _stream()))


def rdkv_cache_generations(cache):
    return int(lib.rdkv_cache_generations(cache.h))


def rdkv_cache_generation(cache, index, cfg):
    h = lib.rdkv_cache_generation(cache.h, int(index))
    if not h:
        raise IndexError(f"generation {index} does not exist")
    return _Borrowed(ctypes.c_void_p(h), cfg, cache)


def rdkv_calibrate_eps(cfg, K, V):
    """(eps_k, eps_v): float64 [items, 3] for b = 2, 4, 8."""
    n = len(cfg.seq_lens) * cfg.hkv
    eps_k = np.zeros((n, 3), dtype=np.float64)
    eps_v = np.zeros((n, 3), dtype=np.float64)
    _check(lib.rdkv_calibrate_eps(cfg.ref(), _ptr(K), _ptr(V), eps_k.ctypes.data_as(ctypes.c_void_p),
                                  eps_v.ctypes.data_as(ctypes.c_void_p), _stream()))
    return eps_k, eps_v


def rdkv_decode_bf16_workspace_bytes(seq_lens, hq, hkv, head_dim=128):
    arr = (ctypes.c_int32 * len(seq_lens))(*[int(x) for x in seq_lens])
    return lib.rdkv_decode_bf16_workspace_bytes(arr, len(seq_lens), hq, hkv, head_dim)


def rdkv_decode_attn_bf16(K, V, seq_lens, hq, hkv, q, head_dim=128, out=None, lse=None, workspace=None):
    arr = (ctypes.c_int32 * len(seq_lens))(*map(int, seq_lens))
    if workspace is None:
        n = lib.rdkv_decode_bf16_workspace_bytes(arr, len(seq_lens), hq, hkv, head_dim)
        workspace = torch.empty(max(n, 16), dtype=torch.uint8, device=q.device)
    if out is None:
        out = _empty_f32((len(seq_lens), hq, head_dim), (hq * head_dim, head_dim, 1), q.device)
    if lse is None:
        lse = _empty_f32((len(seq_lens), hq), (hq, 1), q.device)
    _check(lib.rdkv_decode_attn_bf16(_ptr(K), _ptr(V), arr, len(seq_lens), hq, hkv, head_dim, _ptr(q), _ptr(out),
                                     _ptr(lse), _ptr(workspace), workspace.numel(), _stream()))
    return out, lse


def rdkv_decode_attn_bf16_noalloc(K, V, seq_lens, hq, hkv, q, out, lse=None, head_dim=128):
    """The caller passes every buffer; nothing is allocated here or in the library."""
    arr = (ctypes.c_int32 * len(seq_lens))(*[int(x) for x in seq_lens])
    _check(lib.rdkv_decode_attn_bf16_noalloc(_ptr(K), _ptr(V), arr, len(seq_lens), hq, hkv, head_dim, _ptr(q),
                                             _ptr(out), _ptr(lse), _stream()))
    return out, lse


def _int32(name, x):
    """A number that ctypes would otherwise cut to 32 bits, or int() to a whole one."""
    if x != x or int(x) != x or not -2 ** 31 <= int(x) < 2 ** 31:
        raise ValueError(f"{name} = {x} is no whole 32-bit number")
    return int(x)


def _rows_of(t, name, tokens, heads, d, device):
    """The stride that names a tensor's layout: 0 of a flat ragged one, or that of rows [tokens, heads, d] whose heads lie side by side, and one row behind
    another (rows of an expanded view have a stride of 0 as well, which would name the other layout)."""
    if t.dtype != torch.bfloat16 or t.device != device:
        raise ValueError(f"{name} must be a torch.bfloat16 tensor on {device}: got {t.dtype} on {t.device}")
    if t.dim() in (1, 2):
        if not t.is_contiguous() or t.numel() != tokens * heads * d or t.dim() == 2 and t.shape[1] != d:
            raise ValueError(f"{name} must be {tokens * heads} contiguous rows of {d}, flat, or [tokens, heads, {d}]: got {tuple(t.shape)}")
        return 0
    if tuple(t.shape) != (tokens, heads, d) or t.numel() > 0 and (t.stride(2) != 1 or heads > 1 and t.stride(1) != d):
        raise ValueError(f"{name} must be [{tokens}, {heads}, {d}] with a row's heads side by side, or flat: got {tuple(t.shape)}, strides {t.stride()}")
    if tokens > 1 and t.stride(0) < heads * d:
        raise ValueError(f"{name}: the rows of its tokens overlap: strides {t.stride()} of [{tokens}, {heads}, {d}]")
    return t.stride(0) if tokens > 1 else heads * d


def rdkv_prompt_attn_bf16(Q, K, V, seq_lens, hq, hkv, head_dim=128, window=0, sinks=0, score_cap=0.0, slopes=None, out=None, lse=None):
    """(out, lse).  Each of Q, K, V and out is either flat (ragged [heads][T_s][head_dim] blocks: one dimension, or rows of head_dim) or
    [tokens, heads, head_dim] (tokens of the batch one after another; a view of wider rows will do); out is laid out as Q unless it is given.
    lse: float32, ragged [hq][T_s]."""
    done = _fast(Q) and _call.prompt(_stream(), Q.device.index, Q, K, V, seq_lens, hq, hkv, head_dim, window, sinks, score_cap, slopes, out, lse)
    if done:
        if done[0] != RDKV_OK:
            _check(done[0])
        return done[1:]
    n, hq, hkv, d = len(seq_lens), _int32("hq", hq), _int32("hkv", hkv), _int32("head_dim", head_dim)
    lens = (ctypes.c_int32 * max(n, 1))(*[_int32("seq_lens", x) for x in seq_lens])
    cap = float(score_cap)
    if cap != 0 and ctypes.c_float(cap).value == 0:    # (0 is no cap)
        raise ValueError(f"score_cap = {score_cap} is 0 in 32 bits")
    device, tokens = Q.device, sum(max(x, 0) for x in lens[:n])
    strides = _rows_of(Q, "Q", tokens, hq, d, device), _rows_of(K, "K", tokens, hkv, d, device), _rows_of(V, "V", tokens, hkv, d, device)
    if slopes is not None:
        _tensor(slopes, (hq,), torch.float32, device, "slopes")
    if out is None:
        out = torch.empty((tokens, hq, d) if Q.dim() == 3 else Q.shape, dtype=torch.bfloat16, device=device)
    out_stride = _rows_of(out, "out", tokens, hq, d, device)
    if lse is None:
        lse = torch.empty(tokens * hq, dtype=torch.float32, device=device)
    else:
        _tensor(lse.view(-1), (tokens * hq,), torch.float32, device, "lse")
    c = rdkv_prompt(n, hq, hkv, d, lens, _int32("window", window), _int32("sinks", sinks), cap, _ptr(slopes), *strides, out_stride)
    with _at(device):
        _check(lib.rdkv_prompt_attn_bf16(ctypes.byref(c), Q.data_ptr(), K.data_ptr(), V.data_ptr(), out.data_ptr(), lse.data_ptr(), _stream()))
    return out, lse


class Slots:
    """A slot cache (rdkv_slots): its parameters and the device tensors that hold it, made here unless the caller brings them.

      k, v      bits 16: bfloat16 [batch, hkv, capacity, 128]; bits 4: uint8 [batch, hkv, ceil(capacity / 64), 5120]
      pos       int32 [batch, hkv, capacity]
      weight    float32 [batch, hkv, capacity], or None with track=False: no attention weights are kept
      lens      int32 [batch, hkv]: slots in use;  next_pos: int32 [batch, hkv]: position of the next token
      slopes    float32 [hq] or None

    The calls on it run on the current stream of its device.  A call leaves tensors it was given where they are, so that views
    of them stay good.  A tensor assigned to one of these names takes the place of the one before from the next call on (graphs
    that were captured go on with the one before); what shapes follow from stays as it was made."""

    _FIELDS = {"k": "k", "v": "v", "pos": "pos", "weight": "weight", "lens": "len", "next_pos": "next", "slopes": "slopes"}
    _FIXED = ("c", "device", "batch", "hq", "hkv", "capacity", "bits", "d", "workspace_bytes", "address")

    def __setattr__(self, name, value):
        if name in self._FIELDS:
            if value is not None:
                _tensor(value, *self._shapes[name], self.device, name)
            elif name not in ("weight", "slopes"):
                raise ValueError(f"{name} must be a tensor")
            setattr(self.c, self._FIELDS[name], None if value is None else value.data_ptr())
            if name == "weight":                       # (a step keeps scores for them)
                self.__dict__["workspace_bytes"] = lib.rdkv_slots_decode_workspace_bytes(ctypes.byref(self.c))
        elif name in self._FIXED and name in self.__dict__:
            raise AttributeError(f"{name} of a slot cache stays as it was made")
        super().__setattr__(name, value)

    def __delattr__(self, name):
        if name in self._FIELDS or name in self._FIXED:
            raise AttributeError(f"{name} belongs to the slot cache")
        super().__delattr__(name)

    def __copy__(self):
        """Another with the same tensors."""
        c = self.c
        return Slots(c.batch, c.hq, c.hkv, c.capacity, bits=c.bits, head_dim=c.head_dim, sinks=c.sinks, recent=c.recent, window=c.window,
                     score_cap=c.score_cap, decay=c.decay, track=self.weight is not None, device=self.device,
                     **{name: getattr(self, name) for name in self._FIELDS})

    def __init__(self, batch, hq, hkv, capacity, bits=16, head_dim=128, sinks=0, recent=0, window=0, score_cap=0.0, decay=1.0,
                 slopes=None, k=None, v=None, pos=None, weight=None, lens=None, next_pos=None, track=True, device=None):
        self.c = rdkv_slots()
        _check(lib.rdkv_slots_default(ctypes.byref(self.c)))
        c = self.c
        for name, x in (("batch", batch), ("hq", hq), ("hkv", hkv), ("head_dim", head_dim), ("capacity", capacity), ("bits", bits),
                        ("sinks", sinks), ("recent", recent), ("window", window)):
            setattr(c, name, _int32(name, x))
        c.score_cap, c.decay = float(score_cap), float(decay)
        if c.score_cap == 0 and score_cap != 0:        # (0 is no cap)
            raise ValueError(f"score_cap = {score_cap} is 0 in 32 bits")
        c.k = c.v = c.pos = c.len = c.next = 16        # (what the library checks of memory is that there is some)
        _check(lib.rdkv_slots_read(ctypes.byref(c), None, 0, None, None, None))
        held = [t for t in (k, v, pos, weight, lens, next_pos) if t is not None]
        device = torch.device(device) if device is not None else held[0].device if held else torch.device("cuda")
        self.device = torch.device("cuda", torch.cuda.current_device()) if device.type == "cuda" and device.index is None else device
        self.batch, self.hq, self.hkv, self.capacity, self.bits, self.d = c.batch, c.hq, c.hkv, c.capacity, c.bits, c.head_dim
        items = (c.batch, c.hkv)
        side = items + ((c.capacity, c.head_dim) if c.bits == 16 else ((c.capacity + 63) // 64, 5120))
        kind = torch.bfloat16 if c.bits == 16 else torch.uint8

        self._shapes = {"k": (side, kind), "v": (side, kind), "pos": (items + (c.capacity,), torch.int32),
                        "weight": (items + (c.capacity,), torch.float32), "lens": (items, torch.int32), "next_pos": (items, torch.int32),
                        "slopes": ((c.hq,), torch.float32)}

        def tensor(t, name):
            return torch.zeros(self._shapes[name][0], dtype=self._shapes[name][1], device=self.device) if t is None else t

        self.k, self.v, self.pos = tensor(k, "k"), tensor(v, "v"), tensor(pos, "pos")
        self.weight = tensor(weight, "weight") if track or weight is not None else None
        self.lens, self.next_pos = tensor(lens, "lens"), tensor(next_pos, "next_pos")
        self.slopes = slopes
        self.address = ctypes.addressof(c)

    def ref(self):
        return ctypes.byref(self.c)

    def workspace(self):
        """Scratch of a decode step, for callers that keep it."""
        return torch.empty(max(self.workspace_bytes, 16), dtype=torch.uint8, device=self.device)

    def tree_workspace(self, n):
        """Scratch of rdkv_slots_tree_attn with n drafted tokens, for callers that keep it."""
        need = lib.rdkv_slots_tree_workspace_bytes(self.ref(), _int32("n", n))
        return torch.empty(max(need, 16), dtype=torch.uint8, device=self.device)

    def accept_workspace(self):
        """Scratch of rdkv_slots_accept, for callers that keep it."""
        return torch.empty(max(lib.rdkv_slots_accept_workspace_bytes(self.ref()), 16), dtype=torch.uint8, device=self.device)


def _tensor(t, shape, dtype, device, name):
    """`t`, if it is what the library takes for `name`: it reads and writes plain memory."""
    if t.dtype != dtype or t.device != device or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {device}: "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}" + ("" if t.is_contiguous() else ", not contiguous"))
    return t


def _on(slots):
    """The slots' device as the current one."""
    if slots.device.type != "cuda":
        raise ValueError(f"the slots lie on {slots.device}: the calls on them run on a GPU")
    return _at(slots.device)


def _at(device):
    """A GPU as the current one."""
    if device.type != "cuda":
        raise ValueError(f"the tensors lie on {device}: the call runs on a GPU")
    index = device.index
    return _SAME if index is None or _current_device is None or _current_device() == index else torch.cuda.device(index)


def _fast(slots):
    """Whether a call may go through the native code, which looks at the tensors itself: the slots (or a tensor) lie on the current device."""
    index = slots.device.index
    return _call is not None and index is not None and _current_device is not None and _current_device() == index


class _Same:
    def __enter__(self):
        pass

    def __exit__(self, *exc):
        pass


_SAME = _Same()


def rdkv_slots_fill(slots, K, V, seq_lens, w_tok=None, first=0):
    """Prompts of len(seq_lens) sequences into the slots of sequences first, first + 1, ..: K, V bfloat16, w_tok float32 or
    None, ragged as everywhere."""
    status = _call.slots_fill(slots.address, _stream(), slots.device.index, K, V, seq_lens, w_tok, first) if _fast(slots) else None
    if status is not None:
        return _check(status)
    n, first = len(seq_lens), _int32("first", first)
    lens = (ctypes.c_int32 * max(n, 1))(*[_int32("seq_lens", x) for x in seq_lens])
    rows = sum(max(x, 0) for x in lens[:n]) * slots.hkv
    for t, name in ((K, "K"), (V, "V")):
        _tensor(t.view(-1), (rows * slots.d,), torch.bfloat16, slots.device, name)
    if w_tok is not None:
        _tensor(w_tok.view(-1), (rows,), torch.float32, slots.device, "w_tok")
    with _on(slots):
        need = lib.rdkv_slots_fill_workspace_bytes(slots.ref(), n, lens)
        workspace = torch.empty(need, dtype=torch.uint8, device=slots.device) if need else None
        _check(lib.rdkv_slots_fill(slots.ref(), first, n, lens, _ptr(K), _ptr(V), _ptr(w_tok), _ptr(workspace), need, _stream()))


def rdkv_slots_append(slots, k_new, v_new, slot=None):
    """The slot that each item's new token took: int32 [batch, hkv]."""
    done = _fast(slots) and _call.slots_append(slots.address, _stream(), slots.device.index, k_new, v_new, slot)
    if done:
        if done[0] != RDKV_OK:
            _check(done[0])
        return done[1]
    items = (slots.batch, slots.hkv)
    _tensor(k_new, items + (slots.d,), torch.bfloat16, slots.device, "k_new")
    _tensor(v_new, items + (slots.d,), torch.bfloat16, slots.device, "v_new")
    if slot is None:
        slot = torch.empty(items, dtype=torch.int32, device=slots.device)
    else:
        _tensor(slot, items, torch.int32, slots.device, "slot")
    with _on(slots):
        _check(lib.rdkv_slots_append(slots.ref(), k_new.data_ptr(), v_new.data_ptr(), slot.data_ptr(), _stream()))
    return slot


def rdkv_slots_decode_attn(slots, q, out=None, lse=None, workspace=None):
    done = _fast(slots) and _call.slots_decode(slots.address, _stream(), slots.device.index, q, out, lse, workspace, slots.workspace_bytes)
    if done:
        if done[0] != RDKV_OK:
            _check(done[0])
        return done[1:]
    rows = (slots.batch, slots.hq)
    _tensor(q, rows + (slots.d,), torch.bfloat16, slots.device, "q")
    if out is None:
        out = _empty_f32(rows + (slots.d,), (slots.hq * slots.d, slots.d, 1), slots.device)
    else:
        _tensor(out, rows + (slots.d,), torch.float32, slots.device, "out")
    if lse is None:
        lse = _empty_f32(rows, (slots.hq, 1), slots.device)
    else:
        _tensor(lse, rows, torch.float32, slots.device, "lse")
    if workspace is None:
        workspace = slots.workspace()
    elif workspace.dtype != torch.uint8 or workspace.device != slots.device or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous uint8 tensor on {slots.device}")
    with _on(slots):
        _check(lib.rdkv_slots_decode_attn(slots.ref(), q.data_ptr(), out.data_ptr(), lse.data_ptr(), workspace.data_ptr(),
                                          workspace.numel(), _stream()))
    return out, lse


def _drafted(slots, q, k_draft, v_draft):
    """The number of drafted tokens per sequence."""
    if k_draft.dim() != 4:
        raise ValueError(f"k_draft must be [batch, n, hkv, {slots.d}]: got {tuple(k_draft.shape)}")
    n = k_draft.shape[1]
    for t, name, heads in ((q, "q", slots.hq), (k_draft, "k_draft", slots.hkv), (v_draft, "v_draft", slots.hkv)):
        if t is not None:
            _tensor(t, (slots.batch, n, heads, slots.d), torch.bfloat16, slots.device, name)
    return n


def rdkv_slots_tree_attn(slots, q, k_draft, v_draft, parent, counts=None, out=None, stats=None, workspace=None):
    """(out, stats): bfloat16 [batch, n, hq, 128], float32 [batch, n, hq, 2]; what belongs to drafted tokens from counts on stays as it was."""
    done = _fast(slots) and _call.slots_tree(slots.address, _stream(), slots.device.index, q, k_draft, v_draft, parent, counts, out, stats, workspace)
    if done:
        if done[0] != RDKV_OK:
            _check(done[0])
        return done[1:]
    n = _drafted(slots, q, k_draft, v_draft)
    _tensor(parent, (slots.batch, n), torch.int32, slots.device, "parent")
    if counts is not None:
        _tensor(counts, (slots.batch,), torch.int32, slots.device, "counts")
    rows = (slots.batch, n, slots.hq)
    out = torch.empty_like(q) if out is None else _tensor(out, rows + (slots.d,), torch.bfloat16, slots.device, "out")
    if stats is None:
        stats = torch.empty(rows + (2,), dtype=torch.float32, device=slots.device)
    else:
        _tensor(stats, rows + (2,), torch.float32, slots.device, "stats")
    if workspace is None:
        workspace = slots.tree_workspace(n)
    elif workspace.dtype != torch.uint8 or workspace.device != slots.device or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous uint8 tensor on {slots.device}")
    with _on(slots):
        _check(lib.rdkv_slots_tree_attn(slots.ref(), n, q.data_ptr(), k_draft.data_ptr(), v_draft.data_ptr(), parent.data_ptr(), _ptr(counts),
                                        out.data_ptr(), stats.data_ptr(), workspace.data_ptr(), workspace.numel(), _stream()))
    return out, stats


def rdkv_slots_accept(slots, q, k_draft, v_draft, path, stats, slot=None, workspace=None):
    """The slots that the accepted tokens took: int32 [batch, hkv, m], -1 behind a path's end.  A cache without weights needs neither q nor stats (None)."""
    done = _fast(slots) and _call.slots_accept(slots.address, _stream(), slots.device.index, q, k_draft, v_draft, path, stats, slot, workspace)
    if done:
        if done[0] != RDKV_OK:
            _check(done[0])
        return done[1]
    n = _drafted(slots, q, k_draft, v_draft)
    if path.dim() != 2:
        raise ValueError(f"path must be [batch, m]: got {tuple(path.shape)}")
    m = path.shape[1]
    _tensor(path, (slots.batch, m), torch.int32, slots.device, "path")
    if stats is not None:
        _tensor(stats, (slots.batch, n, slots.hq, 2), torch.float32, slots.device, "stats")
    shape = (slots.batch, slots.hkv, m)
    slot = torch.empty(shape, dtype=torch.int32, device=slots.device) if slot is None else _tensor(slot, shape, torch.int32, slots.device, "slot")
    if workspace is None:
        workspace = slots.accept_workspace()
    elif workspace.dtype != torch.uint8 or workspace.device != slots.device or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous uint8 tensor on {slots.device}")
    with _on(slots):
        _check(lib.rdkv_slots_accept(slots.ref(), n, m, _ptr(q), k_draft.data_ptr(), v_draft.data_ptr(), path.data_ptr(), _ptr(stats), slot.data_ptr(),
                                     workspace.data_ptr(), workspace.numel(), _stream()))
    return slot


def rdkv_slots_read(slots, index=None, n=None, K=None, V=None):
    """(K, V) bfloat16 [batch, hkv, n, 128]: rows of slots `index` (int32 [batch, hkv, n]), or of the first n slots (all)."""
    done = _fast(slots) and _call.slots_read(slots.address, _stream(), slots.device.index, index, n, K, V)
    if done:
        if done[0] != RDKV_OK:
            _check(done[0])
        return done[1:]
    if index is not None:
        if index.dim() != 3 or n not in (None, index.shape[2]):
            raise ValueError(f"index must be [batch, hkv, n]: got {tuple(index.shape)}")
        n = index.shape[2]
        _tensor(index, (slots.batch, slots.hkv, n), torch.int32, slots.device, "index")
    elif n is None:
        n = slots.capacity
    n = _int32("n", n)
    shape = (slots.batch, slots.hkv, max(n, 0), slots.d)
    K = torch.empty(shape, dtype=torch.bfloat16, device=slots.device) if K is None else _tensor(K, shape, torch.bfloat16, slots.device, "K")
    V = torch.empty(shape, dtype=torch.bfloat16, device=slots.device) if V is None else _tensor(V, shape, torch.bfloat16, slots.device, "V")
    with _on(slots):
        _check(lib.rdkv_slots_read(slots.ref(), _ptr(index), n, K.data_ptr(), V.data_ptr(), _stream()))
    return K, V


def rdkv_kernel_timing_enable(enable):
    _check(lib.rdkv_kernel_timing_enable(1 if enable else 0))


def rdkv_kernel_timing_read(kind):
    """(launches, total_ms) of the bracketed main kernel of one kind since the last read."""
    n, ms = ctypes.c_int64(), ctypes.c_double()
    _check(lib.rdkv_kernel_timing_read(kind, ctypes.byref(n), ctypes.byref(ms)))
    return n.value, ms.value
