"""ctypes binding of libdmc.so (the gfx950 DMC decode-path library).

Argument marshalling only: every step of the path runs in the library's HIP
kernels.  PyTorch supplies device memory and the current HIP stream.  If the
library is missing or fails to load, importing this module raises -- there
is no fallback implementation.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import POINTER, byref, c_char_p, c_float, c_int32, c_int64, c_size_t, c_void_p

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libdmc.so")

DMC_OK, DMC_ERR_INVALID_ARG, DMC_ERR_UNSUPPORTED, DMC_ERR_CAPACITY, DMC_ERR_HIP = range(5)
DMC_BF16, DMC_FP32 = 0, 1
DMC_OMEGA_LEAD_QHEAD, DMC_OMEGA_GROUP_MEAN, DMC_OMEGA_UNIFORM = 0, 1, 2
DMC_DECISION_PER_HEAD, DMC_DECISION_SHARED_LAYER = 0, 1
OMEGA_SRC = {"lead": DMC_OMEGA_LEAD_QHEAD, "group_mean": DMC_OMEGA_GROUP_MEAN,
             "uniform": DMC_OMEGA_UNIFORM}
DECISION_SRC = {"per_head": DMC_DECISION_PER_HEAD, "shared_layer": DMC_DECISION_SHARED_LAYER}
DMC_PAIRS_HALVES, DMC_PAIRS_ADJACENT = 0, 1
PAIRS = {"halves": DMC_PAIRS_HALVES, "adjacent": DMC_PAIRS_ADJACENT}
DMC_FULL_COUNTER_BYTES = 8192
DMC_FLAG_ROW_FULL, DMC_FLAG_BAD_ROWS, DMC_FLAG_BAD_PAGE = 2, 4, 8
STATUS_NAMES = {0: "DMC_OK", 1: "DMC_ERR_INVALID_ARG", 2: "DMC_ERR_UNSUPPORTED",
                3: "DMC_ERR_CAPACITY", 4: "DMC_ERR_HIP"}

#: Every entry point declared in include/dmc.h.
EXPORTS = ("dmc_cache_workspace_bytes", "dmc_cache_alloc", "dmc_cache_free", "dmc_cache_reset",
           "dmc_prefill_compress", "dmc_prefill_attend", "dmc_decode_step", "dmc_decode_step_static",
           "dmc_cache_lengths", "dmc_cache_export",
           "dmc_cache_import", "dmc_cache_check", "dmc_cache_pages_used", "dmc_last_error",
           "dmc_train_workspace_bytes", "dmc_train_forward", "dmc_train_backward",
           "dmc_chunk_workspace_bytes", "dmc_chunk_attend", "dmc_chunk_append",
           "dmc_causal_workspace_bytes", "dmc_causal_forward", "dmc_causal_backward",
           "dmc_rotate", "dmc_full_append", "dmc_full_workspace_bytes", "dmc_full_attend")


class CacheConfig(ctypes.Structure):
    """Mirror of dmc_cache_config."""
    _fields_ = [("num_layers", c_int32), ("batch", c_int32), ("num_q_heads", c_int32),
                ("num_kv_heads", c_int32), ("head_dim", c_int32), ("dtype", c_int32),
                ("page_size", c_int32), ("max_slots_per_seq", c_int32), ("num_pages", c_int64),
                ("decision_bias", c_float), ("omega_src", c_int32), ("split_tile", c_int32),
                ("max_prompt_len", c_int32), ("decision_src", c_int32), ("window", c_int32)]


class TrainConfig(ctypes.Structure):
    """Mirror of dmc_train_config."""
    _fields_ = [("batch", c_int32), ("seq_len", c_int32), ("num_q_heads", c_int32),
                ("num_kv_heads", c_int32), ("head_dim", c_int32), ("dtype", c_int32),
                ("decision_bias", c_float), ("temperature", c_float), ("window", c_int32),
                ("omega_src", c_int32)]


class CausalConfig(ctypes.Structure):
    """Mirror of dmc_causal_config."""
    _fields_ = [("num_q_heads", c_int32), ("num_kv_heads", c_int32), ("head_dim", c_int32),
                ("dtype", c_int32)]


class RotaryConfig(ctypes.Structure):
    """Mirror of dmc_rotary_config."""
    _fields_ = [("num_q_heads", c_int32), ("num_kv_heads", c_int32), ("head_dim", c_int32),
                ("dtype", c_int32), ("rotary_dim", c_int32), ("rotary_pairs", c_int32)]


class FullConfig(ctypes.Structure):
    """Mirror of dmc_full_config."""
    _fields_ = [("batch", c_int32), ("num_q_heads", c_int32), ("num_kv_heads", c_int32),
                ("head_dim", c_int32), ("dtype", c_int32), ("page_size", c_int32), ("max_pages", c_int32),
                ("num_pages", c_int32), ("rotary_dim", c_int32), ("rotary_pairs", c_int32)]


class DMCError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


def _load():
    # torch first: its HIP runtime is then the one the library binds to (one
    # runtime per process; loading the library first can bring in a second
    # copy, which then finds no device)
    import torch  # noqa: F401
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run __graft_entry__.build() "
                          "or python paper_2403_09636_amd/csrc/build.py")
    lib = ctypes.CDLL(LIB_PATH)
    i64p = POINTER(c_int64)
    lib.dmc_cache_workspace_bytes.argtypes = [POINTER(CacheConfig)]
    lib.dmc_cache_workspace_bytes.restype = c_size_t
    lib.dmc_cache_alloc.argtypes = [POINTER(CacheConfig), c_void_p, c_size_t, c_void_p,
                                    POINTER(c_void_p)]
    lib.dmc_cache_free.argtypes = [c_void_p]
    lib.dmc_cache_reset.argtypes = [c_void_p, c_void_p]
    lib.dmc_prefill_compress.argtypes = [c_void_p, c_int32, c_void_p, i64p, c_void_p, i64p,
                                         c_void_p, i64p, c_int32, c_void_p, c_void_p, c_void_p]
    lib.dmc_prefill_attend.argtypes = [c_void_p, c_int32, c_void_p, i64p, c_void_p, i64p,
                                       c_void_p, i64p, c_int32, c_void_p, c_void_p, i64p,
                                       c_void_p, c_void_p]
    lib.dmc_decode_step.argtypes = [c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_void_p,
                                    c_void_p, c_void_p]
    lib.dmc_decode_step_static.argtypes = lib.dmc_decode_step.argtypes
    lib.dmc_cache_lengths.argtypes = [c_void_p, c_int32, c_void_p, c_void_p]
    lib.dmc_cache_export.argtypes = [c_void_p, c_int32, c_void_p, c_void_p, c_int32, c_void_p,
                                     c_void_p]
    lib.dmc_cache_import.argtypes = [c_void_p, c_int32, c_void_p, c_void_p, c_int32, c_void_p,
                                     c_void_p, c_void_p]
    lib.dmc_cache_check.argtypes = [c_void_p, c_void_p]
    lib.dmc_cache_pages_used.argtypes = [c_void_p, i64p, c_void_p]
    lib.dmc_last_error.argtypes = []
    lib.dmc_last_error.restype = c_char_p
    lib.dmc_train_workspace_bytes.argtypes = [POINTER(TrainConfig)]
    lib.dmc_train_workspace_bytes.restype = c_size_t
    lib.dmc_train_forward.argtypes = [POINTER(TrainConfig), c_void_p, c_void_p, c_void_p, c_void_p,
                                      c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.dmc_train_backward.argtypes = [POINTER(TrainConfig), c_void_p, c_void_p, c_void_p, c_void_p,
                                       c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                       c_void_p, c_size_t, c_void_p]
    packed = [c_void_p, c_void_p]   # a tensor [tokens, heads, d] and its strides (int64 [2])
    lib.dmc_chunk_workspace_bytes.argtypes = [c_void_p, c_int32, c_int32]
    lib.dmc_chunk_workspace_bytes.restype = c_size_t
    lib.dmc_chunk_attend.argtypes = [c_void_p, c_int32, *packed * 3, c_void_p, c_int32, c_int32,
                                     *packed, c_void_p, c_size_t, c_void_p]
    lib.dmc_chunk_append.argtypes = [c_void_p, c_int32, *packed * 3, c_void_p, c_void_p, c_int32,
                                     c_int32, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.dmc_causal_workspace_bytes.argtypes = [POINTER(CausalConfig), c_int32]
    lib.dmc_causal_workspace_bytes.restype = c_size_t
    lib.dmc_causal_forward.argtypes = [POINTER(CausalConfig), *packed * 3, c_void_p, c_int32, c_int32,
                                       *packed, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.dmc_causal_backward.argtypes = [POINTER(CausalConfig), *packed * 3, c_void_p, c_int32, c_int32,
                                        *packed, c_void_p, *packed * 4, c_void_p, c_size_t, c_void_p]
    lib.dmc_rotate.argtypes = [POINTER(RotaryConfig), *packed * 2, c_void_p, c_void_p, c_int32, c_int32, *packed * 2,
                               c_void_p]
    lib.dmc_full_append.argtypes = [POINTER(FullConfig), *packed * 3, c_void_p, c_void_p, c_int32, c_void_p, c_void_p,
                                    c_void_p, c_void_p, *packed, c_void_p, c_void_p]
    lib.dmc_full_workspace_bytes.argtypes = [POINTER(FullConfig), c_int32, c_int32]
    lib.dmc_full_workspace_bytes.restype = c_size_t
    lib.dmc_full_attend.argtypes = [POINTER(FullConfig), *packed, c_void_p, c_int32, c_int32, c_void_p, c_void_p,
                                    c_void_p, c_void_p, *packed, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    for name in EXPORTS:
        if not name.endswith("workspace_bytes") and name != "dmc_last_error":
            getattr(lib, name).restype = c_int32
    return lib


lib = _load()


def last_error() -> str:
    msg = lib.dmc_last_error()
    return msg.decode() if msg else ""


def check(status: int):
    if status != DMC_OK:
        raise DMCError(status, last_error())


def make_config(num_layers, batch, num_q_heads, num_kv_heads, head_dim, dtype="bf16",
                page_size=32, max_slots_per_seq=4096, num_pages=None, decision_bias=0.0,
                omega_src="lead", split_tile=0, max_prompt_len=0,
                decision_src="per_head", window=0) -> CacheConfig:
    """A dmc_cache_config; num_pages defaults to room for every unit at capacity.

    omega_src: 'lead' | 'group_mean' | 'uniform'; decision_src: 'per_head' |
    'shared_layer' (DMC-HardC); window: 0 (exact) or the window-grouping width."""
    units = num_layers * batch * num_kv_heads
    if num_pages is None:
        num_pages = units * -(-max_slots_per_seq // page_size)
    return CacheConfig(num_layers, batch, num_q_heads, num_kv_heads, head_dim,
                       DMC_FP32 if dtype in ("fp32", "float32") else DMC_BF16, page_size,
                       max_slots_per_seq, num_pages, decision_bias, OMEGA_SRC[omega_src],
                       split_tile, max_prompt_len, DECISION_SRC[decision_src], window)


def workspace_bytes(cfg: CacheConfig) -> int:
    n = lib.dmc_cache_workspace_bytes(ctypes.byref(cfg))
    if n == 0:
        raise DMCError(DMC_ERR_INVALID_ARG, last_error())
    return n


def _ptr(t):
    return None if t is None else c_void_p(t.data_ptr())


# -- argument validation ------------------------------------------------------
# The C ABI receives raw pointers and cannot see shapes, dtypes or devices, so
# everything the header requires of a tensor is checked here, before any call
# into the library.  Checks run in a fixed order (dtype, shape, layout,
# alignment, then device), so each rejection can be exercised with CPU tensors.

def _fail(msg):
    raise DMCError(DMC_ERR_INVALID_ARG, msg)


def cache_dtype(cfg):
    import torch
    return torch.float32 if cfg.dtype == DMC_FP32 else torch.bfloat16


def _check(name, t, dtype, shape=None, contiguous=True, align16=True,
           last_dim_contiguous=False, stride_mult=None):
    """Validate one tensor argument (not its device, see _on_device); shape
    entries of None match any size."""
    import torch
    if not isinstance(t, torch.Tensor):
        _fail(f"{name} must be a torch.Tensor")
    if t.dtype != dtype:
        _fail(f"{name} has dtype {t.dtype}, expected {dtype}")
    if shape is not None:
        if t.dim() != len(shape) or any(w is not None and g != w for g, w in zip(t.shape, shape)):
            want = "[" + ", ".join("*" if w is None else str(w) for w in shape) + "]"
            _fail(f"{name} has shape {list(t.shape)}, expected {want}")
    if contiguous and not t.is_contiguous():
        _fail(f"{name} must be contiguous")
    if last_dim_contiguous and t.dim() > 0 and t.shape[-1] > 1 and t.stride(-1) != 1:
        _fail(f"{name} must have a contiguous last dimension")
    if stride_mult and any(st % stride_mult for st in t.stride()[:-1]):
        _fail(f"{name} strides {tuple(t.stride())} must be multiples of {stride_mult} elements")
    if align16 and t.numel() > 0 and t.data_ptr() % 16:
        _fail(f"{name} must be 16-byte aligned")


def _on_device(device, **tensors):
    """Last check of every entry point: all tensors on the cache's device."""
    for name, t in tensors.items():
        if t is not None and t.device != device:
            _fail(f"{name} is on {t.device}, the cache is on {device}")


def check_decode_args(cfg, device, q, k, v, out, slot_index=None):
    """dmc_decode_step: q, out [B, Hq, d]; k, v [B, Hkv, d]; contiguous, cache
    dtype, 16-byte aligned; slot_index int32 [B, Hkv]."""
    import torch
    dt = cache_dtype(cfg)
    B, Hq, Hkv, d = cfg.batch, cfg.num_q_heads, cfg.num_kv_heads, cfg.head_dim
    _check("q", q, dt, (B, Hq, d))
    _check("k", k, dt, (B, Hkv, d))
    _check("v", v, dt, (B, Hkv, d))
    _check("out", out, dt, (B, Hq, d))
    if slot_index is not None:
        _check("slot_index", slot_index, torch.int32, (B, Hkv), align16=False)
    for name, t in (("q", q), ("k", k), ("v", v)):
        if _overlap(out, t):
            _fail(f"out overlaps {name}")
    _on_device(device, q=q, k=k, v=v, out=out, slot_index=slot_index)


class _DecodeCall:
    """The tensor checks of a decode step in one pass, for steps whose GPU time
    is a few microseconds: the same conditions as check_decode_args, tested on
    every call against the configuration's dtype and shapes, without a message.
    pointers() returns the addresses of q, k, v, out and slot_index, or None if
    any condition fails (check_decode_args then names it)."""

    def __init__(self, cfg, device):
        import torch
        self.Tensor = torch.Tensor
        self.device, self.dtype, self.i32 = device, cache_dtype(cfg), torch.int32
        self.q_shape = (cfg.batch, cfg.num_q_heads, cfg.head_dim)
        self.kv_shape = (cfg.batch, cfg.num_kv_heads, cfg.head_dim)
        self.slot_shape = (cfg.batch, cfg.num_kv_heads)
        es = 4 if cfg.dtype == DMC_FP32 else 2
        self.q_bytes = cfg.batch * cfg.num_q_heads * cfg.head_dim * es
        self.kv_bytes = cfg.batch * cfg.num_kv_heads * cfg.head_dim * es

    def pointers(self, q, k, v, out, slot_index):
        device, dtype, tensor = self.device, self.dtype, self.Tensor
        for t, shape in ((q, self.q_shape), (k, self.kv_shape), (v, self.kv_shape), (out, self.q_shape)):
            if not (isinstance(t, tensor) and t.dtype is dtype and t.shape == shape
                    and t.is_contiguous() and t.device == device):
                return None
        sp = None
        if slot_index is not None:
            if not (isinstance(slot_index, tensor) and slot_index.dtype is self.i32
                    and slot_index.shape == self.slot_shape and slot_index.is_contiguous()
                    and slot_index.device == device):
                return None
            sp = slot_index.data_ptr()
        qp, kp, vp, op = q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr()
        if (qp | kp | vp | op) & 15:
            return None
        end = op + self.q_bytes
        if ((op < qp + self.q_bytes and qp < end) or (op < kp + self.kv_bytes and kp < end)
                or (op < vp + self.kv_bytes and vp < end)):
            return None
        return qp, kp, vp, op, sp


def _overlap(x, y):
    if x.numel() == 0 or y.numel() == 0:
        return False
    x0, x1 = x.data_ptr(), x.data_ptr() + x.numel() * x.element_size()
    y0, y1 = y.data_ptr(), y.data_ptr() + y.numel() * y.element_size()
    return x0 < y1 and y0 < x1


def check_prefill_args(cfg, device, k, v, q, n, prompt_lens=None, slot_index=None,
                       full_q=False, out=None):
    """dmc_prefill_compress / dmc_prefill_attend: k, v [B, >= n, Hkv, d] with a
    contiguous last dimension and strides that are multiples of 8 elements,
    16-byte aligned; q [B, >= n, Hq, d] likewise when every element is read
    (prompt attention, full_q), else [B, >= n, Hq] or [B, >= n, Hq, *] (only
    element 0 is read); out like q; prompt_lens int32 [B]; slot_index int32
    [B, Hkv, n] contiguous."""
    import torch
    dt = cache_dtype(cfg)
    B, Hq, Hkv, d = cfg.batch, cfg.num_q_heads, cfg.num_kv_heads, cfg.head_dim
    maxn = cfg.max_prompt_len if cfg.max_prompt_len > 0 else cfg.max_slots_per_seq
    if not 0 <= n <= maxn:
        _fail(f"prompt length {n} outside [0, {maxn}]")
    for name, t in (("k", k), ("v", v)):
        _check(name, t, dt, (B, None, Hkv, d), contiguous=False, last_dim_contiguous=True,
               stride_mult=8)
        if t.shape[1] < n:
            _fail(f"{name} holds {t.shape[1]} tokens, fewer than n = {n}")
    if full_q:
        _check("q", q, dt, (B, None, Hq, d), contiguous=False, last_dim_contiguous=True,
               stride_mult=8)
    else:
        if q.dim() == 3:
            _check("q", q, dt, (B, None, Hq), contiguous=False, align16=False)
        else:
            _check("q", q, dt, (B, None, Hq, None), contiguous=False, align16=False)
    if q.shape[1] < n:
        _fail(f"q holds {q.shape[1]} tokens, fewer than n = {n}")
    if out is not None:
        _check("out", out, dt, (B, None, Hq, d), contiguous=False,
               last_dim_contiguous=True, stride_mult=8)
        if out.shape[1] < n:
            _fail(f"out holds {out.shape[1]} tokens, fewer than n = {n}")
        for name, t in (("q", q), ("k", k), ("v", v)):
            if _overlap(out, t):
                _fail(f"out overlaps {name}")
    if prompt_lens is not None:
        _check("prompt_lens", prompt_lens, torch.int32, (B,), align16=False)
    if slot_index is not None:
        _check("slot_index", slot_index, torch.int32, (B, Hkv, n), align16=False)
    _on_device(device, k=k, v=v, q=q, out=out, prompt_lens=prompt_lens, slot_index=slot_index)


def check_import_args(cfg, device, K, V, lengths, z):
    """dmc_cache_import: K, V [B, Hkv, dense_slots, d] contiguous cache dtype,
    16-byte aligned; lengths int32 [B, Hkv]; z float32 [B, Hkv]."""
    import torch
    dt = cache_dtype(cfg)
    B, Hkv, d = cfg.batch, cfg.num_kv_heads, cfg.head_dim
    _check("K", K, dt, (B, Hkv, None, d))
    _check("V", V, dt, (B, Hkv, K.shape[2], d))
    _check("lengths", lengths, torch.int32, (B, Hkv), align16=False)
    _check("z", z, torch.float32, (B, Hkv), align16=False)
    _on_device(device, K=K, V=V, lengths=lengths, z=z)


def check_train_args(cfg, device, q, k, v, noise, extra=()):
    """dmc_train_forward / dmc_train_backward: q-shaped [B, n, Hq, d] and
    k-shaped [B, n, Hkv, d] tensors contiguous in the config dtype and 16-byte
    aligned; noise and the per-token fp32 arrays [B, n, Hkv] contiguous.
    extra: (name, tensor, kind) with kind 'q', 'k' or 'tok' (None tensors skip)."""
    import torch
    dt = torch.float32 if cfg.dtype == DMC_FP32 else torch.bfloat16
    B, n, Hq, Hkv, d = cfg.batch, cfg.seq_len, cfg.num_q_heads, cfg.num_kv_heads, cfg.head_dim
    shapes = {"q": (dt, (B, n, Hq, d), True), "k": (dt, (B, n, Hkv, d), True),
              "tok": (torch.float32, (B, n, Hkv), False)}
    items = [("q", q, "q"), ("k", k, "k"), ("v", v, "k"), ("noise", noise, "tok"), *extra]
    for name, t, kind in items:
        if t is None:
            continue
        dtype, shape, a16 = shapes[kind]
        _check(name, t, dtype, shape, align16=a16)
    _on_device(device, **{name: t for name, t, _ in items})


def _spans(t):
    """Byte range of a tensor [tokens, heads, d], and of its first token in it."""
    es = t.element_size()
    row = ((t.shape[1] - 1) * t.stride(1) + t.shape[2]) * es
    return t.data_ptr(), t.data_ptr() + (t.shape[0] - 1) * t.stride(0) * es + row, row


def _packed_overlap(x, y):
    """Whether two tensors [tokens, heads, d] share memory; views of one projection whose tokens
    interleave without sharing any element do not."""
    if x.numel() == 0 or y.numel() == 0:
        return False
    x0, x1, xr = _spans(x)
    y0, y1, yr = _spans(y)
    if x0 >= y1 or y0 >= x1:
        return False
    step = x.stride(0) * x.element_size()
    if step != y.stride(0) * y.element_size() or step < max(xr, yr):
        return True
    shift = (y0 - x0) % step   # y's tokens start this far behind x's
    return shift < xr or shift + yr > step


def _touches(x, lo, hi):
    """Whether a tensor [tokens, heads, d] has an element in the bytes lo .. hi - 1."""
    x0, x1, _ = _spans(x)
    if x.numel() == 0 or x0 >= hi or lo >= x1:
        return False
    es, row, step = x.element_size(), x.shape[2] * x.element_size(), x.stride(0) * x.element_size()
    for h in range(x.shape[1]):
        at = x0 + h * x.stride(1) * es   # rows at + t * step
        if step == 0:
            if at < hi and at + row > lo:
                return True
        else:
            first = max(0, -(-(lo - row + 1 - at) // step))   # the first row that ends behind lo
            if first < x.shape[0] and at + first * step < hi:
                return True
    return False


def _shared(x, y):
    """Whether two tensors share memory: packed ones (three dimensions) or contiguous arrays."""
    if x.dim() != 3:
        x, y = y, x
    if x.dim() != 3:
        return _overlap(x, y)
    if y.dim() == 3:
        return _packed_overlap(x, y)
    return y.numel() > 0 and _touches(x, y.data_ptr(), y.data_ptr() + y.numel() * y.element_size())


def _check_apart(written, read):
    """No tensor that a call writes (name, tensor or None) shares memory with another one of it."""
    for i, (name, x) in enumerate(written):
        for other, y in (*read, *written[:i]):
            if x is not None and y is not None and _shared(x, y):
                _fail(f"{name} overlaps {other}")


def _check_rows(name, t, dtype, tokens, heads, d):
    some = getattr(t, "shape", (1,))[:1] != (0,)   # (an empty tensor's strides mean nothing)
    _check(name, t, dtype, (tokens, heads, d), contiguous=False, last_dim_contiguous=some,
           stride_mult=8 if some else None)


def _check_packed(inputs, outputs, dtype, d):
    """Packed tensors (name, tensor, tokens, heads): [tokens, heads, d], contiguous last dimension,
    strides multiples of 8 elements, 16-byte aligned; an output shares memory with no other one."""
    for name, t, tokens, heads in (*inputs, *outputs):
        _check_rows(name, t, dtype, tokens, heads, d)
    _check_apart([x[:2] for x in outputs], [x[:2] for x in inputs])


def _check_cu(cu_seqlens, rows=None):
    import torch
    _check("cu_seqlens", cu_seqlens, torch.int32, (None if rows is None else rows + 1,), align16=False)
    if cu_seqlens.numel() < 1:
        _fail("cu_seqlens is empty")


class _PackedCall:
    """The checks of a packed call's tensors in one pass, for calls whose GPU time is a few
    microseconds: the conditions of _check_packed and _check_apart, tested without a message.  tensors()
    returns the addresses of the tensors and their strides as one int64 array, or None if any condition
    fails (the caller's full check then names it, or finds that nothing is wrong)."""

    def __init__(self, dtype, device, d, es):
        import torch
        self.Tensor, self.f32, self.i32 = torch.Tensor, torch.float32, torch.int32
        self.dtype, self.device, self.d, self.es = dtype, device, d, es
        self.strides = {n: c_int64 * (2 * n) for n in range(1, 9)}

    def tensors(self, T, inputs, outputs, read=(), written=()):
        """inputs, outputs: (tensor, heads) each; read, written: the byte ranges of the
        call's arrays, as addresses.  What is written must lie apart from everything."""
        dtype, device, d, es, tensor = self.dtype, self.device, self.d, self.es, self.Tensor
        ptrs, strides, spans = [], [], [*read]
        for t, heads in (*inputs, *outputs):
            if not (isinstance(t, tensor) and t.dtype is dtype and t.shape == (T, heads, d) and t.device == device):
                return None
            s0, s1, s2 = t.stride()
            p = t.data_ptr()
            if s2 != 1 or (s0 | s1) & 7 or p & 15:
                return None
            ptrs.append(p)
            strides += (s0, s1)
            spans.append((p, p + ((T - 1) * s0 + (heads - 1) * s1 + d) * es))
        spans += written
        for i in range(len(read) + len(inputs), len(spans)):
            lo, hi = spans[i]
            for a, b in spans[:i]:
                if lo < b and a < hi:
                    return None
        return ptrs, self.strides[len(ptrs)](*strides)

    def rows(self, t):
        return t.shape[0] if isinstance(t, self.Tensor) and t.dim() else 0

    def array(self, t, dtype, shape=None):
        """Address of a contiguous tensor of this type and shape (None: of one dimension and not
        empty), or None."""
        if not (isinstance(t, self.Tensor) and t.dtype is dtype and t.device == self.device and t.is_contiguous()):
            return None
        if (t.dim() != 1 or t.shape[0] < 1) if shape is None else t.shape != shape:
            return None
        return t.data_ptr()


class _RowsCall:
    """Like _PackedCall, for calls of a few tensors whose host time is the larger part of a step: every
    condition is tested on every call, the strides' array is kept while the strides stay the same."""

    def __init__(self, dtype, device, d, es):
        import torch
        self.Tensor, self.dtype, self.device, self.d, self.es = torch.Tensor, dtype, device, d, es
        self.f32, self.i32 = torch.float32, torch.int32
        self.kept = None, None

    def take(self, t, shape):
        """(address, token stride, head stride, end) of a tensor of this shape [T, heads, d], or None."""
        if not (isinstance(t, self.Tensor) and t.dtype is self.dtype and t.shape == shape and t.device == self.device):
            return None
        s0, s1, s2 = t.stride()
        p = t.data_ptr()
        if s2 != 1 or (s0 | s1) & 7 or p & 15:
            return None
        return p, s0, s1, p + ((shape[0] - 1) * s0 + (shape[1] - 1) * s1 + self.d) * self.es

    def flat(self, t, dtype, shape):
        """Address of a contiguous tensor of this type and shape, or None."""
        if isinstance(t, self.Tensor) and t.dtype is dtype and t.shape == shape and t.device == self.device and t.is_contiguous():
            return t.data_ptr()
        return None

    def strides(self, *values):
        kept = self.kept   # (one attribute: threads that share the object get their own call's)
        if values != kept[0]:
            self.kept = kept = values, (c_int64 * len(values))(*values)
        return kept[1]


def check_chunk_args(cfg, device, q, k, v, cu_seqlens, out=None, accepted=None, slot_index=None):
    """dmc_chunk_attend (with out) and dmc_chunk_append: packed k, v [T, Hkv, d] and, for attention,
    q, out [T, Hq, d]; otherwise q [T, Hq] or [T, Hq, *] (only element 0 is read); cu_seqlens int32
    [B + 1]; accepted int32 [B]; slot_index int32 [T, Hkv]."""
    import torch
    dt = cache_dtype(cfg)
    Hq, Hkv, d = cfg.num_q_heads, cfg.num_kv_heads, cfg.head_dim
    _check_rows("k", k, dt, None, Hkv, d)
    T = k.shape[0]
    inputs = [("k", k, T, Hkv), ("v", v, T, Hkv)]
    if out is not None:
        _check_packed([("q", q, T, Hq), *inputs], [("out", out, T, Hq)], dt, d)
    else:
        _check_packed(inputs, (), dt, d)
        _check("q", q, dt, (T, Hq) if isinstance(q, torch.Tensor) and q.dim() == 2 else (T, Hq, None),
               contiguous=False, align16=False)
    _check_cu(cu_seqlens, cfg.batch)
    if accepted is not None:
        _check("accepted", accepted, torch.int32, (cfg.batch,), align16=False)
    if slot_index is not None:
        _check("slot_index", slot_index, torch.int32, (T, Hkv), align16=False)
        q0 = q.unsqueeze(-1) if q.dim() == 2 else q[..., :1]   # what is read of it
        _check_apart([("slot_index", slot_index)], [("k", k), ("v", v), ("q", q0)])
    _check_apart([("out", out), ("slot_index", slot_index)], [("cu_seqlens", cu_seqlens), ("accepted", accepted)])
    _on_device(device, q=q, k=k, v=v, cu_seqlens=cu_seqlens, out=out, accepted=accepted,
               slot_index=slot_index)


def check_causal_args(cfg, device, q, k, v, cu_seqlens, out, lse, dout=None, dq=None, dk=None, dv=None):
    """dmc_causal_forward / dmc_causal_backward (with dout and the gradients): q-shaped [T, Hq, d] and
    k-shaped [T, Hkv, d] packed tensors, cu_seqlens int32 [sequences + 1], lse float32 [T, Hq]."""
    import torch
    dt = torch.float32 if cfg.dtype == DMC_FP32 else torch.bfloat16
    Hq, Hkv, d = cfg.num_q_heads, cfg.num_kv_heads, cfg.head_dim
    _check_rows("q", q, dt, None, Hq, d)
    T = q.shape[0]
    inputs = [("q", q, T, Hq), ("k", k, T, Hkv), ("v", v, T, Hkv)]
    outputs = [("out", out, T, Hq)]
    if dout is not None:
        inputs += [*outputs, ("dout", dout, T, Hq)]
        outputs = [("dq", dq, T, Hq), ("dk", dk, T, Hkv), ("dv", dv, T, Hkv)]
    _check_packed(inputs, outputs, dt, d)
    _check_cu(cu_seqlens)
    _check("lse", lse, torch.float32, (T, Hq), align16=False)
    tensors, written = [x[:2] for x in inputs], [x[:2] for x in outputs]
    if dout is None:
        _check_apart([("lse", lse)], [*tensors, *written])
        _check_apart([*written, ("lse", lse)], [("cu_seqlens", cu_seqlens)])
    else:
        _check_apart(written, [("lse", lse), ("cu_seqlens", cu_seqlens)])
    _on_device(device, cu_seqlens=cu_seqlens, lse=lse,
               **{name: t for name, t, _, _ in (*inputs, *outputs)})


def _check_in_place(pairs, read, arrays):
    """Outputs share no memory with another tensor, but with the input of their own if both are the same
    rows: pairs of (name, input, output name, output), other tensors read, contiguous arrays."""
    for i, (name, x, out_name, out) in enumerate(pairs):
        same = out.data_ptr() == x.data_ptr() and out.stride() == x.stride()
        others = [(n, t) for j, (n, t, _, _) in enumerate(pairs) if j != i]
        others += [(n, t) for _, _, n, t in pairs[:i]]
        _check_apart([(out_name, out)], [*([] if same else [(name, x)]), *others, *read, *arrays])


def check_rotary_args(cfg, device, q, k, positions, inv_freq, q_out, k_out):
    """dmc_rotate: packed q, q_out [T, Hq, d] and k, k_out [T, Hkv, d], positions int32 [T], inv_freq
    float32 [rotary_dim / 2] (None if that is 0); an output may be its own input."""
    import torch
    dt = torch.float32 if cfg.dtype == DMC_FP32 else torch.bfloat16
    Hq, Hkv, d = cfg.num_q_heads, cfg.num_kv_heads, cfg.head_dim
    _check_rows("q", q, dt, None, Hq, d)
    T = q.shape[0]
    _check_rows("k", k, dt, T, Hkv, d)
    _check_rows("q_out", q_out, dt, T, Hq, d)
    _check_rows("k_out", k_out, dt, T, Hkv, d)
    _check("positions", positions, torch.int32, (T,), align16=False)
    arrays = [("positions", positions)]
    if cfg.rotary_dim:
        _check("inv_freq", inv_freq, torch.float32, (cfg.rotary_dim // 2,), align16=False)
        arrays.append(("inv_freq", inv_freq))
    _check_in_place([("q", q, "q_out", q_out), ("k", k, "k_out", k_out)], [], arrays)
    _on_device(device, q=q, k=k, q_out=q_out, k_out=k_out, **dict(arrays))


def _check_full_tokens(cfg, T, cu_seqlens):
    if cu_seqlens is not None:
        _check_cu(cu_seqlens, cfg.batch)
    elif T != cfg.batch:
        _fail(f"{T} tokens without cu_seqlens, one for each of {cfg.batch} rows expected")


def check_full_append_args(cfg, device, storage, k, v, q=None, q_out=None, cu_seqlens=None):
    """dmc_full_append: packed k, v [T, Hkv, d], q, q_out [T, Hq, d] (both or none; q_out may be q),
    cu_seqlens int32 [batch + 1] or None (T = batch); storage: the cache's own tensors, by name."""
    import torch
    dt = cache_dtype(cfg)
    Hq, Hkv, d = cfg.num_q_heads, cfg.num_kv_heads, cfg.head_dim
    _check_rows("k", k, dt, None, Hkv, d)
    T = k.shape[0]
    _check_rows("v", v, dt, T, Hkv, d)
    if (q is None) != (q_out is None):
        _fail("q and q_out go together")
    read = [("k", k), ("v", v)]
    if q is not None:
        _check_rows("q", q, dt, T, Hq, d)
        _check_rows("q_out", q_out, dt, T, Hq, d)
    _check_full_tokens(cfg, T, cu_seqlens)
    own = list(storage.items())
    if q is not None:
        _check_in_place([("q", q, "q_out", q_out)], read, [*own, ("cu_seqlens", cu_seqlens)])
        read.append(("q", q))
    _check_apart([x for x in own if x[0] in ("k_pages", "v_pages")], [*read, ("cu_seqlens", cu_seqlens)])
    _on_device(device, k=k, v=v, q=q, q_out=q_out, cu_seqlens=cu_seqlens)


def check_full_attend_args(cfg, device, storage, q, out, lse=None, cu_seqlens=None):
    """dmc_full_attend: packed q, out [T, Hq, d], lse float32 [T, Hq] or None, cu_seqlens int32 [batch + 1]
    or None (T = batch); storage: the cache's own tensors, by name."""
    import torch
    dt = cache_dtype(cfg)
    Hq, d = cfg.num_q_heads, cfg.head_dim
    _check_rows("q", q, dt, None, Hq, d)
    T = q.shape[0]
    _check_rows("out", out, dt, T, Hq, d)
    if lse is not None:
        _check("lse", lse, torch.float32, (T, Hq), align16=False)
    _check_full_tokens(cfg, T, cu_seqlens)
    read = [("q", q), *storage.items(), ("cu_seqlens", cu_seqlens)]
    _check_apart([("out", out), ("lse", lse)], read)
    _on_device(device, q=q, out=out, lse=lse, cu_seqlens=cu_seqlens)


def _stream(stream, device):
    """The handle of a stream, or of the current one of the device that the call's tensors are on
    (which need not be the current device)."""
    import torch
    if stream is not None:
        return stream.cuda_stream
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)   # no Stream object around the handle
    return raw(device.index) if raw else torch.cuda.current_stream(device).cuda_stream


def _cuda_device(device):
    import torch
    dev = torch.device(device)
    if dev.type == "cuda" and dev.index is None:
        dev = torch.device("cuda", torch.cuda.current_device())
    return dev


class DMCCache:
    """A paged DMC cache in one torch-allocated workspace on the current GPU.

    Thin wrapper over the C ABI.  The library checks pointers, alignment,
    strides, layer and prompt length; the shapes, dtypes, devices and layouts
    of the tensors, which it cannot see, are checked here before each call
    (check_*_args), raising DMCError.
    """

    def __init__(self, cfg: CacheConfig, device="cuda", stream=None):
        import torch
        self.cfg = cfg
        self.device = _cuda_device(device)
        self.dtype = torch.float32 if cfg.dtype == DMC_FP32 else torch.bfloat16
        self.G = cfg.num_q_heads // cfg.num_kv_heads
        nbytes = workspace_bytes(cfg)
        self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
        base = self.workspace.data_ptr()
        self._ws_ptr = (base + 255) // 256 * 256
        self._ws_bytes = nbytes
        handle = c_void_p()
        check(lib.dmc_cache_alloc(ctypes.byref(cfg), c_void_p(self._ws_ptr), nbytes,
                                  _stream(stream, self.device), ctypes.byref(handle)))
        self.handle = handle
        self._decode_call = _DecodeCall(cfg, self.device)

    def close(self):
        if getattr(self, "handle", None):
            lib.dmc_cache_free(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- hot path -------------------------------------------------------------
    def _decode(self, step, layer, q, k, v, out, slot_index, stream):
        ptrs = self._decode_call.pointers(q, k, v, out, slot_index)
        if ptrs is None:
            check_decode_args(self.cfg, self.device, q, k, v, out, slot_index)
            ptrs = (q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
                    None if slot_index is None else slot_index.data_ptr())
        check(step(self.handle, layer, *ptrs, _stream(stream, self.device)))
        return out

    def decode_step(self, layer, q, k, v, out=None, slot_index=None, stream=None):
        """Algorithm 1 update + attention for one layer; returns out [B, Hq, d]."""
        if out is None:
            out = torch_empty_like(q)
        return self._decode(lib.dmc_decode_step, layer, q, k, v, out, slot_index, stream)

    def decode_step_static(self, layer, q, k, v, out, slot_index=None, stream=None):
        """dmc_decode_step_static: as decode_step, with the split-K records in the
        library's static device scratch; allocates nothing (`out` is required)."""
        return self._decode(lib.dmc_decode_step_static, layer, q, k, v, out, slot_index, stream)

    def prefill(self, layer, k, v, q, n=None, prompt_lens=None, slot_index=None, stream=None):
        """Compress a prompt: k, v [B, n, Hkv, d] (strided), q [B, n, Hq, (d)]."""
        n = k.shape[1] if n is None else n
        check_prefill_args(self.cfg, self.device, k, v, q, n, prompt_lens, slot_index)
        ks = (c_int64 * 3)(k.stride(0), k.stride(1), k.stride(2))
        vs = (c_int64 * 3)(v.stride(0), v.stride(1), v.stride(2))
        qs = (c_int64 * 3)(q.stride(0), q.stride(1), q.stride(2))
        check(lib.dmc_prefill_compress(self.handle, layer, _ptr(k), ks, _ptr(v), vs, _ptr(q), qs,
                                       n, _ptr(prompt_lens), _ptr(slot_index), _stream(stream, self.device)))

    def prefill_attend(self, layer, k, v, q, out=None, n=None, prompt_lens=None, slot_index=None,
                       stream=None):
        """Compress a prompt and attend every prompt query: k, v [B, n, Hkv, d],
        q [B, n, Hq, d] (strided, d contiguous); returns out [B, n, Hq, d]."""
        n = k.shape[1] if n is None else n
        if out is None:
            import torch
            out = torch.empty((q.shape[0], n, q.shape[2], q.shape[3]), dtype=q.dtype,
                              device=q.device)
        check_prefill_args(self.cfg, self.device, k, v, q, n, prompt_lens, slot_index,
                           full_q=True, out=out)
        ks = (c_int64 * 3)(k.stride(0), k.stride(1), k.stride(2))
        vs = (c_int64 * 3)(v.stride(0), v.stride(1), v.stride(2))
        qs = (c_int64 * 3)(q.stride(0), q.stride(1), q.stride(2))
        os_ = (c_int64 * 3)(out.stride(0), out.stride(1), out.stride(2))
        check(lib.dmc_prefill_attend(self.handle, layer, _ptr(k), ks, _ptr(v), vs, _ptr(q), qs, n,
                                     _ptr(prompt_lens), _ptr(out), os_, _ptr(slot_index),
                                     _stream(stream, self.device)))
        return out

    # -- accessors --------------------------------------------------------------
    def lengths(self, layer, stream=None):
        import torch
        out = torch.empty((self.cfg.batch, self.cfg.num_kv_heads), dtype=torch.int32,
                          device=self.device)
        check(lib.dmc_cache_lengths(self.handle, layer, _ptr(out), _stream(stream, self.device)))
        return out

    def export(self, layer, dense_slots=None, stream=None):
        import torch
        dense_slots = self.cfg.max_slots_per_seq if dense_slots is None else dense_slots
        shape = (self.cfg.batch, self.cfg.num_kv_heads, dense_slots, self.cfg.head_dim)
        K = torch.empty(shape, dtype=self.dtype, device=self.device)
        V = torch.empty(shape, dtype=self.dtype, device=self.device)
        z = torch.empty(shape[:2], dtype=torch.float32, device=self.device)
        check(lib.dmc_cache_export(self.handle, layer, _ptr(K), _ptr(V), dense_slots, _ptr(z),
                                   _stream(stream, self.device)))
        return K, V, z

    def import_(self, layer, K, V, lengths, z, stream=None):
        check_import_args(self.cfg, self.device, K, V, lengths, z)
        check(lib.dmc_cache_import(self.handle, layer, _ptr(K), _ptr(V), K.shape[2],
                                   _ptr(lengths), _ptr(z), _stream(stream, self.device)))

    def check(self, stream=None):
        check(lib.dmc_cache_check(self.handle, _stream(stream, self.device)))

    def status(self, stream=None) -> int:
        return lib.dmc_cache_check(self.handle, _stream(stream, self.device))

    def pages_used(self, stream=None) -> int:
        n = c_int64()
        check(lib.dmc_cache_pages_used(self.handle, ctypes.byref(n), _stream(stream, self.device)))
        return n.value

    def reset(self, stream=None):
        check(lib.dmc_cache_reset(self.handle, _stream(stream, self.device)))


class DMCChunk:
    """Chunks of new tokens on top of a cache (pieces of prompts, later turns, packed prompts,
    drafted tokens): the workspace for up to max_tokens tokens in a call, at most max_chunk of them
    in a batch row, in one torch allocation.  Keeps the cache alive."""

    def __init__(self, cache: DMCCache, max_tokens, max_chunk=None):
        import torch
        self.cache = cache
        self.max_tokens = max_tokens
        self.max_chunk = max(1, max_tokens if max_chunk is None else max_chunk)
        n = lib.dmc_chunk_workspace_bytes(cache.handle, max_tokens, self.max_chunk)
        if n == 0:
            raise DMCError(DMC_ERR_INVALID_ARG, last_error())
        self.workspace = torch.empty(n + 256, dtype=torch.uint8, device=cache.device)
        self._ws = c_void_p((self.workspace.data_ptr() + 255) // 256 * 256)
        self._ws_bytes = n

        self._call = _PackedCall(cache.dtype, cache.device, cache.cfg.head_dim, 4 if cache.cfg.dtype == DMC_FP32 else 2)
        self._cu_shape = (cache.cfg.batch + 1,)

    def _tokens(self, T):
        if T > self.max_tokens:
            _fail(f"{T} tokens, the workspace holds {self.max_tokens}")
        return T

    def attend(self, layer, q, k, v, cu_seqlens, out=None, stream=None):
        """Attention of packed new tokens q [T, Hq, d], k, v [T, Hkv, d] over the layer's cache and
        themselves, row b's chunk being the tokens cu_seqlens[b] .. cu_seqlens[b + 1] - 1; the cache
        stays as it is.  Returns out [T, Hq, d]; rows outside every chunk stay as they are."""
        if out is None:
            out = torch_empty_like(q)
        call, cfg = self._call, self.cache.cfg
        T = call.rows(k)
        Hq, Hkv = cfg.num_q_heads, cfg.num_kv_heads
        cu, args = call.array(cu_seqlens, call.i32, self._cu_shape), None
        if cu is not None and T > 0:
            args = call.tensors(T, ((q, Hq), (k, Hkv), (v, Hkv)), ((out, Hq),), ((cu, cu + 4 * cfg.batch + 4),))
        if args is None:
            check_chunk_args(cfg, self.cache.device, q, k, v, cu_seqlens, out)
            args, cu = _packed_args(q, k, v, out), cu_seqlens.data_ptr()
        (qp, kp, vp, op), st = args
        check(lib.dmc_chunk_attend(self.cache.handle, layer, qp, st, kp, byref(st, 16), vp, byref(st, 32), cu,
                                   self._tokens(T), self.max_chunk, op, byref(st, 48), self._ws,
                                   self._ws_bytes, _stream(stream, self.cache.device)))
        return out

    def append(self, layer, k, v, q, cu_seqlens, accepted=None, slot_index=None, stream=None):
        """Append the chunk (of row b only its first accepted[b] tokens) to the layer's cache; only
        q[..., 0] is read.  slot_index [T, Hkv] receives each token's slot, -1 if not appended."""
        call, cfg = self._call, self.cache.cfg
        T = call.rows(k)
        Hq, Hkv = cfg.num_q_heads, cfg.num_kv_heads
        cu, args = call.array(cu_seqlens, call.i32, self._cu_shape), None
        acc = None if accepted is None else call.array(accepted, call.i32, (cfg.batch,))
        slots = None if slot_index is None else call.array(slot_index, call.i32, (T, Hkv))
        if cu is not None and (acc is None) == (accepted is None) and (slots is None) == (slot_index is None) and T > 0:
            read, written = [(cu, cu + 4 * cfg.batch + 4)], ()
            if acc is not None:
                read.append((acc, acc + 4 * cfg.batch))
            if slots is not None:
                written = ((slots, slots + 4 * T * Hkv),)
            args = call.tensors(T, ((q, Hq), (k, Hkv), (v, Hkv)), (), read, written)
        if args is None:
            check_chunk_args(cfg, self.cache.device, q, k, v, cu_seqlens, None, accepted, slot_index)
            args, cu = _packed_args(q, k, v), cu_seqlens.data_ptr()
            acc, slots = _ptr(accepted), _ptr(slot_index)
        (qp, kp, vp), st = args
        check(lib.dmc_chunk_append(self.cache.handle, layer, kp, byref(st, 16), vp, byref(st, 32), qp, st, cu, acc,
                                   self._tokens(T), self.max_chunk, slots, self._ws, self._ws_bytes,
                                   _stream(stream, self.cache.device)))


def torch_empty_like(t):
    import torch
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def _new_like(name, t):
    """An output for a call that got none: contiguous, like the tensor t of this name."""
    import torch
    if not isinstance(t, torch.Tensor):
        _fail(f"{name} must be a torch.Tensor")
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def make_train_config(batch, seq_len, num_q_heads, num_kv_heads, head_dim, dtype="bf16",
                      decision_bias=5.0, temperature=0.1, window=12, omega_src="lead") -> TrainConfig:
    """A dmc_train_config (defaults: the paper's c = 5, tau = 0.1, w = 12)."""
    return TrainConfig(batch, seq_len, num_q_heads, num_kv_heads, head_dim,
                       DMC_FP32 if dtype in ("fp32", "float32") else DMC_BF16, decision_bias,
                       temperature, window, OMEGA_SRC[omega_src])


class DMCTrainer:
    """Training-time DMC attention of one layer shape (forward + backward)
    with its workspace in one torch allocation on the current GPU."""

    def __init__(self, cfg: TrainConfig, device="cuda"):
        import torch
        self.cfg = cfg
        n = lib.dmc_train_workspace_bytes(ctypes.byref(cfg))
        if n == 0:
            raise DMCError(DMC_ERR_INVALID_ARG, last_error())
        self.device = _cuda_device(device)
        self.workspace = torch.empty(n + 256, dtype=torch.uint8, device=self.device)
        self._ws = c_void_p((self.workspace.data_ptr() + 255) // 256 * 256)
        self._ws_bytes = n

    def forward(self, q, k, v, noise, out=None, alpha=None, stream=None):
        """out [B, n, Hq, d] (and alpha [B, n, Hkv] fp32 if given)."""
        if out is None:
            out = torch_empty_like(q)
        check_train_args(self.cfg, self.device, q, k, v, noise,
                         (("out", out, "q"), ("alpha", alpha, "tok")))
        check(lib.dmc_train_forward(ctypes.byref(self.cfg), _ptr(q), _ptr(k), _ptr(v), _ptr(noise),
                                    _ptr(out), _ptr(alpha), self._ws, self._ws_bytes,
                                    _stream(stream, self.device)))
        return out

    def backward(self, q, k, v, noise, out, dout, dalpha=None, dq=None, dk=None, dv=None,
                 stream=None):
        """(dq, dk, dv) of sum(out * dout) + sum(alpha * dalpha)."""
        dq = torch_empty_like(q) if dq is None else dq
        dk = torch_empty_like(k) if dk is None else dk
        dv = torch_empty_like(v) if dv is None else dv
        check_train_args(self.cfg, self.device, q, k, v, noise,
                         (("out", out, "q"), ("dout", dout, "q"), ("dalpha", dalpha, "tok"),
                          ("dq", dq, "q"), ("dk", dk, "k"), ("dv", dv, "k")))
        check(lib.dmc_train_backward(ctypes.byref(self.cfg), _ptr(q), _ptr(k), _ptr(v),
                                     _ptr(noise), _ptr(out), _ptr(dout), _ptr(dalpha), _ptr(dq),
                                     _ptr(dk), _ptr(dv), self._ws, self._ws_bytes,
                                     _stream(stream, self.device)))
        return dq, dk, dv


def make_causal_config(num_q_heads, num_kv_heads, head_dim, dtype="bf16") -> CausalConfig:
    """A dmc_causal_config: plain causal attention (no cache, no compression)."""
    return CausalConfig(num_q_heads, num_kv_heads, head_dim,
                        DMC_FP32 if dtype in ("fp32", "float32") else DMC_BF16)


def _packed_args(*tensors):
    """Addresses and strides of packed tensors that have passed the full check."""
    strides = [x for t in tensors for x in t.stride()[:2]]
    return [t.data_ptr() for t in tensors], (c_int64 * len(strides))(*strides)


class DMCCausal:
    """Plain causal attention of packed sequences (forward + backward), for layers without
    compression; the workspace, for up to max_tokens tokens, is one torch allocation."""

    def __init__(self, cfg: CausalConfig, max_tokens, device="cuda"):
        import torch
        self.cfg = cfg
        self._cfg_ref = byref(cfg)
        n = lib.dmc_causal_workspace_bytes(self._cfg_ref, max_tokens)
        if n == 0:
            raise DMCError(DMC_ERR_INVALID_ARG, last_error())
        self.max_tokens = max_tokens
        self.device = _cuda_device(device)
        fp32 = cfg.dtype == DMC_FP32
        self._call = _PackedCall(torch.float32 if fp32 else torch.bfloat16, self.device, cfg.head_dim, 4 if fp32 else 2)
        self.workspace = torch.empty(n + 256, dtype=torch.uint8, device=self.device)
        self._ws = c_void_p((self.workspace.data_ptr() + 255) // 256 * 256)
        self._ws_bytes = n

    def forward(self, q, k, v, cu_seqlens, out=None, lse=None, stream=None):
        """(out [T, Hq, d], lse [T, Hq] fp32) of q [T, Hq, d], k, v [T, Hkv, d], sequence b holding
        the tokens cu_seqlens[b] .. cu_seqlens[b + 1] - 1; other rows of out and lse stay as they
        are."""
        import torch
        if out is None:
            out = torch_empty_like(q)
        if lse is None:
            lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
        call = self._call
        T = call.rows(q)
        Hq, Hkv = self.cfg.num_q_heads, self.cfg.num_kv_heads
        lp, cu, args = call.array(lse, call.f32, (T, Hq)), call.array(cu_seqlens, call.i32), None
        if lp is not None and cu is not None and T > 0:
            args = call.tensors(T, ((q, Hq), (k, Hkv), (v, Hkv)), ((out, Hq),),
                                ((cu, cu + 4 * cu_seqlens.shape[0]),), ((lp, lp + 4 * T * Hq),))
        if args is None:
            check_causal_args(self.cfg, self.device, q, k, v, cu_seqlens, out, lse)
            args, lp, cu = _packed_args(q, k, v, out), lse.data_ptr(), cu_seqlens.data_ptr()
        if T > self.max_tokens:
            _fail(f"{T} tokens, the workspace holds {self.max_tokens}")
        (qp, kp, vp, op), st = args
        check(lib.dmc_causal_forward(self._cfg_ref, qp, st, kp, byref(st, 16), vp, byref(st, 32), cu,
                                     cu_seqlens.numel() - 1, T, op, byref(st, 48), lp, self._ws,
                                     self._ws_bytes, _stream(stream, self.device)))
        return out, lse

    def backward(self, q, k, v, cu_seqlens, out, lse, dout, dq=None, dk=None, dv=None, stream=None):
        """(dq, dk, dv) of sum(out * dout), given the forward's inputs and outputs."""
        dq = torch_empty_like(q) if dq is None else dq
        dk = torch_empty_like(k) if dk is None else dk
        dv = torch_empty_like(v) if dv is None else dv
        call = self._call
        T = call.rows(q)
        Hq, Hkv = self.cfg.num_q_heads, self.cfg.num_kv_heads
        lp, cu, args = call.array(lse, call.f32, (T, Hq)), call.array(cu_seqlens, call.i32), None
        if lp is not None and cu is not None and T > 0:
            args = call.tensors(T, ((q, Hq), (k, Hkv), (v, Hkv), (out, Hq), (dout, Hq)),
                                ((dq, Hq), (dk, Hkv), (dv, Hkv)),
                                ((cu, cu + 4 * cu_seqlens.shape[0]), (lp, lp + 4 * T * Hq)))
        if args is None:
            check_causal_args(self.cfg, self.device, q, k, v, cu_seqlens, out, lse, dout, dq, dk, dv)
            args = _packed_args(q, k, v, out, dout, dq, dk, dv)
            lp, cu = lse.data_ptr(), cu_seqlens.data_ptr()
        if T > self.max_tokens:
            _fail(f"{T} tokens, the workspace holds {self.max_tokens}")
        (qp, kp, vp, op, dop, dqp, dkp, dvp), st = args
        check(lib.dmc_causal_backward(self._cfg_ref, qp, st, kp, byref(st, 16), vp, byref(st, 32), cu,
                                      cu_seqlens.numel() - 1, T, op, byref(st, 48), lp, dop, byref(st, 64),
                                      dqp, byref(st, 80), dkp, byref(st, 96), dvp, byref(st, 112), self._ws,
                                      self._ws_bytes, _stream(stream, self.device)))
        return dq, dk, dv


def make_rotary_config(num_q_heads, num_kv_heads, head_dim, dtype="bf16", rotary_dim=None, pairs="halves") -> RotaryConfig:
    """A dmc_rotary_config: rotary_dim elements of every head turn (default: all of them), in pairs
    (i, i + rotary_dim / 2) ('halves') or (2 i, 2 i + 1) ('adjacent')."""
    return RotaryConfig(num_q_heads, num_kv_heads, head_dim, DMC_FP32 if dtype in ("fp32", "float32") else DMC_BF16,
                        head_dim if rotary_dim is None else rotary_dim, PAIRS[pairs])


class DMCRotation:
    """The position rotation of packed queries and keys (forward + backward), for the inputs of DMCCausal.
    inv_freq float32 [rotary_dim / 2]: radians per position of every pair."""

    def __init__(self, cfg: RotaryConfig, inv_freq=None, device="cuda"):
        import torch
        self.cfg = cfg
        self._cfg_ref = byref(cfg)
        self.device = _cuda_device(device)
        fp32 = cfg.dtype == DMC_FP32
        self._call = _RowsCall(torch.float32 if fp32 else torch.bfloat16, self.device, cfg.head_dim, 4 if fp32 else 2)
        self._inv_freq, self._freq_span = None, (0, 0)
        if cfg.rotary_dim:
            _check("inv_freq", inv_freq, torch.float32, (cfg.rotary_dim // 2,), align16=False)
            _on_device(self.device, inv_freq=inv_freq)
            self._inv_freq, self._freq_span = inv_freq, (inv_freq.data_ptr(), inv_freq.data_ptr() + 2 * cfg.rotary_dim)

    inv_freq = property(lambda self: self._inv_freq)

    def _quick(self, q, k, positions, q_out, k_out):
        """Addresses and strides of the call's tensors, or None if the full check has to look at them."""
        call, cfg = self._call, self.cfg
        if not (isinstance(q, call.Tensor) and q.dim() == 3 and q.shape[0] > 0):
            return None
        T = q.shape[0]
        q_shape, k_shape = (T, cfg.num_q_heads, cfg.head_dim), (T, cfg.num_kv_heads, cfg.head_dim)
        a, b, x, y = call.take(q, q_shape), call.take(k, k_shape), call.take(q_out, q_shape), call.take(k_out, k_shape)
        pos = call.flat(positions, call.i32, (T,))
        if a is None or b is None or x is None or y is None or pos is None:
            return None
        q0, q1, k0, k1, x0, x1, y0, y1 = a[0], a[3], b[0], b[3], x[0], x[3], y[0], y[3]
        p1, (f0, f1) = pos + 4 * T, self._freq_span
        if (x0 < q1 and q0 < x1 or x0 < k1 and k0 < x1 or x0 < p1 and pos < x1 or x0 < f1 and f0 < x1 or y0 < q1 and q0 < y1
                or y0 < k1 and k0 < y1 or y0 < p1 and pos < y1 or y0 < f1 and f0 < y1 or y0 < x1 and x0 < y1):
            return None
        return T, q0, k0, pos, x0, y0, call.strides(a[1], a[2], b[1], b[2], x[1], x[2], y[1], y[2])

    def _rotate(self, q, k, positions, q_out, k_out, inverse, stream):
        q_out = _new_like("q", q) if q_out is None else q_out
        k_out = _new_like("k", k) if k_out is None else k_out
        args = self._quick(q, k, positions, q_out, k_out)
        if args is None:
            check_rotary_args(self.cfg, self.device, q, k, positions, self.inv_freq, q_out, k_out)
            (q0, k0, x0, y0), st = _packed_args(q, k, q_out, k_out)
            args = q.shape[0], q0, k0, positions.data_ptr(), x0, y0, st
        T, q0, k0, pos, x0, y0, st = args
        check(lib.dmc_rotate(self._cfg_ref, q0, st, k0, byref(st, 16), pos, self._freq_span[0], T, inverse, x0, byref(st, 32), y0,
                             byref(st, 48), _stream(stream, self.device)))
        return q_out, k_out

    def forward(self, q, k, positions, q_out=None, k_out=None, stream=None):
        """(q_out [T, Hq, d], k_out [T, Hkv, d]): q and k turned by positions int32 [T]; q_out may be q
        itself, k_out k."""
        return self._rotate(q, k, positions, q_out, k_out, 0, stream)

    def backward(self, dq_out, dk_out, positions, dq=None, dk=None, stream=None):
        """(dq, dk): gradients with respect to q and k, given those with respect to q_out and k_out."""
        return self._rotate(dq_out, dk_out, positions, dq, dk, 1, stream)


def make_full_config(batch, num_q_heads, num_kv_heads, head_dim, dtype="bf16", page_size=32, max_pages=128, num_pages=None,
                     rotary_dim=0, pairs="halves") -> FullConfig:
    """A dmc_full_config: rows of up to max_pages * page_size tokens; num_pages defaults to room for every row at
    capacity.  rotary_dim elements of every head are turned by append (0: keys and queries are stored as they are)."""
    return FullConfig(batch, num_q_heads, num_kv_heads, head_dim, DMC_FP32 if dtype in ("fp32", "float32") else DMC_BF16,
                      page_size, max_pages, batch * max_pages if num_pages is None else num_pages, rotary_dim, PAIRS[pairs])


class DMCFull:
    """Paged caches of layers that keep every token, with the workspace for attention of up to max_tokens new tokens
    (default: one per row), at most max_chunk in a row; append needs none, and is not bound by it.  The program owns
    what a scheduler decides and writes it in place:

    - page_table, int32 [batch, max_pages]: the pages of every row, shared by the layers; -1 (no page: calls that need
      it find and flag it) until the program writes it;
    - lengths, int32 [batch]: the tokens that every row holds before a call (negative: row not in use); the
      program adds the new ones once all layers have appended and attended;
    - k_pages, v_pages [num_layers, num_pages, Hkv, page_size, d], to copy whole pages in or out.

    Calls of attend share the object's workspace: those that may run at the same time, on two streams, need objects
    of their own.  A new object is ready for calls on any stream (the constructor waits for its own; one made while a
    graph is captured belongs to that graph)."""

    def __init__(self, cfg: FullConfig, max_tokens=None, max_chunk=1, inv_freq=None, num_layers=1, device="cuda"):
        import torch
        self.cfg, self.num_layers = cfg, num_layers
        self._cfg_ref = byref(cfg)
        self.device = _cuda_device(device)
        self.dtype = cache_dtype(cfg)
        self.max_tokens = cfg.batch if max_tokens is None else max_tokens
        self.max_chunk = max_chunk
        n = lib.dmc_full_workspace_bytes(self._cfg_ref, self.max_tokens, max_chunk)
        if n == 0:
            raise DMCError(DMC_ERR_INVALID_ARG, last_error())
        if num_layers < 1:
            _fail("num_layers must be >= 1")
        if cfg.rotary_dim:
            _check("inv_freq", inv_freq, torch.float32, (cfg.rotary_dim // 2,), align16=False)
            _on_device(self.device, inv_freq=inv_freq)
        # pools, page table, lengths and flags in one allocation: one range to keep the calls' tensors apart from
        dev, es = self.device, 4 if cfg.dtype == DMC_FP32 else 2
        self._layer_bytes = cfg.num_pages * cfg.num_kv_heads * cfg.page_size * cfg.head_dim * es
        pools = num_layers * self._layer_bytes
        sizes = [pools, pools, 4 * cfg.batch * cfg.max_pages, 4 * cfg.batch, 4]
        starts = [0]
        for n_bytes in sizes:
            starts.append(starts[-1] + (n_bytes + 255) // 256 * 256)
        self._buffer = torch.empty(starts[-1] + 256, dtype=torch.uint8, device=dev)
        at = -self._buffer.data_ptr() % 256
        parts = [self._buffer[at + lo:at + lo + n_bytes] for lo, n_bytes in zip(starts, sizes)]
        shape = (num_layers, cfg.num_pages, cfg.num_kv_heads, cfg.page_size, cfg.head_dim)
        self._storage = dict(k_pages=parts[0].view(self.dtype).view(shape), v_pages=parts[1].view(self.dtype).view(shape),
                             page_table=parts[2].view(torch.int32).view(cfg.batch, cfg.max_pages),
                             lengths=parts[3].view(torch.int32), flags=parts[4].view(torch.int32))
        self._storage["page_table"].fill_(-1)   # (no page: rows that the program has not given pages yet share none)
        for name in ("lengths", "flags"):
            self._storage[name].zero_()
        self._kp, self._vp, self._table, self._lens, self._flags = (t.data_ptr() for t in self._storage.values())
        self._span = self._buffer.data_ptr(), self._buffer.data_ptr() + self._buffer.numel()
        self._freq_span = 0, 0
        if cfg.rotary_dim:
            self._storage["inv_freq"] = inv_freq
            self._freq_span = inv_freq.data_ptr(), inv_freq.data_ptr() + 2 * cfg.rotary_dim
        self.workspace = torch.empty(n + 256, dtype=torch.uint8, device=dev)
        at = -self.workspace.data_ptr() % 256
        self.workspace[at:at + DMC_FULL_COUNTER_BYTES].zero_()
        self._ws = c_void_p(self.workspace.data_ptr() + at)
        self._ws_bytes = n
        self._call = _RowsCall(self.dtype, dev, cfg.head_dim, es)
        self._cu_shape = (cfg.batch + 1,)
        # the fills above are done before any call, on whichever stream that comes; in a captured graph they come before
        # the graph's calls
        if dev.type == "cuda":
            with torch.cuda.device(dev):
                if not torch.cuda.is_current_stream_capturing():
                    torch.cuda.current_stream().synchronize()

    k_pages = property(lambda self: self._storage["k_pages"])
    v_pages = property(lambda self: self._storage["v_pages"])
    page_table = property(lambda self: self._storage["page_table"])
    lengths = property(lambda self: self._storage["lengths"])
    flags = property(lambda self: self._storage["flags"])

    def _pages(self, layer):
        if not 0 <= layer < self.num_layers:
            _fail(f"layer {layer} outside [0, {self.num_layers})")
        return self._kp + layer * self._layer_bytes, self._vp + layer * self._layer_bytes

    def _rows(self, t, cu_seqlens):
        """(tokens, address of the boundaries or 0) of a call, or None if the full check has to look at them."""
        call = self._call
        if not (isinstance(t, call.Tensor) and t.dim() == 3):
            return None
        T = t.shape[0]
        if T == 0:
            return None
        if cu_seqlens is None:
            return (T, 0) if T == self.cfg.batch else None
        cu = call.flat(cu_seqlens, call.i32, self._cu_shape)
        return None if cu is None else (T, cu)

    def _quick_append(self, k, v, q, q_out, cu_seqlens):
        rows = self._rows(k, cu_seqlens)
        if rows is None:
            return None
        (T, cu), call, cfg, (o0, o1) = rows, self._call, self.cfg, self._span
        shape = T, cfg.num_kv_heads, cfg.head_dim
        a, b = call.take(k, shape), call.take(v, shape)
        if a is None or b is None:
            return None
        k0, k1, v0, v1, c1 = a[0], a[3], b[0], b[3], cu + 4 * cfg.batch + 4
        if o0 < k1 and k0 < o1 or o0 < v1 and v0 < o1 or o0 < c1 and cu < o1:
            return None
        if q is None:
            return (T, cu or None, k0, v0, None, None, call.strides(a[1], a[2], b[1], b[2])) if q_out is None else None
        shape = T, cfg.num_q_heads, cfg.head_dim
        c, x = call.take(q, shape), call.take(q_out, shape)
        if c is None or x is None:
            return None
        q0, q1, x0, x1, (f0, f1) = c[0], c[3], x[0], x[3], self._freq_span
        if (o0 < q1 and q0 < o1 or o0 < x1 and x0 < o1 or x0 < k1 and k0 < x1 or x0 < v1 and v0 < x1 or x0 < q1 and q0 < x1
                or x0 < c1 and cu < x1 or x0 < f1 and f0 < x1):
            return None
        return T, cu or None, k0, v0, q0, x0, call.strides(a[1], a[2], b[1], b[2], c[1], c[2], x[1], x[2])

    def _quick_attend(self, q, out, lse, cu_seqlens):
        rows = self._rows(q, cu_seqlens)
        if rows is None:
            return None
        (T, cu), call, cfg, (o0, o1) = rows, self._call, self.cfg, self._span
        Hq = cfg.num_q_heads
        shape = T, Hq, cfg.head_dim
        a, x, l0 = call.take(q, shape), call.take(out, shape), call.flat(lse, call.f32, (T, Hq))
        if a is None or x is None or l0 is None:
            return None
        q0, q1, x0, x1, l1, c1, (f0, f1) = a[0], a[3], x[0], x[3], l0 + 4 * T * Hq, cu + 4 * cfg.batch + 4, self._freq_span
        if (x0 < q1 and q0 < x1 or x0 < o1 and o0 < x1 or x0 < l1 and l0 < x1 or x0 < c1 and cu < x1 or l0 < q1 and q0 < l1
                or l0 < o1 and o0 < l1 or l0 < c1 and cu < l1 or x0 < f1 and f0 < x1 or l0 < f1 and f0 < l1):
            return None
        return T, cu or None, q0, x0, l0, call.strides(a[1], a[2], x[1], x[2])

    def append(self, layer, k, v, q=None, q_out=None, cu_seqlens=None, stream=None):
        """Append new tokens' keys, turned by their positions, and values [T, Hkv, d] to the layer's pages: one per
        row, or with cu_seqlens int32 [batch + 1] row b's being the tokens cu_seqlens[b] .. cu_seqlens[b + 1] - 1.
        With q [T, Hq, d], returns q_out, the queries turned likewise (q_out may be q itself)."""
        if q is not None and q_out is None:
            q_out = _new_like("q", q)
        kp, vp = self._pages(layer)
        args = self._quick_append(k, v, q, q_out, cu_seqlens)
        if args is None:
            check_full_append_args(self.cfg, self.device, self._storage, k, v, q, q_out, cu_seqlens)
            ptrs, st = _packed_args(k, v) if q is None else _packed_args(k, v, q, q_out)
            args = (k.shape[0], None if cu_seqlens is None else cu_seqlens.data_ptr(), *ptrs[:2],
                    *(ptrs[2:] if q is not None else (None, None)), st)
        T, cu, k0, v0, q0, x0, st = args
        check(lib.dmc_full_append(self._cfg_ref, k0, st, v0, byref(st, 16), q0, byref(st, 32) if q0 else None,
                                  self._freq_span[0], cu, T, self._lens, self._table, kp, vp, x0,
                                  byref(st, 48) if q0 else None, self._flags, _stream(stream, self.device)))
        return q_out

    def attend(self, layer, q, cu_seqlens=None, max_chunk=None, out=None, lse=None, stream=None):
        """Attention of new tokens' queries [T, Hq, d], whose keys and values are in the pages already, over their
        rows' caches up to themselves; at most max_chunk (default: the object's) of them in a row.  Returns (out
        [T, Hq, d], lse [T, Hq] fp32); rows of tokens outside every chunk stay as they are."""
        import torch
        if not isinstance(q, torch.Tensor):
            _fail("q must be a torch.Tensor")
        if out is None:
            out = torch_empty_like(q)
        if lse is None:
            lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
        kp, vp = self._pages(layer)
        max_chunk = 1 if cu_seqlens is None else self.max_chunk if max_chunk is None else max_chunk
        if max_chunk > self.max_chunk:
            _fail(f"chunks of {max_chunk} tokens, the workspace holds {self.max_chunk}")
        args = self._quick_attend(q, out, lse, cu_seqlens)
        if args is None:
            check_full_attend_args(self.cfg, self.device, self._storage, q, out, lse, cu_seqlens)
            (q0, x0), st = _packed_args(q, out)
            args = q.shape[0], None if cu_seqlens is None else cu_seqlens.data_ptr(), q0, x0, lse.data_ptr(), st
        T, cu, q0, x0, l0, st = args
        if T > self.max_tokens:
            _fail(f"{T} tokens, the workspace holds {self.max_tokens}")
        check(lib.dmc_full_attend(self._cfg_ref, q0, st, cu, T, max_chunk, self._lens, self._table, kp, vp, x0,
                                  byref(st, 16), l0, self._flags, self._ws, self._ws_bytes, _stream(stream, self.device)))
        return out, lse

    def check(self):
        """Raise what the calls so far have found on the device (waits for them)."""
        found = int(self.flags.item())
        if found & DMC_FLAG_ROW_FULL:
            raise DMCError(DMC_ERR_CAPACITY, f"a row is full (flags 0x{found:x})")
        if found:
            _fail(f"boundaries or lengths out of range, or page ids outside the pool (flags 0x{found:x})")
