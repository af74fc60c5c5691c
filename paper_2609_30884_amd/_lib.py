"""ctypes binding of libcrf.so (include/crf.h).

Argument marshalling only: every step of the recomputation runs inside the
library's HIP kernels.  Tensors are torch device tensors (ROCm); their device
pointers and the current HIP stream are handed to the C ABI.  There is no
fallback: if the library is missing or fails to load, every call raises.
"""
from __future__ import annotations

import ctypes
import os
import sys
from typing import Dict, Iterable, List, Mapping, Optional, Sequence, Tuple

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("CRF_LIBRARY") or os.path.join(HERE, "libcrf.so")

TARGETS = ("q", "k", "v", "o", "gate", "up", "down")
NUM_TARGETS = 7

CRF_F32, CRF_BF16 = 0, 1
KERNEL_KINDS = ("norm", "lora_down", "gemm_qkv", "attn", "gemm_o", "gemm_gateup", "gemm_down", "drift", "other")

STATUS = {0: "CRF_OK", 1: "CRF_ERR_INVALID_ARG", 2: "CRF_ERR_SHAPE", 3: "CRF_ERR_RANGE", 4: "CRF_ERR_UNSUPPORTED",
          5: "CRF_ERR_WORKSPACE", 6: "CRF_ERR_HIP", 7: "CRF_ERR_DEVICE"}


class CrfError(RuntimeError):
    def __init__(self, status: int, message: str):
        self.status = status
        super().__init__(f"{STATUS.get(status, status)}: {message}")


# ----------------------------------------------------------------------------- structs

class ModelDims(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("d_model", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("d_ffn", ctypes.c_int32),
                ("rms_eps", ctypes.c_float), ("rope_theta", ctypes.c_float), ("dtype", ctypes.c_int32)]


class LayerWeights(ctypes.Structure):
    _fields_ = [("attn_norm", ctypes.c_void_p), ("mlp_norm", ctypes.c_void_p),
                ("w", ctypes.c_void_p * NUM_TARGETS),
                ("bias_q", ctypes.c_void_p), ("bias_k", ctypes.c_void_p), ("bias_v", ctypes.c_void_p)]


class LoraLayer(ctypes.Structure):
    _fields_ = [("rank", ctypes.c_int32), ("scale", ctypes.c_float),
                ("A", ctypes.c_void_p * NUM_TARGETS), ("B", ctypes.c_void_p * NUM_TARGETS)]


class KVCache(ctypes.Structure):
    _fields_ = [("k_pool", ctypes.c_void_p), ("v_pool", ctypes.c_void_p),
                ("layer_stride", ctypes.c_int64), ("page_stride", ctypes.c_int64),
                ("block_table", ctypes.c_void_p),
                ("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("n_tokens", ctypes.c_int32)]


class WindowItem(ctypes.Structure):
    _fields_ = [("hidden_at_boundary", ctypes.c_void_p), ("lora", ctypes.POINTER(LoraLayer)),
                ("l0", ctypes.c_int32), ("h", ctypes.c_int32), ("kv", KVCache),
                ("hidden_out", ctypes.c_void_p)]


class PagePool(ctypes.Structure):
    _fields_ = [("k_pool", ctypes.c_void_p), ("v_pool", ctypes.c_void_p),
                ("layer_stride", ctypes.c_int64), ("page_stride", ctypes.c_int64),
                ("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32)]


class SeqBatch(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("n_rows", ctypes.c_int32), ("max_new", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("table_stride", ctypes.c_int64),
                ("row_start", ctypes.c_void_p), ("length", ctypes.c_void_p), ("block_tables", ctypes.c_void_p)]


class Rope(ctypes.Structure):
    _fields_ = [("layout", ctypes.c_int32), ("rotary_dim", ctypes.c_int32), ("mscale", ctypes.c_float),
                ("freq", ctypes.c_double * 64)]


class RopeScaling(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("factor", ctypes.c_double), ("original_len", ctypes.c_double),
                ("low_turns", ctypes.c_double), ("high_turns", ctypes.c_double), ("mscale", ctypes.c_double)]


class PageMap(ctypes.Structure):
    _fields_ = [("refs", ctypes.c_void_p), ("block_tables", ctypes.c_void_p), ("lengths", ctypes.c_void_p),
                ("table_stride", ctypes.c_int64), ("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("n_seqs", ctypes.c_int32), ("max_pages", ctypes.c_int32)]


# ----------------------------------------------------------------------------- loading

_LIB: Optional[ctypes.CDLL] = None

EXPORTS = ("crf_status_string", "crf_abi_version", "crf_context_create", "crf_context_destroy", "crf_last_error",
           "crf_validate_dims", "crf_validate_window", "crf_recompute_window", "crf_recompute_window_batched",
           "crf_layer_drift", "crf_context_device_errors", "crf_context_set_timing", "crf_context_set_timing_classes",
           "crf_context_read_timing",
           "crf_device_info", "crf_decode_logits", "crf_layer_drift_noalloc", "crf_rope_init", "crf_rope_append",
           "crf_paged_attention", "crf_pages_copy", "crf_pages_fork", "crf_pages_extend", "crf_pages_free",
           "crf_pages_compact")


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libcrf.so (once).  Raises if it is missing: there is no fallback."""
    global _LIB
    if _LIB is not None:
        return _LIB
    if not os.path.exists(path):
        raise ImportError(f"libcrf.so not built at {path}; run `python -m paper_2609_30884_amd.build`")
    lib = ctypes.CDLL(path)
    P, I32, VP = ctypes.POINTER, ctypes.c_int32, ctypes.c_void_p
    lib.crf_status_string.restype = ctypes.c_char_p
    lib.crf_status_string.argtypes = [I32]
    lib.crf_abi_version.restype = I32
    lib.crf_last_error.restype = ctypes.c_char_p
    lib.crf_last_error.argtypes = [VP]
    lib.crf_context_create.restype = I32
    lib.crf_context_create.argtypes = [P(ModelDims), I32, I32, P(VP)]
    lib.crf_context_destroy.restype = None
    lib.crf_context_destroy.argtypes = [VP]
    lib.crf_validate_dims.restype = I32
    lib.crf_validate_dims.argtypes = [P(ModelDims)]
    lib.crf_validate_window.restype = I32
    lib.crf_validate_window.argtypes = [P(ModelDims), I32, I32, P(KVCache)]
    lib.crf_recompute_window.restype = I32
    lib.crf_recompute_window.argtypes = [VP, P(ModelDims), VP, P(LayerWeights), P(LoraLayer), I32, I32, P(KVCache),
                                         VP, VP]
    lib.crf_recompute_window_batched.restype = I32
    lib.crf_recompute_window_batched.argtypes = [VP, P(ModelDims), P(LayerWeights), I32, P(WindowItem), VP]
    lib.crf_layer_drift.restype = I32
    lib.crf_layer_drift.argtypes = [VP, P(ModelDims), P(LoraLayer), I32, P(P(LoraLayer)), P(I32), VP, I32, VP, VP,
                                    VP, VP]
    lib.crf_layer_drift_noalloc.restype = I32
    lib.crf_layer_drift_noalloc.argtypes = [P(ModelDims), P(LoraLayer), I32, P(P(LoraLayer)), P(I32), VP, I32, VP,
                                            VP, VP, VP]
    lib.crf_context_device_errors.restype = I32
    lib.crf_context_device_errors.argtypes = [VP, P(I32)]
    lib.crf_context_set_timing.restype = I32
    lib.crf_context_set_timing.argtypes = [VP, I32]
    lib.crf_context_set_timing_classes.restype = I32
    lib.crf_context_set_timing_classes.argtypes = [VP, ctypes.c_uint32]
    lib.crf_context_read_timing.restype = I32
    lib.crf_context_read_timing.argtypes = [VP, P(ctypes.c_float), P(I32), I32]
    lib.crf_decode_logits.restype = I32
    lib.crf_decode_logits.argtypes = [VP, P(ModelDims), VP, I32, P(LayerWeights), P(LoraLayer), P(KVCache), VP, VP,
                                      I32, VP, VP]
    lib.crf_device_info.restype = I32
    lib.crf_device_info.argtypes = [I32, P(I32), P(I32), ctypes.c_char_p, I32]
    I64 = ctypes.c_int64
    for name, args in (
            ("rope_init", [P(Rope), I32, I32, ctypes.c_double, P(RopeScaling)]),
            ("rope_append", [VP, P(Rope), P(SeqBatch), VP, VP, I64, VP, I64, VP, I64, VP, I64, P(PagePool), I32, VP]),
            ("paged_attention", [VP, P(SeqBatch), VP, I64, P(PagePool), I32, ctypes.c_float, I32, VP, I64, VP, VP]),
            ("pages_copy", [VP, P(PagePool), I32, P(PagePool), I32, I32, I32, VP, VP, VP]),
            ("pages_fork", [VP, P(PagePool), P(PageMap), I32, VP, VP, VP]),
            ("pages_extend", [VP, P(PageMap), VP, VP]),
            ("pages_free", [VP, P(PageMap), I32, VP, VP]),
            ("pages_compact", [VP, P(PagePool), P(PageMap), P(PageMap), VP, VP, VP])):
        fn = getattr(lib, "crf_" + name)
        fn.restype, fn.argtypes = I32, args
    _LIB = lib
    return lib


def _err(lib, ctx, st: int):
    if st != 0:
        msg = lib.crf_last_error(ctx)
        raise CrfError(st, msg.decode() if msg else "")


# ----------------------------------------------------------------------------- marshalling

def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return int(t.data_ptr())


def make_dims(n_layers, d_model, n_q_heads, n_kv_heads, head_dim, d_ffn, rms_eps=1e-6, rope_theta=1e6,
              dtype="bf16") -> ModelDims:
    return ModelDims(n_layers, d_model, n_q_heads, n_kv_heads, head_dim, d_ffn, rms_eps, rope_theta,
                     CRF_BF16 if dtype == "bf16" else CRF_F32)


def layer_weights_array(layers: Sequence[Optional[Mapping]]) -> ctypes.Array:
    """layers[l]: {"attn_norm", "mlp_norm", "w_q" ... "w_down", optional "bias_q/k/v"} of
    device tensors, or None for layers outside every window."""
    arr = (LayerWeights * len(layers))()
    for l, w in enumerate(layers):
        if w is None:
            continue
        arr[l].attn_norm = _ptr(w["attn_norm"])
        arr[l].mlp_norm = _ptr(w["mlp_norm"])
        for i, t in enumerate(TARGETS):
            arr[l].w[i] = _ptr(w["w_" + t])
        arr[l].bias_q = _ptr(w.get("bias_q"))
        arr[l].bias_k = _ptr(w.get("bias_k"))
        arr[l].bias_v = _ptr(w.get("bias_v"))
    return arr


def lora_array(layers: Optional[Sequence[Optional[Mapping]]], n_layers: int) -> Optional[ctypes.Array]:
    """layers[l]: {"rank": r, "scale": s, "targets": {name: (A [r, d_in], B [d_out, r])}} or None."""
    if layers is None:
        return None
    arr = (LoraLayer * n_layers)()
    for l, ll in enumerate(layers):
        if not ll:
            continue
        arr[l].rank = int(ll["rank"])
        arr[l].scale = float(ll.get("scale", 1.0))
        for i, t in enumerate(TARGETS):
            ab = ll["targets"].get(t)
            if ab is not None:
                arr[l].A[i] = _ptr(ab[0])
                arr[l].B[i] = _ptr(ab[1])
    return arr


def kv_cache(k_pool, v_pool, block_table, n_tokens: int, page_size: int) -> KVCache:
    """k_pool/v_pool: [n_layers, n_pages, n_kv_heads, page_size, head_dim] device tensors."""
    n_pages = int(k_pool.shape[1])
    return KVCache(_ptr(k_pool), _ptr(v_pool), int(k_pool.stride(0)), int(k_pool.stride(1)), _ptr(block_table),
                   n_pages, int(page_size), int(n_tokens))


def _stream(stream) -> Optional[int]:
    if stream is None:
        # (the pointer itself: a torch.cuda.Stream object around it takes 3 us to make)
        import torch
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    if isinstance(stream, int):
        return stream
    return int(stream.cuda_stream)


# ----------------------------------------------------------------------------- API

class Context:
    """crf_context: workspace for windows of up to max_tokens tokens."""

    def __init__(self, dims: ModelDims, max_tokens: int, max_lora_rank: int = 16):
        self.lib = load()
        self.dims = dims
        h = ctypes.c_void_p()
        _err(self.lib, None, self.lib.crf_context_create(ctypes.byref(dims), int(max_tokens), int(max_lora_rank),
                                                          ctypes.byref(h)))
        self.handle = h
        # (a program that has not imported torch, which brings a HIP runtime of its own, gets along without it)
        self._device = sys.modules["torch"].cuda.current_device() if "torch" in sys.modules else None

    @property
    def device(self) -> int:
        """The device current when the context was made, for checks of the page-pool operators' tensors."""
        if self._device is None:
            import torch
            self._device = torch.cuda.current_device()
        return self._device

    def close(self):
        if getattr(self, "handle", None) and self.handle.value:
            self.lib.crf_context_destroy(self.handle)
            self.handle = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def device_errors(self) -> int:
        out = ctypes.c_int32()
        _err(self.lib, self.handle, self.lib.crf_context_device_errors(self.handle, ctypes.byref(out)))
        return int(out.value)

    def set_timing(self, on: bool, classes=None):
        """Event timing of every kernel class (on), of none, or of the named
        classes only (KERNEL_KINDS names)."""
        if classes is None:
            _err(self.lib, self.handle, self.lib.crf_context_set_timing(self.handle, 1 if on else 0))
            return
        mask = 0
        for name in classes if on else ():
            mask |= 1 << KERNEL_KINDS.index(name)
        _err(self.lib, self.handle, self.lib.crf_context_set_timing_classes(self.handle, mask))

    def read_timing(self) -> Dict[str, Tuple[float, int]]:
        n = len(KERNEL_KINDS)
        ms = (ctypes.c_float * n)()
        cnt = (ctypes.c_int32 * n)()
        _err(self.lib, self.handle, self.lib.crf_context_read_timing(self.handle, ms, cnt, n))
        return {k: (float(ms[i]), int(cnt[i])) for i, k in enumerate(KERNEL_KINDS)}


def device_info(device: int = 0) -> Dict[str, object]:
    """Compute-unit count, peak engine clock and architecture of a device."""
    lib = load()
    cu, mhz = ctypes.c_int32(), ctypes.c_int32()
    name = ctypes.create_string_buffer(64)
    _err(lib, None, lib.crf_device_info(device, ctypes.byref(cu), ctypes.byref(mhz), name, 64))
    return {"arch": name.value.decode(), "compute_units": int(cu.value), "max_sclk_mhz": int(mhz.value)}


def status_string(st: int) -> str:
    return load().crf_status_string(int(st)).decode()


def abi_version() -> int:
    return int(load().crf_abi_version())


def validate_dims(dims: ModelDims) -> int:
    return int(load().crf_validate_dims(ctypes.byref(dims)))


def validate_window(dims: ModelDims, l0: int, h: int, kv: KVCache) -> int:
    """Host-only check (no device needed); returns the status code."""
    return int(load().crf_validate_window(ctypes.byref(dims), int(l0), int(h), ctypes.byref(kv)))


def last_error(ctx: Optional[Context] = None) -> str:
    lib = load()
    return lib.crf_last_error(ctx.handle if ctx else None).decode()


def recompute_window(ctx: Context, dims: ModelDims, hidden_at_boundary, base_weights: ctypes.Array,
                     lora: Optional[ctypes.Array], l0: int, h: int, kv: KVCache, hidden_out=None, stream=None):
    """crf_recompute_window: refresh layers [l0, l0+h) of `kv` from H_{l0-1}."""
    lib = ctx.lib
    st = lib.crf_recompute_window(ctx.handle, ctypes.byref(dims), _ptr(hidden_at_boundary), base_weights,
                                  lora, int(l0), int(h), ctypes.byref(kv), _ptr(hidden_out), _stream(stream))
    _err(lib, ctx.handle, st)


def window_item(hidden_at_boundary, lora: Optional[ctypes.Array], l0: int, h: int, kv: KVCache,
                hidden_out=None) -> WindowItem:
    it = WindowItem()
    it.hidden_at_boundary = _ptr(hidden_at_boundary)
    it.lora = ctypes.cast(lora, ctypes.POINTER(LoraLayer)) if lora is not None else None
    it.l0, it.h, it.kv = int(l0), int(h), kv
    it.hidden_out = _ptr(hidden_out)
    return it


def recompute_window_batched(ctx: Context, dims: ModelDims, base_weights: ctypes.Array, items: Sequence[WindowItem],
                             stream=None):
    """crf_recompute_window_batched over independent stale caches."""
    arr = (WindowItem * len(items))(*items)
    st = ctx.lib.crf_recompute_window_batched(ctx.handle, ctypes.byref(dims), base_weights, len(items), arr,
                                              _stream(stream))
    _err(ctx.lib, ctx.handle, st)


def decode_logits(ctx: Context, dims: ModelDims, new_tokens, base_weights: ctypes.Array,
                  lora: Optional[ctypes.Array], kv: KVCache, final_norm, lm_head, logits_out, stream=None):
    """crf_decode_logits: first-step next-token logits of the last of new_tokens
    [n_new, d] over the cached prefix kv (kv.n_tokens tokens)."""
    lib = ctx.lib
    st = lib.crf_decode_logits(ctx.handle, ctypes.byref(dims), _ptr(new_tokens), int(new_tokens.shape[0]),
                               base_weights, lora, ctypes.byref(kv), _ptr(final_norm), _ptr(lm_head),
                               int(lm_head.shape[0]), _ptr(logits_out), _stream(stream))
    _err(lib, ctx.handle, st)


def layer_drift(ctx: Context, dims: ModelDims, current: ctypes.Array, versions: Sequence[ctypes.Array],
                anchor_version: Sequence[int], sensitivity, drift_out, risk_out, sq_partial_out=None,
                per_layer_only: bool = False, stream=None):
    """crf_layer_drift: d_l = ||theta_t - theta_anchor(l)||_2 and q_l = s_l d_l."""
    n_layers = dims.n_layers
    vp = (ctypes.POINTER(LoraLayer) * len(versions))(*[ctypes.cast(v, ctypes.POINTER(LoraLayer)) for v in versions])
    anc = (ctypes.c_int32 * n_layers)(*[int(a) for a in anchor_version])
    st = ctx.lib.crf_layer_drift(ctx.handle, ctypes.byref(dims), current, len(versions), vp, anc, _ptr(sensitivity),
                                 1 if per_layer_only else 0, _ptr(drift_out), _ptr(risk_out), _ptr(sq_partial_out),
                                 _stream(stream))
    _err(ctx.lib, ctx.handle, st)


def layer_drift_noalloc(dims: ModelDims, current: ctypes.Array, versions: Sequence[ctypes.Array],
                        anchor_version: Sequence[int], sensitivity, drift_out, risk_out, sq_partial_out=None,
                        per_layer_only: bool = False, stream=None):
    """crf_layer_drift_noalloc: crf_layer_drift without a context, in the library's fixed device scratch."""
    lib = load()
    n_layers = dims.n_layers
    vp = (ctypes.POINTER(LoraLayer) * len(versions))(*[ctypes.cast(v, ctypes.POINTER(LoraLayer)) for v in versions])
    anc = (ctypes.c_int32 * n_layers)(*[int(a) for a in anchor_version])
    st = lib.crf_layer_drift_noalloc(ctypes.byref(dims), current, len(versions), vp, anc, _ptr(sensitivity),
                                     1 if per_layer_only else 0, _ptr(drift_out), _ptr(risk_out),
                                     _ptr(sq_partial_out), _stream(stream))
    _err(lib, None, st)


# ----------------------------------------------------------------------------- many sequences in one cache

ROPE_LAYOUTS = ("half", "interleaved")
ROPE_SCALINGS = ("none", "linear", "base", "parts")


def _same_device(*tensors) -> int:
    """The device of a descriptor's tensors (-1: host memory, which no call takes)."""
    dev = tensors[0].get_device()
    if any(t.get_device() != dev for t in tensors):
        raise CrfError(1, "tensors of one descriptor lie on different devices")
    return dev


def _check_device(ctx: Context, descriptors, tensors):
    """Descriptors and tensors of a call lie on the context's device."""
    dev = ctx.device
    for d in descriptors:
        if d.device != dev:
            raise CrfError(1, f"tensors {'on the host' if d.device < 0 else f'of device {d.device}'}, context of device {dev}")
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise CrfError(1, f"a tensor {'on the host' if not t.is_cuda else f'of {t.device}'}, context of device {dev}")


def _int32(t, n: Optional[int], name: str):
    """A contiguous int32 device vector (of n values)."""
    import torch
    if t.dtype is not torch.int32 or t.dim() != 1 or (n is not None and t.shape[0] != n) or not t.is_contiguous():
        raise CrfError(2, f"{name} must be a contiguous int32 vector" + (f" of {n}" if n is not None else ""))
    return t


def _tables(t):
    import torch
    if t.dtype is not torch.int32 or t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1) or \
            (t.shape[0] > 1 and t.stride(0) < t.shape[1]):
        raise CrfError(2, "block tables must be int32 [sequences, entries], entries contiguous, rows that do not overlap")
    return t


def _storage(dims: ModelDims):
    """The torch type of the context's storage type."""
    import torch
    return torch.bfloat16 if dims.dtype == CRF_BF16 else torch.float32


def _head_rows(d: ModelDims, t, n_rows: int, heads: int, name: str):
    """Pointer and row stride of [rows, heads, head_dim] or [rows, heads * head_dim] whose rows are contiguous."""
    shape, stride, hd = t.shape, t.stride(), d.head_dim
    if t.dtype is not _storage(d):
        raise CrfError(1, f"{name} is {t.dtype}, the context's storage type differs")
    if len(shape) == 3:
        ok = shape[1] == heads and shape[2] == hd and (heads == 1 or stride[1] == hd)
    else:
        ok = len(shape) == 2 and shape[1] == heads * hd
    if not ok or shape[0] != n_rows or stride[-1] != 1:
        raise CrfError(2, f"{name} {tuple(shape)} (strides {stride}) is not {n_rows} rows of {heads} heads of {hd}")
    return t.data_ptr(), stride[0] if n_rows > 1 else heads * hd


def page_pool(k_pool, v_pool, page_size: int) -> PagePool:
    """k_pool, v_pool: [n_layers, n_pages, n_kv_heads, page_size, head_dim] device tensors."""
    if k_pool.dtype is not v_pool.dtype or k_pool.shape != v_pool.shape or k_pool.stride() != v_pool.stride() or \
            k_pool.dim() != 5 or (k_pool.numel() and not k_pool[0, 0].is_contiguous()) or k_pool.shape[3] != page_size:
        raise CrfError(2, "pools must be two like tensors [layers, pages, kv heads, page_size, head_dim], pages contiguous")
    p = PagePool(k_pool.data_ptr(), v_pool.data_ptr(), k_pool.stride(0), k_pool.stride(1), k_pool.shape[1], page_size)
    p.tensors, p.device = (k_pool, v_pool), _same_device(k_pool, v_pool)
    p.layers, p.heads, p.head_dim = k_pool.shape[0], k_pool.shape[2], k_pool.shape[4]
    return p


def _check_pool(d: ModelDims, pool: PagePool, layers: int):
    """The pool's storage type and heads are the context's, and it has that many layers."""
    if pool.tensors[0].dtype is not _storage(d):
        raise CrfError(1, f"the pool is {pool.tensors[0].dtype}, the context's storage type differs")
    if pool.heads != d.n_kv_heads or pool.head_dim != d.head_dim:
        raise CrfError(2, f"the pool has {pool.heads} heads of {pool.head_dim}, the context {d.n_kv_heads} of {d.head_dim}")
    if not 0 <= layers <= pool.layers:
        raise CrfError(3, f"{layers} layers of a pool of {pool.layers}")


def seq_batch(row_start, length, block_tables, n_rows: int, max_new: int = 0) -> SeqBatch:
    """row_start [S + 1], length [S], block_tables [S, pages]: int32 device tensors; n_rows: rows of the
    calls' tensors; max_new: the most new tokens of a sequence (0: n_rows).  max_new and the tables' width are what
    paged_attention chooses its kernel by: a batch of single tokens should pass max_new=1."""
    t = _tables(block_tables)
    n = t.shape[0]
    b = SeqBatch(n, int(n_rows), int(max_new), t.shape[1], t.stride(0) if n > 1 else t.shape[1],
                 _int32(row_start, n + 1, "row_start").data_ptr(), _int32(length, n, "length").data_ptr(), t.data_ptr())
    b.tensors, b.device = (row_start, length, block_tables), _same_device(row_start, length, block_tables)
    return b


def rope(rotary_dim: int, theta: float, layout: str = "half", scaling: str = "none", factor: float = 1.0,
         original_len: float = 0, low_turns: float = 0, high_turns: float = 0, mscale: float = 0) -> Rope:
    """crf_rope_init: the rotary plan of a model (host only)."""
    if layout not in ROPE_LAYOUTS or scaling not in ROPE_SCALINGS:
        raise CrfError(1, f"layout {layout!r} or scaling {scaling!r} unknown")
    lib, out = load(), Rope()
    sc = RopeScaling(ROPE_SCALINGS.index(scaling), factor, original_len, low_turns, high_turns, mscale)
    _err(lib, None, lib.crf_rope_init(ctypes.byref(out), ROPE_LAYOUTS.index(layout), int(rotary_dim), theta,
                                      ctypes.byref(sc)))
    return out


def rope_append(ctx: Context, rope: Rope, batch: SeqBatch, q, k, v, pool: PagePool, layer: int, q_out=None,
                positions=None, stream=None):
    """crf_rope_append: q rotated into q_out (both None: keys and values only), k rotated and v into the pages."""
    d, n = ctx.dims, batch.n_rows
    _check_pool(ctx.dims, pool, layer + 1)
    qp, qs = _head_rows(d, q, n, d.n_q_heads, "q") if q is not None else (None, 0)
    op, os_ = _head_rows(d, q_out, n, d.n_q_heads, "q_out") if q_out is not None else (None, 0)
    kp, ks = _head_rows(d, k, n, d.n_kv_heads, "k")
    vp, vs = _head_rows(d, v, n, d.n_kv_heads, "v")
    pp = _int32(positions, n, "positions").data_ptr() if positions is not None else None
    _check_device(ctx, (batch, pool), (q, k, v, q_out, positions))
    st = ctx.lib.crf_rope_append(ctx.handle, rope, batch, pp, qp, qs, kp, ks, vp, vs, op, os_, pool, layer,
                                 _stream(stream))
    _err(ctx.lib, ctx.handle, st)


def paged_attention(ctx: Context, batch: SeqBatch, q, pool: PagePool, layer: int, out, lse=None, scale: float = 0.0,
                    window: int = 0, stream=None):
    """crf_paged_attention: out [rows, heads, head_dim] (and lse, fp32 [rows, heads]) of the new tokens' queries q."""
    d, n = ctx.dims, batch.n_rows
    _check_pool(ctx.dims, pool, layer + 1)
    qp, qs = _head_rows(d, q, n, d.n_q_heads, "q")
    op, os_ = _head_rows(d, out, n, d.n_q_heads, "out")
    if lse is not None:
        if not lse.is_floating_point() or lse.element_size() != 4 or lse.shape != (n, d.n_q_heads) or not lse.is_contiguous():
            raise CrfError(2, f"lse must be contiguous float32 [{n}, {d.n_q_heads}]")
    _check_device(ctx, (batch, pool), (q, out, lse))
    # (ctypes would take an int's low 32 bits; past the longest sequence a window is none)
    st = ctx.lib.crf_paged_attention(ctx.handle, batch, qp, qs, pool, layer, scale, min(window, 0x7fffffff), op, os_,
                                     _ptr(lse), _stream(stream))
    _err(ctx.lib, ctx.handle, st)


def pages_copy(ctx: Context, pool: PagePool, src, dst, l0: int = 0, h: Optional[int] = None,
               to: Optional[PagePool] = None, to_l0: Optional[int] = None, stream=None):
    """crf_pages_copy: pages src of `pool` to pages dst of `to` (None: the same pool), layers [l0, l0 + h)."""
    h = pool.tensors[0].shape[0] - l0 if h is None else h
    to, to_l0 = pool if to is None else to, l0 if to_l0 is None else to_l0
    _check_pool(ctx.dims, pool, l0 + h)
    _check_pool(ctx.dims, to, to_l0 + h)
    n = src.numel()
    sp, dp = _int32(src, n, "src").data_ptr(), _int32(dst, n, "dst").data_ptr()
    _check_device(ctx, (pool, to), (src, dst))
    st = ctx.lib.crf_pages_copy(ctx.handle, pool, l0, to, to_l0, h, n, sp, dp, _stream(stream))
    _err(ctx.lib, ctx.handle, st)


def page_map(refs, block_tables, lengths, page_size: int) -> PageMap:
    """refs [pages], block_tables [S, pages of a sequence], lengths [S]: int32 device tensors."""
    t = _tables(block_tables)
    n = t.shape[0]
    m = PageMap(_int32(refs, None, "refs").data_ptr(), t.data_ptr(), _int32(lengths, n, "lengths").data_ptr(),
                t.stride(0) if n > 1 else t.shape[1], refs.numel(), int(page_size), n, t.shape[1])
    m.tensors, m.device = (refs, block_tables, lengths), _same_device(refs, block_tables, lengths)
    return m


def pages_fork(ctx: Context, pool: PagePool, map: PageMap, parents, children, stream=None):
    """crf_pages_fork: children[i] becomes a copy of parents[i] that shares its full pages."""
    _check_pool(ctx.dims, pool, ctx.dims.n_layers)
    n = parents.numel()
    pp, cp = _int32(parents, n, "parents").data_ptr(), _int32(children, n, "children").data_ptr()
    _check_device(ctx, (pool, map), (parents, children))
    st = ctx.lib.crf_pages_fork(ctx.handle, pool, map, n, pp, cp, _stream(stream))
    _err(ctx.lib, ctx.handle, st)


def pages_extend(ctx: Context, map: PageMap, n_new, stream=None):
    """crf_pages_extend: every sequence s grows by n_new[s] tokens."""
    gp = _int32(n_new, map.n_seqs, "n_new").data_ptr()
    _check_device(ctx, (map,), (n_new,))
    st = ctx.lib.crf_pages_extend(ctx.handle, map, gp, _stream(stream))
    _err(ctx.lib, ctx.handle, st)


def pages_free(ctx: Context, map: PageMap, seqs, stream=None):
    """crf_pages_free: the sequences end."""
    n = seqs.numel()
    sp = _int32(seqs, n, "seqs").data_ptr()
    _check_device(ctx, (map,), (seqs,))
    st = ctx.lib.crf_pages_free(ctx.handle, map, n, sp, _stream(stream))
    _err(ctx.lib, ctx.handle, st)


def pages_compact(ctx: Context, pool: PagePool, map: PageMap, map_out: PageMap, remap, counts, stream=None):
    """crf_pages_compact: the pages in use move to the front of the pool; map_out may be map."""
    _check_pool(ctx.dims, pool, ctx.dims.n_layers)
    rp, cp = _int32(remap, map.n_pages, "remap").data_ptr(), _int32(counts, 2, "counts").data_ptr()
    _check_device(ctx, (pool, map, map_out), (remap, counts))
    st = ctx.lib.crf_pages_compact(ctx.handle, pool, map, map_out, rp, cp, _stream(stream))
    _err(ctx.lib, ctx.handle, st)
