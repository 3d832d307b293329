"""ctypes binding of libbaklava.so: argument marshalling only.

Function names and argument order follow include/baklava.h.  Device buffers are
torch tensors (torch is used for device memory and streams, nothing else); every
step of the method runs inside the library.  If the library is missing the
first call raises: there is no other path.
"""
import ctypes
import functools
import os
import struct
from ctypes import POINTER, c_char_p, c_double, c_float, c_int32, c_int64, c_size_t, c_uint32, c_void_p

import numpy as np
import torch

OK = 0
FLAG_NO_APPEND, FLAG_NO_SCORE, FLAG_NO_EVICT = 1, 2, 4
FLAG_OVERLAP_PREV = 8
FLAG_ROW_QUOTIENT = 16
FLAG_TEST_STALL = 256
SCOPE_LAYER, SCOPE_MODEL = 0, 1
STATUS_OVERFLOW, STATUS_BAD_STATE, STATUS_TIMEOUT = 1, 2, 4
KV_BF16, KV_FP8_E4M3, KV_INT4 = 0, 1, 2
ROPE_INTERLEAVED = 1
MAX_TREE = 64
PROB_F32, PROB_BF16 = 0, 1
VERIFY_DISTINCT = 1

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libbaklava.so")
_lib = None


class BaklavaError(RuntimeError):
    def __init__(self, code, what):
        super().__init__("%s failed: %s (%d)" % (what, strerror(code), code))
        self.code = code


class Shape(ctypes.Structure):
    _fields_ = [(n, c_int32) for n in ("L", "Hq", "Hkv", "D", "page", "n_sink", "recent_num", "recent_den")]

    @property
    def g(self):
        return self.Hq // self.Hkv


class CacheStruct(ctypes.Structure):
    _fields_ = [("k_slab", c_void_p), ("v_slab", c_void_p), ("pos", c_void_p), ("score", c_void_p),
                ("len", c_void_p), ("free_slot", c_void_p), ("cap", c_void_p), ("slab_off", c_void_p),
                ("seq_stride_tokens", c_int64), ("B", c_int32), ("status", c_void_p), ("kv_dtype", c_int32),
                ("kv_scale", c_void_p), ("row_scale", c_void_p)]


class Strides(ctypes.Structure):
    _fields_ = [("seq", c_int64), ("head", c_int64), ("token", c_int64)]


class AllocParams(ctypes.Structure):
    _fields_ = [("t", c_double), ("r_num", c_int32), ("r_den", c_int32), ("scope", c_int32),
                ("min_tokens", c_int32), ("max_tokens", c_int32), ("layer_importance", POINTER(c_double)),
                ("t_layer", c_double), ("rl_num", c_int32), ("rl_den", c_int32)]


class PlanInfo(ctypes.Structure):
    _fields_ = [("n_items", c_int32), ("n_score_items", c_int32), ("n_units", c_int32), ("chunk_tokens", c_int32),
                ("layer_begin", c_int32), ("layer_end", c_int32), ("B", c_int32), ("ws_bytes", c_int64)]


def lib():
    """The loaded library.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError("libbaklava.so is not built (run `python -m paper_2502_13176_b200.build`); "
                               "there is no fallback path")
        L = ctypes.CDLL(_LIB_PATH)
        L.baklava_strerror.restype = c_char_p
        L.baklava_strerror.argtypes = [ctypes.c_int]
        L.baklava_importance.argtypes = [POINTER(Shape), POINTER(c_float), c_int32, POINTER(c_double)]
        L.baklava_allocate.argtypes = [POINTER(Shape), POINTER(c_double), POINTER(AllocParams), c_int64,
                                       POINTER(c_int32), POINTER(c_int64), POINTER(c_int64)]
        L.baklava_decode_plan.argtypes = [POINTER(Shape), POINTER(c_int32), c_int32, c_int32, c_int32, c_int32,
                                          c_int32, c_int32, c_int64, POINTER(c_int32), c_int64, POINTER(PlanInfo)]
        L.baklava_decode_attn.argtypes = [POINTER(Shape), POINTER(CacheStruct), c_void_p, c_void_p, c_void_p, c_int32,
                                          c_void_p, c_void_p, c_uint32, c_void_p, POINTER(PlanInfo),
                                          c_void_p, c_size_t, c_void_p]
        L.baklava_decode_attn_varlen.argtypes = [POINTER(Shape), POINTER(CacheStruct), c_void_p, c_void_p, c_void_p,
                                                 c_void_p, c_void_p, c_void_p, c_uint32, c_void_p, POINTER(PlanInfo),
                                                 c_void_p, c_size_t, c_void_p]
        L.baklava_evict_varlen.argtypes = [POINTER(Shape), POINTER(CacheStruct), c_int32, c_int32, c_void_p, c_void_p,
                                           c_void_p, c_int32, c_void_p, c_int64, c_int64, c_int64, c_int32, c_void_p,
                                           c_size_t, c_void_p]
        L.baklava_evict.argtypes = [POINTER(Shape), POINTER(CacheStruct), c_int32, c_int32, c_void_p, c_void_p,
                                    c_void_p, c_int32, c_int64, c_int64, c_int64, c_int32, c_void_p, c_size_t, c_void_p]
        L.baklava_evict_workspace_size.restype = c_size_t
        L.baklava_evict_workspace_size.argtypes = [POINTER(Shape), c_int32, c_int32, c_int32]
        L.baklava_evict_static.argtypes = [POINTER(Shape), POINTER(CacheStruct), c_int32, c_int32, c_void_p, c_void_p,
                                           c_void_p, c_int32, c_int64, c_int64, c_int64, c_int32, c_void_p]
        L.baklava_profile_heads.argtypes = [POINTER(Shape), c_void_p, c_void_p, c_void_p, c_void_p, c_int32, c_int32,
                                            c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
        L.baklava_prefill_scores.argtypes = [POINTER(Shape), c_void_p, c_void_p, c_void_p, c_void_p, c_int32, c_int32,
                                             c_void_p, c_void_p, c_size_t, c_void_p]
        L.baklava_prefill_workspace_size.restype = c_size_t
        L.baklava_prefill_workspace_size.argtypes = [POINTER(Shape), c_int32, c_int32]
        L.baklava_qk_norm_rope.argtypes = [POINTER(Shape), c_void_p, POINTER(Strides), c_void_p, POINTER(Strides), c_void_p,
                                           c_int32, c_int32, c_void_p, c_int32, c_void_p, c_void_p, c_float, c_uint32,
                                           c_void_p, POINTER(Strides), c_void_p, POINTER(Strides), c_void_p]
        prompt = [POINTER(Shape)] + [c_void_p, POINTER(Strides)] * 3 + [c_void_p, c_int32, c_int32]
        L.baklava_prefill_attn.argtypes = prompt + [c_void_p, POINTER(Strides), c_void_p, c_void_p, c_void_p]
        L.baklava_prefill_attn_packed.argtypes = prompt + [c_int64, c_void_p, POINTER(Strides), c_void_p, c_void_p, c_void_p]
        L.baklava_tree_plan.argtypes = [POINTER(Shape), POINTER(c_int32)] + [c_int32] * 6 + [POINTER(c_int32), c_int64, POINTER(PlanInfo)]
        L.baklava_tree_attn.argtypes = [POINTER(Shape), POINTER(CacheStruct)] + [c_void_p, POINTER(Strides)] * 3 + [
            c_void_p, c_void_p, c_int32, c_void_p, POINTER(Strides), c_void_p, c_void_p, POINTER(PlanInfo), c_void_p, c_size_t, c_void_p]
        L.baklava_tree_verify.argtypes = [c_void_p, c_int64, c_void_p, c_int64, c_int32] + [c_void_p] * 3 + [c_int32] * 3 + [
            c_void_p, c_void_p, c_uint32] + [c_void_p] * 5
        L.baklava_tree_commit.argtypes = [POINTER(Shape), POINTER(CacheStruct)] + [c_void_p] * 4 + [
            c_int32, c_void_p, c_void_p, c_int32, c_void_p, c_void_p, c_uint32, c_void_p, POINTER(PlanInfo), c_void_p, c_size_t, c_void_p]
        L.baklava_tree_commit_workspace_size.restype = c_size_t
        L.baklava_tree_commit_workspace_size.argtypes = [POINTER(Shape), POINTER(PlanInfo), c_int32]
        L.baklava_tree_call.argtypes = [c_int32, c_char_p, c_int32]
        L.baklava_output_error.argtypes = [c_void_p, c_void_p, c_int64, c_int32, c_void_p, c_void_p, c_size_t, c_void_p]
        L.baklava_output_error_workspace_size.restype = c_size_t
        L.baklava_output_error_workspace_size.argtypes = [c_int64]
        L.baklava_search_pick.argtypes = [POINTER(c_double), c_int32, POINTER(c_int32)]
        L.baklava_set_wait_limit.argtypes = [c_int64]
        L.baklava_profile_workspace_size.restype = c_size_t
        L.baklava_profile_workspace_size.argtypes = [POINTER(Shape), c_int32, c_int32]
        _lib = L
    return _lib


def strerror(code):
    return lib().baklava_strerror(int(code)).decode()


def _check(rc, what):
    if rc != OK:
        raise BaklavaError(rc, what)


def _ptr(t):
    return None if t is None else c_void_p(t.data_ptr())


def _stream(stream, dev=None):
    if stream is not None:
        return stream.cuda_stream
    # the current stream's handle without building a Stream object for it (3 us of a call that launches in 4)
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device() if dev is None else dev)


def make_shape(L, Hq, Hkv, D, page=16, n_sink=4, recent_num=1, recent_den=2):
    return Shape(L, Hq, Hkv, D, page, n_sink, recent_num, recent_den)


# ------------------------------------------------------------------ host entry points
def baklava_importance(shape, head_cos):
    """head_cos: float32 array [P, L, Hq] -> float64 array [L, Hkv]."""
    hc = np.ascontiguousarray(head_cos, dtype=np.float32)
    P = hc.shape[0]
    assert hc.shape == (P, shape.L, shape.Hq)
    out = np.empty((shape.L, shape.Hkv), dtype=np.float64)
    _check(lib().baklava_importance(ctypes.byref(shape), hc.ctypes.data_as(POINTER(c_float)), P,
                                    out.ctypes.data_as(POINTER(c_double))), "baklava_importance")
    return out


def baklava_allocate(shape, kv_importance, t, r_num, r_den, total_tokens, min_tokens, max_tokens,
                     scope=SCOPE_LAYER, layer_importance=None, t_layer=0.0, rl_num=0, rl_den=1):
    """Returns (cap int32 [L, Hkv], slab_off int64 [L, Hkv], seq_stride int)."""
    imp = np.ascontiguousarray(kv_importance, dtype=np.float64).reshape(shape.L, shape.Hkv)
    li = None if layer_importance is None else np.ascontiguousarray(layer_importance, dtype=np.float64)
    params = AllocParams(t, r_num, r_den, scope, min_tokens, max_tokens,
                         None if li is None else li.ctypes.data_as(POINTER(c_double)), t_layer, rl_num, rl_den)
    cap = np.empty((shape.L, shape.Hkv), dtype=np.int32)
    off = np.empty((shape.L, shape.Hkv), dtype=np.int64)
    stride = c_int64(0)
    _check(lib().baklava_allocate(ctypes.byref(shape), imp.ctypes.data_as(POINTER(c_double)), ctypes.byref(params),
                                  int(total_tokens), cap.ctypes.data_as(POINTER(c_int32)),
                                  off.ctypes.data_as(POINTER(c_int64)), ctypes.byref(stride)), "baklava_allocate")
    return cap, off, int(stride.value)


class Plan:
    """The decode work plan: `items` (int32 [n_items + n_score_items, 4], host) and `info`; `items_dev` after `.to(device)`."""

    def __init__(self, items, info):
        self.items, self.info, self.items_dev = items, info, None

    def to(self, device):
        self.items_dev = torch.from_numpy(self.items).to(device)
        return self


def baklava_decode_plan(shape, cap, B, layer_begin, layer_end, seq_stride_tokens, chunk_tokens=0, n_sm=148, kv_dtype=0):
    cap = np.ascontiguousarray(cap, dtype=np.int32).reshape(shape.L, shape.Hkv)
    info = PlanInfo()
    capp = cap.ctypes.data_as(POINTER(c_int32))
    _check(lib().baklava_decode_plan(ctypes.byref(shape), capp, B, layer_begin, layer_end, chunk_tokens, n_sm, kv_dtype,
                                     int(seq_stride_tokens), None, 0, ctypes.byref(info)), "baklava_decode_plan")
    total = info.n_items + info.n_score_items
    items = np.empty((total, 4), dtype=np.int32)
    _check(lib().baklava_decode_plan(ctypes.byref(shape), capp, B, layer_begin, layer_end, chunk_tokens, n_sm, kv_dtype,
                                     int(seq_stride_tokens), items.ctypes.data_as(POINTER(c_int32)), total,
                                     ctypes.byref(info)), "baklava_decode_plan")
    return Plan(items, info)


# ------------------------------------------------------------------ device state
def kv_row_bytes(D, kv_dtype):
    """Bytes of one cached token's K and V (4-bit rows with their two scales)."""
    return {KV_BF16: 4 * D, KV_FP8_E4M3: 2 * D, KV_INT4: D + 8}[kv_dtype]


class Cache:
    """Device buffers of a budgeted cache plus the struct the library reads.  Memory only."""

    def __init__(self, shape, cap, slab_off, seq_stride, B, device="cuda", kv_dtype=KV_BF16, kv_scale=None):
        """kv_scale: float32 array [L, Hkv, 4] = (K scale, 1 / K scale, V scale, 1 / V scale) per head, for FP8
        slabs; [L, Hkv, 4, D], the same per channel, for 4-bit slabs; passed to the library as given."""
        self.shape, self.B, self.seq_stride = shape, int(B), int(seq_stride)
        self.kv_dtype = int(kv_dtype)
        self.cap_host = np.ascontiguousarray(cap, dtype=np.int32).reshape(shape.L, shape.Hkv)
        self.off_host = np.ascontiguousarray(slab_off, dtype=np.int64).reshape(shape.L, shape.Hkv)
        rows = self.B * self.seq_stride
        slab_type = torch.bfloat16 if self.kv_dtype == KV_BF16 else torch.uint8
        width = shape.D // 2 if self.kv_dtype == KV_INT4 else shape.D
        self.k_slab = torch.empty((rows, width), dtype=slab_type, device=device)
        self.v_slab = torch.empty((rows, width), dtype=slab_type, device=device)
        self.kv_scale = self.row_scale = None
        if self.kv_dtype != KV_BF16:
            per_head = (4, shape.D) if self.kv_dtype == KV_INT4 else (4,)
            self.kv_scale_host = np.ascontiguousarray(kv_scale, dtype=np.float32).reshape((shape.L, shape.Hkv) + per_head).copy()
            self.kv_scale = torch.from_numpy(self.kv_scale_host).to(device)
        if self.kv_dtype == KV_INT4:
            self.row_scale = torch.zeros((rows, 2), dtype=torch.float32, device=device)
        self.pos = torch.full((rows,), -1, dtype=torch.int32, device=device)
        self.score = torch.zeros((rows,), dtype=torch.float32, device=device)
        self.len = torch.zeros((self.B, shape.L, shape.Hkv), dtype=torch.int32, device=device)
        self.free_slot = torch.zeros((self.B, shape.L, shape.Hkv), dtype=torch.int32, device=device)
        self.cap = torch.from_numpy(self.cap_host).to(device)
        self.slab_off = torch.from_numpy(self.off_host).to(device)
        self.status = torch.zeros((1,), dtype=torch.int32, device=device)
        self.struct = CacheStruct(self.k_slab.data_ptr(), self.v_slab.data_ptr(), self.pos.data_ptr(),
                                  self.score.data_ptr(), self.len.data_ptr(), self.free_slot.data_ptr(),
                                  self.cap.data_ptr(), self.slab_off.data_ptr(), self.seq_stride, self.B,
                                  self.status.data_ptr(), self.kv_dtype,
                                  None if self.kv_scale is None else self.kv_scale.data_ptr(),
                                  None if self.row_scale is None else self.row_scale.data_ptr())

    def reset(self):
        self.len.zero_()
        self.free_slot.zero_()
        self.status.zero_()

    def rows(self, b, l, h):
        """Row range [lo, hi) of head (l, h) of sequence b inside the slabs."""
        lo = b * self.seq_stride + int(self.off_host[l, h])
        return lo, lo + int(self.cap_host[l, h])

    def kv_bytes_retained(self):
        """Bytes of K and V rows currently valid (the metric's numerator for one step)."""
        return int(self.len.sum().item()) * kv_row_bytes(self.shape.D, self.kv_dtype)


def decode_workspace(plan, device="cuda"):
    return torch.zeros((int(plan.info.ws_bytes),), dtype=torch.uint8, device=device)


def baklava_decode_attn(shape, cache, q, k_new, v_new, t_pos, out, lse, flags, plan, ws, stream=None):
    _check(lib().baklava_decode_attn(ctypes.byref(shape), ctypes.byref(cache.struct), _ptr(q), _ptr(k_new), _ptr(v_new),
                                     int(t_pos), _ptr(out), _ptr(lse), int(flags), _ptr(plan.items_dev),
                                     ctypes.byref(plan.info), _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)),
           "baklava_decode_attn")


def baklava_decode_attn_varlen(shape, cache, q, k_new, v_new, t_pos, out, lse, flags, plan, ws, stream=None):
    """t_pos: device int32 [B]; a negative entry idles that sequence for the step."""
    assert t_pos.dtype == torch.int32 and t_pos.numel() == cache.B and t_pos.is_cuda
    _check(lib().baklava_decode_attn_varlen(ctypes.byref(shape), ctypes.byref(cache.struct), _ptr(q), _ptr(k_new),
                                            _ptr(v_new), _ptr(t_pos), _ptr(out), _ptr(lse), int(flags),
                                            _ptr(plan.items_dev), ctypes.byref(plan.info), _ptr(ws),
                                            ws.numel() * ws.element_size(), _stream(stream)),
           "baklava_decode_attn_varlen")


def baklava_set_wait_limit(sm_cycles):
    _check(lib().baklava_set_wait_limit(int(sm_cycles)), "baklava_set_wait_limit")


def workspace_error(ws):
    """The error word baklava_profile_heads / baklava_prefill_scores leave in their workspace (0 = none);
    synchronises."""
    return int(ws[:4].view(torch.int32).item())


def baklava_evict_workspace_size(shape, B, layers, T):
    return int(lib().baklava_evict_workspace_size(ctypes.byref(shape), B, layers, T))


def baklava_evict(shape, cache, layer_begin, layer_end, k_dense, v_dense, score_dense, T,
                  stride_layer, stride_seq, stride_head, reserve, ws, stream=None):
    _check(lib().baklava_evict(ctypes.byref(shape), ctypes.byref(cache.struct), layer_begin, layer_end,
                               _ptr(k_dense), _ptr(v_dense), _ptr(score_dense), int(T), int(stride_layer),
                               int(stride_seq), int(stride_head), int(reserve), _ptr(ws),
                               ws.numel() * ws.element_size(), _stream(stream)), "baklava_evict")


def baklava_evict_varlen(shape, cache, layer_begin, layer_end, k_dense, v_dense, score_dense, T, prompt_len,
                         stride_layer, stride_seq, stride_head, reserve, ws, stream=None):
    """prompt_len: device int32 [B] or None."""
    _check(lib().baklava_evict_varlen(ctypes.byref(shape), ctypes.byref(cache.struct), layer_begin, layer_end,
                                      _ptr(k_dense), _ptr(v_dense), _ptr(score_dense), int(T), _ptr(prompt_len),
                                      int(stride_layer), int(stride_seq), int(stride_head), int(reserve), _ptr(ws),
                                      ws.numel() * ws.element_size(), _stream(stream)), "baklava_evict_varlen")


EVICT_STATIC_MAX_ENTRIES = 1 << 20


def baklava_evict_static(shape, cache, layer_begin, layer_end, k_dense, v_dense, score_dense, T,
                         stride_layer, stride_seq, stride_head, reserve, stream=None):
    """baklava_evict for callers that cannot allocate a workspace: the kept-row list lives in a
    fixed 4 MiB array inside the library.  Calls on one device must not overlap in time."""
    _check(lib().baklava_evict_static(ctypes.byref(shape), ctypes.byref(cache.struct), layer_begin, layer_end,
                                      _ptr(k_dense), _ptr(v_dense), _ptr(score_dense), int(T), int(stride_layer),
                                      int(stride_seq), int(stride_head), int(reserve), _stream(stream)),
           "baklava_evict_static")


def baklava_profile_workspace_size(shape, P, T):
    return int(lib().baklava_profile_workspace_size(ctypes.byref(shape), P, T))


def baklava_profile_heads(shape, q, k, v, prompt_len, P, T, head_cos, token_cos, ws, stream=None):
    _check(lib().baklava_profile_heads(ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(prompt_len), P, T,
                                       _ptr(head_cos), _ptr(token_cos), _ptr(ws),
                                       0 if ws is None else ws.numel() * ws.element_size(), _stream(stream)),
           "baklava_profile_heads")


def baklava_prefill_workspace_size(shape, B, T):
    return int(lib().baklava_prefill_workspace_size(ctypes.byref(shape), B, T))


def baklava_prefill_scores(shape, q, k, prompt_len, B, T, score, ws, stream=None, lse=None):
    _check(lib().baklava_prefill_scores(ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(prompt_len), _ptr(lse), B, T, _ptr(score),
                                        _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)),
           "baklava_prefill_scores")


def _device():
    if torch.cuda._initialized:                      # (the two calls below take a microsecond)
        return torch._C._cuda_getDevice()
    return torch.cuda.current_device() if torch.cuda.is_initialized() or torch.cuda.is_available() else -2   # -2: none


def _elsewhere(t, what, dev):
    raise ValueError("%s is on %s; the current device is cuda:%d" % (what, t.device, dev))


@functools.lru_cache(maxsize=256)
def _strides(st):
    return Strides(st[0], st[1], st[2])              # (the library only reads it)


_BF16 = torch.bfloat16


def _rows(t, what, dev, shape):
    """Pointer and strides of a bf16 tensor [seqs, heads, tokens, D] (any view whose last dimension is contiguous)."""
    st = t.stride()
    if t.dtype is not _BF16 or t.shape != shape or st[3] != 1:
        raise ValueError("%s: expected bf16 [%d, %d, %d, %d] with contiguous rows, got %s %s with strides %s"
                         % ((what,) + shape + (t.dtype, tuple(t.shape), st)))
    if t.get_device() != dev:
        _elsewhere(t, what, dev)
    return t.data_ptr(), _strides(st)


def _dense(t, what, dev, dtype, shape):
    """Pointer of a contiguous tensor, NULL for None."""
    if t is None:
        return None
    if t.dtype is dtype and t.shape == shape and t.is_contiguous() and t.get_device() == dev:
        return t.data_ptr()
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError("%s: expected a contiguous %s tensor %s, got %s %s" % (what, dtype, shape, t.dtype, tuple(t.shape)))
    _elsewhere(t, what, dev)


def baklava_qk_norm_rope(shape, q, k, positions, inv_freq, q_weight, k_weight, eps, q_out, k_out, flags=0, stream=None):
    """q, q_out: bf16 [B, Hq, T, D], k, k_out: bf16 [B, Hkv, T, D], each any view with contiguous rows; positions: int32
    [B, T]; inv_freq: float32 [rotary_dim / 2]; weights: bf16 [D] or None."""
    B, _, T, _ = q.shape
    D = shape.D
    dev, n = _device(), inv_freq.numel()
    queries, keys = (B, shape.Hq, T, D), (B, shape.Hkv, T, D)
    _check(lib().baklava_qk_norm_rope(shape, *_rows(q, "q", dev, queries), *_rows(k, "k", dev, keys),
                                      _dense(positions, "positions", dev, torch.int32, (B, T)), B, T,
                                      _dense(inv_freq, "inv_freq", dev, torch.float32, (n,)), 2 * n,
                                      _dense(q_weight, "q_weight", dev, _BF16, (D,)),
                                      _dense(k_weight, "k_weight", dev, _BF16, (D,)), eps, flags,
                                      *_rows(q_out, "q_out", dev, queries), *_rows(k_out, "k_out", dev, keys),
                                      _stream(stream, dev)), "baklava_qk_norm_rope")


def baklava_prefill_attn(shape, q, k, v, prompt_len, out, lse, status, stream=None):
    """q, out: bf16 [B, Hq, T, D], k, v: bf16 [B, Hkv, T, D], any views with contiguous rows; prompt_len: int32 [B] or None;
    lse: float32 [B, Hq, T] or None; status: int32 [1]."""
    B, _, T, _ = q.shape
    D = shape.D
    dev = _device()
    queries, keys = (B, shape.Hq, T, D), (B, shape.Hkv, T, D)
    _check(lib().baklava_prefill_attn(shape, *_rows(q, "q", dev, queries), *_rows(k, "k", dev, keys),
                                      *_rows(v, "v", dev, keys), _dense(prompt_len, "prompt_len", dev, torch.int32, (B,)),
                                      B, T, *_rows(out, "out", dev, queries),
                                      _dense(lse, "lse", dev, torch.float32, queries[:3]),
                                      _dense(status, "status", dev, torch.int32, (1,)), _stream(stream, dev)),
           "baklava_prefill_attn")


def baklava_prefill_attn_packed(shape, q, k, v, cu_seqlens, max_len, out, lse, status, stream=None):
    """q, out: bf16 [Hq, total, D], k, v: bf16 [Hkv, total, D], any views with contiguous rows; cu_seqlens: int32 [B + 1];
    lse: float32 [Hq, total] or None; status: int32 [1]."""
    total, D, Hq = q.shape[1], shape.D, shape.Hq
    dev, n = _device(), cu_seqlens.numel()
    queries, keys = (1, Hq, total, D), (1, shape.Hkv, total, D)
    _check(lib().baklava_prefill_attn_packed(shape, *_rows(q.unsqueeze(0), "q", dev, queries),
                                             *_rows(k.unsqueeze(0), "k", dev, keys),
                                             *_rows(v.unsqueeze(0), "v", dev, keys),
                                             _dense(cu_seqlens, "cu_seqlens", dev, torch.int32, (n,)), n - 1, max_len, total,
                                             *_rows(out.unsqueeze(0), "out", dev, queries),
                                             _dense(lse, "lse", dev, torch.float32, (Hq, total)),
                                             _dense(status, "status", dev, torch.int32, (1,)), _stream(stream, dev)),
           "baklava_prefill_attn_packed")


# ------------------------------------------------------------------ drafted tokens
def baklava_tree_plan(shape, cap, B, layer, T, chunk_tokens=0, n_sm=148, kv_dtype=KV_BF16):
    """cap: int32 array [L, Hkv].  The plan of baklava_tree_attn for one layer; `decode_workspace(plan)` is its workspace."""
    cap = np.ascontiguousarray(cap, dtype=np.int32).reshape(shape.L, shape.Hkv)
    info = PlanInfo()
    args = (ctypes.byref(shape), cap.ctypes.data_as(POINTER(c_int32)), B, layer, T, chunk_tokens, n_sm, kv_dtype)
    _check(lib().baklava_tree_plan(*args, None, 0, ctypes.byref(info)), "baklava_tree_plan")
    items = np.empty((info.n_items, 4), dtype=np.int32)
    _check(lib().baklava_tree_plan(*args, items.ctypes.data_as(POINTER(c_int32)), info.n_items, ctypes.byref(info)),
           "baklava_tree_plan")
    return Plan(items, info)


_address = ctypes.addressof
_words = {n: struct.Struct("%dq" % n).pack for n in (18, 19, 27)}
_CALL_ATTN, _CALL_VERIFY, _CALL_COMMIT = 0, 1, 2
_I32, _F32 = torch.int32, torch.float32


def _tree_call(call, what, *args):
    n = len(args)
    rc = lib().baklava_tree_call(call, _words[n](*args), n)
    if rc != OK:
        raise BaklavaError(rc, what)


def _row_words(t, what, dev, shape):
    """Pointer and strides of a bf16 tensor [seqs, heads, tokens, D] (any view whose last dimension is contiguous)."""
    st = t.stride()
    if t.dtype is _BF16 and t.shape == shape and st[3] == 1 and t.get_device() == dev:
        return t.data_ptr(), st[0], st[1], st[2]
    _rows(t, what, dev, shape)
    return t.data_ptr(), st[0], st[1], st[2]


def _planned(plan, dev):
    items = plan.items_dev
    if items is None or items.get_device() != dev:
        raise ValueError("the plan's items are not on the current device (Plan.to)")
    return items.data_ptr(), _address(plan.info)


def _workspace(ws, dev):
    if not ws.is_contiguous():
        raise ValueError("ws: expected a contiguous tensor")
    if ws.get_device() != dev:
        _elsewhere(ws, "ws", dev)
    return ws.data_ptr(), ws.numel() * ws.element_size()


def _cache_here(cache, B, dev):
    if cache.B != B:
        raise ValueError("the cache holds %d sequences, the tensors %d" % (cache.B, B))
    if cache.k_slab.get_device() != dev:
        _elsewhere(cache.k_slab, "the cache", dev)
    return _address(cache.struct)


def baklava_tree_attn(shape, cache, q, k, v, parent, n_nodes, out, lse, plan, ws, stream=None):
    """q, out: bf16 [B, Hq, T, D], k, v: bf16 [B, Hkv, T, D], any views with contiguous rows; parent: int32 [B, T]; n_nodes:
    int32 [B] or None; lse: float32 [B, Hq, T] or None; plan: baklava_tree_plan's for the layer."""
    B, Hq, T, _ = q.shape
    D = shape.D
    dev = _device()
    queries, keys = (B, shape.Hq, T, D), (B, shape.Hkv, T, D)
    _tree_call(_CALL_ATTN, "baklava_tree_attn", _address(shape), _cache_here(cache, B, dev), *_row_words(q, "q", dev, queries),
               *_row_words(k, "k", dev, keys), *_row_words(v, "v", dev, keys), _dense(parent, "parent", dev, _I32, (B, T)),
               _dense(n_nodes, "n_nodes", dev, _I32, (B,)) or 0, T, *_row_words(out, "out", dev, queries),
               _dense(lse, "lse", dev, _F32, (B, Hq, T)) or 0, *_planned(plan, dev), *_workspace(ws, dev), _stream(stream, dev))


def _probabilities(t, what, dev, shape, dtype):
    """Pointer and row stride of probabilities [B, T, V]: rows contiguous, all the same distance apart, at least a row (rows that
    repeat, as expand() makes them, or overlap are none that a stride could reach)."""
    B, T, V = shape
    st = t.stride()
    row = st[1] if T > 1 else st[0] if B > 1 else V           # (the stride of a single row means nothing)
    if t.dtype is not dtype or t.shape != shape or st[2] != 1 and V > 1 or B > 1 and T > 1 and st[0] != T * st[1] or row < V:
        raise ValueError("%s: expected %s [%d, %d, %d] with contiguous rows at one distance of at least a row, got %s %s with strides %s"
                         % (what, dtype, B, T, V, t.dtype, tuple(t.shape), st))
    if t.get_device() != dev:
        _elsewhere(t, what, dev)
    return t.data_ptr(), row


def baklava_tree_verify(target, draft, tokens, parent, n_nodes, u_accept, u_sample, path, n_path, next_token, status, flags=0,
                        stream=None):
    """target: float32 or bf16 [B, T, V]; draft: the same or None; tokens, parent, path: int32 [B, T]; n_nodes, n_path,
    next_token: int32 [B] (n_nodes may be None); u_accept: float32 [B, T]; u_sample: float32 [B]; status: int32 [1]."""
    probs, kind = target.shape, target.dtype
    B, T, V = probs
    dev = _device()
    if kind is not _F32 and kind is not _BF16:
        raise ValueError("target: expected float32 or bfloat16, got %s" % kind)
    per_node, per_seq = (B, T), (B,)
    _tree_call(_CALL_VERIFY, "baklava_tree_verify", *_probabilities(target, "target", dev, probs, kind),
               *((0, 0) if draft is None else _probabilities(draft, "draft", dev, probs, kind)), PROB_F32 if kind is _F32 else PROB_BF16,
               _dense(tokens, "tokens", dev, _I32, per_node), _dense(parent, "parent", dev, _I32, per_node),
               _dense(n_nodes, "n_nodes", dev, _I32, per_seq) or 0, B, T, V, _dense(u_accept, "u_accept", dev, _F32, per_node),
               _dense(u_sample, "u_sample", dev, _F32, per_seq), flags, _dense(path, "path", dev, _I32, per_node),
               _dense(n_path, "n_path", dev, _I32, per_seq), _dense(next_token, "next_token", dev, _I32, per_seq),
               _dense(status, "status", dev, _I32, (1,)), _stream(stream, dev))


def tree_commit_workspace(shape, plan, max_path, device="cuda"):
    n = int(lib().baklava_tree_commit_workspace_size(ctypes.byref(shape), ctypes.byref(plan.info), max_path))
    return torch.empty((n,), dtype=torch.uint8, device=device)


def baklava_tree_commit(shape, cache, q, k, v, lse, path, n_path, max_path, t_pos, t_next, flags, plan, ws, stream=None):
    """q: bf16 [layers, B, Hq, T, D], k, v: bf16 [layers, B, Hkv, T, D], lse: float32 [layers, B, Hq, T], contiguous (q and lse
    may be None with FLAG_NO_SCORE); path: int32 [B, T]; n_path, t_pos, t_next: int32 [B] (t_next may be None); plan: one of
    baklava_decode_plan for the layers; ws: tree_commit_workspace."""
    n, B, _, T, _ = k.shape
    dev, info = _device(), plan.info
    if n != info.layer_end - info.layer_begin:
        raise ValueError("k has %d layers, the plan %d" % (n, info.layer_end - info.layer_begin))
    Hq, keys = shape.Hq, (n, B, shape.Hkv, T, shape.D)
    _tree_call(_CALL_COMMIT, "baklava_tree_commit", _address(shape), _cache_here(cache, B, dev),
               _dense(q, "q", dev, _BF16, (n, B, Hq, T, shape.D)) or 0, _dense(k, "k", dev, _BF16, keys), _dense(v, "v", dev, _BF16, keys),
               _dense(lse, "lse", dev, _F32, (n, B, Hq, T)) or 0, T, _dense(path, "path", dev, _I32, (B, T)),
               _dense(n_path, "n_path", dev, _I32, (B,)), max_path, _dense(t_pos, "t_pos", dev, _I32, (B,)),
               _dense(t_next, "t_next", dev, _I32, (B,)) or 0, flags, *_planned(plan, dev), *_workspace(ws, dev), _stream(stream, dev))


def baklava_output_error(out, ref, loss, ws, stream=None):
    """out, ref: bf16 tensors of the same shape [..., D]; loss: float64 tensor [1] (device), overwritten."""
    assert out.shape == ref.shape and out.dtype == torch.bfloat16 and ref.dtype == torch.bfloat16
    assert out.is_contiguous() and ref.is_contiguous() and loss.dtype == torch.float64
    D = out.shape[-1]
    rows = out.numel() // D
    _check(lib().baklava_output_error(_ptr(out), _ptr(ref), rows, D, _ptr(loss), _ptr(ws),
                                      ws.numel() * ws.element_size(), _stream(stream)), "baklava_output_error")


def baklava_output_error_workspace_size(rows):
    return int(lib().baklava_output_error_workspace_size(int(rows)))


def baklava_search_pick(avg_loss):
    a = np.ascontiguousarray(avg_loss, dtype=np.float64)
    best = c_int32(-2)
    _check(lib().baklava_search_pick(a.ctypes.data_as(POINTER(c_double)), len(a), ctypes.byref(best)),
           "baklava_search_pick")
    return int(best.value)
