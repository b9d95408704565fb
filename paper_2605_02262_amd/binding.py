"""Thin ctypes binding over libwq.so: argument marshalling only.

PyTorch is used for device memory (``torch.empty(..., device="cuda")``, ``.data_ptr()``) and for the current
stream; every step of the path runs in the library's kernels.  Loading fails loudly when the library has
not been built (``python -m paper_2605_02262_amd.build``): there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import operator
import os
from typing import Optional, Sequence

import torch

F32, BF16, F16 = 0, 1, 2
SCORE_AUTO, SCORE_PAIRWISE_MFMA, SCORE_POOLED = 0, 1, 2
MODE_QUOTA, MODE_THRESHOLD = 0, 1
DECODE_AUTO, DECODE_GENERIC, DECODE_MFMA = 0, 1, 2
DECODE_PARTIALS_ONLY = 0x100
DECODE_FIXED_SHARES = 0x200
DECODE_BY_LENGTH = 0x400
DECODE_SEPARATE_MERGE = 0x800
ROPE_HALF, ROPE_PAIRS = 0, 1
ROPE_PLAIN, ROPE_EVEN, ROPE_BASE, ROPE_PARTS = 0, 1, 2, 3
CLASS_BITS = (2, 4, 8)
DEV_CLASS_OVERFLOW, DEV_SEG16_OVERFLOW, DEV_APPEND_TIMEOUT, DEV_TOO_MANY_WINDOWS, DEV_BAD_ASSIGNMENT = 1, 2, 4, 16, 32
DEV_TOO_MANY_ROWS, DEV_BAD_INDEX = 64, 128

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libwq.so")
_lib = None


class WQError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"wq error {code}: {msg}")
        self.code = code


class _PackedKV(C.Structure):
    _fields_ = [("B", C.c_int32), ("Hkv", C.c_int32), ("hd", C.c_int32), ("group", C.c_int32),
                ("dtype16", C.c_int32), ("reserved", C.c_int32),
                ("codes", C.c_void_p * 3), ("meta", C.c_void_p * 3), ("cap", C.c_int64 * 3),
                ("cls_off", C.c_void_p * 3), ("cls_len", C.c_void_p * 3),
                ("k16", C.c_void_p), ("v16", C.c_void_p), ("cap16", C.c_int64),
                ("off16", C.c_void_p), ("len16", C.c_void_p), ("v_scale_max", C.c_void_p)]


def lib() -> C.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2605_02262_amd.build`")
        L = C.CDLL(_LIB_PATH)
        vp, i32, i64, f32 = C.c_void_p, C.c_int, C.c_int64, C.c_float
        L.wq_create.argtypes = [C.POINTER(vp), vp, vp, C.c_size_t]
        L.wq_destroy.argtypes = [vp]
        L.wq_set_stream.argtypes = [vp, vp]
        L.wq_last_error.argtypes = [vp]
        L.wq_last_error.restype = C.c_char_p
        L.wq_device_status.argtypes = [vp, C.POINTER(C.c_uint32)]
        L.wq_v_scale_floats.argtypes = [i32, i32, C.POINTER(C.c_int64)]
        L.wq_v_scale_floats.restype = C.c_size_t
        L.wq_workspace_bytes.argtypes = [i32, i32, i32, i32, i64, i64, i32]
        L.wq_workspace_bytes.restype = C.c_size_t
        L.wq_packed_bytes.argtypes = [i32, i64, i32, i32, i32, C.POINTER(C.c_size_t)]
        L.wq_packed_bytes.restype = C.c_size_t
        L.wq_auto_splits.argtypes = [i32, i32, i64]
        L.wq_auto_splits_ragged.argtypes = [i32, i32, i64, i64]
        L.wq_window_scores.argtypes = [vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, i64, i64, i64, i32, vp]
        L.wq_assign_bits.argtypes = [vp, vp, i32, vp, i32, i32, vp, vp, i32, i32, vp, vp, vp]
        L.wq_layer_thresholds.argtypes = [C.POINTER(C.c_double), i32, C.c_double, C.POINTER(C.c_float), C.POINTER(C.c_float)]
        L.wq_vote_bits.argtypes = [vp, vp, i32, vp, i32, vp, vp, vp]
        L.wq_validate_assignment.argtypes = [vp, i32, vp, i32, vp, vp]
        L.wq_reorder_quantize.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp, vp, vp, i64, C.POINTER(_PackedKV)]
        L.wq_append_kv.argtypes = [vp, vp, vp, i32, i32, C.POINTER(_PackedKV)]
        L.wq_dequantize.argtypes = [vp, i32, C.POINTER(_PackedKV), C.POINTER(_PackedKV)]
        L.wq_decode_append_attention.argtypes = [vp, vp, i32, i32, i32, C.POINTER(_PackedKV), vp, vp, i32, f32, i32, i64, i32, vp, vp]
        L.wq_decode_attention.argtypes = [vp, vp, i32, i32, i32, C.POINTER(_PackedKV), f32, i32, i64, i32, vp, vp]
        L.wq_decode_attention_static.argtypes = [vp, vp, i32, i32, i32, C.POINTER(_PackedKV), f32, i32, i64, i32, vp, vp]
        L.wq_static_last_error.argtypes = []
        L.wq_static_last_error.restype = C.c_char_p
        L.wq_rope.argtypes = [vp, vp, i64, vp, i64, i32, i64, i32, i32, i32, i32, i32, vp, vp, f32, vp, i64, vp, i64]
        L.wq_rope_append_kv.argtypes = [vp, vp, i64, vp, i64, vp, i64, i32, i32, i32, i32, i32, vp, vp, f32, vp, i64, C.POINTER(_PackedKV)]
        L.wq_rope_frequencies.argtypes = [i32, C.c_double, i32, C.c_double, i64, C.POINTER(C.c_float), C.POINTER(C.c_float)]
        L.wq_prefill_attention.argtypes = [vp, vp, i64, vp, i64, vp, i64, i32, i32, i32, i32, i32, vp, vp, vp, i64, i64, i64, f32, i32, vp, vp]
        L.wq_prefill_workspace_bytes.argtypes = [i64, i32, i32, i32, i32, i64, i32]
        L.wq_prefill_workspace_bytes.restype = C.c_size_t
        L.wq_decode_attention_shared.argtypes = [vp, vp, i32, i32, i32, C.POINTER(_PackedKV), vp, C.POINTER(_PackedKV), f32, i32, i64, i64, vp, vp]
        L.wq_shared_workspace_bytes.argtypes = [i32, i32, i32, i32, i32, i64, i64, i32]
        L.wq_shared_workspace_bytes.restype = C.c_size_t
        L.wq_tree_attention.argtypes = [vp, vp, i64, vp, i64, vp, i64, i32, i32, i32, C.POINTER(_PackedKV), vp, vp, i64, i32, f32, i32, i64, vp, vp]
        L.wq_tree_workspace_bytes.argtypes = [i64, i32, i32, i32, i32, i64, i32, i32]
        L.wq_tree_workspace_bytes.restype = C.c_size_t
        L.wq_tree_accept.argtypes = [vp, vp, vp, vp, i32, vp, i64, i32, i32, vp, vp, vp]
        L.wq_append_rows.argtypes = [vp, i32, vp, i64, vp, i64, i32, i32, vp, i64, vp, vp, i32, vp]
        L.wq_copy_sequences.argtypes = [vp, i32, vp, vp, vp]
        L.wq_probe_stream.argtypes = [vp, vp, vp, i64, i32]
        L.wq_probe_mfma.argtypes = [vp, i32, i32, i32, C.POINTER(C.c_double)]
        L.wq_decode_timing.argtypes = [vp, i32]
        L.wq_decode_times_us.argtypes = [vp, C.POINTER(C.c_float), i32]
        _lib = L
    return _lib


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()      # (of an empty tensor: 0, a view's too)


_DTYPE_ID = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}


def _dtype_id(t: torch.Tensor) -> int:
    return _DTYPE_ID[t.dtype]


def workspace_bytes(B=0, Hq=0, hd=0, max_splits=0, total_vis=0, total_txt=0, D=0) -> int:
    return int(lib().wq_workspace_bytes(B, Hq, hd, max_splits, total_vis, total_txt, D))


def packed_bytes(bits: int, cap_tokens: int, Hkv: int, hd: int, group: int):
    mb = C.c_size_t(0)
    cb = lib().wq_packed_bytes(bits, cap_tokens, Hkv, hd, group, C.byref(mb))
    return int(cb), int(mb.value)


def auto_splits(B: int, Hkv: int, max_seq_tokens: int) -> int:
    return int(lib().wq_auto_splits(B, Hkv, max_seq_tokens))


def auto_splits_ragged(B: int, Hkv: int, max_seq_tokens: int, total_tokens: int) -> int:
    return int(lib().wq_auto_splits_ragged(B, Hkv, max_seq_tokens, total_tokens))


class Context:
    """wq_ctx plus the torch tensor that backs its workspace (first 256 bytes zero = clean status word)."""

    def __init__(self, workspace_bytes_: int, device: str = "cuda", stream: Optional[torch.cuda.Stream] = None):
        self.device = torch.device(device)
        self.ws = torch.zeros(max(int(workspace_bytes_), 16384), dtype=torch.uint8, device=self.device)
        self.index = self.ws.get_device()
        self.handle = C.c_void_p()
        st = (stream or torch.cuda.current_stream(self.device)).cuda_stream
        rc = lib().wq_create(C.byref(self.handle), C.c_void_p(st), self.ws.data_ptr(), self.ws.numel())
        if rc != 0:
            raise WQError(rc, "wq_create failed")

    def set_stream(self, stream: torch.cuda.Stream):
        lib().wq_set_stream(self.handle, C.c_void_p(stream.cuda_stream))

    def check(self, rc: int):
        if rc != 0:
            raise WQError(rc, lib().wq_last_error(self.handle).decode())

    def decode_timing(self, enable: bool = True):
        self.check(lib().wq_decode_timing(self.handle, 1 if enable else 0))

    def decode_times_us(self, n: int):
        buf = (C.c_float * n)()
        self.check(lib().wq_decode_times_us(self.handle, buf, n))
        return [float(x) for x in buf]

    def device_status(self) -> int:
        bits = C.c_uint32(0)
        self.check(lib().wq_device_status(self.handle, C.byref(bits)))
        return int(bits.value)

    def __del__(self):
        try:
            if self.handle:
                lib().wq_destroy(self.handle)
                self.handle = C.c_void_p()
        except Exception:
            pass


class PackedKV:
    """Device buffers of one layer's packed cache plus the C descriptor that points at them."""

    def __init__(self, B: int, Hkv: int, hd: int, group: int, dtype16: torch.dtype, cap: Sequence[int], off16: Sequence[int],
                 device: str = "cuda", fill: Optional[int] = None):
        dev = torch.device(device)
        self.B, self.Hkv, self.hd, self.group = B, Hkv, hd, group
        self.cap = [(int(c) + 31) // 32 * 32 for c in cap]
        self.dtype16 = dtype16
        G = hd // group
        mk = (lambda *s, dtype: torch.empty(*s, dtype=dtype, device=dev)) if fill is None else \
             (lambda *s, dtype: torch.full(s, fill, dtype=dtype, device=dev))
        self.codes = [mk(2, Hkv, self.cap[c] * hd * b // 8, dtype=torch.uint8) for c, b in enumerate(CLASS_BITS)]
        self.meta = [mk(2, Hkv, self.cap[c] * G, dtype=torch.int32) for c in range(3)]
        self.cls_off = [torch.zeros(B + 1, dtype=torch.int32, device=dev) for _ in range(3)]
        self.cls_len = [torch.zeros(B, dtype=torch.int32, device=dev) for _ in range(3)]
        self.off16 = torch.as_tensor(list(off16), dtype=torch.int32).to(dev)
        assert self.off16.numel() == B + 1
        self.cap16 = int(off16[-1]) if len(off16) else 0
        self.k16 = torch.zeros(self.cap16, Hkv, hd, dtype=dtype16, device=dev)
        self.v16 = torch.zeros(self.cap16, Hkv, hd, dtype=dtype16, device=dev)
        self.len16 = torch.zeros(B, dtype=torch.int32, device=dev)
        n_vs = lib().wq_v_scale_floats(B, Hkv, (C.c_int64 * 3)(*[int(c) for c in self.cap]))
        self.v_scale_max = torch.zeros(n_vs, dtype=torch.float32, device=dev)
        d = _PackedKV()
        d.B, d.Hkv, d.hd, d.group = B, Hkv, hd, group
        d.dtype16 = _dtype_id(self.k16)
        for c in range(3):
            d.codes[c] = _ptr(self.codes[c])
            d.meta[c] = _ptr(self.meta[c])
            d.cap[c] = self.cap[c]
            d.cls_off[c] = self.cls_off[c].data_ptr()
            d.cls_len[c] = _ptr(self.cls_len[c])
        d.k16, d.v16, d.cap16 = _ptr(self.k16), _ptr(self.v16), self.cap16
        d.off16, d.len16 = self.off16.data_ptr(), _ptr(self.len16)
        d.v_scale_max = _ptr(self.v_scale_max)
        self.desc = d
        self.index = self.off16.get_device()

    def bytes_algorithmic(self) -> int:
        """Bytes a decode step has to read: codes + metadata of the real tokens and the 16-bit rows in use."""
        G = self.hd // self.group
        n = 0
        for c, b in enumerate(CLASS_BITS):
            t = int(self.cls_len[c].sum().item())
            n += t * self.Hkv * 2 * (self.hd * b // 8 + G * 4)
        n += int(self.len16.sum().item()) * self.Hkv * self.hd * 2 * 2
        return n


# ------------------------------------------------------------------------------------------------------------
# the four calls (same names as the C ABI)
# ------------------------------------------------------------------------------------------------------------
def wq_window_scores(ctx: Context, vis_emb, txt_emb, vis_off, txt_off, win_size, win_off, total_vis: int,
                     total_txt: int, total_win: int, algo: int = SCORE_AUTO, scores: Optional[torch.Tensor] = None):
    B = win_size.numel()
    D = vis_emb.shape[1] if vis_emb.numel() else txt_emb.shape[1]
    if scores is None:
        scores = torch.empty(total_win, dtype=torch.float32, device=ctx.device)
    ctx.check(lib().wq_window_scores(ctx.handle, _ptr(vis_emb), _ptr(txt_emb), _dtype_id(vis_emb), B, D, _ptr(vis_off),
                                     _ptr(txt_off), _ptr(win_size), _ptr(win_off), total_vis, total_txt, total_win, algo,
                                     _ptr(scores)))
    return scores


def wq_assign_bits(ctx: Context, scores, win_off, max_windows: int, mode: int = MODE_QUOTA, quota=None, thresholds=None,
                   top_bits: int = 8, pin_first: int = 1):
    B = win_off.numel() - 1
    W = scores.numel()
    bits = torch.empty(W, dtype=torch.uint8, device=ctx.device)
    perm = torch.empty(W, dtype=torch.int32, device=ctx.device)
    seg = torch.empty(B, 4, dtype=torch.int32, device=ctx.device)
    ctx.check(lib().wq_assign_bits(ctx.handle, _ptr(scores), B, _ptr(win_off), max_windows, mode, _ptr(quota),
                                   _ptr(thresholds), top_bits, pin_first, _ptr(bits), _ptr(perm), _ptr(seg)))
    return bits, perm, seg


def wq_layer_thresholds(s, alpha: float):
    """(T_low, T_high) per layer as fp32 lists (host-only call)."""
    n = len(s)
    sa = (C.c_double * n)(*[float(x) for x in s])
    lo, hi = (C.c_float * n)(), (C.c_float * n)()
    rc = lib().wq_layer_thresholds(sa, n, float(alpha), lo, hi)
    if rc != 0:
        raise WQError(rc, "wq_layer_thresholds: bad argument")
    return [float(x) for x in lo], [float(x) for x in hi]


def wq_vote_bits(ctx: Context, bits, win_off, max_windows: int):
    B = win_off.numel() - 1
    W = bits.numel()
    out = torch.empty(W, dtype=torch.uint8, device=ctx.device)
    perm = torch.empty(W, dtype=torch.int32, device=ctx.device)
    seg = torch.empty(B, 4, dtype=torch.int32, device=ctx.device)
    ctx.check(lib().wq_vote_bits(ctx.handle, _ptr(bits), B, _ptr(win_off), max_windows, _ptr(out), _ptr(perm), _ptr(seg)))
    return out, perm, seg


def wq_validate_assignment(ctx: Context, win_off, max_windows: int, perm, seg_windows):
    B = win_off.numel() - 1
    ctx.check(lib().wq_validate_assignment(ctx.handle, B, _ptr(win_off), max_windows, _ptr(perm), _ptr(seg_windows)))


def wq_reorder_quantize(ctx: Context, K, V, kv_off, win_size, win_off, perm, seg_windows, total_rows: int, out: PackedKV):
    B = win_size.numel()
    # a batch without any window has an empty perm: the library still wants a valid pointer (it cannot see the window
    # count on the host), which is never read then
    perm_ptr = _ptr(perm) if perm.numel() else _ptr(seg_windows)
    ctx.check(lib().wq_reorder_quantize(ctx.handle, _ptr(K), _ptr(V), _dtype_id(K), B, _ptr(kv_off), _ptr(win_size),
                                        _ptr(win_off), perm_ptr, _ptr(seg_windows), total_rows, C.byref(out.desc)))
    return out


def wq_append_kv(ctx: Context, k_new, v_new, kv: PackedKV):
    B = k_new.shape[0]
    ctx.check(lib().wq_append_kv(ctx.handle, _ptr(k_new), _ptr(v_new), _dtype_id(k_new), B, C.byref(kv.desc)))


def wq_decode_append_attention(ctx: Context, q, kv: PackedKV, k_new, v_new, sm_scale: float, num_splits: int = 0,
                               max_seq_tokens: int = 0, algo: int = DECODE_AUTO, out: Optional[torch.Tensor] = None,
                               lse: Optional[torch.Tensor] = None):
    B, Hq, hd = q.shape
    if out is None:
        out = torch.empty(B, Hq, hd, dtype=torch.float32, device=ctx.device)
    ctx.check(lib().wq_decode_append_attention(ctx.handle, _ptr(q), _dtype_id(q), B, Hq, C.byref(kv.desc), _ptr(k_new), _ptr(v_new),
                                               _dtype_id(k_new), sm_scale, num_splits, max_seq_tokens, algo, _ptr(out), _ptr(lse)))
    return out


def wq_dequantize(ctx: Context, src: PackedKV, dst: PackedKV):
    ctx.check(lib().wq_dequantize(ctx.handle, src.B, C.byref(src.desc), C.byref(dst.desc)))


def wq_decode_attention(ctx: Context, q, kv: PackedKV, sm_scale: float, num_splits: int = 0, max_seq_tokens: int = 0,
                        algo: int = DECODE_AUTO, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None):
    B, Hq, hd = q.shape
    if out is None:
        out = torch.empty(B, Hq, hd, dtype=torch.float32, device=ctx.device)
    ctx.check(lib().wq_decode_attention(ctx.handle, _ptr(q), _dtype_id(q), B, Hq, C.byref(kv.desc), sm_scale, num_splits,
                                        max_seq_tokens, algo, _ptr(out), _ptr(lse)))
    return out


def wq_decode_attention_static(q, kv: PackedKV, sm_scale: float, num_splits: int = 0, max_seq_tokens: int = 0,
                               algo: int = DECODE_AUTO, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                               stream: Optional[torch.cuda.Stream] = None):
    """wq_decode_attention without a context: the library's own static scratch array is the workspace."""
    B, Hq, hd = q.shape
    if out is None:
        out = torch.empty(B, Hq, hd, dtype=torch.float32, device=q.device)
    st = (stream or torch.cuda.current_stream(q.device)).cuda_stream
    rc = lib().wq_decode_attention_static(C.c_void_p(st), _ptr(q), _dtype_id(q), B, Hq, C.byref(kv.desc), sm_scale, num_splits,
                                          max_seq_tokens, algo, _ptr(out), _ptr(lse))
    if rc != 0:
        raise WQError(rc, lib().wq_static_last_error().decode())
    return out


# ------------------------------------------------------------------------------------------------------------
# rotary positions, prompt attention, decode over shared caches
# ------------------------------------------------------------------------------------------------------------
# (A call's checks cost about as much as its launch: a tensor's attributes are read once, 0.1 us each, and outputs made here are not checked.)
def _rows(name: str, t: torch.Tensor, like: Optional[torch.Tensor] = None, shape=None):
    """(rows, heads, hd, elements from row to row) of [rows, heads, hd] whose rows are contiguous inside; like: of its type, shape: of that."""
    have = tuple(t.shape)
    if len(have) != 3 or (shape is not None and have != shape):
        raise ValueError(f"{name}: {shape or '[rows, heads, head_dim]'} expected, got shape {have}")
    if like is not None and t.dtype != like.dtype:
        raise ValueError(f"{name}: type differs from the queries'")
    rows, heads, hd = have
    if t.is_contiguous():
        return rows, heads, hd, heads * hd
    row, head, channel = t.stride()
    if channel != 1 or (heads > 1 and head != hd):
        raise ValueError(f"{name}: [rows, heads, head_dim] with contiguous rows expected, got shape {have}, strides {t.stride()}")
    return rows, heads, hd, max(row, heads * hd) if rows <= 1 else row


def _here(ctx: Context, *tensors: Optional[torch.Tensor]):
    """Every tensor on the context's device: a kernel given a host pointer would fault."""
    for t in tensors:
        if t is not None and t.get_device() != ctx.index:
            raise ValueError(f"a tensor of shape {tuple(t.shape)} on {t.device}: the context's device, cuda:{ctx.index}, expected")


def _like(t: torch.Tensor) -> torch.Tensor:
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def _contiguous(name: str, t: torch.Tensor, dtype: torch.dtype, numel: int):
    if t.dtype != dtype or not t.is_contiguous() or t.numel() != numel:
        raise ValueError(f"{name}: {numel} contiguous elements of {dtype} expected, got {tuple(t.shape)} of {t.dtype}")


def wq_rope_frequencies(rot_dim: int, base: float, scaling: int = ROPE_PLAIN, factor: float = 1.0, trained_context: int = 0):
    """(inv_freq as an fp32 list, mscale) (host-only call)."""
    f, m = (C.c_float * max(rot_dim // 2, 1))(), C.c_float(0.0)
    rc = lib().wq_rope_frequencies(rot_dim, float(base), scaling, float(factor), trained_context, f, C.byref(m))
    if rc != 0:
        raise WQError(rc, "wq_rope_frequencies: bad argument")
    return [float(x) for x in f], float(m.value)


def wq_rope(ctx: Context, q, k, positions, inv_freq, layout: int = ROPE_HALF, mscale: float = 1.0, q_out: Optional[torch.Tensor] = None,
            k_out: Optional[torch.Tensor] = None):
    """Turns q [rows, Hq, hd] and k [rows, Hkv, hd] (or None); 2 * inv_freq.numel() channels of every head."""
    _here(ctx, q, k, positions, inv_freq, q_out, k_out)
    rows, Hq, hd, qs = _rows("q", q)
    _contiguous("positions", positions, torch.int32, rows)
    half = inv_freq.numel()
    _contiguous("inv_freq", inv_freq, torch.float32, half)
    if q_out is None:
        q_out, qo = _like(q), Hq * hd
    else:
        qo = _rows("q_out", q_out, q, (rows, Hq, hd))[3]
    ks = ko = Hkv = 0
    if k is not None:
        k_rows, Hkv, k_hd, ks = _rows("k", k, q)
        if k_rows != rows or k_hd != hd:
            raise ValueError("k: the rows and head_dim of q expected")
        if k_out is None:
            k_out, ko = _like(k), Hkv * hd
        else:
            ko = _rows("k_out", k_out, q, (rows, Hkv, hd))[3]
    ctx.check(lib().wq_rope(ctx.handle, _ptr(q), qs, _ptr(k), ks, _dtype_id(q), rows, Hq, Hkv, hd, 2 * half, layout, _ptr(positions),
                            _ptr(inv_freq), mscale, _ptr(q_out), qo, _ptr(k_out) if k is not None else None, ko))
    return q_out, k_out


def wq_rope_append_kv(ctx: Context, q, k, v, positions, inv_freq, kv: PackedKV, layout: int = ROPE_HALF, mscale: float = 1.0,
                      q_out: Optional[torch.Tensor] = None):
    """Turns q [B, Hq, hd] (returned) and k [B, Hkv, hd]; k and v become the cache's next rows."""
    _here(ctx, q, k, v, positions, inv_freq, q_out, kv.off16)
    B, Hq, hd, qs = _rows("q", q)
    shape = (B, kv.Hkv, kv.hd)
    if hd != kv.hd:
        raise ValueError("q: the head_dim of the cache expected")
    ks, vs = _rows("k", k, q, shape)[3], _rows("v", v, q, shape)[3]
    _contiguous("positions", positions, torch.int32, B)
    half = inv_freq.numel()
    _contiguous("inv_freq", inv_freq, torch.float32, half)
    if q_out is None:
        q_out, qo = _like(q), Hq * hd
    else:
        qo = _rows("q_out", q_out, q, (B, Hq, hd))[3]
    ctx.check(lib().wq_rope_append_kv(ctx.handle, _ptr(q), qs, _ptr(k), ks, _ptr(v), vs, _dtype_id(q), B, Hq, 2 * half, layout, _ptr(positions),
                                      _ptr(inv_freq), mscale, _ptr(q_out), qo, C.byref(kv.desc)))
    return q_out


def prefill_workspace_bytes(total_q: int, B: int, Hq: int, Hkv: int, hd: int, max_kv_rows: int, num_splits: int = 0) -> int:
    return int(lib().wq_prefill_workspace_bytes(total_q, B, Hq, Hkv, hd, max_kv_rows, num_splits))


def wq_prefill_attention(ctx: Context, q, k, v, q_off, kv_off, sm_scale: float, prefix_len: Optional[torch.Tensor] = None, max_kv_rows: int = 0,
                         num_splits: int = 0, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None):
    """q [total_q, Hq, hd] over k, v [total_kv, Hkv, hd]; q_off, kv_off [B+1], prefix_len [B] int32.  max_kv_rows 0: few rows get one part."""
    _here(ctx, q, k, v, q_off, kv_off, prefix_len, out, lse)
    total_q, Hq, hd, qs = _rows("q", q)
    total_kv, Hkv, k_hd, ks = _rows("k", k, q)
    if k_hd != hd:
        raise ValueError("k: the head_dim of q expected")
    vs = _rows("v", v, q, (total_kv, Hkv, hd))[3]
    B = q_off.numel() - 1
    _contiguous("q_off", q_off, torch.int32, B + 1)
    _contiguous("kv_off", kv_off, torch.int32, B + 1)
    if prefix_len is not None:
        _contiguous("prefix_len", prefix_len, torch.int32, B)
    if out is None:
        out = _like(q)
    else:
        _contiguous("out", out, q.dtype, q.numel())
    if lse is not None:
        _contiguous("lse", lse, torch.float32, total_q * Hq)
    ctx.check(lib().wq_prefill_attention(ctx.handle, _ptr(q), qs, _ptr(k), ks, _ptr(v), vs, _dtype_id(q), B, Hq, Hkv, hd, _ptr(q_off), _ptr(kv_off),
                                         _ptr(prefix_len), total_q, total_kv, max_kv_rows, sm_scale, num_splits, _ptr(out), _ptr(lse)))
    return out


def shared_workspace_bytes(B: int, P: int, Hq: int, Hkv: int, hd: int, max_prefix_tokens: int, max_own_tokens: int = 0, num_splits: int = 0) -> int:
    return int(lib().wq_shared_workspace_bytes(B, P, Hq, Hkv, hd, max_prefix_tokens, max_own_tokens, num_splits))


def wq_decode_attention_shared(ctx: Context, q, prefix: PackedKV, req_off, own: Optional[PackedKV], sm_scale: float, num_splits: int = 0,
                               max_prefix_tokens: int = 0, max_own_tokens: int = 0, out: Optional[torch.Tensor] = None,
                               lse: Optional[torch.Tensor] = None):
    """q [B, Hq, hd]; requests req_off[p] .. req_off[p+1]-1 share sequence p of prefix, request b has sequence b of own (or None).
    max_prefix_tokens 0: one part."""
    _here(ctx, q, req_off, out, lse, prefix.off16, None if own is None else own.off16)
    B, Hq, hd = q.shape
    if hd != prefix.hd:
        raise ValueError("q: the head_dim of the cache expected")
    _contiguous("q", q, q.dtype, q.numel())
    _contiguous("req_off", req_off, torch.int32, prefix.B + 1)
    if out is None:
        out = _like(q)
    else:
        _contiguous("out", out, q.dtype, q.numel())
    if lse is not None:
        _contiguous("lse", lse, torch.float32, B * Hq)
    ctx.check(lib().wq_decode_attention_shared(ctx.handle, _ptr(q), _dtype_id(q), B, Hq, C.byref(prefix.desc), _ptr(req_off),
                                               None if own is None else C.byref(own.desc), sm_scale, num_splits, max_prefix_tokens, max_own_tokens,
                                               _ptr(out), _ptr(lse)))
    return out


# ------------------------------------------------------------------------------------------------------------
# several new rows per sequence, copies of sequences
# ------------------------------------------------------------------------------------------------------------
def tree_workspace_bytes(total_rows: int, B: int, Hq: int, Hkv: int, hd: int, max_cache_tokens: int, max_rows: int, num_splits: int = 0) -> int:
    return int(lib().wq_tree_workspace_bytes(total_rows, B, Hq, Hkv, hd, max_cache_tokens, max_rows, num_splits))


def wq_tree_attention(ctx: Context, q, k, v, kv: PackedKV, row_off, sm_scale: float, parent: Optional[torch.Tensor] = None, max_rows: int = 0,
                      max_cache_tokens: int = 0, num_splits: int = 0, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None):
    """New rows q [rows, Hq, hd], k, v [rows, Hkv, hd], row_off[b] .. row_off[b+1]-1 those of sequence b, over its cache and each other: along
    parent [rows] (a tree; numbered within the sequence, -1: none), or every row the ones before it (None).  max_rows, max_cache_tokens 0: few parts."""
    _here(ctx, q, k, v, row_off, parent, out, lse, kv.off16)
    rows, Hq, hd, qs = _rows("q", q)
    if hd != kv.hd:
        raise ValueError("q: the head_dim of the cache expected")
    shape = (rows, kv.Hkv, hd)
    ks, vs = _rows("k", k, q, shape)[3], _rows("v", v, q, shape)[3]
    _contiguous("row_off", row_off, torch.int32, kv.B + 1)
    if parent is not None:
        _contiguous("parent", parent, torch.int32, rows)
    if out is None:
        out = _like(q)
    else:
        _contiguous("out", out, q.dtype, q.numel())
    if lse is not None:
        _contiguous("lse", lse, torch.float32, rows * Hq)
    ctx.check(lib().wq_tree_attention(ctx.handle, _ptr(q), qs, _ptr(k), ks, _ptr(v), vs, _dtype_id(q), kv.B, Hq, C.byref(kv.desc), _ptr(row_off), _ptr(parent),
                                      rows, max_rows, sm_scale, num_splits, max_cache_tokens, _ptr(out), _ptr(lse)))
    return out


def wq_tree_accept(ctx: Context, tokens, target, row_off, parent: Optional[torch.Tensor] = None, max_rows: int = 1024, max_path: int = 64):
    """(path [B, max_path], n_path [B], next_token [B]): the rows whose tokens the model agrees with, from every sequence's first row on."""
    _here(ctx, tokens, target, row_off, parent)
    rows, B = tokens.numel(), row_off.numel() - 1
    for name, t, n in (("tokens", tokens, rows), ("target", target, rows), ("row_off", row_off, B + 1)) + ((("parent", parent, rows),) if parent is not None else ()):
        _contiguous(name, t, torch.int32, n)
    path = torch.empty(B, max(max_path, 0), dtype=torch.int32, device=ctx.device)
    n_path, next_token = torch.empty(B, dtype=torch.int32, device=ctx.device), torch.empty(B, dtype=torch.int32, device=ctx.device)
    ctx.check(lib().wq_tree_accept(ctx.handle, _ptr(tokens), _ptr(target), _ptr(parent), B, _ptr(row_off), rows, max_rows, max_path, _ptr(path), _ptr(n_path),
                                   _ptr(next_token)))
    return path, n_path, next_token


# (Many layers: what is checked of every tensor is read by loops in C, 0.1 to 0.2 us each, and descriptors are joined as bytes.)
_dtype_of = operator.attrgetter("dtype")


def _layers_alike(ctx: Context, name: str, tensors: Sequence[torch.Tensor], like: torch.Tensor) -> int:
    """Every layer's rows like the first layer's keys, and like the first of their own in strides: elements from row to row."""
    n, first = len(tensors), tensors[0]
    stride = _rows(name, first, like, tuple(like.shape))[3]
    if [*map(torch.Tensor.size, tensors)] != [first.shape] * n or [*map(_dtype_of, tensors)] != [like.dtype] * n:
        raise ValueError(f"{name}: shapes or types of the layers' rows differ")
    if [*map(torch.Tensor.stride, tensors)] != [first.stride()] * n:        # (of a dimension of one they say nothing)
        for t in tensors:
            if _rows(name, t)[3] != stride and t.shape[0] > 1:
                raise ValueError(f"{name}: the layers' rows are not equally far apart")
    if [*map(torch.Tensor.get_device, tensors)] != [ctx.index] * n:
        raise ValueError(f"{name}: the context's device, cuda:{ctx.index}, expected")
    return stride


def _descs(ctx: Context, kvs: Sequence[PackedKV]) -> bytes:
    for kv in kvs:
        if kv.index != ctx.index:
            raise ValueError(f"a cache on another device than the context's, cuda:{ctx.index}")
    return b"".join([kv.desc for kv in kvs])


def wq_append_rows(ctx: Context, k: Sequence[torch.Tensor], v: Sequence[torch.Tensor], kv: Sequence[PackedKV], row_off, max_take: int,
                   take: Optional[torch.Tensor] = None, n_take: Optional[torch.Tensor] = None):
    """Layer l's rows k[l], v[l] [rows, Hkv, hd] into kv[l]: those that take [B, max_take] and n_take [B] name, or all of a sequence's (None)."""
    n = len(kv)
    if n == 0 or len(k) != n or len(v) != n:
        raise ValueError("k, v, kv: one of each for every layer expected")
    first, B = k[0], kv[0].B
    _here(ctx, row_off, take, n_take)
    ks, vs = _layers_alike(ctx, "k", k, first), _layers_alike(ctx, "v", v, first)
    rows, Hkv, hd = first.shape
    for c in kv:
        if c.Hkv != Hkv or c.hd != hd:
            raise ValueError("k: the KV heads and head_dim of the caches expected")
    _contiguous("row_off", row_off, torch.int32, B + 1)
    if (take is None) != (n_take is None):
        raise ValueError("take and n_take go together")
    if take is not None:
        _contiguous("take", take, torch.int32, B * max_take)
        _contiguous("n_take", n_take, torch.int32, B)
    pointers = C.c_void_p * n
    ctx.check(lib().wq_append_rows(ctx.handle, n, pointers(*map(torch.Tensor.data_ptr, k)), ks, pointers(*map(torch.Tensor.data_ptr, v)), vs, _dtype_id(first), B,
                                   _ptr(row_off), rows, _ptr(take), _ptr(n_take), max_take, _descs(ctx, kv)))


def wq_copy_sequences(ctx: Context, src: Sequence[PackedKV], dst: Sequence[PackedKV], from_seq):
    """Sequence d of every layer's dst becomes a copy of sequence from_seq[d] of that layer's src (-1: an empty one); src and dst share no memory."""
    if len(src) != len(dst) or not src:
        raise ValueError("src, dst: one of each for every layer expected")
    _here(ctx, from_seq)
    _contiguous("from_seq", from_seq, torch.int32, dst[0].B)
    ctx.check(lib().wq_copy_sequences(ctx.handle, len(src), _descs(ctx, src), _descs(ctx, dst), _ptr(from_seq)))


def wq_probe_mfma(ctx: Context, random_operands: bool, workgroups: int = 2048, iters: int = 1000) -> float:
    """Launches the matrix-core rate probe; returns the floating-point operations of the launch."""
    fl = C.c_double(0.0)
    ctx.check(lib().wq_probe_mfma(ctx.handle, int(random_operands), workgroups, iters, C.byref(fl)))
    return fl.value


def wq_probe_stream(ctx: Context, src: torch.Tensor, dst: Optional[torch.Tensor] = None, blocks: int = 4096):
    nbytes = src.numel() * src.element_size() // 16 * 16
    ctx.check(lib().wq_probe_stream(ctx.handle, src.data_ptr(), None if dst is None else dst.data_ptr(), nbytes, blocks))
    return nbytes
