"""Thin ctypes binding of ``liblvlm.so`` (declared in ``include/lvlm.h``).

Each function marshals torch CUDA tensors into the C call of the same name and returns the
output tensors; no step of the method runs in Python.  torch is used for device memory and
streams only.  There is no CPU path: a missing library or a non-CUDA tensor is an error.
"""
from __future__ import annotations

import ctypes
import math
import os
from typing import Optional

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_PKG, "liblvlm.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_ALIGNMENT, ERR_WORKSPACE, ERR_CUDA = range(6)
DEV_NONFINITE, DEV_TIMEOUT, DEV_BOUNDS = 1, 2, 4
W_LINEAR_RANK, W_GEOMETRIC, W_UNIFORM, W_CUSTOM, W_NEAREST_KEPT = range(5)
OP_SCORE_TOKENS, OP_SELECT_TOPK, OP_MERGE_COMPACT, OP_KV_COMPRESS, OP_DECODE_ATTN, OP_PREFILL_ATTN, OP_TREE_ATTN = range(7)

EXPORTS = ("lvlm_version", "lvlm_status_string", "lvlm_workspace_bytes", "lvlm_score_tokens",
           "lvlm_select_topk", "lvlm_merge_compact", "lvlm_kv_compress", "lvlm_decode_attn",
           "lvlm_decode_attn_static", "lvlm_prefill_attn", "lvlm_rope_append", "lvlm_commit_rows", "lvlm_tree_attn")
STATIC_SCRATCH_BYTES = 4 << 20


class Dims(ctypes.Structure):
    """Mirror of ``lvlm_dims``."""
    _fields_ = [(n, ctypes.c_int32) for n in
                ("B", "H", "Hkv", "D", "N", "C", "cap", "i0", "n", "k", "q_lo", "q_hi", "causal",
                 "recent", "merge_mode", "cache_stable")] + \
               [(n, ctypes.c_int64) for n in
                ("q_stride_b", "q_stride_n", "q_stride_h", "kv_stride_b", "kv_stride_h",
                 "hid_stride_b", "out_stride_b", "head_stride")] + \
               [(n, ctypes.c_int32) for n in
                ("T", "page", "n_pages", "max_pages", "draft_cap", "rot", "interleaved", "n_pos", "axes", "sect0", "sect1",
                 "count_heads", "mask_shared")] + \
               [(n, ctypes.c_int64) for n in
                ("new_stride_b", "new_stride_n", "new_stride_h", "page_stride", "draft_stride_b", "draft_stride_h")]


class LvlmError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {status_string(code)} (lvlm_status {code})")


_lib = None


def use_library(path: Optional[str]) -> None:
    """Makes the binding load another build of the library at its next use (the tests load the build
    with test hooks this way); None goes back to ``liblvlm.so``."""
    global _lib, _LIB_PATH
    _lib = None
    _LIB_PATH = path or os.path.join(_PKG, "liblvlm.so")


def lib() -> ctypes.CDLL:
    """The loaded library.  Raises if ``liblvlm.so`` has not been built (see build.py)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(
                f"{_LIB_PATH} is missing: build it with `python -m paper_2509_00419_b200.build` "
                "(there is no fallback implementation)")
        L = ctypes.CDLL(_LIB_PATH)
        vp, i32, i64, f32, sz = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float,
                                 ctypes.c_size_t)
        dp = ctypes.POINTER(Dims)
        L.lvlm_version.restype = ctypes.c_char_p
        L.lvlm_version.argtypes = []
        L.lvlm_status_string.restype = ctypes.c_char_p
        L.lvlm_status_string.argtypes = [ctypes.c_int]
        L.lvlm_workspace_bytes.restype = sz
        L.lvlm_workspace_bytes.argtypes = [ctypes.c_int, dp]
        L.lvlm_score_tokens.restype = ctypes.c_int
        L.lvlm_score_tokens.argtypes = [vp, vp, vp, dp, f32, vp, vp, vp, sz, vp, vp]
        L.lvlm_select_topk.restype = ctypes.c_int
        L.lvlm_select_topk.argtypes = [vp, i32, i32, i64, i32, vp, vp, vp, vp, sz, vp, vp]
        L.lvlm_merge_compact.restype = ctypes.c_int
        L.lvlm_merge_compact.argtypes = [vp, vp, vp, vp, vp, vp, dp, ctypes.c_int, vp, vp, vp, vp,
                                         sz, vp, vp]
        L.lvlm_kv_compress.restype = ctypes.c_int
        L.lvlm_kv_compress.argtypes = [vp, vp, vp, vp, vp, vp, vp, dp, f32, i32, vp, sz, vp, vp]
        L.lvlm_decode_attn.restype = ctypes.c_int
        L.lvlm_decode_attn.argtypes = [vp, vp, vp, vp, vp, vp, vp, dp, f32, vp, vp, sz, vp, vp]
        L.lvlm_decode_attn_static.restype = ctypes.c_int
        L.lvlm_decode_attn_static.argtypes = [vp, vp, vp, vp, vp, vp, vp, dp, f32, vp, vp, vp]
        L.lvlm_prefill_attn.restype = ctypes.c_int
        L.lvlm_prefill_attn.argtypes = [vp, vp, vp, dp, f32, vp, vp, vp, vp, vp, sz, vp, vp]
        L.lvlm_rope_append.restype = ctypes.c_int
        L.lvlm_rope_append.argtypes = [vp] * 14 + [dp, vp, vp]
        L.lvlm_commit_rows.restype = ctypes.c_int
        L.lvlm_commit_rows.argtypes = [vp] * 12 + [dp, vp, vp]
        L.lvlm_tree_attn.restype = ctypes.c_int
        L.lvlm_tree_attn.argtypes = [vp] * 9 + [dp, f32, vp, vp, vp, sz, vp, vp]
        _lib = L
    return _lib


def version() -> str:
    return lib().lvlm_version().decode()


def status_string(code: int) -> str:
    return lib().lvlm_status_string(int(code)).decode()


def workspace_bytes(op: int, dims: Dims) -> int:
    return int(lib().lvlm_workspace_bytes(int(op), ctypes.byref(dims)))


# The helpers below run for every argument of every call, so they hand plain ints to ctypes (the argtypes convert them;
# building c_void_p objects costs more than the conversion) and ask for the raw stream handle (0.1 us; the Stream object
# of torch.cuda.current_stream() takes 3 us to make).  Host time of a call around the library's own, before and now:
# score_tokens 10.2 -> 3.9 us, select_topk 5.7 -> 1.8 us, merge_compact 9.8 -> 5.6 us.
def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda:
        raise TypeError("lvlm works on CUDA tensors only; there is no CPU path")
    return t.data_ptr()


def _stream(stream) -> int:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream


def _check(code: int, where: str):
    if code != OK:
        raise LvlmError(code, where)


def alloc_workspace(op: int, dims: Dims, device) -> torch.Tensor:
    nbytes = max(workspace_bytes(op, dims), 256)
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _ws(ws, op, dims, device):
    if ws is None:
        ws = alloc_workspace(op, dims, device)
    return ws, ws.data_ptr(), ws.numel() * ws.element_size()


# ----------------------------------------------------------------------------------------------
def score_tokens(Q, K, *, N, i0, n, q_lo, q_hi, causal=True, scale=None, lse=None,
                 want_head=False, score_out=None, head_out=None, ws=None, dev_status=None,
                 stream=None):
    """lvlm_score_tokens.  Q [B,q_hi-q_lo,H,D] (a view with strides is fine), K [B,Hkv,cap,D].
    Returns (score [B,n], score_head [B,Hkv,n] or None)."""
    B, Nq, H, D = Q.shape
    Hkv, cap = K.shape[1], K.shape[2]
    d = Dims(B=B, H=H, Hkv=Hkv, D=D, N=N, cap=cap, i0=i0, n=n, q_lo=q_lo, q_hi=q_hi,
             causal=int(causal))
    d.q_stride_b, d.q_stride_n, d.q_stride_h, q_inner = Q.stride()
    d.kv_stride_b, d.kv_stride_h, k_row, k_inner = K.stride()
    assert q_inner == 1 and k_inner == 1 and k_row == D
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    score = score_out if score_out is not None else \
        torch.empty(B, n, dtype=torch.float32, device=Q.device)
    head = head_out
    if head is None and want_head:
        head = torch.empty(B, Hkv, n, dtype=torch.float32, device=Q.device)
    if head is not None:
        assert head.stride(2) == 1 and head.stride(0) == Hkv * head.stride(1)
        d.head_stride = head.stride(1)
    ws, wsp, wsn = _ws(ws, OP_SCORE_TOKENS, d, Q.device)
    _check(lib().lvlm_score_tokens(_ptr(Q), _ptr(K), _ptr(lse), ctypes.byref(d),
                                   scale, _ptr(score), _ptr(head), wsp, wsn,
                                   _ptr(dev_status), _stream(stream)), "lvlm_score_tokens")
    return score, head


def prefill_attn(Q, K, V, *, N, causal=True, scale=None, window=None, i0=0, n=0, want_head=False,
                 out=None, lse=None, score_out=None, head_out=None, ws=None, dev_status=None, stream=None):
    """lvlm_prefill_attn.  Q [B,N,H,D], K, V [B,Hkv,cap,D].  Returns (out [B,N,H,D] bf16, lse [B,H,N],
    score [B,n] or None, score_head [B,Hkv,n] or None); the scores are asked for with
    ``window=(q_lo, q_hi)`` and the image span ``i0, n``."""
    B, Nq, H, D = Q.shape
    Hkv, cap = K.shape[1], K.shape[2]
    assert Nq == N and Q.stride(3) == 1 and K.stride(3) == 1 and K.stride(2) == D and V.stride() == K.stride()
    d = Dims(B=B, H=H, Hkv=Hkv, D=D, N=N, cap=cap, causal=int(causal))
    d.q_stride_b, d.q_stride_n, d.q_stride_h = Q.stride(0), Q.stride(1), Q.stride(2)
    d.kv_stride_b, d.kv_stride_h = K.stride(0), K.stride(1)
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    if out is None:
        out = torch.empty(B, N, H, D, dtype=Q.dtype, device=Q.device)
    if lse is None:
        lse = torch.empty(B, H, N, dtype=torch.float32, device=Q.device)
    score = head = None
    wsp, wsn = None, 0
    if window is not None:
        d.q_lo, d.q_hi, d.i0, d.n = window[0], window[1], i0, n
        score = score_out if score_out is not None else torch.empty(B, n, dtype=torch.float32, device=Q.device)
        head = head_out
        if head is None and want_head:
            head = torch.empty(B, Hkv, n, dtype=torch.float32, device=Q.device)
        if head is not None:
            assert head.stride(2) == 1 and head.stride(0) == Hkv * head.stride(1)
            d.head_stride = head.stride(1)
        ws, wsp, wsn = _ws(ws, OP_PREFILL_ATTN, d, Q.device)
    _check(lib().lvlm_prefill_attn(_ptr(Q), _ptr(K), _ptr(V), ctypes.byref(d), scale, _ptr(out),
                                   _ptr(lse), _ptr(score), _ptr(head), wsp, wsn, _ptr(dev_status),
                                   _stream(stream)), "lvlm_prefill_attn")
    return out, lse, score, head


def select_topk(score, k, *, want_kept=True, want_near=False, rank_out=None, kept_out=None,
                dev_status=None, stream=None):
    """lvlm_select_topk.  score [B,n] fp32 (row stride may exceed n).
    Returns (rank [B,n], kept_idx [B,k] or None, near_tie [B] or None)."""
    B, n = score.shape
    assert score.stride(1) == 1
    rank = rank_out if rank_out is not None else \
        torch.empty(B, n, dtype=torch.int32, device=score.device)
    kept = kept_out
    if kept is None and want_kept:
        kept = torch.empty(B, k, dtype=torch.int32, device=score.device)
    near = torch.empty(B, dtype=torch.int32, device=score.device) if want_near else None
    _check(lib().lvlm_select_topk(_ptr(score), B, n, score.stride(0), k, _ptr(rank), _ptr(kept),
                                  _ptr(near), None, 0, _ptr(dev_status), _stream(stream)),
           "lvlm_select_topk")
    return rank, kept, near


def merge_dims(hidden, rank, *, i0, k, Kc=None) -> Dims:
    B, N, C = hidden.shape
    n = rank.shape[1]
    d = Dims(B=B, N=N, C=C, i0=i0, n=n, k=k, D=128)
    d.hid_stride_b = hidden.stride(0)
    if Kc is not None:
        d.Hkv, d.cap, d.D = Kc.shape[1], Kc.shape[2], Kc.shape[3]
        d.kv_stride_b, d.kv_stride_h = Kc.stride(0), Kc.stride(1)
    return d


def merged_rows(N, n, k, mode=W_LINEAR_RANK) -> int:
    """Rows of a sequence after lvlm_merge_compact."""
    if mode == W_NEAREST_KEPT:
        return N - (n - k)
    return N - max(n - k - 1, 0)


def merge_compact(hidden, rank, *, i0, k, mode=W_LINEAR_RANK, Kc=None, Vc=None, pos_ids=None,
                  w_custom=None, mass=None, in_place=False, out=None, new_len=None, ws=None,
                  dev_status=None, stream=None):
    """lvlm_merge_compact.  Returns (hidden_out or the compacted `hidden`, new_len [B]).
    With in_place=True `hidden` is compacted in place and its first new_len rows are valid.
    Kc, Vc and pos_ids are always compacted in place."""
    B, N, C = hidden.shape
    n = rank.shape[1]
    d = merge_dims(hidden, rank, i0=i0, k=k, Kc=Kc)
    d.merge_mode = int(mode)
    rows = merged_rows(N, n, k, mode)
    if in_place:
        out = None
    elif out is None:
        out = torch.empty(B, rows, C, dtype=hidden.dtype, device=hidden.device)
    if out is not None:
        d.out_stride_b = out.stride(0)
    if new_len is None:
        new_len = torch.empty(B, dtype=torch.int32, device=hidden.device)
    ws, wsp, wsn = _ws(ws, OP_MERGE_COMPACT, d, hidden.device)
    _check(lib().lvlm_merge_compact(_ptr(hidden), _ptr(out), _ptr(Kc), _ptr(Vc), _ptr(pos_ids),
                                    _ptr(rank), ctypes.byref(d), int(mode), _ptr(w_custom),
                                    _ptr(mass), _ptr(new_len), wsp, wsn, _ptr(dev_status),
                                    _stream(stream)), "lvlm_merge_compact")
    return (hidden if in_place else out), new_len


def nearest_assignment(ws: torch.Tensor, B: int, r: int) -> torch.Tensor:
    """Assignment lvlm_merge_compact leaves at the start of its workspace in mode NEAREST_KEPT:
    [B, r] int32, for the dropped tokens in ascending order the index of their kept token."""
    return ws[:B * r * 4].view(torch.int32).view(B, r)


def kv_dims(Kc, *, H=None, recent=0, max_len=None) -> Dims:
    B, Hkv, cap, D = Kc.shape
    d = Dims(B=B, Hkv=Hkv, H=H if H is not None else Hkv, D=D, N=max_len or 0, cap=cap, recent=recent)
    d.kv_stride_b, d.kv_stride_h = Kc.stride(0), Kc.stride(1)
    return d


def kv_compress(Kc, Vc, acc_score, length, *, beta=1.0, budget=0, recent=0, e_lo=None, e_hi=None,
                pos=None, ws=None, dev_status=None, stream=None):
    """lvlm_kv_compress: everything is updated in place (Kc, Vc, acc_score, pos, length)."""
    d = kv_dims(Kc, recent=recent)
    ws, wsp, wsn = _ws(ws, OP_KV_COMPRESS, d, Kc.device)
    _check(lib().lvlm_kv_compress(_ptr(Kc), _ptr(Vc), _ptr(acc_score), _ptr(pos), _ptr(length),
                                  _ptr(e_lo), _ptr(e_hi), ctypes.byref(d), float(beta),
                                  int(budget), wsp, wsn, _ptr(dev_status), _stream(stream)),
           "lvlm_kv_compress")


def decode_attn(q, Kc, Vc, length, *, k_new=None, v_new=None, acc_score=None, scale=None, out=None,
                ws=None, dev_status=None, stream=None, cache_stable=False, max_len=None):
    """lvlm_decode_attn.  q [B,H,D]; returns out [B,H,D] bf16.  Kc, Vc, length and acc_score are
    updated in place when k_new/v_new or acc_score are given.  max_len: rows a head is expected to hold at most, where the
    caller knows (it decides the form of the kernel, not the result)."""
    B, H, D = q.shape
    d = kv_dims(Kc, H=H, max_len=max_len)
    d.cache_stable = int(bool(cache_stable))
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    if out is None:
        out = torch.empty(B, H, D, dtype=q.dtype, device=q.device)
    ws, wsp, wsn = _ws(ws, OP_DECODE_ATTN, d, q.device)
    _check(lib().lvlm_decode_attn(_ptr(q), _ptr(Kc), _ptr(Vc), _ptr(length), _ptr(k_new),
                                  _ptr(v_new), _ptr(acc_score), ctypes.byref(d),
                                  scale, _ptr(out), wsp, wsn, _ptr(dev_status),
                                  _stream(stream)), "lvlm_decode_attn")
    return out


def decode_attn_static(q, Kc, Vc, length, *, k_new=None, v_new=None, acc_score=None, scale=None,
                       out=None, dev_status=None, stream=None, max_len=None):
    """lvlm_decode_attn_static: lvlm_decode_attn for callers that have no way to get device
    scratch memory (all of it belongs to someone else's pool, or allocating would stall the
    device).  The scratch is a fixed array inside the library, at most STATIC_SCRATCH_BYTES per
    problem, shared by every call on the device: calls must not overlap on the GPU.  ``out`` is
    required to come from the caller as well when nothing may be allocated; it is created here
    only as a convenience when omitted."""
    B, H, D = q.shape
    d = kv_dims(Kc, H=H, max_len=max_len)
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    if out is None:
        out = torch.empty(B, H, D, dtype=q.dtype, device=q.device)
    _check(lib().lvlm_decode_attn_static(_ptr(q), _ptr(Kc), _ptr(Vc), _ptr(length), _ptr(k_new),
                                         _ptr(v_new), _ptr(acc_score), ctypes.byref(d),
                                         scale, _ptr(out), _ptr(dev_status),
                                         _stream(stream)), "lvlm_decode_attn_static")
    return out


# ---- several new tokens at a time, and paged caches -------------------------------------------
# A cache is contiguous, [B,Hkv,cap,D] (table None), or paged, [n_pages,page,D] with table [B,Hkv,max_pages] int32.
_BF16, _I32, _F32 = torch.bfloat16, torch.int32, torch.float32


def _refuse(t: torch.Tensor, name: str, dtype, shape, device: int, rows: bool):
    """Says what is wrong with an argument."""
    if not t.is_cuda:
        raise TypeError("lvlm works on CUDA tensors only; there is no CPU path")
    if t.dtype != dtype:
        raise TypeError(f"{name} has to be {dtype}, not {t.dtype}")
    if t.get_device() != device:
        raise ValueError(f"{name} is on {t.device}, the current device is cuda:{device}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} has to have the shape {tuple(shape)}, not {tuple(t.shape)}")
    raise ValueError(f"{name} has to be " + ("contiguous in its last dimension" if rows else "contiguous"))


# One comparison an argument on the way through: of 11 to 13 us of host time a call the C entry takes 3.4 (appends) to 4.3 (attention).
def _arg(t: Optional[torch.Tensor], name: str, dtype, shape, device: int):
    """Pointer of an optional contiguous argument after the checks that the C call cannot make."""
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != device or (shape is not None and t.shape != shape) or not t.is_contiguous():
        _refuse(t, name, dtype, shape, device, False)
    return t.data_ptr()


def _pair(K: torch.Tensor, V: torch.Tensor, names, D: int, device: int):
    """Shape, strides and pointers of two bf16 tensors laid out alike, of which only the rows of D channels have to be contiguous."""
    shape, st = K.shape, K.stride()
    if (K.dtype is not _BF16 or V.dtype is not _BF16 or K.get_device() != device or V.get_device() != device or V.shape != shape
            or V.stride() != st or st[-1] != 1 or shape[-1] != D):
        for t, name in zip((K, V), names):
            if t.dtype != _BF16 or t.get_device() != device or t.shape != shape or t.stride(-1) != 1:
                _refuse(t, name, _BF16, shape, device, True)
        if shape[-1] != D:
            raise ValueError(f"{names[0]} has rows of {shape[-1]} channels, the other tensors of {D}")
        raise ValueError(f"{names[0]} and {names[1]} have to have the same strides")
    return shape, st, K.data_ptr(), V.data_ptr()


def _queries(d: Dims, q: torch.Tensor, shape, device: int):
    """Pointer of the queries [B,T,H,D], whose rows of D channels have to be contiguous; fills their strides."""
    st = q.stride()
    if q.dtype is not _BF16 or q.get_device() != device or q.shape != shape or st[3] != 1:
        _refuse(q, "q", _BF16, shape, device, True)
    d.q_stride_b, d.q_stride_n, d.q_stride_h = _outer(q, "q", st, 3)
    return q.data_ptr()


def _outer(t: torch.Tensor, name: str, strides, n: int):
    """The first n strides (2 or 3) for the C call: 0 (packed) for a dimension of one element, whose stride means nothing."""
    a, b, c = strides[0], strides[1], strides[n - 1]
    if a and b and c and not (a | b | c) & 7:
        return strides[:n]
    st = tuple([x if size > 1 else 0 for x, size in zip(strides[:n], t.shape)])
    if any(x == 0 and size > 1 for x, size in zip(st, t.shape)):
        raise ValueError(f"{name} repeats its elements along a dimension (an expanded view)")
    return st


def _packed(names, shape, st):
    if st[-2] != shape[-1] and shape[-2] > 1:
        raise ValueError(f"the rows of {names[0]} and {names[1]} have to be packed")


def _cache(d: Dims, Kc, Vc, table, B, Hkv, D, device: int):
    """Fills the cache's fields of ``d``; returns the three pointers."""
    shape, st, kp, vp = _pair(Kc, Vc, ("Kc", "Vc"), D, device)
    _packed(("Kc", "Vc"), shape, st)
    if table is None:
        if len(shape) != 4 or shape[0] != B or shape[1] != Hkv:
            raise ValueError(f"a contiguous cache has the shape [{B}, {Hkv}, cap, D], not {tuple(shape)}")
        d.cap = shape[2]
        d.kv_stride_b, d.kv_stride_h = _outer(Kc, "Kc", st, 2)
        return kp, vp, None
    t_shape = table.shape
    if len(shape) != 3 or len(t_shape) != 3:
        raise ValueError("a paged cache has the shape [n_pages, page, D], its table [B, Hkv, max_pages]")
    d.n_pages, d.page, _ = shape
    d.page_stride = st[0] if st[0] and not st[0] & 7 else _outer(Kc, "Kc", st, 2)[0]
    d.max_pages = n = t_shape[2]
    return kp, vp, _arg(table, "table", _I32, (B, Hkv, n), device)


def _drafts(d: Dims, Kd, Vd, B, Hkv, D, device: int):
    """The same for a draft cache [B,Hkv,draft_cap,D]."""
    if Kd is None or Vd is None:
        raise ValueError("Kd and Vd go together")
    shape, st, kp, vp = _pair(Kd, Vd, ("Kd", "Vd"), D, device)
    if len(shape) != 4 or shape[0] != B or shape[1] != Hkv:
        raise ValueError(f"a draft cache has the shape [{B}, {Hkv}, rows, D], not {tuple(shape)}")
    _packed(("Kd", "Vd"), shape, st)
    d.draft_cap = shape[2]
    d.draft_stride_b, d.draft_stride_h = _outer(Kd, "Kd", st, 2)
    return kp, vp


def _here(t: torch.Tensor) -> int:
    """The current device, on which every tensor has to be."""
    if not t.is_cuda:
        raise TypeError("lvlm works on CUDA tensors only; there is no CPU path")
    return torch._C._cuda_getDevice()


def _new(make, stream):
    """What ``make`` allocates, on the stream that will use it: memory of the current stream may still be read there, and is handed
    out again there as soon as it is freed."""
    if stream is None:
        return make()
    with torch.cuda.stream(stream):
        return make()


def rope_table(n_pos: int, rot: int = 128, base: float = 10000.0, device="cuda") -> torch.Tensor:
    """cos_sin [n_pos, rot] fp32 for ``rope_append``: cosines of the rot/2 frequencies base^(-2i/rot), then their sines.
    The angles are formed in 64 bits: in 32 an angle of position p is off by p 2^-24 radians."""
    freq = torch.tensor(base, dtype=torch.float64) ** (torch.arange(0, rot, 2, dtype=torch.float64) / -rot)
    angle = torch.arange(n_pos, dtype=torch.float64)[:, None] * freq
    return torch.cat([angle.cos(), angle.sin()], 1).to(_F32).to(device)


def tree_mask(parents: torch.Tensor) -> torch.Tensor:
    """Mask words for ``tree_attn`` of trees given by their parents [..., T]: draft t (parent < t, negative = the last token of
    the cache) sees itself and what it descends from.  Returns [..., T, ceil(T/32)] int32 on the device of ``parents``."""
    T, lead = parents.shape[-1], parents.shape[:-1]
    par = parents.reshape(-1, T).cpu().tolist()
    W = (T + 31) // 32
    words = []
    for row in par:
        seen = []
        for t, p in enumerate(row):
            if p >= t:
                raise ValueError(f"the parent of draft {t} is {p}: parents come before their children")
            seen.append((seen[p] if p >= 0 else 0) | 1 << t)
        words += [[(x >> (32 * w)) & 0xFFFFFFFF for w in range(W)] for x in seen]
    m = torch.tensor(words, dtype=torch.int64).reshape(*lead, T, W)
    return torch.where(m >= 1 << 31, m - (1 << 32), m).to(torch.int32).to(parents.device)


def rope_append(k_new, v_new, pos, cos_sin, Kc, Vc, length=None, *, q=None, q_out=None, table=None, count=None, len_out=None,
                sections=None, interleaved=False, acc_score=None, pos_cache=None, dev_status=None, stream=None):
    """lvlm_rope_append.  k_new, v_new [B,T,Hkv,D] and q [B,T,H,D] (views with strides are fine) are rotated by
    cos_sin[pos] and k_new, v_new are appended behind ``length`` [B,Hkv], which grows by ``count`` [B] (None = T): in place, or
    into ``len_out``.  length None: the rows start at 0 (a draft cache), and no length is written unless len_out is given.
    pos is [B,T], or [3,B,T] with ``sections`` (the frequencies that follow each axis); cos_sin None: nothing is rotated.
    Returns q_out [B,T,H,D] (``q_out=q`` rotates in place) or None without q."""
    dev = _here(k_new)
    B, T, Hkv, D = k_new.shape
    _, st, knp, vnp = _pair(k_new, v_new, ("k_new", "v_new"), D, dev)
    d = Dims()
    d.B, d.Hkv, d.D, d.T, d.interleaved = B, Hkv, D, T, bool(interleaved)
    kp, vp, tp = _cache(d, Kc, Vc, table, B, Hkv, D, dev)
    d.new_stride_b, d.new_stride_n, d.new_stride_h = _outer(k_new, "k_new", st, 3)
    qp = qop = None
    if q is not None:
        d.H = H = q.shape[2]
        q_shape = (B, T, H, D)
        qp = _queries(d, q, q_shape, dev)
        if q_out is q:
            qop = qp
        else:
            if q_out is None:
                q_out = _new(lambda: torch.empty(q_shape, dtype=_BF16, device=q.device), stream)
            qop = _arg(q_out, "q_out", _BF16, q_shape, dev)
            if qop == qp and q_out.stride() != q.stride():
                raise ValueError("q_out starts where q does but is laid out differently")
    elif q_out is not None:
        raise ValueError("q_out without q")
    if cos_sin is not None:
        d.n_pos, d.rot = cos_sin.shape
    pos_shape = (B, T)
    if sections is not None:
        if len(sections) != 3 or sum(sections) != d.rot // 2:
            raise ValueError(f"sections {tuple(sections)} do not share out {d.rot // 2} frequencies")
        d.axes, d.sect0, d.sect1 = 3, sections[0], sections[1]
        pos_shape = (3, B, T)
    hs = (B, Hkv)
    lp = _arg(length, "length", _I32, hs, dev)
    ap = pcp = None
    if acc_score is not None or pos_cache is not None:
        side = (B, Hkv, d.cap or d.page * d.max_pages)
        ap, pcp = _arg(acc_score, "acc_score", _F32, side, dev), _arg(pos_cache, "pos_cache", _I32, side, dev)
    _check(lib().lvlm_rope_append(
        qp, knp, vnp, _arg(pos, "pos", _I32, pos_shape, dev), _arg(cos_sin, "cos_sin", _F32, None, dev),
        _arg(count, "count", _I32, (B,), dev), qop, kp, vp, tp, lp, lp if len_out is None else _arg(len_out, "len_out", _I32, hs, dev),
        ap, pcp, ctypes.byref(d), _arg(dev_status, "dev_status", _I32, None, dev), torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream), "lvlm_rope_append")
    return q_out


def commit_rows(Kd, Vd, Kc, Vc, length, count=None, *, index=None, table=None, len_out=None, pos=None, acc_score=None,
                pos_cache=None, dev_status=None, stream=None):
    """lvlm_commit_rows.  Rows index[b,i] of Kd, Vd [B,Hkv,draft_cap,D] are appended to a cache behind ``length`` [B,Hkv], which
    grows by ``count``: in place, or into ``len_out``.  count [B] (None = all) or, to move a ragged cache, [B,Hkv];
    index [B,T] int32, None = the first rows."""
    dev = _here(Kd)
    B, Hkv, rows, D = Kd.shape
    T = rows if index is None else index.shape[-1]
    d = Dims()
    d.B, d.Hkv, d.D, d.T = B, Hkv, D, T
    kp, vp, tp = _cache(d, Kc, Vc, table, B, Hkv, D, dev)
    kdp, vdp = _drafts(d, Kd, Vd, B, Hkv, D, dev)
    hs = (B, Hkv)
    d.count_heads = count is not None and count.dim() == 2
    lp = _arg(length, "length", _I32, hs, dev)
    ap = pcp = None
    if acc_score is not None or pos_cache is not None:
        side = (B, Hkv, d.cap or d.page * d.max_pages)
        ap, pcp = _arg(acc_score, "acc_score", _F32, side, dev), _arg(pos_cache, "pos_cache", _I32, side, dev)
    _check(lib().lvlm_commit_rows(
        kdp, vdp, _arg(index, "index", _I32, (B, T), dev), _arg(count, "count", _I32, hs if d.count_heads else (B,), dev),
        _arg(pos, "pos", _I32, (B, rows), dev), kp, vp, tp, lp, lp if len_out is None else _arg(len_out, "len_out", _I32, hs, dev),
        ap, pcp, ctypes.byref(d), _arg(dev_status, "dev_status", _I32, None, dev), torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream), "lvlm_commit_rows")


def tree_dims(q, Kc, table=None, Kd=None, *, max_len=None) -> Dims:
    """Sizes for ``alloc_workspace(OP_TREE_ATTN, ...)``."""
    B, T, H, D = q.shape
    d = Dims(B=B, H=H, T=T, D=D, N=max_len or 0)
    if table is None:
        d.Hkv, d.cap = Kc.shape[1], Kc.shape[2]
    else:
        d.Hkv, d.n_pages, d.page, d.max_pages = table.shape[1], Kc.shape[0], Kc.shape[1], table.shape[2]
    if Kd is not None:
        d.draft_cap = Kd.shape[2]
    return d


def tree_attn(q, Kc, Vc, length, *, Kd=None, Vd=None, mask=None, count=None, table=None, scale=None, out=None, lse=None,
              want_lse=False, max_len=None, ws=None, dev_status=None, stream=None):
    """lvlm_tree_attn.  q [B,T,H,D] (a view with strides is fine) attends to ``length`` [B,Hkv] rows of a cache and to the
    drafts Kd, Vd [B,Hkv,>=T,D] that ``mask`` lets it see ([B,T,W] or [T,W] int32 words from ``tree_mask``; None = a chain).  count
    [B]: drafts of each sequence (None = T).  max_len: rows a head is expected to hold at most, where the caller knows (it decides
    how the work is split, not the result).  out may be q itself where q is contiguous.  Returns (out [B,T,H,D], lse [B,H,T] or None);
    rows behind count are left as they were."""
    dev = _here(q)
    shape = q.shape
    B, T, H, D = shape
    Hkv = Kc.shape[1] if table is None else table.shape[1]
    d = Dims()
    d.B, d.H, d.Hkv, d.D, d.T, d.N = B, H, Hkv, D, T, max_len or 0
    qp = _queries(d, q, shape, dev)
    kp, vp, tp = _cache(d, Kc, Vc, table, B, Hkv, D, dev)
    kdp = vdp = None
    if Kd is not None or Vd is not None:
        kdp, vdp = _drafts(d, Kd, Vd, B, Hkv, D, dev)
    mp = None
    if mask is not None:
        W = (T + 31) // 32
        d.mask_shared = mask.dim() == 2
        mp = _arg(mask, "mask", _I32, (T, W) if d.mask_shared else (B, T, W), dev)
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    if out is None:
        out = _new(lambda: torch.empty(B, T, H, D, dtype=_BF16, device=q.device), stream)
    if lse is None and want_lse:
        lse = _new(lambda: torch.empty(B, H, T, dtype=_F32, device=q.device), stream)
    if ws is None:
        ws = _new(lambda: alloc_workspace(OP_TREE_ATTN, d, q.device), stream)
    elif ws.get_device() != dev:
        raise ValueError(f"ws is on {ws.device}, the current device is cuda:{dev}")
    _check(lib().lvlm_tree_attn(qp, kp, vp, tp, _arg(length, "length", _I32, (B, Hkv), dev), kdp, vdp, mp,
                                _arg(count, "count", _I32, (B,), dev), ctypes.byref(d), scale, _arg(out, "out", _BF16, shape, dev),
                                _arg(lse, "lse", _F32, (B, H, T), dev), ws.data_ptr(), ws.numel() * ws.element_size(),
                                _arg(dev_status, "dev_status", _I32, None, dev), torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream), "lvlm_tree_attn")
    return out, lse
