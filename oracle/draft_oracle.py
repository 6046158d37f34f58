"""CPU oracle for decoding several drafted tokens at a time: rotation and append, tree attention, commit of rows.

TEST INFRASTRUCTURE ONLY, like ``lvlm_oracle``.  float64 throughout; what a caller rounds once to bf16 is returned unrounded here.
Caches are logical, [B][Hkv][cap][D]; ``to_pages`` / ``from_pages`` lay one out in pages and back.
Pins (tests/test_drafts_host.py): a rotation keeps norms and makes q . k a function of the distance; a chain over an empty cache is
the causal attention of ``lvlm_oracle``; one draft is its decode attention; a tree's node is a decode step over its path.
"""
from __future__ import annotations

import numpy as np


def rotate(x, pos, cos_sin, interleaved=False, sections=None):
    """x [B, T, heads, D], pos [B, T] or [3, B, T] with sections, cos_sin [n_pos, rot].  An angle whose position is outside the
    table is zero."""
    y = np.array(x, dtype=np.float64)
    rot = cos_sin.shape[1]
    h = rot // 2
    for f in range(h):
        axis = 0 if sections is None else int(f >= sections[0]) + int(f >= sections[0] + sections[1])
        p = pos if sections is None else pos[axis]
        ok = (p >= 0) & (p < cos_sin.shape[0])
        c = np.where(ok, cos_sin[np.where(ok, p, 0), f].astype(np.float64), 1.0)[:, :, None]
        s = np.where(ok, cos_sin[np.where(ok, p, 0), h + f].astype(np.float64), 0.0)[:, :, None]
        i, j = (2 * f, 2 * f + 1) if interleaved else (f, f + h)
        a, b = np.array(x[..., i], np.float64), np.array(x[..., j], np.float64)
        y[..., i], y[..., j] = a * c - b * s, b * c + a * s
    return y


def append(K, V, length, k_new, v_new, count):
    """Rows k_new, v_new [B, T, Hkv, D] behind length [B, Hkv]; a head whose rows do not fit stays as it is."""
    K, V, length = np.array(K), np.array(V), np.array(length)
    for b in range(K.shape[0]):
        for g in range(K.shape[1]):
            n, ln = int(count[b]), int(length[b, g])
            if n < 0 or n > k_new.shape[1] or ln < 0 or ln + n > K.shape[2]:
                continue
            K[b, g, ln:ln + n], V[b, g, ln:ln + n] = k_new[b, :n, g], v_new[b, :n, g]
            length[b, g] = ln + n
    return K, V, length


def commit(K, V, length, Kd, Vd, index, count):
    """Rows index[b] (None = the first) of Kd, Vd [B, Hkv, rows, D]; count [B] or [B, Hkv]."""
    K, V, length = np.array(K), np.array(V), np.array(length)
    count = np.asarray(count)
    for b in range(K.shape[0]):
        for g in range(K.shape[1]):
            n, ln = int(count[b] if count.ndim == 1 else count[b, g]), int(length[b, g])
            if n < 0 or ln < 0 or ln + n > K.shape[2]:
                continue
            at = np.arange(n) if index is None else index[b, :n]
            K[b, g, ln:ln + n], V[b, g, ln:ln + n] = Kd[b, g, at], Vd[b, g, at]
            length[b, g] = ln + n
    return K, V, length


def tree_attn(q, K, V, length, Kd, Vd, see, count, scale=None):
    """q [B, T, H, D]; see [B, T, T] truth values.  Returns (out [B, T, H, D], lse [B, H, T]); rows behind count are NaN."""
    q = np.asarray(q, np.float64)
    B, T, H, D = q.shape
    Hkv = K.shape[1]
    scale = 1.0 / np.sqrt(D) if scale is None else scale
    out, lse = np.full((B, T, H, D), np.nan), np.full((B, H, T), np.nan)
    for b in range(B):
        n = int(count[b])
        for h in range(H):
            g = h // (H // Hkv)
            ln = int(length[b, g])
            for t in range(n):
                keys, vals = np.asarray(K[b, g, :ln], np.float64), np.asarray(V[b, g, :ln], np.float64)
                if Kd is not None:
                    u = np.flatnonzero(see[b, t, :n])
                    keys, vals = np.concatenate([keys, Kd[b, g, u]]), np.concatenate([vals, Vd[b, g, u]])
                if not len(keys):
                    out[b, t, h], lse[b, h, t] = 0.0, -np.inf
                    continue
                x = keys @ q[b, t, h] * scale
                e = np.exp(x - x.max())
                out[b, t, h] = e @ vals / e.sum()
                lse[b, h, t] = x.max() + np.log(e.sum())
    return out, lse


def to_pages(K, V, page, table, n_pages, fill=np.nan):
    """A logical cache in pages: table [B][Hkv][max_pages]; what belongs to no head is `fill`."""
    B, Hkv, cap, D = K.shape
    kp, vp = np.full((n_pages, page, D), fill), np.full((n_pages, page, D), fill)
    for b in range(B):
        for g in range(Hkv):
            for j in range(cap):
                kp[table[b, g, j // page], j % page] = K[b, g, j]
                vp[table[b, g, j // page], j % page] = V[b, g, j]
    return kp, vp


def from_pages(kp, table, cap):
    page = kp.shape[1]
    j = np.arange(cap)
    return kp[table[:, :, j // page], j % page]
