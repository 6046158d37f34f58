"""Measured cases of the operators for decoding several drafted tokens at a time over ragged, paged caches.

``rope_append`` rotates new queries and keys by their positions and appends keys and values to a cache,
``tree_attn`` is the attention of a tree of drafted tokens over a cache, ``commit_rows`` appends chosen rows
of a contiguous cache (the accepted drafts, or a whole compressed cache) to another one.  A cache is
contiguous, ``[B][Hkv][cap][128]``, or paged, ``[pages][page][128]`` with a page table per (sequence, KV head).

``run`` computes them in plain torch, or, where ``own`` is set, by the library's calls.  Head layouts and
lengths are those of the 7B-, 8B- and 26B-class workloads of this repository.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

D = 128
HEADS = {"small": (8, 8), "7b": (28, 4), "8b": (32, 8), "26b": (48, 8)}
BASE = 1e6                   # of the rotation's frequencies


def _append(name, heads, B, T, rows, page, rot=128, axes=1, interleaved=False, ragged=False):
    return dict(name=name, kind="append", heads=heads, B=B, T=T, rows=rows, page=page, rot=rot, axes=axes, interleaved=interleaved, ragged=ragged)


def _tree(name, heads, B, T, rows, page, mask="tree", ragged=False):
    return dict(name=name, kind="tree", heads=heads, B=B, T=T, rows=rows, page=page, mask=mask, ragged=ragged)


def _commit(name, heads, B, T, rows, page, pack=False):
    return dict(name=name, kind="commit", heads=heads, B=B, T=T, rows=rows, page=page, pack=pack)


def listed():
    return [
        # One generated token of one sequence on the 7B class, its layer's cache in pages: nothing but latency.
        _append("append_token", "7b", 1, 1, 1100, 64),
        # Trees of drafted tokens of eight sequences, not all of them full, into their own small contiguous caches.
        _append("append_drafts", "8b", 8, 26, 0, 0, ragged=True),
        # Sixteen prompts of the 8B class entering small pages behind a shared system prompt, three position axes, padded.
        _append("append_prompts", "8b", 16, 1888, 35, 16, axes=3, ragged=True),
        # One long prompt of the 26B class into a contiguous cache, half of the channels rotated, neighbours paired.
        _append("append_long", "26b", 1, 16640, 0, 0, rot=64, interleaved=True),
        # One token over the short ragged cache that token reduction leaves (contiguous).
        _tree("tree_token", "7b", 1, 1, 216, 0, ragged=True),
        # Five tokens in a row for eight sequences near the cache budget, in pages.
        _tree("tree_chain", "8b", 8, 5, 1100, 64, mask="chain", ragged=True),
        # A tree of 26 drafts over an uncompressed prompt in small pages.
        _tree("tree_prompt", "7b", 1, 26, 3008, 16),
        # Trees of up to 61 drafts for sixteen requests: between memory and tensor cores.
        _tree("tree_batch", "8b", 16, 61, 1888, 64, ragged=True),
        # A small tree over a video prompt's cache that is not compressed: one sequence, four heads, long.
        _tree("tree_video", "7b", 1, 13, 32898, 0),
        # The widest trees over the longest caches of the 26B class: the largest call.
        _tree("tree_wide", "26b", 4, 256, 16640, 128),
        # The accepted path of 7 drafts enters the caches of 28 layers (folded into the batch).
        _commit("commit_path", "7b", 28, 7, 1100, 64),
        # Compressed contiguous caches of 22 layers of four prompts move into pages, so that what was evicted is free memory.
        _commit("commit_pack", "8b", 88, 1059, 0, 64, pack=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    while True:
        kind = rng.choice(["append", "append", "tree", "tree", "tree", "commit"])
        heads = rng.choice(sorted(HEADS))
        H, Hkv = HEADS[heads]
        page = rng.choice([0, 16, 32, 64, 128])
        ragged = rng.random() < 0.6
        if kind == "append":
            c = _append("", heads, _log(rng, 1, 32), _log(rng, 1, 16640), rng.choice([0, 0, _log(rng, 1, 4000)]), page, rng.choice([128, 128, 64]),
                        rng.choice([1, 3]), rng.random() < 0.3, ragged)
            cost = c["B"] * c["T"] * (H + 2 * Hkv) / (16640 * 64)
            size = c["B"] * Hkv * (c["rows"] + c["T"]) / (16 * 8 * 2000)
        elif kind == "tree":
            c = _tree("", heads, _log(rng, 1, 32), _log(rng, 1, 256), _log(rng, 1, 33000), page, rng.choice(["tree", "chain"]), ragged)
            cost = c["B"] * c["T"] * H * (c["rows"] + c["T"]) / (4 * 256 * 48 * 16640)
            size = c["B"] * Hkv * c["rows"] / (4 * 8 * 16640)
        else:
            pack = rng.random() < 0.4
            c = _commit("", heads, _log(rng, 1, 96), _log(rng, 1, 1500 if pack else 128), 0 if pack else _log(rng, 1, 1200), page, pack)
            cost = c["B"] * Hkv * c["T"] / (88 * 8 * 1059)
            size = c["B"] * Hkv * (c["rows"] + c["T"]) / (88 * 8 * 1200)
        if cost <= 1 and size <= 1:
            del c["name"]
            return c


# ---- sizes that vary inside a case: the same for every seed ------------------------------------------------
def _sizes(case):
    """(rows a head holds before the call [B][Hkv], new rows a sequence [B] or, packing, a head [B][Hkv])."""
    H, Hkv = HEADS[case["heads"]]
    r = random.Random("%s %d %d %d" % (case["kind"], case["B"], case["T"], case["rows"]))
    B, T, rows = case["B"], case["T"], case["rows"]
    if case["kind"] == "commit":
        lens = [[max(0, rows - r.randrange(1 + rows // 3)) for _ in range(Hkv)] for _ in range(B)]
        if case["pack"]:
            return lens, [[max(1, T - r.randrange(1 + T // 2)) for _ in range(Hkv)] for _ in range(B)]
        return lens, [max(1, T - r.randrange(1 + T // 2)) for _ in range(B)]
    if not case["ragged"]:
        return [[rows] * Hkv for _ in range(B)], [T] * B
    lens = [[max(0, rows - r.randrange(1 + rows // 3)) for _ in range(Hkv)] for _ in range(B)]
    return lens, [T if b == 0 else max(1, T - r.randrange(1 + T // 4)) for b in range(B)]


def work(case):
    H, Hkv = HEADS[case["heads"]]
    lens, count = _sizes(case)
    row = 2 * D                                                      # bytes of a row of one head
    if case["kind"] == "append":
        tokens = sum(count)
        # queries, keys and values in and out; a position per axis and token; the table's rows once
        positions = min(tokens * case["axes"], case["rows"] + case["T"])
        return {"bytes": tokens * (H + 2 * Hkv) * row * 2 + tokens * 4 * case["axes"] + positions * case["rot"] * 4 + 8 * len(count) * Hkv,
                "flops": tokens * (H + Hkv) * case["rot"] * 3}
    if case["kind"] == "tree":
        kv = sum((n + c) * 2 * row for ln, c in zip(lens, count) for n in ln)
        qo = sum(c * H * 2 * row + c * H * 4 for c in count)
        flops = sum(4 * D * c * (H // Hkv) * (n + (c + 1) // 2) for ln, c in zip(lens, count) for n in ln)
        return {"bytes": kv + qo, "flops": flops}
    moved = sum(sum(c) for c in count) if case["pack"] else sum(count) * Hkv
    return {"bytes": moved * row * 2 * 2 + 8 * len(lens) * Hkv, "flops": 0}


# ---- inputs ----------------------------------------------------------------------------------------------------
def _ancestors(parents):
    """[T][T] truth values: draft t sees itself and the drafts it descends from."""
    T = len(parents)
    m = np.zeros((T, T), bool)
    for t, p in enumerate(parents):
        if p >= 0:
            m[t] = m[p]
        m[t, t] = True
    return m


def _words(m):
    """Truth values [..., T, T] as 32-bit words, bit u % 32 of word u / 32 of a row for draft u."""
    T = m.shape[-1]
    W = (T + 31) // 32
    pad = np.zeros(m.shape[:-1] + (W * 32,), bool)
    pad[..., :T] = m
    return np.packbits(pad, axis=-1, bitorder="little").view(np.uint32).reshape(m.shape[:-1] + (W,)).view(np.int32)


def prepare(case, seed):
    H, Hkv = HEADS[case["heads"]]
    B, T, page = case["B"], case["T"], case["page"]
    lens, count = _sizes(case)
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    host = np.random.default_rng(seed)
    bf = torch.bfloat16

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev, dtype=torch.float32).to(bf)

    s = {"case": case, "status": torch.zeros(1, dtype=torch.int32, device=dev),
         "len": torch.tensor(lens, dtype=torch.int32, device=dev),
         "count": torch.tensor(count, dtype=torch.int32, device=dev)}
    kind = case["kind"]
    top = max(max(x) for x in lens) + (0 if kind == "tree" else T)   # rows a head has to have room for
    if page:
        mp = (top + page - 1) // page + 1
        n_pages = B * Hkv * mp + 3
        s["table"] = torch.from_numpy(host.permutation(n_pages)[:B * Hkv * mp].reshape(B, Hkv, mp).astype(np.int32)).to(dev)
        shape = (n_pages, page, D)
    else:
        s["table"] = None
        shape = (B, Hkv, top + 5 if kind == "tree" else top, D)
    s["K"], s["V"] = normal(*shape), normal(*shape)
    if kind == "tree":
        # Attention mass as the rest of the repository draws it: every query leans towards a direction of its KV head, and
        # so do a few of the keys.
        u = torch.randn(B, Hkv, 1, D, generator=gen, device=dev)
        u = u / u.norm(dim=-1, keepdim=True)
        q = torch.randn(B, T, Hkv, H // Hkv, D, generator=gen, device=dev) + 4 * u.view(B, 1, Hkv, 1, D)
        s["q"] = q.view(B, T, H, D).to(bf)
        rows = _rows(s["K"], s["table"], torch.arange(top, device=dev))         # [B][Hkv][top] places
        heavy = torch.rand(B, Hkv, top, generator=gen, device=dev) < 0.02
        flat = s["K"].view(-1, D)
        k = flat[rows].float() + 16 * u * heavy[..., None]
        flat[rows] = k.to(bf)
        s["Kd"], s["Vd"] = normal(B, Hkv, T, D), normal(B, Hkv, T, D)
        if case["mask"] == "tree":
            parents = [[int(host.integers(-1, t)) if t else -1 for t in range(T)] for _ in range(B)]
            s["mask"] = torch.from_numpy(_words(np.stack([_ancestors(p) for p in parents]))).to(dev)
        else:
            s["mask"] = None
        s["out"] = torch.zeros(B, T, H, D, dtype=bf, device=dev)
        s["lse"] = torch.zeros(B, H, T, dtype=torch.float32, device=dev)
        s["max_len"] = max(max(x) for x in lens)
        s["ws"] = torch.empty(32 << 20, dtype=torch.uint8, device=dev)          # one workspace for every call of a program
        return s
    s["len_out"] = torch.empty(B, Hkv, dtype=torch.int32, device=dev)
    if kind == "append":
        # queries, keys and values lie side by side, as a fused projection leaves them
        qkv = normal(B, T, H + 2 * Hkv, D)
        s["q"], s["k"], s["v"] = qkv[:, :, :H], qkv[:, :, H:H + Hkv], qkv[:, :, H + Hkv:]
        s["q_out"] = torch.zeros(B, T, H, D, dtype=bf, device=dev)
        n_pos, rot = top + 1, case["rot"]
        freq = BASE ** (-np.arange(rot // 2) * 2.0 / rot)
        angle = np.arange(n_pos)[:, None] * freq[None]
        s["cos_sin"] = torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)).to(dev)
        pos = case["rows"] + np.arange(T)[None].repeat(B, 0)
        if case["axes"] == 3:                                        # time, row and column of an image token
            side = max(1, int(math.isqrt(T)))
            t = np.arange(T)
            pos = case["rows"] + np.stack([t // (side * side), t // side % side, t % side])[:, None].repeat(B, 1)
            s["sections"] = (rot // 8, rot * 3 // 16, rot * 3 // 16)
        else:
            s["sections"] = None
        s["pos"] = torch.from_numpy(pos.astype(np.int32)).to(dev)
    else:
        s["Kd"], s["Vd"] = normal(B, Hkv, T, D), normal(B, Hkv, T, D)
        s["index"] = None
        if not case["pack"]:                                         # the accepted path of every sequence
            path = np.zeros((B, T), np.int32)
            for b, c in enumerate(count):
                path[b, :c] = np.sort(host.permutation(T)[:c])
            s["index"] = torch.from_numpy(path).to(dev)
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------
def _rows(K, table, j):
    """Places of the rows j ([n], or [B][Hkv][n]) of every head in a cache seen as rows of 128 channels."""
    if table is None:
        B, Hkv, cap, _ = K.shape
        first = (torch.arange(B * Hkv, device=K.device) * cap).view(B, Hkv, 1)
        return first + j
    page = K.shape[1]
    at = (j // page).expand(*table.shape[:2], j.shape[-1]).long()
    return torch.gather(table.long(), 2, at) * page + j % page


def _store(cache, rows, new, valid):
    flat = cache.view(-1, D)
    flat[rows] = torch.where(valid[..., None], new, flat[rows])


def _plain_append(s):
    c = s["case"]
    B, T, H = s["q"].shape[:3]
    Hkv, rot = s["k"].shape[2], c["rot"]
    h = rot // 2
    cs = s["cos_sin"][s["pos"].long()]                               # [(axes)][B][T][rot]
    if s["sections"]:
        cos = torch.cat([x[..., :h].split(s["sections"], -1)[a] for a, x in enumerate(cs)], -1)
        sin = torch.cat([x[..., h:].split(s["sections"], -1)[a] for a, x in enumerate(cs)], -1)
    else:
        cos, sin = cs[..., :h], cs[..., h:]
    cos, sin = cos[:, :, None], sin[:, :, None]

    def rotate(x):
        x = x.float()
        if c["interleaved"]:
            a, b = x[..., 0:rot:2], x[..., 1:rot:2]
            return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., rot:]], -1)
        a, b = x[..., :h], x[..., h:rot]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., rot:]], -1)

    t = torch.arange(T, device=s["q"].device)
    valid = t[None] < s["count"][:, None]                            # [B][T]
    q = torch.where(valid[..., None, None], rotate(s["q"]).to(torch.bfloat16), s["q_out"])
    rows = _rows(s["K"], s["table"], s["len"][..., None].long() + t)
    to = valid[:, None].expand(B, Hkv, T)
    _store(s["K"], rows, rotate(s["k"]).to(torch.bfloat16).transpose(1, 2), to)
    _store(s["V"], rows, s["v"].transpose(1, 2), to)
    return {"q": q, "K": s["K"], "V": s["V"], "len": s["len"] + s["count"][:, None]}


def _plain_tree(s):
    B, T, H, _ = s["q"].shape
    Hkv = s["Kd"].shape[1]
    dev = s["q"].device
    j = torch.arange(s["max_len"], device=dev)
    rows = _rows(s["K"], s["table"], j)
    t = torch.arange(T, device=dev)
    seen_cache = j < s["len"][..., None]                             # [B][Hkv][rows]
    if s["mask"] is None:
        bits = (t[None] <= t[:, None])[None].expand(B, T, T)
    else:
        bits = (s["mask"][:, :, t // 32] >> (t % 32)) & 1 != 0
    seen_draft = bits & (t < s["count"][:, None])[:, None]           # [B][T][T]
    K = torch.cat([s["K"].view(-1, D)[rows].float(), s["Kd"].float()], 2)
    V = torch.cat([s["V"].view(-1, D)[rows].float(), s["Vd"].float()], 2)
    q = s["q"].float().view(B, T, Hkv, H // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, D)
    x = (q @ K.transpose(2, 3) * D ** -0.5).view(B, Hkv, H // Hkv, T, -1)
    del K, q
    seen = torch.cat([seen_cache[:, :, None].expand(B, Hkv, T, j.numel()), seen_draft[:, None].expand(B, Hkv, T, T)], 3)[:, :, None]
    x = torch.where(seen, x, -math.inf)
    m = x.amax(-1, keepdim=True).clamp_min(-1e30)
    x = torch.exp(x - m)
    total = x.sum(-1, keepdim=True)
    out = (x.view(B, Hkv, -1, x.shape[-1]) @ V).view(B, Hkv, H // Hkv, T, D) / total.clamp_min(1e-30)
    lse = (m + torch.log(total)).view(B, H, T)
    valid = t[None] < s["count"][:, None]
    out = out.permute(0, 3, 1, 2, 4).reshape(B, T, H, D).to(torch.bfloat16)
    return {"out": torch.where(valid[..., None, None], out, s["out"]), "lse": torch.where(valid[:, None], lse, s["lse"])}


def _plain_commit(s):
    B, Hkv, T, _ = s["Kd"].shape
    t = torch.arange(T, device=s["Kd"].device)
    count = s["count"] if s["case"]["pack"] else s["count"][:, None].expand(B, Hkv)
    valid = t < count[..., None]
    at = (t if s["index"] is None else s["index"].long()[:, None]).expand(B, Hkv, T)[..., None].expand(B, Hkv, T, D)
    rows = _rows(s["K"], s["table"], s["len"][..., None].long() + t)
    _store(s["K"], rows, torch.gather(s["Kd"], 2, at), valid)
    _store(s["V"], rows, torch.gather(s["Vd"], 2, at), valid)
    return {"K": s["K"], "V": s["V"], "len": s["len"] + count}


def run(s):
    kind = s["case"]["kind"]
    if not own:
        return {"append": _plain_append, "tree": _plain_tree, "commit": _plain_commit}[kind](s)
    from paper_2509_00419_b200 import binding as L
    if kind == "append":
        L.rope_append(s["k"], s["v"], s["pos"], s["cos_sin"], s["K"], s["V"], s["len"], q=s["q"], q_out=s["q_out"], table=s["table"],
                      count=s["count"], len_out=s["len_out"], sections=s["sections"], interleaved=s["case"]["interleaved"],
                      dev_status=s["status"])
        return {"q": s["q_out"], "K": s["K"], "V": s["V"], "len": s["len_out"]}
    if kind == "tree":
        out, lse = L.tree_attn(s["q"], s["K"], s["V"], s["len"], Kd=s["Kd"], Vd=s["Vd"], mask=s["mask"], count=s["count"],
                               table=s["table"], out=s["out"], lse=s["lse"], max_len=s["max_len"], ws=s["ws"], dev_status=s["status"])
        return {"out": out, "lse": lse}
    L.commit_rows(s["Kd"], s["Vd"], s["K"], s["V"], s["len"], s["count"], index=s["index"], table=s["table"], len_out=s["len_out"],
                  dev_status=s["status"])
    return {"K": s["K"], "V": s["V"], "len": s["len_out"]}


# ---- the definition in 64 bits, head by head -----------------------------------------------------------------------
def _exact_place(s, b, g, j):
    """Where row j (numbers on the host) of a head lies: index into the cache as rows."""
    if s["table"] is None:
        Hkv, cap = s["K"].shape[1:3]
        return (b * Hkv + g) * cap + j
    page = s["K"].shape[1]
    return s["table"][b, g].cpu().numpy().astype(np.int64)[j // page] * page + j % page


def exact(case, seed):
    s = prepare(case, seed)
    H, Hkv = HEADS[case["heads"]]
    G = H // Hkv
    B, T = case["B"], case["T"]
    lens, count = _sizes(case)
    dev = s["K"].device
    if case["kind"] == "tree":
        if B * Hkv > 512:
            return None
        out = torch.zeros(B, T, H, D, dtype=torch.float64, device=dev)
        lse = torch.zeros(B, H, T, dtype=torch.float64, device=dev)
        words = None if s["mask"] is None else s["mask"].cpu().numpy().astype(np.int64)
        for b in range(B):
            n = count[b]
            see = np.zeros((n, n), bool)
            for u in range(n):
                see[:, u] = np.arange(n) >= u if words is None else words[b, :n, u // 32] >> (u % 32) & 1 == 1
            see = torch.from_numpy(see).to(dev)
            for g in range(Hkv):
                at = torch.from_numpy(_exact_place(s, b, g, np.arange(lens[b][g]))).to(dev)
                k = torch.cat([s["K"].reshape(-1, D)[at], s["Kd"][b, g, :n]]).double()
                v = torch.cat([s["V"].reshape(-1, D)[at], s["Vd"][b, g, :n]]).double()
                for h in range(g * G, g * G + G):
                    logit = s["q"][b, :n, h].double() @ k.T / math.sqrt(D)
                    logit[:, lens[b][g]:].masked_fill_(~see, -math.inf)
                    lse[b, h, :n] = torch.logsumexp(logit, 1)
                    out[b, :n, h] = torch.softmax(logit, 1).nan_to_num(0.0) @ v
        return {"out": out, "lse": lse}
    K, V = s["K"].double().view(-1, D), s["V"].double().view(-1, D)
    if case["kind"] == "append":
        rot = case["rot"]
        q = torch.zeros(B, T, H, D, dtype=torch.float64, device=dev)
        pair = np.arange(rot // 2)
        first = torch.from_numpy(2 * pair if case["interleaved"] else pair).to(dev)
        second = first + (1 if case["interleaved"] else rot // 2)
        axis = torch.zeros(rot // 2, dtype=torch.long, device=dev)
        if s["sections"]:
            axis = torch.repeat_interleave(torch.arange(3, device=dev), torch.tensor(s["sections"], device=dev))
        table = s["cos_sin"].double()
        for b in range(B):
            n = count[b]
            p = s["pos"][:, b, :n].long().T[:, axis] if case["axes"] == 3 else s["pos"][b, :n].long()[:, None].expand(n, rot // 2)
            i = torch.arange(rot // 2, device=dev)
            turn = torch.complex(table[p, i], table[p, rot // 2 + i])[:, None]

            def rotated(x):
                y = x.double().clone()
                z = torch.complex(y[..., first], y[..., second]) * turn
                y[..., first], y[..., second] = z.real, z.imag
                return y

            q[b, :n] = rotated(s["q"][b, :n])
            kr = rotated(s["k"][b, :n])
            for g in range(Hkv):
                at = torch.from_numpy(_exact_place(s, b, g, lens[b][g] + np.arange(n))).to(dev)
                K[at], V[at] = kr[:, g], s["v"][b, :n, g].double()
        return {"q": q, "K": K.view(s["K"].shape), "V": V.view(s["V"].shape), "len": s["len"].double() + s["count"][:, None]}
    for b in range(B):
        for g in range(Hkv):
            n = count[b][g] if case["pack"] else count[b]
            at = torch.from_numpy(_exact_place(s, b, g, lens[b][g] + np.arange(n))).to(dev)
            src = torch.arange(n, device=dev) if s["index"] is None else s["index"][b, :n].long()
            K[at], V[at] = s["Kd"][b, g, src].double(), s["Vd"][b, g, src].double()
    grown = s["count"] if case["pack"] else s["count"][:, None]
    return {"K": K.view(s["K"].shape), "V": V.view(s["V"].shape), "len": s["len"].double() + grown}
