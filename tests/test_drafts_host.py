"""Decoding several drafted tokens at a time, without a GPU: pins of the oracle, refusals of the entry points and the binding."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import draft_oracle as DO
from oracle import lvlm_oracle as O
from paper_2509_00419_b200 import binding as L
from paper_2509_00419_b200 import build as B


@pytest.fixture(scope="module")
def lib():
    B.build()
    return L.lib()


# ---- the oracle ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_keeps_norms_and_depends_on_distance(interleaved):
    r = np.random.default_rng(1)
    table = L.rope_table(40, 32, 100.0, device="cpu").numpy()
    x, y = r.normal(size=(2, 1, 1, 1, 48))
    turned = lambda v, p: DO.rotate(v, np.array([[p]]), table, interleaved)[0, 0, 0]
    # the table is rounded to fp32: cos^2 + sin^2 is off by 2 x 2^-24 at most, products of two such by four times that
    assert np.isclose(np.linalg.norm(turned(x, 17)), np.linalg.norm(x), rtol=2.0 ** -22)
    dots = [turned(x, p + 5) @ turned(y, p) for p in (0, 3, 30)]
    assert np.allclose(dots, dots[0], atol=2.0 ** -21 * np.linalg.norm(x) * np.linalg.norm(y))
    assert np.array_equal(turned(x, 0), x[0, 0, 0]) and np.array_equal(turned(x, 9)[32:], x[0, 0, 0, 32:])
    assert np.array_equal(turned(x, 40), x[0, 0, 0])           # a position outside the table turns nothing


def test_rotation_pairs_and_sections():
    r = np.random.default_rng(2)
    table = L.rope_table(64, 32, 50.0, device="cpu").numpy()
    x = r.normal(size=(1, 2, 3, 32))
    pos = np.array([[7, 9]])
    order = np.concatenate([np.arange(0, 32, 2), np.arange(1, 32, 2)])
    assert np.array_equal(DO.rotate(x, pos, table, True)[..., order], DO.rotate(x[..., order], pos, table))
    same = DO.rotate(x, np.stack([pos] * 3), table, sections=(4, 6, 6))
    assert np.array_equal(same, DO.rotate(x, pos, table))
    mixed = DO.rotate(x, np.stack([pos, pos + 3, pos + 11]), table, sections=(4, 6, 6))
    for lo, hi, d in ((0, 4, 0), (4, 10, 3), (10, 16, 11)):
        assert np.array_equal(mixed[..., lo:hi], DO.rotate(x, pos + d, table)[..., lo:hi])


def test_rope_table_far_positions():
    t = L.rope_table(200001, 64, 10000.0, device="cpu")
    freq = 10000.0 ** (-np.arange(32) / 32)
    assert np.abs(t[200000].numpy() - np.concatenate([np.cos(200000 * freq), np.sin(200000 * freq)])).max() <= 2.0 ** -24 + 2e-10


def test_chain_over_an_empty_cache_is_causal_attention():
    r = np.random.default_rng(3)
    q, k, v = r.normal(size=(2, 6, 4, 16)), r.normal(size=(2, 2, 6, 16)), r.normal(size=(2, 2, 6, 16))
    see = np.tril(np.ones((6, 6), bool))[None].repeat(2, 0)
    out, lse = DO.tree_attn(q, k[:, :, :0], v[:, :, :0], np.zeros((2, 2), int), k, v, see, [6, 6])
    want = O.attention_with_scores(q, k, v, 0, 6, 0, 6)
    assert np.abs(out - want["out"]).max() <= 2.0 ** -8 * np.abs(out).max()
    assert np.allclose(lse, want["lse"], atol=1e-6)


def test_a_node_is_a_decode_step_over_its_path():
    r = np.random.default_rng(4)
    B_, H, Hkv, T, cap = 1, 4, 2, 5, 9
    q, K, V = r.normal(size=(B_, T, H, 8)), r.normal(size=(B_, Hkv, cap, 8)), r.normal(size=(B_, Hkv, cap, 8))
    Kd, Vd = r.normal(size=(B_, Hkv, T, 8)), r.normal(size=(B_, Hkv, T, 8))
    length = np.array([[9, 4]])
    parents = [-1, 0, 0, 2, -1]
    words = L.tree_mask(torch.tensor([parents])).numpy()
    see = (words[:, :, :1] >> np.arange(T)) & 1 == 1
    out, _ = DO.tree_attn(q, K, V, length, Kd, Vd, see, [T])
    for t, path in enumerate([[0], [0, 1], [0, 2], [0, 2, 3], [4]]):
        K1 = np.concatenate([K, np.zeros((B_, Hkv, T, 8))], 2)
        V1 = np.concatenate([V, np.zeros((B_, Hkv, T, 8))], 2)
        K1, V1, l1 = DO.commit(K1, V1, length, Kd, Vd, np.array([path]), [len(path)])
        want = O.decode_attn(q[:, t], K1, V1, l1)["out"]
        assert np.abs(out[0, t] - want).max() <= 2.0 ** -8 * np.abs(want).max() + 1e-6


# ---- helpers of the binding ---------------------------------------------------------------------------------
def test_tree_mask_words():
    r = np.random.default_rng(5)
    for T in (1, 31, 32, 33, 70, 256):
        par = torch.tensor([[int(r.integers(-1, t)) if t else -1 for t in range(T)] for _ in range(2)])
        words = L.tree_mask(par).numpy().astype(np.int64) & 0xFFFFFFFF
        assert words.shape == (2, T, (T + 31) // 32)
        for b in range(2):
            for t in range(T):
                path, u = set(), t
                while u >= 0:
                    path.add(u)
                    u = int(par[b, u])
                assert {u for u in range(words.shape[2] * 32) if words[b, t, u // 32] >> (u % 32) & 1} == path
    with pytest.raises(ValueError):
        L.tree_mask(torch.tensor([0]))
    assert torch.equal(L.tree_mask(torch.tensor([-1, 0, 1])), torch.tensor([[1], [3], [7]], dtype=torch.int32))


def test_binding_refuses_cpu_tensors_and_wrong_types():
    z = torch.zeros(1, 1, 1, 128, dtype=torch.bfloat16)
    i = torch.zeros(1, 1, dtype=torch.int32)
    with pytest.raises(TypeError):
        L.rope_append(z, z, i, None, z, z, i)
    with pytest.raises(TypeError):
        L.commit_rows(z, z, z, z, i)
    with pytest.raises(TypeError):
        L.tree_attn(z, z, z, i)


# ---- refusals: nothing below is ever dereferenced ---------------------------------------------------------------
P, P2, ODD = ctypes.c_void_p(0x100000), ctypes.c_void_p(0x9000000), ctypes.c_void_p(0x100008)
WS, N_WS = ctypes.c_void_p(0x10000), ctypes.c_size_t(1 << 40)


def _dims(**kw):
    d = L.Dims(B=2, H=8, Hkv=2, D=128, T=5, cap=100, draft_cap=8, rot=128, n_pos=1000)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


PAGED = dict(page=64, n_pages=30, max_pages=4)


def test_rope_append_refusals(lib):
    def call(d, q=P, k=P, v=P, pos=P, cs=P, q_out=P2, K=P, V=P, table=None, ln=P, pc=None):
        return lib.lvlm_rope_append(q, k, v, pos, cs, None, q_out, K, V, table, ln, None, None, pc, ctypes.byref(d), None, None)

    for kw in (dict(k=None), dict(v=None), dict(K=None), dict(V=None), dict(q=None), dict(q_out=None), dict(pos=None), dict(cs=None), dict(table=P)):
        assert call(_dims(), **kw) == L.ERR_INVALID_ARG, kw
    for kw in (dict(B=0), dict(Hkv=0), dict(T=0), dict(H=7), dict(cap=0), dict(rot=-16), dict(rot=144), dict(n_pos=0), dict(axes=2),
               dict(axes=3, sect0=40, sect1=30), dict(axes=3, sect0=-1), dict(page=64)):
        assert call(_dims(**kw)) == L.ERR_INVALID_ARG, kw
    assert call(_dims(rot=0), pos=None, pc=P) == L.ERR_INVALID_ARG
    for kw in (dict(n_pages=0), dict(max_pages=0), dict(page=0), dict(page_stride=63 * 128)):
        assert call(_dims(**{**PAGED, **kw}), table=P) == L.ERR_INVALID_ARG, kw
    assert call(_dims(D=64)) == L.ERR_UNSUPPORTED and call(_dims(rot=24)) == L.ERR_UNSUPPORTED
    for page in (8, 48):
        assert call(_dims(**{**PAGED, "page": page}), table=P) == L.ERR_UNSUPPORTED
    assert call(_dims(page=1 << 20, n_pages=4, max_pages=1 << 12), table=P) == L.ERR_UNSUPPORTED      # a capacity beyond 32 bits
    for kw in (dict(q=ODD), dict(k=ODD), dict(v=ODD), dict(q_out=ODD), dict(K=ODD), dict(V=ODD), dict(cs=ODD)):
        assert call(_dims(), **kw) == L.ERR_ALIGNMENT, kw
    for kw in (dict(q_stride_n=1028), dict(new_stride_h=132), dict(kv_stride_h=100 * 128 + 4)):
        assert call(_dims(**kw)) == L.ERR_ALIGNMENT, kw
    # q_out behind the start of q but before its end
    assert call(_dims(), q_out=ctypes.c_void_p(0x100000 + 256)) == L.ERR_INVALID_ARG


def test_commit_rows_refusals(lib):
    def call(d, Kd=P, Vd=P, index=P, pos=None, K=P2, V=P2, table=None, pc=None):
        return lib.lvlm_commit_rows(Kd, Vd, index, None, pos, K, V, table, P, None, None, pc, ctypes.byref(d), None, None)

    for kw in (dict(Kd=None), dict(Vd=None), dict(K=None), dict(V=None), dict(K=P), dict(V=P), dict(pos=P), dict(pc=P), dict(table=P)):
        assert call(_dims(), **kw) == L.ERR_INVALID_ARG, kw
    for kw in (dict(B=0), dict(Hkv=0), dict(T=0), dict(draft_cap=0), dict(cap=0)):
        assert call(_dims(**kw)) == L.ERR_INVALID_ARG, kw
    assert call(_dims(T=9), index=None) == L.ERR_INVALID_ARG                          # more rows than the drafts have
    assert call(_dims(D=256)) == L.ERR_UNSUPPORTED and call(_dims(**{**PAGED, "page": 24}), table=P) == L.ERR_UNSUPPORTED
    for kw in (dict(Kd=ODD), dict(Vd=ODD), dict(K=ODD), dict(V=ODD)):
        assert call(_dims(), **kw) == L.ERR_ALIGNMENT, kw
    assert call(_dims(draft_stride_b=2052)) == L.ERR_ALIGNMENT


def test_tree_attn_refusals(lib):
    def call(d, q=P, K=P, V=P, table=None, ln=P, Kd=P, Vd=P, mask=None, scale=0.1, out=P, ws=WS, n_ws=N_WS):
        return lib.lvlm_tree_attn(q, K, V, table, ln, Kd, Vd, mask, None, ctypes.byref(d), ctypes.c_float(scale), out, None, ws, n_ws, None, None)

    for kw in (dict(q=None), dict(K=None), dict(V=None), dict(ln=None), dict(out=None), dict(Kd=None), dict(Vd=None), dict(table=P),
               dict(Kd=None, Vd=None, mask=P), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan"))):
        assert call(_dims(), **kw) == L.ERR_INVALID_ARG, kw
    for kw in (dict(B=0), dict(H=0), dict(Hkv=0), dict(H=7), dict(T=0), dict(draft_cap=4), dict(cap=0)):
        assert call(_dims(**kw)) == L.ERR_INVALID_ARG, kw
    for kw in (dict(D=64), dict(T=257, draft_cap=257), dict(H=130, Hkv=2)):
        assert call(_dims(**kw)) == L.ERR_UNSUPPORTED, kw
    assert call(_dims(**{**PAGED, "page": 8}), table=P) == L.ERR_UNSUPPORTED
    for kw in (dict(q=ODD), dict(K=ODD), dict(V=ODD), dict(Kd=ODD), dict(Vd=ODD), dict(out=ODD)):
        assert call(_dims(), **kw) == L.ERR_ALIGNMENT, kw
    for kw in (dict(q_stride_b=5121), dict(draft_stride_h=8 * 128 + 4), dict(kv_stride_b=100 * 256 + 2)):
        assert call(_dims(**kw)) == L.ERR_ALIGNMENT, kw
    d = _dims(cap=5000)                                                               # long enough to be split
    need = L.workspace_bytes(L.OP_TREE_ATTN, d)
    assert need > 256 and need % 256 == 0
    assert call(d, ws=None) == L.ERR_WORKSPACE and call(d, n_ws=ctypes.c_size_t(need - 256)) == L.ERR_WORKSPACE
    assert call(d, ws=ctypes.c_void_p(0x10010)) == L.ERR_WORKSPACE
    assert L.workspace_bytes(L.OP_TREE_ATTN, _dims(T=0)) == 0


def test_appends_refuse_lengths_over_what_others_read(lib):
    """len_out is len, or shares nothing with len or count: only then has every thread read what another writes."""
    at = lambda n: ctypes.c_void_p(0x9100000 + n)

    def append(ln, lo, count, **kw):
        return lib.lvlm_rope_append(None, P, P, None, None, count, None, P2, P2, None, ln, lo, None, None, ctypes.byref(_dims(rot=0, **kw)), None, None)

    def commit(ln, lo, count, **kw):
        return lib.lvlm_commit_rows(P, P, P, count, None, P2, P2, None, ln, lo, None, None, ctypes.byref(_dims(**kw)), None, None)

    for call in (append, commit):                                    # two sequences of two heads: 16 bytes of lengths, 8 of counts
        for n in (4, 8, 12, -4, -12):
            assert call(at(0), at(n), None) == L.ERR_INVALID_ARG, n
        for n in (0, 4, 8, 12, -4):
            assert call(at(64), at(0), at(n)) == call(at(0), at(0), at(n)) == call(None, at(0), at(n)) == L.ERR_INVALID_ARG, n
    for n in (4, 12, -12):
        assert commit(at(0), at(0), at(n), count_heads=1) == L.ERR_INVALID_ARG
    assert commit(at(64), at(0), at(0), count_heads=1) == L.ERR_INVALID_ARG
    assert append(at(64), at(0), at(0), Hkv=1) == L.ERR_INVALID_ARG


def test_tree_attn_refuses_more_tiles_than_it_can_count(lib):
    """128 row tiles a head (64 query heads of 256 drafts) over 2^31 rows, in a few large pages that lie in the table many times."""
    def call(max_pages):
        d = _dims(B=1, H=64, Hkv=1, T=256, page=1 << 20, n_pages=4, max_pages=max_pages)
        return lib.lvlm_tree_attn(P, P2, P2, P, P, None, None, None, None, ctypes.byref(d), ctypes.c_float(0.1), P2, None, ctypes.c_void_p(8), 8, None, None)

    assert call(2047) == call(1025) == L.ERR_UNSUPPORTED


def test_tree_attn_refuses_results_over_other_queries(lib):
    """out is q, row for row, or lies elsewhere."""
    def call(d, q=P, out=P):
        return lib.lvlm_tree_attn(q, P2, P2, None, P, None, None, None, None, ctypes.byref(d), ctypes.c_float(0.1), out, None, None, 0, None, None)

    at = lambda n: ctypes.c_void_p(0x100000 + n)
    size = 2 * 5 * 8 * 128 * 2
    split = _dims(cap=5000)                                                           # (refused for its workspace where nothing else is wrong)
    for n in (16, 256, size - 16):
        assert call(split, out=at(n)) == call(split, q=at(n)) == L.ERR_INVALID_ARG, n
    assert call(split) == call(split, out=at(size)) == call(split, q=at(size)) == L.ERR_WORKSPACE
    for kw in (dict(q_stride_n=9 * 128), dict(q_stride_b=6 * 8 * 128), dict(q_stride_h=256)):
        assert call(_dims(cap=5000, **kw)) == L.ERR_INVALID_ARG, kw
    assert call(_dims(cap=5000, q_stride_n=9 * 128), out=at(2 * 5 * 9 * 128 * 2)) == L.ERR_WORKSPACE


# a program sizes a workspace once, for its widest batch, longest cache and largest tree: nothing smaller may ask for more
@pytest.mark.parametrize("heads", [(8, 8), (28, 4), (32, 8), (48, 8), (1, 1), (64, 1)])
def test_tree_workspace_never_shrinks(lib, heads):
    H, Hkv = heads

    def size(B_, n, T):
        return L.workspace_bytes(L.OP_TREE_ATTN, L.Dims(B=B_, H=H, Hkv=Hkv, D=128, T=T, draft_cap=T, cap=n))

    Bs = [1, 2, 3, 4, 5, 7, 8, 9, 10, 16, 32, 74, 75, 149, 300]
    ns = [1, 16, 63, 64, 65, 127, 128, 129, 200, 500, 1000, 1100, 3008, 5000, 16640, 33000, 100000]
    Ts = [1, 2, 3, 5, 8, 13, 16, 17, 26, 31, 32, 33, 61, 64, 65, 100, 128, 200, 256]
    for line in ([[(b, n, T) for n in ns] for b in Bs for T in Ts] + [[(b, n, T) for b in Bs] for n in ns for T in Ts] +
                 [[(b, n, T) for T in Ts] for b in Bs for n in ns]):
        sizes = [size(*x) for x in line]
        for i in range(1, len(line)):
            assert sizes[i] >= sizes[i - 1], (line[i - 1], line[i])


def test_records_of_cut_units():
    """Any two words that a workspace may hold: what is taken for a record names CTAs of the grid only."""
    t = ctypes.CDLL(B.build_test())
    ok = lambda first, more: bool(t.lvlm_debug_tree_record(ctypes.c_int(first), ctypes.c_int(more)))
    for first in range(-2, 150):
        for more in range(-2, 150):
            assert ok(first, more) == (0 <= first and 0 < more and first + more <= 147), (first, more)
    far = [-(1 << 31), (1 << 31) - 1, 0x7F7F7F7F, -0x7F7F7F7F, 1 << 30, 148, 147, 1, 0, -1]
    for x in far:
        for y in far:
            assert ok(x, y) == (0 <= x and 0 < y and x + y <= 147), (x, y)


def test_room_follows_the_pages():
    """What the commits are held against: the rows of the pages that a head has."""
    from paper_2509_00419_b200.pipeline import PagedLayers

    c = PagedLayers(2, 2, 4, 2, n_pages=20, page=16, max_pages=3, T=4, device="cpu")
    rows = torch.tensor([[[17, 0], [16, 48]], [[1, 33], [32, 5]]])
    c.reserve(rows)
    assert torch.equal(c.room.long(), (rows + 15) // 16 * 16) and torch.equal(c.room, (c.table >= 0).sum(3).int() * 16)
    c.reserve(rows.clamp_max(20) + 1)                  # what a head has it keeps
    assert torch.equal(c.room, (c.table >= 0).sum(3).int() * 16) and (c.room.long() >= (rows + 15) // 16 * 16).all()
    c.release(0)
    assert (c.room[:, 0] == 0).all() and torch.equal(c.room[:, 1], (c.table[:, 1] >= 0).sum(2).int() * 16)
    c.check()
    c.status.fill_(L.DEV_BOUNDS)
    with pytest.raises(RuntimeError):
        c.check()
    c.check()


def test_tree_workspace_is_small(lib):
    """The widest trees over the longest caches fit 32 MiB, a token over a short cache asks for little."""
    for H, Hkv in ((8, 8), (28, 4), (32, 8), (48, 8), (64, 1)):
        for B_ in (1, 4, 32, 96):
            for T in (1, 26, 61, 256):
                for n in (216, 1888, 16640, 33000, 1 << 20):
                    assert L.workspace_bytes(L.OP_TREE_ATTN, L.Dims(B=B_, H=H, Hkv=Hkv, D=128, T=T, draft_cap=T, cap=n)) <= 32 << 20
    assert L.workspace_bytes(L.OP_TREE_ATTN, L.Dims(B=1, H=28, Hkv=4, D=128, T=1, draft_cap=1, cap=216)) <= 1 << 20


def test_pages_come_back():
    """Pages are handed out once, a finished sequence gives all of its own back, and the others keep theirs."""
    from paper_2509_00419_b200.pipeline import PagedLayers

    c = PagedLayers(2, 3, 4, 2, n_pages=40, page=16, max_pages=5, T=4, device="cpu")
    rows = torch.tensor([[[17, 1], [0, 80], [33, 16]]] * 2)
    c.reserve(rows)
    need = (rows + 15) // 16
    used = c.table[c.table >= 0].tolist()
    assert len(used) == len(set(used)) == int(need.sum()) and c.pages_free() == 40 - len(used)
    assert torch.equal((c.table >= 0).sum(3), need)
    c.len.copy_(rows)
    before = c.table.clone()
    c.release(1)
    assert (c.table[:, 1] == -1).all() and (c.len[:, 1] == 0).all() and c.pages_free() == 40 - int(need[:, [0, 2]].sum())
    for b in (0, 2):
        assert torch.equal(c.table[:, b], before[:, b]) and torch.equal(c.len[:, b].long(), rows[:, b])
    c.release(1)                                       # nothing is given back twice
    assert c.pages_free() == 40 - int(need[:, [0, 2]].sum())
    c.reserve(rows)
    used = c.table[c.table >= 0].tolist()
    assert len(used) == len(set(used)) == int(need.sum())
    with pytest.raises(IndexError):
        c.release(3)
    free, table = c.pages_free(), c.table.clone()
    with pytest.raises(RuntimeError):
        c.reserve(torch.full((2, 3, 2), 80))           # more than there are: nothing is handed out
    with pytest.raises(ValueError):
        c.reserve(torch.full((2, 3, 2), 81))
    assert c.pages_free() == free and torch.equal(c.table, table)
