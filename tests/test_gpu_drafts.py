"""Decoding several drafted tokens at a time on the GPU against the 64-bit oracle: append with rotation, tree attention, commit."""
import numpy as np
import pytest
import torch

from bench import count_launches
from oracle import draft_oracle as DO
from paper_2509_00419_b200 import binding as L
from paper_2509_00419_b200 import build as BU
from tests.util import f64, i32

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def bf(r, *shape):
    return torch.from_numpy(r.normal(size=shape).astype(np.float32)).to(BF)


def dev(x, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, dtype))).cuda()


def flag():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def paged(r, K, V, page, fill=float("nan"), spare=3):
    """A logical cache [B][Hkv][cap][D] (cap a multiple of page) in shuffled pages: (Kp, Vp, table)."""
    B, Hkv, cap, D = K.shape
    mp = cap // page
    n_pages = B * Hkv * mp + spare
    table = r.permutation(n_pages)[:B * Hkv * mp].reshape(B, Hkv, mp)
    kp, vp = (torch.full((n_pages, page, D), fill, dtype=BF) for _ in range(2))
    at = torch.from_numpy(table).reshape(-1)
    kp[at], vp[at] = K.reshape(-1, page, D), V.reshape(-1, page, D)
    return kp.cuda(), vp.cuda(), dev(table)


def logical(Kp, table):
    """Back to [B][Hkv][cap][D]."""
    t = table.long()
    return Kp[t.reshape(-1)].reshape(*t.shape[:2], -1, Kp.shape[-1])


def same(a, b):
    """Bit for bit, NaN included."""
    return torch.equal(a.cpu().contiguous().view(torch.int16), b.cpu().contiguous().view(torch.int16))


# ---- append with rotation ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("B,H,Hkv,T,cap,page,rot,interleaved,sections,inplace", [
    (1, 28, 4, 1, 37, 0, 128, False, None, True), (2, 8, 8, 1, 64, 16, 128, True, None, False), (3, 8, 2, 37, 100, 0, 64, False, None, False),
    (2, 7, 1, 130, 256, 64, 128, False, (16, 24, 24), True), (2, 4, 4, 17, 64, 32, 32, True, (3, 7, 6), False),
    (1, 2, 1, 5, 16, 16, 16, False, None, True), (2, 6, 2, 9, 128, 128, 0, False, None, True), (4, 48, 8, 3, 40, 0, 112, False, (0, 56, 0), False)])
def test_rope_append(B, H, Hkv, T, cap, page, rot, interleaved, sections, inplace):
    r = np.random.default_rng(B * 1000 + T * 10 + rot)
    n_pos = 300
    qkv = bf(r, B, T, H + 2 * Hkv, 128)
    K, V = bf(r, B, Hkv, cap, 128), bf(r, B, Hkv, cap, 128)
    ln = r.integers(0, cap - T + 1, size=(B, Hkv))
    ln.reshape(-1)[0] = cap - T                                       # filled to the last row
    count = r.integers(0, T + 1, size=B)
    count[0] = T
    pos = r.integers(0, n_pos, size=(3, B, T) if sections else (B, T))
    table_cs = L.rope_table(n_pos, rot, 1000.0, device="cpu") if rot else None
    cs = np.zeros((1, 0), np.float32) if rot == 0 else table_cs.numpy()
    x = f64(qkv)
    turn = (lambda v: v) if rot == 0 else (lambda v: DO.rotate(v, pos, cs, interleaved, sections))
    want_q, k_rot = turn(x[:, :, :H]), turn(x[:, :, H:H + Hkv])
    want_K, want_V, want_len = DO.append(f64(K), f64(V), ln, k_rot, x[:, :, H + Hkv:], count)

    d = qkv.cuda()
    q, kn, vn = d[:, :, :H], d[:, :, H:H + Hkv], d[:, :, H + Hkv:]
    Kd, Vd, tab = paged(r, K, V, page) if page else (K.cuda(), V.cuda(), None)
    ld, st = dev(ln), flag()
    acc = torch.full((B, Hkv, cap), 5.0, device="cuda")
    pc = torch.full((B, Hkv, cap), -7, dtype=torch.int32, device="cuda")
    q_out = q if inplace else torch.full((B, T, H, 128), 3.0, dtype=BF, device="cuda")
    len_out = None if inplace else torch.empty_like(ld)
    got = L.rope_append(kn, vn, dev(pos), None if rot == 0 else table_cs.cuda(), Kd, Vd, ld, q=q, q_out=q_out, table=tab, count=dev(count),
                        len_out=len_out, sections=sections, interleaved=interleaved, acc_score=acc, pos_cache=pc, dev_status=st)
    torch.cuda.synchronize()
    assert st.item() == 0 and got is q_out
    assert np.array_equal(i32(ld if inplace else len_out), want_len) and (inplace or np.array_equal(i32(ld), ln))
    # a rounding to bf16 (2^-8 of the value), two products and a sum in fp32 (2^-24 of a and b each, a and b below 2^3)
    close = lambda a, b: np.abs(a - b) <= 2.0 ** -8 * np.abs(b) + 2.0 ** -20
    for b in range(B):
        n = count[b]
        assert close(f64(q_out)[b, :n], want_q[b, :n]).all()
        assert same(q_out[b, n:], d[b, n:, :H] if inplace else torch.full_like(q_out[b, n:], 3.0))
    Kl, Vl = (Kd, Vd) if not page else (logical(Kd, tab), logical(Vd, tab))
    assert close(f64(Kl), want_K).all() and np.array_equal(f64(Vl), want_V)
    p0 = pos[0] if sections else pos
    for b in range(B):
        for g in range(Hkv):
            lo, hi = ln[b, g], ln[b, g] + count[b]
            assert same(Kl[b, g, :lo], K[b, g, :lo]) and same(Kl[b, g, hi:], K[b, g, hi:])
            assert (acc[b, g, lo:hi] == 0).all() and (acc[b, g, :lo] == 5).all() and (acc[b, g, hi:] == 5).all()
            assert np.array_equal(i32(pc[b, g, lo:hi]), p0[b, :count[b]]) and (pc[b, g, :lo] == -7).all() and (pc[b, g, hi:] == -7).all()
    if not inplace:
        assert same(d[:, :, :H], qkv[:, :, :H])
    if page:
        other = sorted(set(range(Kd.shape[0])) - set(i32(tab).reshape(-1).tolist()))
        assert torch.isnan(Kd[other]).all() and torch.isnan(Vd[other]).all()


# more tokens than the few that get a large CTA each (296): another instance of the kernel
@pytest.mark.parametrize("B,H,Hkv,T,cap,page,rot,interleaved,sections,inplace", [
    (1, 4, 2, 296, 300, 0, 128, False, None, True), (1, 4, 2, 297, 320, 16, 128, False, None, True), (2, 28, 4, 200, 512, 16, 128, False, (16, 24, 24), True),
    (1, 48, 8, 333, 350, 0, 64, True, None, False), (3, 8, 2, 150, 256, 64, 112, False, (0, 56, 0), True), (1, 8, 8, 301, 320, 32, 128, True, (20, 21, 23), False),
    (298, 2, 1, 1, 48, 16, 128, False, None, True), (5, 7, 1, 120, 128, 128, 0, False, None, False)])
def test_rope_append_of_prompts(B, H, Hkv, T, cap, page, rot, interleaved, sections, inplace):
    test_rope_append(B, H, Hkv, T, cap, page, rot, interleaved, sections, inplace)


def test_rope_append_into_a_draft_cache_without_queries():
    r = np.random.default_rng(7)
    kn, vn = bf(r, 2, 6, 3, 128), bf(r, 2, 6, 3, 128)
    Kd, Vd = (torch.full((2, 3, 9, 128), 2.0, dtype=BF, device="cuda") for _ in range(2))
    st = flag()
    assert L.rope_append(kn.cuda(), vn.cuda(), None, None, Kd, Vd, dev_status=st) is None
    assert st.item() == 0 and same(Kd[:, :, :6], kn.transpose(1, 2)) and same(Vd[:, :, :6], vn.transpose(1, 2))
    assert (Kd[:, :, 6:] == 2).all() and (Vd[:, :, 6:] == 2).all()


def test_rope_append_flags():
    """Heads and tokens that cannot be served are skipped and flagged; the others are served."""
    r = np.random.default_rng(8)
    B, Hkv, T, page = 5, 2, 4, 16
    K, V = bf(r, B, Hkv, 32, 128), bf(r, B, Hkv, 32, 128)
    kn, vn, q = bf(r, B, T, Hkv, 128), bf(r, B, T, Hkv, 128), bf(r, B, T, 4, 128)
    cs = L.rope_table(50, 128, 100.0)
    good_len = np.array([[0, 5], [28, 3], [12, 20], [7, 7], [14, 1]])
    pos = np.arange(B * T).reshape(B, T)

    def go(ln=good_len, count=np.full(B, T), p=pos, broken=None):
        Kp, Vp, tab = paged(np.random.default_rng(9), K, V, page)
        if broken is not None:
            tab[broken[0], broken[1], broken[2]] = broken[3]
        ld, st, qo = dev(ln), flag(), torch.zeros_like(q).cuda()
        L.rope_append(kn.cuda(), vn.cuda(), dev(p), cs, Kp, Vp, ld, q=q.cuda(), q_out=qo, table=tab, count=dev(count), dev_status=st)
        return st.item(), i32(ld), Kp, Vp, tab, qo

    s0, l0, K0, V0, t0, q0 = go()
    assert s0 == 0 and np.array_equal(l0, good_len + T)
    for bad in (-1, 33, 29, 1 << 30, -(1 << 31)):                    # 29: the rows do not fit
        ln = good_len.copy()
        ln[1, 1] = bad
        s, l, K1, V1, t, q1 = go(ln)
        assert s == L.DEV_BOUNDS and l[1, 1] == bad and same(q1, q0)
        keep = np.ones((B, Hkv), bool)
        keep[1, 1] = False
        assert np.array_equal(l[keep], l0[keep])
        lg, lg0 = logical(K1, t), logical(K0, t0)
        assert same(lg[1, 1], K[1, 1]) and same(lg[torch.from_numpy(keep)], lg0[torch.from_numpy(keep)])
    for bad in (-1, 5):
        c = np.full(B, T)
        c[2] = bad
        s, l, K1, _, t, q1 = go(count=c)
        assert s == L.DEV_BOUNDS and np.array_equal(l[2], good_len[2]) and same(logical(K1, t)[2], K[2]) and (q1[2] == 0).all()
        assert same(q1[3], q0[3]) and np.array_equal(l[3], l0[3])
    for bad in (-1, 23, 1 << 30):                                    # 20 pages and 3 spare ones: 23 is the first that is none
        s, l, K1, _, t, q1 = go(broken=(4, 0, 0, bad))               # rows 14, 15 of this head are lost, 16 and 17 arrive
        assert s == L.DEV_BOUNDS and l[4, 0] == 18 and same(q1, q0)
        assert same(K1[t0[4, 0, 1].item(), :2], K0[t0[4, 0, 1].item(), :2]) and same(K1[t0[4, 0, 0].item()], K[4, 0, :16])
    p = pos.copy()
    p[3, 2] = 50
    s, _, K1, _, t, q1 = go(p=p)
    assert s == L.DEV_BOUNDS and same(q1[3, 2], q[3, 2]) and same(logical(K1, t)[3, 0, 9], kn[3, 2, 0]) and same(q1[3, 1], q0[3, 1])


# ---- commit ----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("B,Hkv,rows,T,cap,page,inplace", [
    (1, 1, 1, 1, 3, 0, True), (3, 4, 7, 7, 48, 16, True), (2, 2, 9, 30, 96, 32, False), (2, 3, 65, 65, 192, 64, True), (2, 1, 300, 300, 400, 0, False),
    (1, 2, 130, 64, 128, 128, True)])
def test_commit_path(B, Hkv, rows, T, cap, page, inplace):
    r = np.random.default_rng(rows + T)
    K, V, Kd, Vd = bf(r, B, Hkv, cap, 128), bf(r, B, Hkv, cap, 128), bf(r, B, Hkv, rows, 128), bf(r, B, Hkv, rows, 128)
    ln = r.integers(0, cap - T + 1, size=(B, Hkv))
    ln.reshape(-1)[-1] = cap - T
    count = r.integers(0, T + 1, size=B)
    count[-1] = T
    index = r.integers(0, rows, size=(B, T))                          # any order, the same row twice
    pos = r.integers(0, 9999, size=(B, rows))
    want = DO.commit(f64(K), f64(V), ln, f64(Kd), f64(Vd), index, count)
    Kc, Vc, tab = paged(r, K, V, page) if page else (K.cuda(), V.cuda(), None)
    ld, st = dev(ln), flag()
    lo = None if inplace else torch.empty_like(ld)
    acc = torch.full((B, Hkv, cap), 5.0, device="cuda")
    pc = torch.full((B, Hkv, cap), -7, dtype=torch.int32, device="cuda")
    bad = index.copy()
    for b in range(B):
        bad[b, count[b]:] = 1 << 30                                   # entries behind count are not read
    L.commit_rows(Kd.cuda(), Vd.cuda(), Kc, Vc, ld, dev(count), index=dev(bad), table=tab, len_out=lo, pos=dev(pos), acc_score=acc,
                  pos_cache=pc, dev_status=st)
    torch.cuda.synchronize()
    assert st.item() == 0
    Kl, Vl = (Kc, Vc) if not page else (logical(Kc, tab), logical(Vc, tab))
    assert np.array_equal(f64(Kl), want[0]) and np.array_equal(f64(Vl), want[1]) and np.array_equal(i32(ld if inplace else lo), want[2])
    for b in range(B):
        for g in range(Hkv):
            a, z = ln[b, g], ln[b, g] + count[b]
            assert (acc[b, g, a:z] == 0).all() and (acc[b, g, :a] == 5).all() and (acc[b, g, z:] == 5).all()
            assert np.array_equal(i32(pc[b, g, a:z]), pos[b, index[b, :count[b]]]) and (pc[b, g, z:] == -7).all()


@pytest.mark.parametrize("rows,page", [(40, 16), (200, 64), (200, 0), (64, 32)])
def test_commit_moves_a_ragged_cache(rows, page):
    r = np.random.default_rng(rows)
    B, Hkv, cap = 3, 2, 256
    Kd, Vd = bf(r, B, Hkv, rows, 128), bf(r, B, Hkv, rows, 128)
    ln = r.integers(0, rows + 1, size=(B, Hkv))
    ln.reshape(-1)[:3] = [0, rows, 1]
    K, V = bf(r, B, Hkv, cap, 128), bf(r, B, Hkv, cap, 128)
    want = DO.commit(f64(K), f64(V), np.zeros((B, Hkv), int), f64(Kd), f64(Vd), None, ln)
    Kc, Vc, tab = paged(r, K, V, page) if page else (K.cuda(), V.cuda(), None)
    ld, st = dev(np.zeros((B, Hkv))), flag()
    # the source is a part of a larger cache, as compression leaves it
    wide = torch.full((B, Hkv, rows + 9, 128), float("nan"), dtype=BF, device="cuda")
    wide2 = wide.clone()
    wide[:, :, :rows], wide2[:, :, :rows] = Kd.cuda(), Vd.cuda()
    L.commit_rows(wide[:, :, :rows], wide2[:, :, :rows], Kc, Vc, ld, dev(ln), table=tab, dev_status=st)
    torch.cuda.synchronize()
    Kl, Vl = (Kc, Vc) if not page else (logical(Kc, tab), logical(Vc, tab))
    assert st.item() == 0 and np.array_equal(i32(ld), ln)
    assert np.array_equal(f64(Kl), want[0]) and np.array_equal(f64(Vl), want[1])


@pytest.mark.parametrize("rows", [20, 100])
def test_commit_by_the_lengths_themselves(rows):
    """count and length in one tensor: every head doubles."""
    r = np.random.default_rng(rows)
    Kd, Vd, K, V = bf(r, 2, 3, rows, 128), bf(r, 2, 3, rows, 128), bf(r, 2, 3, 2 * rows, 128), bf(r, 2, 3, 2 * rows, 128)
    ln = r.integers(0, rows + 1, size=(2, 3))
    want = DO.commit(f64(K), f64(V), ln, f64(Kd), f64(Vd), None, ln)
    Kc, Vc, ld, st = K.cuda(), V.cuda(), dev(ln), flag()
    L.commit_rows(Kd.cuda(), Vd.cuda(), Kc, Vc, ld, ld, dev_status=st)
    assert st.item() == 0 and np.array_equal(i32(ld), 2 * ln) and np.array_equal(f64(Kc), want[0]) and np.array_equal(f64(Vc), want[1])


def test_commit_flags():
    r = np.random.default_rng(11)
    B, Hkv, T = 4, 2, 5
    Kd, Vd, K, V = bf(r, B, Hkv, T, 128), bf(r, B, Hkv, T, 128), bf(r, B, Hkv, 32, 128), bf(r, B, Hkv, 32, 128)

    def go(ln=np.full((B, Hkv), 3), count=np.full(B, T), index=np.arange(T)[None].repeat(B, 0)):
        Kc, Vc, ld, st = K.cuda(), V.cuda(), dev(ln), flag()
        L.commit_rows(Kd.cuda(), Vd.cuda(), Kc, Vc, ld, dev(count), index=dev(index), dev_status=st)
        return st.item(), i32(ld), Kc, Vc

    s0, l0, K0, V0 = go()
    assert s0 == 0 and (l0 == 8).all()
    for bad in (-1, 28, 33):
        ln = np.full((B, Hkv), 3)
        ln[2, 1] = bad
        s, l, Kc, _ = go(ln=ln)
        assert s == L.DEV_BOUNDS and l[2, 1] == bad and same(Kc[2, 1], K[2, 1]) and same(Kc[2, 0], K0[2, 0]) and (l[:2] == 8).all()
    for bad in (-3, 6):
        s, l, Kc, _ = go(count=np.array([T, bad, T, T]))
        assert s == L.DEV_BOUNDS and (l[1] == 3).all() and same(Kc[1], K[1]) and same(Kc[2], K0[2])
    for bad in (-1, T, 1 << 30):
        index = np.arange(T)[None].repeat(B, 0)
        index[0, 2] = bad
        s, l, Kc, _ = go(index=index)
        assert s == L.DEV_BOUNDS and (l == 8).all() and same(Kc[0, :, 5], K[0, :, 5]) and same(Kc[0, :, 6], K0[0, :, 6]) and same(Kc[1], K0[1])


# ---- tree attention ----------------------------------------------------------------------------------------------
def tree_bound(q, K, V, n_keys, scale):
    """What a result may be off beside its rounding, from the arithmetic.  A logit: 128 exact products added in fp32, each addition
    off by at most 2^-23 of the running sum of magnitudes (the tensor core truncates), scaled once.  A probability: that, the
    exponential (2^-22), the remainder of its two bf16 parts (2^-17).  The sums over the keys: 2^-23 an addition."""
    mags = np.sqrt((q ** 2).sum(-1).max()) * np.sqrt((K ** 2).sum(-1).max()) * scale
    logit = mags * 128 * 2.0 ** -23
    prob = logit + 2.0 ** -22 + 2.0 ** -17 + n_keys * 2.0 ** -23
    return 2 * prob * np.abs(V).max(), logit + (n_keys + 8) * 2.0 ** -23


def random_tree(r, T, kind):
    if kind == "chain":
        return np.tril(np.ones((T, T), bool)), None
    if kind == "any":                                                 # no tree at all; some rows see no draft
        see = r.random((T, T)) < 0.4
        see[r.integers(0, T)] = False
        return see, None
    par = [int(r.integers(-1, t)) if t else -1 for t in range(T)]
    see = np.zeros((T, T), bool)
    for t, p in enumerate(par):
        see[t] = see[p] if p >= 0 else False
        see[t, t] = True
    return see, par


def words_of(see):
    T = see.shape[-1]
    W = (T + 31) // 32
    pad = np.zeros((*see.shape[:-1], W * 32), bool)
    pad[..., :T] = see
    return dev(np.packbits(pad, axis=-1, bitorder="little").view(np.uint32).reshape(*see.shape[:-1], W).astype(np.int64).astype(np.uint32).view(np.int32))


def run_tree(B, H, Hkv, T, lens, count, page, kind, seed, max_len=None, shared=False, fill=float("nan"), drafts=True, spread=1.0, cap=None,
             entries=0):
    r = np.random.default_rng(seed)
    lens = np.asarray(lens).reshape(B, Hkv)
    unit = page or 1
    cap = (cap or max(int(lens.max()), 1)) + (0 if page else 3)
    cap = (cap + unit - 1) // unit * unit
    q = (bf(r, B, T, H + 1, 128).float() * spread).to(BF)             # a view with strides
    K, V = bf(r, B, Hkv, cap, 128), bf(r, B, Hkv, cap, 128)
    Kd, Vd = bf(r, B, Hkv, T + 2, 128), bf(r, B, Hkv, T + 2, 128)
    see = np.stack([random_tree(r, T, kind)[0] for _ in range(B)])
    if shared:
        see[:] = see[0]
    count = np.asarray(count)
    qf, scale = f64(q)[:, :, :H], 1 / np.sqrt(128)
    out, lse = DO.tree_attn(qf, f64(K), f64(V), lens, f64(Kd) if drafts else None, f64(Vd), see, count)
    o_tol, l_tol = tree_bound(qf, np.concatenate([f64(K), f64(Kd)], 2), np.concatenate([f64(V), f64(Vd)], 2), cap + T, scale)
    for b in range(B):                                               # what lies behind holds anything
        Kd[b, :, count[b]:], Vd[b, :, count[b]:] = fill, fill
        for g in range(Hkv):
            K[b, g, lens[b, g]:], V[b, g, lens[b, g]:] = fill, fill
    Kc, Vc, tab = paged(r, K, V, page, fill) if page else (K.cuda(), V.cuda(), None)
    if entries:                                                       # a longer table, its entries behind the pages never read
        tab = torch.cat([tab, torch.full((B, Hkv, entries), -1, dtype=torch.int32, device="cuda")], 2).contiguous()
    mask = None if kind == "chain" or not drafts else words_of(see[0] if shared else see)
    o = torch.full((B, T, H, 128), 9.0, dtype=BF, device="cuda")
    ls = torch.full((B, H, T), 9.0, device="cuda")
    st = flag()
    args = dict(Kd=Kd.cuda()[:, :, :T + 2] if drafts else None, Vd=Vd.cuda() if drafts else None, mask=mask, count=dev(count), table=tab,
                max_len=max_len, dev_status=st)
    got, gl = L.tree_attn(q.cuda()[:, :, :H], Kc, Vc, dev(lens), out=o, lse=ls, **args)
    torch.cuda.synchronize()
    assert st.item() == 0 and got is o and gl is ls
    for b in range(B):
        n = count[b]
        a, w = f64(o)[b, :n], out[b, :n]
        err = np.abs(a - w) - 2.0 ** -8 * np.abs(w)
        assert np.isfinite(a).all() and err.size == 0 or err.max() <= o_tol, (b, err.max(), o_tol)
        assert (o[b, n:] == 9).all() and (ls[b, :, n:] == 9).all()
        x, y = f64(ls)[b, :, :n], lse[b, :, :n]
        assert np.array_equal(np.isinf(x), np.isinf(y)) and (x[np.isinf(x)] < 0).all()
        fin = np.isfinite(y)
        assert (np.abs(x[fin] - y[fin]) <= l_tol + 2.0 ** -22 * np.abs(y[fin])).all()
        assert (a[np.isinf(np.transpose(y))] == 0).all()              # a row that sees nothing
    again, _ = L.tree_attn(q.cuda()[:, :, :H], Kc, Vc, dev(lens), out=o.clone(), **args)
    assert same(again, o)                                            # the same bits from run to run
    return o


@pytest.mark.parametrize("page", [0, 16, 32, 64, 128, 256])
@pytest.mark.parametrize("B,H,Hkv,T,lens,count,kind", [
    (1, 1, 1, 1, [0], [1], "chain"), (1, 1, 1, 1, [1], [1], "chain"), (1, 28, 4, 1, [216, 1, 0, 64], [1], "chain"),
    (2, 8, 2, 5, [63, 64, 65, 0], [5, 3], "tree"), (3, 4, 4, 9, [0, 15, 16, 17, 31, 32, 33, 127, 128, 129, 0, 1], [9, 0, 4], "any"),
    (1, 32, 8, 33, [130, 128, 100, 40, 257, 5, 64, 200], [33], "tree"), (2, 7, 1, 61, [300, 20], [61, 32], "tree"),
    (1, 12, 2, 64, [500, 0], [64], "any"), (1, 5, 1, 65, [90], [65], "chain"), (2, 6, 1, 1, [70, 2], [1, 0], "any")])
def test_tree_attn(page, B, H, Hkv, T, lens, count, kind):
    run_tree(B, H, Hkv, T, lens, count, page, kind, seed=T + H)


@pytest.mark.parametrize("B,H,Hkv,T,lens,count,kind,page", [
    (1, 2, 1, 256, [40], [256], "tree", 0), (1, 1, 1, 129, [0], [129], "any", 0), (1, 3, 1, 200, [129], [160], "any", 64),
    (1, 64, 1, 5, [150], [5], "tree", 16), (1, 40, 1, 3, [7], [3], "chain", 0), (1, 8, 1, 17, [1000], [17], "tree", 32)])
def test_tree_attn_wide(B, H, Hkv, T, lens, count, kind, page):
    run_tree(B, H, Hkv, T, lens, count, page, kind, seed=T)


@pytest.mark.parametrize("B,H,Hkv,T,page,seed", [
    (5, 32, 8, 13, 64, 1), (60, 32, 8, 5, 16, 2), (9, 28, 4, 40, 0, 3), (2, 48, 8, 44, 128, 4), (130, 12, 4, 7, 0, 5), (1, 6, 1, 150, 32, 6)])
def test_tree_attn_ragged_over_the_gpu(B, H, Hkv, T, page, seed):
    """Ragged lengths and counts, nothing at all among them: the run of a CTA begins and ends anywhere."""
    r = np.random.default_rng(seed)
    lens = r.integers(0, 700 if B < 20 else 150, size=(B, Hkv))
    lens[r.random((B, Hkv)) < 0.15] = 0
    lens.reshape(-1)[:3] = ([1500, 0, 128] if B < 20 else [300, 0, 128])[:lens.size]
    count = np.where(r.random(B) < 0.2, 0, r.integers(1, T + 1, size=B))
    count[0] = T
    run_tree(B, H, Hkv, T, lens.reshape(-1).tolist(), count.tolist(), page, "any", seed=seed)


@pytest.mark.parametrize("B,H,Hkv,T,page,seed", [(20, 32, 8, 13, 64, 1), (13, 28, 4, 40, 128, 2), (10, 48, 8, 44, 16, 3), (160, 1, 1, 3, 32, 4)])
def test_tree_attn_in_runs(B, H, Hkv, T, page, seed):
    """More units than SMs and caches that may be long: every CTA takes an equal run of all key tiles, and units are cut anywhere."""
    r = np.random.default_rng(seed)
    lens = r.integers(0, 600, size=(B, Hkv))
    lens[r.random((B, Hkv)) < 0.2] = 0
    far = r.random((B, Hkv)) < 0.12
    lens[far] = r.integers(1500, 3500, size=int(far.sum()))
    count = np.where(r.random(B) < 0.2, 0, r.integers(1, T + 1, size=B))
    count[0] = T
    run_tree(B, H, Hkv, T, lens.reshape(-1).tolist(), count.tolist(), page, "any", seed=seed, entries=20000 // page)


@pytest.mark.parametrize("max_len", [None, 1, 100, 3001, 100000])
@pytest.mark.parametrize("T,page", [(1, 0), (3, 64), (20, 16)])
def test_tree_attn_split_however(max_len, T, page):
    """However the keys of a head are split, and whatever length was expected."""
    run_tree(1, 4, 2, T, [3001, 170], [T], page, "tree", seed=T, max_len=max_len)
    run_tree(1, 4, 2, T, [40, 0], [T], page, "tree", seed=T, max_len=max_len, cap=3000)


def test_tree_attn_shared_mask_large_logits_no_drafts():
    run_tree(3, 8, 2, 12, [50, 9, 0, 100, 64, 128], [12, 5, 12], 16, "any", seed=1, shared=True)
    run_tree(2, 8, 2, 12, [50, 9, 0, 100], [12, 5], 0, "any", seed=2, drafts=False)
    run_tree(2, 8, 2, 12, [50, 9, 70, 100], [12, 5], 0, "any", seed=3, spread=30.0)
    run_tree(2, 8, 2, 12, [50, 9, 70, 100], [12, 5], 64, "any", seed=3, fill=float("inf"))


@pytest.mark.parametrize("B,H,Hkv,T,page,shared,max_len", [
    (3, 4, 2, 1, 16, 48, None), (3, 8, 2, 5, 64, 192, None), (2, 8, 1, 40, 32, 128, None), (2, 8, 1, 40, 64, 640, 30000), (160, 1, 1, 40, 16, 16, 20000)])
def test_pages_shared_by_sequences(B, H, Hkv, T, page, shared, max_len):
    """A prompt that all sequences begin with lies in pages that their tables share; what they append lies in pages of their own."""
    r = np.random.default_rng(B + T)
    own, cap = 2 * page, shared + 2 * page
    K, V = bf(r, 1, Hkv, shared, 128), bf(r, 1, Hkv, shared, 128)
    first = shared // page
    n_pages = Hkv * first + B * Hkv * 2 + 1
    place = r.permutation(n_pages)
    head = np.broadcast_to(place[:Hkv * first].reshape(1, Hkv, first), (B, Hkv, first))
    table = np.concatenate([head, place[Hkv * first:Hkv * first + B * Hkv * 2].reshape(B, Hkv, 2)], 2)
    wide = np.concatenate([table, np.full((B, Hkv, (max_len or 0) // page), -1)], 2)      # (a capacity for the length expected)
    Kp, Vp = (torch.full((n_pages, page, 128), float("nan"), dtype=BF) for _ in range(2))
    at = torch.from_numpy(head[0].copy())
    Kp[at.reshape(-1)], Vp[at.reshape(-1)] = K[0].reshape(-1, page, 128), V[0].reshape(-1, page, 128)
    Kp, Vp, tab = Kp.cuda(), Vp.cuda(), dev(wide)
    n_new = own - 3
    kn, vn = bf(r, B, n_new, Hkv, 128), bf(r, B, n_new, Hkv, 128)
    count = r.integers(0, n_new + 1, size=B)
    ln, st = torch.full((B, Hkv), shared, dtype=torch.int32, device="cuda"), flag()
    L.rope_append(kn.cuda(), vn.cuda(), None, None, Kp, Vp, ln, table=tab, count=dev(count), dev_status=st)
    Kw, Vw = np.zeros((B, Hkv, cap, 128)), np.zeros((B, Hkv, cap, 128))
    Kw[:, :, :shared], Vw[:, :, :shared] = f64(K), f64(V)
    Kw, Vw, want_len = DO.append(Kw, Vw, np.full((B, Hkv), shared), f64(kn), f64(vn), count)
    assert st.item() == 0 and np.array_equal(i32(ln), want_len)
    assert same(Kp[at.reshape(-1)], K[0].reshape(-1, page, 128)) and same(Vp[at.reshape(-1)], V[0].reshape(-1, page, 128))
    q, Kd, Vd = bf(r, B, T, H, 128), bf(r, B, Hkv, T, 128), bf(r, B, Hkv, T, 128)
    got, _ = L.tree_attn(q.cuda(), Kp, Vp, ln, Kd=Kd.cuda(), Vd=Vd.cuda(), table=tab, max_len=max_len, dev_status=st)
    see = np.tril(np.ones((T, T), bool))[None].repeat(B, 0)
    want, _ = DO.tree_attn(f64(q), Kw, Vw, want_len, f64(Kd), f64(Vd), see, [T] * B)
    tol, _ = tree_bound(f64(q), np.concatenate([Kw, f64(Kd)], 2), np.concatenate([Vw, f64(Vd)], 2), cap + T, 1 / np.sqrt(128))
    assert st.item() == 0 and (np.abs(f64(got) - want) <= 2.0 ** -8 * np.abs(want) + tol).all()


@pytest.mark.parametrize("T,B", [(1, 20), (17, 20), (40, 20), (40, 200)])
def test_probabilities_keep_sixteen_bits(T, B):
    """Two keys, logits 0 and -x, values -bf16(p) v and v with p = exp(-x): the result is v (p - bf16(p)) / (1 + p), nothing but what the
    first bf16 part of p leaves.  Off by: the logit, whose one product is exact, and its scale, 2^-24 a factor and a rounding, four of
    them of x log2(e) < 4.4 (2^-20); the exponential, 2^-22; the second part, 2^-8 of at most 2^-8 of p <= 1; three sums, 2^-23 each:
    below 2^-15 v in all.  Beside it the result's own rounding."""
    r = np.random.default_rng(T)
    x = r.uniform(0.05, 3.0, size=(B, 4))
    q, K, V = torch.zeros(B, T, 4, 128), torch.zeros(B, 4, 2, 128), torch.zeros(B, 4, 2, 128)
    q[..., 0] = 8.0
    K[:, :, 1, 0] = -torch.from_numpy(x * np.sqrt(128) / 8).float()
    K = K.to(BF)
    p = np.exp(f64(K)[:, :, 1, 0] * 8 / np.sqrt(128))                 # of the key as it was rounded
    v = 2.0 ** (np.arange(128) % 4)
    V[:, :, 1] = torch.from_numpy(v).float()
    V[:, :, 0] = -torch.from_numpy(p).to(BF).float()[..., None] * V[:, :, 1]
    V = V.to(BF)
    want = (f64(V)[:, :, 0] + p[..., None] * f64(V)[:, :, 1]) / (1 + p[..., None])
    assert (np.abs(want) > 2 * 2.0 ** -15 * v).mean() > 0.5           # without the second part the result would be 0, and refused below
    ln = torch.full((B, 4), 2, dtype=torch.int32, device="cuda")
    got, lse = L.tree_attn(q.to(BF).cuda(), K.cuda(), V.cuda(), ln, want_lse=True, max_len=2)
    err = np.abs(f64(got).transpose(0, 2, 1, 3) - want[:, :, None]) - 2.0 ** -8 * np.abs(want[:, :, None])
    assert (err <= 2.0 ** -15 * v).all()
    assert (np.abs(f64(lse) - np.log1p(p)[..., None]) <= 2.0 ** -20).all()


@pytest.mark.parametrize("T", [3, 60])
def test_tree_attn_flags(T):
    """A bad length, count or page number: flagged, nothing outside is read, the other heads are as without it."""
    r = np.random.default_rng(12)
    B, H, Hkv, page = 2, 4, 2, 16
    K, V, Kd, Vd, q = bf(r, B, Hkv, 48, 128), bf(r, B, Hkv, 48, 128), bf(r, B, Hkv, T, 128), bf(r, B, Hkv, T, 128), bf(r, B, T, H, 128)
    Kp, Vp, tab = paged(r, K, V, page, fill=0.0)

    def go(ln=((40, 20), (33, 7)), count=(T, T), broken=None):
        t = tab.clone()
        if broken is not None:
            t[0, 1, 0] = broken
        st, o = flag(), torch.full((B, T, H, 128), 9.0, dtype=BF, device="cuda")
        _, l = L.tree_attn(q.cuda(), Kp, Vp, dev(ln), Kd=Kd.cuda(), Vd=Vd.cuda(), table=t, count=dev(count), out=o, want_lse=True, dev_status=st)
        return st.item(), o, l

    s0, o0, l0 = go()
    assert s0 == 0
    for bad in (-1, 49, 1 << 30):
        s, o, l = go(ln=((40, 20), (bad, 7)))
        assert s == L.DEV_BOUNDS and (o[1, :, :2] == 0).all() and torch.isneginf(l[1, :2]).all()
        assert same(o[0], o0[0]) and same(o[1, :, 2:], o0[1, :, 2:])
    for bad in (-1, T + 1):
        s, o, _ = go(count=(T, bad))
        assert s == L.DEV_BOUNDS and (o[1] == 9).all() and same(o[0], o0[0])
    zeroed = K.clone(), V.clone()
    for x in zeroed:
        x[0, 1, :16] = 0                                             # the page's rows are taken as zeros
    see = np.tril(np.ones((T, T), bool))[None].repeat(B, 0)
    want, _ = DO.tree_attn(f64(q), f64(zeroed[0]), f64(zeroed[1]), np.array([[40, 20], [33, 7]]), f64(Kd), f64(Vd), see, [T, T])
    tol, _ = tree_bound(f64(q), f64(K), f64(V), 48 + T, 1 / np.sqrt(128))
    for bad in (-1, Kp.shape[0], 1 << 30, -(1 << 31)):
        s, o, _ = go(broken=bad)
        assert s == L.DEV_BOUNDS and same(o[1], o0[1]) and same(o[0, :, :2], o0[0, :, :2])
        assert (np.abs(f64(o) - want) <= 2.0 ** -8 * np.abs(want) + tol).all()


def test_far_pages():
    """A pool of more than 2^31 elements: every operator reaches its last page."""
    page, n_pages = 128, (1 << 31) // (128 * 128) + 40
    r = np.random.default_rng(13)
    Kp = torch.empty(n_pages, page, 128, dtype=BF, device="cuda")
    Vp = torch.empty_like(Kp)
    tab = dev([[[n_pages - 1, 3, n_pages - 7]]])
    B, T, H = 1, 40, 2
    kn, vn, q = bf(r, B, 300, 1, 128), bf(r, B, 300, 1, 128), bf(r, B, T, H, 128)
    ln = dev([[0]])
    L.rope_append(kn.cuda(), vn.cuda(), None, None, Kp, Vp, ln, table=tab)
    assert same(Kp[n_pages - 1], kn[0, :128, 0]) and same(Vp[n_pages - 7, :44], vn[0, 256:, 0])
    Kd, Vd = bf(r, B, 1, T, 128), bf(r, B, 1, T, 128)
    L.commit_rows(Kd.cuda(), Vd.cuda(), Kp, Vp, ln, table=tab)
    assert same(Kp[n_pages - 7, 44:84], Kd[0, 0]) and ln.item() == 340
    K = torch.cat([kn[:, :, 0], Kd[:, 0]], 1)[:, None]
    V = torch.cat([vn[:, :, 0], Vd[:, 0]], 1)[:, None]
    o, _ = L.tree_attn(q.cuda(), Kp, Vp, ln, table=tab)
    want, _ = DO.tree_attn(f64(q), f64(K), f64(V), np.array([[340]]), None, None, None, [T])
    tol, _ = tree_bound(f64(q), f64(K), f64(V), 340, 1 / np.sqrt(128))
    assert (np.abs(f64(o) - want) <= 2.0 ** -8 * np.abs(want) + tol).all()


def test_binding_refuses_what_the_call_cannot_see():
    z = torch.zeros(2, 2, 16, 128, dtype=BF, device="cuda")
    i = torch.zeros(2, 2, dtype=torch.int32, device="cuda")
    q = torch.zeros(2, 3, 4, 128, dtype=BF, device="cuda")
    for bad in (dict(q=q.half()), dict(Kc=z.float()), dict(length=i.long()), dict(Kd=z.half(), Vd=z.half()), dict(out=q.float()),
                dict(count=torch.zeros(2, device="cuda"))):
        with pytest.raises(TypeError):
            L.tree_attn(**{**dict(q=q, Kc=z, Vc=z, length=i), **bad})
    for bad in (dict(length=i[:1]), dict(Vc=z[:, :, :8]), dict(Kc=z.transpose(2, 3), Vc=z.transpose(2, 3)), dict(q=q[:, :, :1].expand(2, 3, 4, 128)),
                dict(table=i[None].repeat(2, 1, 1)), dict(Kd=z, Vd=z, mask=torch.zeros(2, 3, 2, dtype=torch.int32, device="cuda")),
                dict(out=q[:, :2]), dict(lse=torch.zeros(2, 4, 4, device="cuda")), dict(q=q[..., ::2])):
        with pytest.raises(ValueError):
            L.tree_attn(**{**dict(q=q, Kc=z, Vc=z, length=i), **bad})
    kn = q[:, :, :2]
    pos = torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    cs = L.rope_table(10)
    for bad in (dict(v_new=kn.contiguous()), dict(pos=pos.T), dict(sections=(16, 24, 24)), dict(q=q, q_out=q[:, :2]), dict(len_out=i.view(-1)),
                dict(acc_score=torch.zeros(2, 2, 15, device="cuda"))):
        with pytest.raises(ValueError):
            L.rope_append(**{**dict(k_new=kn, v_new=kn, pos=pos, cos_sin=cs, Kc=z, Vc=z, length=i), **bad})
    with pytest.raises(ValueError):
        L.commit_rows(z, z, z.clone(), z.clone(), i, torch.zeros(3, dtype=torch.int32, device="cuda"))
    with pytest.raises(L.LvlmError):
        L.commit_rows(z, z, z, z.clone(), i)
    assert (i == 0).all()


# ---- as they are used together -------------------------------------------------------------------------------------
def test_drafts_over_a_compressed_cache():
    """Compression, the caches into pages, two steps of trees, each with its accepted path committed: every output and every
    cache row against the oracle, and a plain decode step over the result."""
    from oracle import lvlm_oracle as O
    from paper_2509_00419_b200 import pipeline as P
    r = np.random.default_rng(21)
    nl, B, H, Hkv, cap, T, page = 2, 3, 8, 2, 96, 9, 16
    src = P.DecodeLayers(nl, B, H, Hkv, cap, "cuda")
    K, V = bf(r, nl, B, Hkv, cap, 128), bf(r, nl, B, Hkv, cap, 128)
    acc = r.random((nl, B, Hkv, cap)).astype(np.float32)
    ln = r.integers(60, cap + 1, size=(nl, B, Hkv)).astype(np.int32)
    src.K.copy_(K); src.V.copy_(V); src.acc.copy_(torch.from_numpy(acc)); src.len.copy_(torch.from_numpy(ln))
    src.compress(beta=0.7)
    shp = (nl * B, Hkv)
    want = O.kv_compress(f64(K).reshape(*shp, cap, 128), f64(V).reshape(*shp, cap, 128), acc.reshape(*shp, cap), ln.reshape(shp), beta=0.7)
    length = want["len"].reshape(nl, B, Hkv).copy()
    assert np.array_equal(i32(src.len), length) and length.min() < length.max()
    used = int(((length + 2 * T + page - 1) // page).sum())
    new = P.PagedLayers(nl, B, H, Hkv, used, page, (cap + 2 * T + page - 1) // page, T, "cuda")
    new.K.fill_(float("nan")); new.V.fill_(float("nan"))
    new.pack(src, extra=2 * T)
    assert new.pages_free() == 0 and used * page < nl * B * Hkv * cap
    room = cap + 2 * T
    Kw, Vw = (np.zeros((nl, B, Hkv, room, 128)) for _ in range(2))
    Kw[:, :, :, :cap], Vw[:, :, :, :cap] = want["Kc"].reshape(nl, B, Hkv, cap, 128), want["Vc"].reshape(nl, B, Hkv, cap, 128)
    cs = L.rope_table(300)
    base = np.array([100, 150, 70])
    for step in range(2):
        par = [[int(r.integers(-1, t)) if t else -1 for t in range(T)] for _ in range(B)]
        mask = L.tree_mask(torch.tensor(par)).cuda()
        see = np.zeros((B, T, T), bool)
        depth = np.zeros((B, T), int)
        for b in range(B):
            for t in range(T):
                if par[b][t] >= 0:
                    see[b, t], depth[b, t] = see[b, par[b][t]], depth[b, par[b][t]] + 1
                see[b, t, t] = True
        count = np.array([T, 4, 7])
        pos = base[:, None] + depth
        last = [int(r.integers(0, c)) for c in count]                  # the leaf whose path is accepted
        index, accepted = np.zeros((B, T), int), np.zeros(B, int)
        for b in range(B):
            path = np.flatnonzero(see[b, last[b]])
            index[b, :len(path)], accepted[b] = path, len(path)
        for l in range(nl):
            q, k, v = bf(r, B, T, H, 128), bf(r, B, T, Hkv, 128), bf(r, B, T, Hkv, 128)
            out = new.draft_layer(l, q.cuda(), k.cuda(), v.cuda(), dev(pos), cs, mask=mask, count=dev(count))
            torch.cuda.synchronize()
            qr, kr = f64(new.q), f64(new.Kd[l]).swapaxes(1, 2)
            wq, wk = DO.rotate(f64(q), pos, cs.cpu().numpy()), DO.rotate(f64(k), pos, cs.cpu().numpy())
            for b in range(B):
                assert (np.abs(qr[b, :count[b]] - wq[b, :count[b]]) <= 2.0 ** -8 * np.abs(wq[b, :count[b]]) + 2.0 ** -20).all()
                assert (np.abs(kr[b, :count[b]] - wk[b, :count[b]]) <= 2.0 ** -8 * np.abs(wk[b, :count[b]]) + 2.0 ** -20).all()
            kd = np.nan_to_num(kr.swapaxes(1, 2))                     # what was rounded to bf16 is what is attended to
            vd = f64(v).swapaxes(1, 2)
            wo, _ = DO.tree_attn(qr, Kw[l], Vw[l], length[l], kd, vd, see, count)
            tol, _ = tree_bound(np.nan_to_num(qr), np.concatenate([Kw[l], kd], 2), np.concatenate([Vw[l], vd], 2), room, 1 / np.sqrt(128))
            for b in range(B):
                assert (np.abs(f64(out)[b, :count[b]] - wo[b, :count[b]]) <= 2.0 ** -8 * np.abs(wo[b, :count[b]]) + tol).all()
            Kw[l], Vw[l], length[l] = DO.commit(Kw[l], Vw[l], length[l], kd, vd, index, accepted)
        new.commit(dev(index), dev(accepted))
        base = base + accepted
        assert new.status.item() == 0 and np.array_equal(i32(new.len), length)
        for l in range(nl):
            lg, lv = f64(logical(new.K, new.table[l].clamp_min(0))), f64(logical(new.V, new.table[l].clamp_min(0)))
            for b in range(B):
                for g in range(Hkv):
                    m = length[l, b, g]
                    assert np.array_equal(lg[b, g, :m], Kw[l, b, g, :m]) and np.array_equal(lv[b, g, :m], Vw[l, b, g, :m])
    q = bf(r, B, 1, H, 128)
    got, _ = L.tree_attn(q.cuda(), new.K, new.V, new.len[1], table=new.table[1])
    want = O.decode_attn(f64(q)[:, 0], Kw[1], Vw[1], length[1])
    tol, _ = tree_bound(f64(q), Kw[1], Vw[1], room, 1 / np.sqrt(128))
    assert (np.abs(f64(got)[:, 0] - want["out"]) <= 2.0 ** -7 * np.abs(want["out"]) + tol).all()       # (the oracle's is rounded too)
    with pytest.raises(RuntimeError):
        new.reserve(new.len.cpu() + 4 * page)


def test_a_commit_without_pages_is_no_commit():
    """Sequences whose drafts do not fit the pages that every head of every layer has stay as they were, in all layers; the others
    are committed, and with pages the rest follows."""
    from paper_2509_00419_b200 import pipeline as P
    r = np.random.default_rng(22)
    nl, B, Hkv, T, page = 2, 3, 2, 5, 16
    c = P.PagedLayers(nl, B, 4, Hkv, 40, page, 4, T, "cuda")
    c.K.fill_(float("nan")); c.V.fill_(float("nan"))
    ln = np.array([[[3, 30], [16, 12], [14, 0]], [[8, 1], [9, 32], [5, 6]]])
    c.reserve(torch.from_numpy(ln))
    K, V = (np.zeros((nl, B, Hkv, 64, 128)) for _ in range(2))
    for l in range(nl):                                              # what the heads hold, by the library's own append
        for b in range(B):
            for g in range(Hkv):
                n = int(ln[l, b, g])
                if n:
                    k, v = bf(r, 1, n, 1, 128), bf(r, 1, n, 1, 128)
                    one = c.len[l, b, g:g + 1].view(1, 1)
                    L.rope_append(k.cuda(), v.cuda(), None, None, c.K, c.V, one, table=c.table[l, b, g].view(1, 1, -1))
                    K[l, b, g, :n], V[l, b, g, :n] = f64(k)[0, :, 0], f64(v)[0, :, 0]
    Kd, Vd = bf(r, nl, B, Hkv, T, 128), bf(r, nl, B, Hkv, T, 128)
    c.Kd.copy_(Kd); c.Vd.copy_(Vd)
    index = np.stack([np.sort(r.permutation(T)) for _ in range(B)])
    count = np.array([2, 4, 2])       # of layer and sequence (0, 1) a head is full, of (1, 1) another; of (0, 2) one is empty and has no page at all

    def compare():
        lens = i32(c.len)
        assert np.array_equal(lens, ln)
        for l in range(nl):
            lk, lv = f64(logical(c.K, c.table[l].clamp_min(0))), f64(logical(c.V, c.table[l].clamp_min(0)))
            for b in range(B):
                for g in range(Hkv):
                    n = lens[l, b, g]
                    assert np.array_equal(lk[b, g, :n], K[l, b, g, :n]) and np.array_equal(lv[b, g, :n], V[l, b, g, :n])

    compare()
    c.check()
    before = c.K.clone(), c.V.clone()
    c.commit(dev(index), dev(count))
    with pytest.raises(RuntimeError):
        c.check()
    own = c.table[:, 1:][c.table[:, 1:] >= 0].long()                 # the pages of the sequences that have to wait
    assert same(c.K[own], before[0][own]) and same(c.V[own], before[1][own])
    for l in range(nl):
        K[l], V[l], ln[l] = DO.commit(K[l], V[l], ln[l], f64(Kd[l]), f64(Vd[l]), index, [2, 0, 0])
    compare()
    c.check()
    c.reserve(c.len.cpu() + T)
    c.commit(dev(index), dev([0, 4, 2]))
    for l in range(nl):
        K[l], V[l], ln[l] = DO.commit(K[l], V[l], ln[l], f64(Kd[l]), f64(Vd[l]), index, [0, 4, 2])
    compare()
    c.check()


@pytest.mark.parametrize("H,Hkv,T,lens", [(8, 2, 3, [700, 33, 5, 129]), (8, 1, 30, [3000, 100]), (2, 2, 200, [300, 40, 0, 511])])
def test_a_step_in_a_graph(H, Hkv, T, lens):
    """Append, attention and commit captured once and replayed over caches that grow: as the same calls made one by one."""
    B = len(lens) // Hkv
    r = np.random.default_rng(T)
    n_pages, page, mp = 60 * B * Hkv, 64, 60
    tab = dev(r.permutation(n_pages).reshape(B, Hkv, mp))
    K, V = bf(r, n_pages, page, 128).cuda(), bf(r, n_pages, page, 128).cuda()
    cs = L.rope_table(500)
    steps = [(bf(r, B, T, H + 2 * Hkv, 128).cuda(), dev(r.integers(0, 500, size=(B, T))), words_of(np.stack([random_tree(r, T, "tree")[0] for _ in range(B)])),
              dev(r.integers(1, T + 1, size=B)), dev(np.sort(r.integers(0, T, size=(B, T)), axis=1))) for _ in range(3)]

    def run(graph):
        Kc, Vc, ln, st = K.clone(), V.clone(), dev(np.reshape(lens, (B, Hkv))), flag()
        qkv, pos, mask, count, index = (x.clone() for x in steps[0])
        Kd, Vd = (torch.zeros(B, Hkv, T, 128, dtype=BF, device="cuda") for _ in range(2))
        qr, out, lse = torch.zeros(B, T, H, 128, dtype=BF, device="cuda"), torch.zeros(B, T, H, 128, dtype=BF, device="cuda"), torch.zeros(B, H, T, device="cuda")
        ws = L.alloc_workspace(L.OP_TREE_ATTN, L.tree_dims(qr, Kc, tab, Kd), "cuda")

        def step():
            L.rope_append(qkv[:, :, H:H + Hkv], qkv[:, :, H + Hkv:], pos, cs, Kd, Vd, q=qkv[:, :, :H], q_out=qr, count=count, dev_status=st)
            L.tree_attn(qr, Kc, Vc, ln, Kd=Kd, Vd=Vd, mask=mask, count=count, table=tab, out=out, lse=lse, ws=ws, dev_status=st)
            L.commit_rows(Kd, Vd, Kc, Vc, ln, count, index=index, table=tab, dev_status=st)

        if graph:
            saved = Kc.clone(), Vc.clone(), ln.clone()
            s = torch.cuda.Stream()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                step()
            torch.cuda.current_stream().wait_stream(s)
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                step()
            for a, b in zip((Kc, Vc, ln), saved):
                a.copy_(b)
            for x in (qr, out, lse):
                x.zero_()
        got = []
        for x in steps:
            for a, b in zip((qkv, pos, mask, count, index), x):
                a.copy_(b)
            g.replay() if graph else step()
            got += [t.clone() for t in (qr, out, lse, ln)]
        torch.cuda.synchronize()
        assert st.item() == 0
        return got + [Kc, Vc]

    for a, b in zip(run(False), run(True)):
        assert torch.equal(a, b)


def test_two_calls_at_once():
    """Two streams, a workspace each: neither disturbs the other."""
    r = np.random.default_rng(5)
    problems = []
    for B, H, Hkv, T, cap in ((2, 8, 2, 40, 3000), (1, 28, 4, 26, 3008)):
        t = [x.cuda() for x in (bf(r, B, T, H, 128), bf(r, B, Hkv, cap, 128), bf(r, B, Hkv, cap, 128), bf(r, B, Hkv, T, 128), bf(r, B, Hkv, T, 128))]
        ln = dev(r.integers(cap // 2, cap, size=(B, Hkv)))
        ws = L.alloc_workspace(L.OP_TREE_ATTN, L.tree_dims(t[0], t[1], None, t[3]), "cuda")
        alone, _ = L.tree_attn(*t[:3], ln, Kd=t[3], Vd=t[4], ws=ws)
        problems.append((t, ln, ws, alone.clone(), torch.cuda.Stream(), torch.empty_like(alone)))
    torch.cuda.synchronize()
    for _ in range(20):
        for t, ln, ws, _, s, out in problems:
            L.tree_attn(*t[:3], ln, Kd=t[3], Vd=t[4], ws=ws, out=out, stream=s)
    torch.cuda.synchronize()
    for t, ln, ws, alone, s, out in problems:
        assert same(out, alone)


def test_what_a_call_allocates_belongs_to_its_stream():
    """Results and workspace that the calls make themselves, on a stream that is behind: memory that the current stream asks for
    meanwhile is other memory."""
    r = np.random.default_rng(6)
    B, H, Hkv, T, cap = 2, 8, 2, 40, 3000
    q, Kc, Vc, Kd, Vd = [x.cuda() for x in (bf(r, B, T, H, 128), bf(r, B, Hkv, cap, 128), bf(r, B, Hkv, cap, 128), bf(r, B, Hkv, T, 128), bf(r, B, Hkv, T, 128))]
    k, v = (bf(r, B, T, Hkv, 128).cuda() for _ in range(2))
    ln, pos, cs = dev(r.integers(cap // 2, cap, size=(B, Hkv))), dev(r.integers(0, 500, size=(B, T))), L.rope_table(512)
    want, want_lse = L.tree_attn(q, Kc, Vc, ln, Kd=Kd, Vd=Vd, want_lse=True)
    Ka, Va = torch.zeros_like(Kd), torch.zeros_like(Vd)
    want_q = L.rope_append(k, v, pos, cs, Ka, Va, q=q)
    size = L.alloc_workspace(L.OP_TREE_ATTN, L.tree_dims(q, Kc, None, Kd), "cuda").numel()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
    got, lse = L.tree_attn(q, Kc, Vc, ln, Kd=Kd, Vd=Vd, want_lse=True, stream=s)
    got_q = L.rope_append(k, v, pos, cs, Ka, Va, q=q, stream=s)
    held = [torch.full((size,), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(3)]      # as large as the workspace that was let go
    torch.cuda.current_stream().synchronize()
    s.synchronize()
    assert len(held) == 3 and same(got, want) and same(got_q, want_q) and torch.equal(lse, want_lse)


# ---- forms, workspaces, waits ----------------------------------------------------------------------------------------
FORMS = [  # B, H, Hkv, T, rows, expected rows, launches
    (1, 28, 4, 1, 300, None, 1), (2, 32, 8, 8, 400, None, 1),          # mma.sync, clusters
    (1, 28, 4, 20, 100, None, 1), (1, 28, 4, 20, 1500, None, 2),       # tcgen05: a part a unit; parts, which a second launch adds
    (1, 28, 4, 1, 300, 30000, 2), (60, 32, 8, 13, 60, None, 1),        # long caches expected; units in waves
    (20, 32, 8, 13, 200, 9000, 2)]                                     # in runs


def _form(B, H, Hkv, T, rows, expected, paged_to=0):
    g = torch.Generator(device="cuda").manual_seed(rows + T)
    bfg = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()
    q, Kd, Vd = bfg(B, T, H, 128), bfg(B, Hkv, T, 128), bfg(B, Hkv, T, 128)
    page, mp = 64, max(rows, expected or 0) // 64 + 1
    used = rows // page + 1
    Kp, Vp = bfg(B * Hkv * used, page, 128), bfg(B * Hkv * used, page, 128)
    tab = torch.full((B, Hkv, mp), -1, dtype=torch.int32, device="cuda")
    tab[:, :, :used] = torch.randperm(B * Hkv * used, generator=g, device="cuda").view(B, Hkv, used).int()
    ln = torch.full((B, Hkv), rows, dtype=torch.int32, device="cuda")
    return dict(q=q, Kc=Kp, Vc=Vp, length=ln, Kd=Kd, Vd=Vd, table=tab, max_len=expected)


@pytest.mark.parametrize("B,H,Hkv,T,rows,expected,launches", FORMS)
def test_tree_form_and_workspace(B, H, Hkv, T, rows, expected, launches):
    """The form goes by the sizes; none reads what the workspace held or writes behind what it asked for."""
    a = _form(B, H, Hkv, T, rows, expected)
    d = L.tree_dims(a["q"], a["Kc"], a["table"], a["Kd"], max_len=expected)
    n = L.workspace_bytes(L.OP_TREE_ATTN, d)
    outs = []
    for fill in (0xFF, 0x00):                                        # NaN, zeros
        ws = torch.full((n + 4096,), fill, dtype=torch.uint8, device="cuda")
        if not outs:
            assert count_launches(lambda: L.tree_attn(**a, ws=ws[:n])) == launches
        outs.append(L.tree_attn(**a, ws=ws[:n], want_lse=True))
        assert ws[n:].eq(fill).all()
    assert same(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    j = torch.arange(rows, device="cuda")
    at = a["table"][:, :, j // 64].long() * 64 + j % 64
    K = torch.cat([a["Kc"].view(-1, 128)[at], a["Kd"]], 2).double().repeat_interleave(H // Hkv, 1)
    V = torch.cat([a["Vc"].view(-1, 128)[at], a["Vd"]], 2).double().repeat_interleave(H // Hkv, 1)
    x = torch.einsum("bthd,bhnd->bhtn", a["q"].double(), K) / 128 ** 0.5
    x[..., rows:].masked_fill_(~torch.ones(T, T, dtype=torch.bool, device="cuda").tril(), -torch.inf)
    want = torch.einsum("bhtn,bhnd->bthd", torch.softmax(x, -1), V)
    o_tol, l_tol = tree_bound(f64(a["q"]), f64(K), f64(V), rows + T, 1 / np.sqrt(128))
    assert ((outs[0][0].double() - want).abs() <= 2.0 ** -8 * want.abs() + o_tol).all()
    lse = torch.logsumexp(x, -1)
    assert ((outs[0][1].double() - lse).abs() <= l_tol + 2.0 ** -22 * lse.abs()).all()


def _least(a):
    """The least workspace that a call is not refused, in steps of 256 bytes."""
    lo, hi = 0, 32 << 12                                              # 32 MiB is enough for every form
    ws = torch.empty(hi * 256, dtype=torch.uint8, device="cuda")
    while lo < hi:
        mid = (lo + hi) // 2
        try:
            L.tree_attn(**a, ws=ws[:mid * 256])
            hi = mid
        except L.LvlmError as e:
            assert e.code == L.ERR_WORKSPACE
            lo = mid + 1
    return lo * 256


@pytest.mark.parametrize("B,H,Hkv,T,rows,expected,launches", FORMS + [(10, 48, 8, 44, 200, 9000, 2), (1, 48, 8, 100, 3000, 20000, 2)])
def test_tree_takes_what_its_form_needs(B, H, Hkv, T, rows, expected, launches):
    """One launch: no workspace at all.  Two: what is said to be enough covers it, and with the least of it the result is the same,
    whatever it held, and nothing behind it is written.  And with out = q."""
    a = _form(B, H, Hkv, T, rows, expected)
    want, want_lse = L.tree_attn(**a, want_lse=True)
    least = _least(a)
    assert (least > 0) == (launches == 2) and count_launches(lambda: L.tree_attn(**a)) == launches
    assert least <= L.workspace_bytes(L.OP_TREE_ATTN, L.tree_dims(a["q"], a["Kc"], a["table"], a["Kd"], max_len=expected))
    for fill in (0xFF, 0x00):
        ws = torch.full((least + 4096,), fill, dtype=torch.uint8, device="cuda")
        got, lse = L.tree_attn(**a, ws=ws[:least], want_lse=True)
        assert same(got, want) and torch.equal(lse, want_lse) and ws[least:].eq(fill).all()
    q = a["q"].clone()
    got, lse = L.tree_attn(**{**a, "q": q}, out=q, want_lse=True)     # (units that would be cut in runs are whole then: other roundings)
    o_tol, l_tol = tree_bound(f64(a["q"]), f64(torch.cat([a["Kc"].view(-1, 128), a["Kd"].view(-1, 128)])),
                              f64(torch.cat([a["Vc"].view(-1, 128), a["Vd"].view(-1, 128)])), rows + T, 1 / np.sqrt(128))
    # (either is off by its rounding and the bound; 1.01: the rounding is of the exact value, not of `want`)
    assert ((got.double() - want.double()).abs() <= 2 * 1.01 * (2.0 ** -8 * want.double().abs() + o_tol)).all()
    assert ((lse - want_lse).double().abs() <= 2 * 1.01 * (l_tol + 2.0 ** -22 * want_lse.double().abs())).all()


@pytest.mark.parametrize("case", [FORMS[0], FORMS[1], FORMS[3], FORMS[5], FORMS[6]])
def test_tree_waits_that_run_out(case):
    """Copies of the keys that never come: the call ends, says so, and the next one is right again."""
    a = _form(*case[:6])
    try:
        L.use_library(BU.build_test())
        st = flag()
        L.lib().lvlm_debug_starve_tree(1)
        L.tree_attn(**a, dev_status=st)
        torch.cuda.synchronize()
        assert st.item() & L.DEV_TIMEOUT
        L.lib().lvlm_debug_starve_tree(0)
        st.zero_()
        got, _ = L.tree_attn(**a, dev_status=st)
        torch.cuda.synchronize()
        assert st.item() == 0
        L.lib().lvlm_debug_set_pdl(0)                                # and programmatic dependent launch changes nothing
        off, _ = L.tree_attn(**a)
        torch.cuda.synchronize()
        assert same(got, off)
    finally:
        L.lib().lvlm_debug_starve_tree(0)
        L.lib().lvlm_debug_set_pdl(1)
        L.use_library(None)
    again, _ = L.tree_attn(**a)
    assert same(again, got)


@pytest.mark.parametrize("fill", [0x00, 0x7F, 0xFF, 0x01])
def test_tree_waits_that_run_out_in_long_runs(fill):
    """Runs of more segments than a scheduler is ahead: it gives up with records of cut units not written, whatever lies in their place."""
    r = np.random.default_rng(33)
    B, H, Hkv, T, page = 25, 32, 8, 13, 64
    rows = np.where(r.random((B, Hkv)) < 0.93, r.integers(0, 60, size=(B, Hkv)), 9000)
    mp = 141
    q, Kp, Vp = bf(r, B, T, H, 128).cuda(), bf(r, 64, page, 128).cuda(), bf(r, 64, page, 128).cuda()
    tab = torch.full((B, Hkv, 150), -1, dtype=torch.int32, device="cuda")
    tab[:, :, :mp] = dev(r.integers(0, 64, size=(B, Hkv, mp)))         # (pages that heads share)
    a = dict(q=q, Kc=Kp, Vc=Vp, length=dev(rows), table=tab)
    assert count_launches(lambda: L.tree_attn(**a)) == 2
    want, _ = L.tree_attn(**a)
    ws = torch.full((L.workspace_bytes(L.OP_TREE_ATTN, L.tree_dims(q, Kp, tab)),), fill, dtype=torch.uint8, device="cuda")
    try:
        L.use_library(BU.build_test())
        st = flag()
        L.lib().lvlm_debug_starve_tree(1)
        L.tree_attn(**a, ws=ws, dev_status=st)
        torch.cuda.synchronize()
        assert st.item() & L.DEV_TIMEOUT
    finally:
        L.lib().lvlm_debug_starve_tree(0)
        L.use_library(None)
    st = flag()
    assert same(L.tree_attn(**a, ws=ws, dev_status=st)[0], want) and st.item() == 0


def test_runs_with_one_half_held_up():
    """Units of one row tile in runs, heads of two and of one key tile in turn: the half that has no key tile in the next unit is through
    with it, as far as it may go, before the other has read what the halves exchanged for this one."""
    r = np.random.default_rng(32)
    B, H, Hkv, T, page = 25, 32, 8, 13, 64
    q, Kp, Vp = bf(r, B, T, H, 128).cuda(), bf(r, B * Hkv * 4, page, 128).cuda(), bf(r, B * Hkv * 4, page, 128).cuda()
    tab = torch.full((B, Hkv, 150), -1, dtype=torch.int32, device="cuda")
    tab[:, :, :4] = dev(r.permutation(B * Hkv * 4).reshape(B, Hkv, 4))
    rows = np.where(np.arange(B * Hkv) % 2 == 0, 250, 100).reshape(B, Hkv)
    a = dict(q=q, Kc=Kp, Vc=Vp, length=dev(rows), table=tab)           # (a capacity of 9600: runs)
    j = torch.arange(256, device="cuda")
    at = tab[:, :, j // page].long() * page + j % page
    K, V = (x.view(-1, 128)[at].double().repeat_interleave(H // Hkv, 1) for x in (Kp, Vp))
    x = torch.einsum("bthd,bhnd->bhtn", q.double(), K) / 128 ** 0.5
    x.masked_fill_((j >= dev(rows)[..., None]).repeat_interleave(H // Hkv, 1)[:, :, None], -torch.inf)
    want, want_lse = torch.einsum("bhtn,bhnd->bthd", torch.softmax(x, -1), V), torch.logsumexp(x, -1)
    o_tol, l_tol = tree_bound(f64(q), f64(K), f64(V), 256, 1 / np.sqrt(128))
    assert count_launches(lambda: L.tree_attn(**a)) == 2
    try:
        L.use_library(BU.build_test())
        L.lib().lvlm_debug_stall_tree(50)
        st = flag()
        got, lse = L.tree_attn(**a, want_lse=True, dev_status=st)
        torch.cuda.synchronize()
        assert st.item() == 0
    finally:
        L.lib().lvlm_debug_stall_tree(0)
        L.use_library(None)
    assert ((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + o_tol).all()
    assert ((lse.double() - want_lse).abs() <= l_tol + 2.0 ** -22 * want_lse.abs()).all()
    assert same(L.tree_attn(**a)[0], got)


def test_lengths_grow_where_they_lie():
    """One token a call into a paged cache, the length read and written by the same kernel, forty times over."""
    r = np.random.default_rng(31)
    B, Hkv, page, mp = 3, 4, 16, 5
    K = torch.zeros(B * Hkv * mp, page, 128, dtype=BF, device="cuda")
    V = torch.zeros_like(K)
    tab = dev(r.permutation(B * Hkv * mp).reshape(B, Hkv, mp))
    start = r.integers(0, 30, size=(B, Hkv))
    ln, st = dev(start), flag()
    new = bf(r, 40, B, 1, Hkv, 128).cuda()
    count = dev([1, 0, 1])
    for i in range(40):
        L.rope_append(new[i], new[i], None, None, K, V, ln, table=tab, count=count, dev_status=st)
    assert st.item() == 0 and np.array_equal(i32(ln), start + 40 * np.array([[1], [0], [1]]))
    lg = logical(K, tab)
    for b in (0, 2):
        for g in range(Hkv):
            assert same(lg[b, g, start[b, g]:start[b, g] + 40], new[:, b, 0, g])
    assert count_launches(lambda: L.rope_append(new[0], new[0], None, None, K, V, ln, table=tab, count=count)) == 1
