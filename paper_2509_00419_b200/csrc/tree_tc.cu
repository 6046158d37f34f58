// lvlm_tree_attn, many query rows or long caches: tcgen05.
//
// The T G query rows of a KV head lie in tiles of up to 128 rows, floor(128 / G) drafts with all heads of the group.  A CTA takes
// a run of the head's key tiles (128 keys: the cache, then the drafts) for two row tiles that take turns at the tensor cores, or
// for one row tile, whose key tiles the two halves of the CTA take in turn and whose results they add at the end:
//   S = Q K_j^T      operands by TMA (128-byte swizzle; a box per page where the cache is paged), 128x128 fp32 in tensor memory
//   softmax          thread = query row, running maximum and sum in the log2 domain; probabilities go back as bf16 head + bf16
//                    remainder over the logits they came from (a plain bf16 would cost as much again as the rounding of the result)
//   O += P V_j       A = P from tensor memory, B = V as it lies in memory
// The keys of a head are cut into S runs, one CTA each, so that the grid fills the SMs; the parts are added by tree_combine_kernel.
// Rows of V behind the end of the cache or of the drafts are zeroed in shared memory before they are multiplied: they may hold
// anything, and their weight of zero would not stop a NaN.
#include "exp2.cuh"
#include "sm100.cuh"
#include "tree_attn.cuh"

namespace lvlm {

using namespace sm100;

constexpr int kTT = kTreeTcRows;             // query rows a tile, keys a tile, head dim
constexpr int kTHalf = kTT * 64 * 2;         // 128 rows x 64 bf16
constexpr int kTTile = 2 * kTHalf;
constexpr int kTStages = 2;
constexpr int kTThreads = 128 + 2 * kTT;     // warp 0 TMA, warp 1 MMA, two idle, four softmax warps a half
// Registers a thread as prefill_attn.cu shares them out: 3 * 168 = 104 + 2 * 200.
constexpr int kTRegsLaunch = 168, kTRegsFew = 104, kTRegsMany = 200;
static_assert(3 * kTRegsLaunch >= kTRegsFew + 2 * kTRegsMany, "the split has to fit the registers the block is launched with");
constexpr uint32_t kTTmemCols = 512;         // S/P of the two halves | O of the two halves
constexpr float kTRescaleStep = 8.0f;

struct TreeTcSmem {
    uint64_t q_full, k_full[kTStages], k_empty[kTStages], v_full[kTStages], v_empty[kTStages], s_full[2], p_ready[2][2], o_done[2];
    uint32_t tmem_base;
    volatile int abort;
    float xm[2][kTT], xl[2][kTT];            // one row tile: (max, sum) of a row over the key tiles of either half
};

__device__ __forceinline__ bool tree_wait(uint64_t* bar, uint32_t parity, TreeTcSmem* sm, const TreeArgs& a) {
    if (mbar_try(bar, parity)) return true;
    if (sm->abort) return false;
    if (mbar_wait(bar, parity)) return true;
    sm->abort = 1;
    tree_flag(a, LVLM_DEV_TIMEOUT);
    return false;
}

// grid.x = heads * S * pairs of row tiles; the pairs of a head and run lie side by side, so that they read the keys from L2
__global__ void __launch_bounds__(kTThreads, 1)
tree_tc_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
               const __grid_constant__ CUtensorMap kdmap, const __grid_constant__ CUtensorMap vdmap, const TreeArgs a) {
    extern __shared__ unsigned char smem_dyn[];
    unsigned char* base = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_dyn) + 1023) & ~(uintptr_t)1023);
    unsigned char* sQ = base;                                     // [2] tiles
    unsigned char* sK = base + 2 * kTTile;                        // [kTStages]
    unsigned char* sV = sK + kTStages * kTTile;                   // [kTStages]
    TreeTcSmem* sm = reinterpret_cast<TreeTcSmem*>(sV + kTStages * kTTile);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        mbar_init(&sm->q_full, 1);
        for (int s = 0; s < kTStages; ++s) {
            mbar_init(&sm->k_full[s], 1); mbar_init(&sm->k_empty[s], 1);
            mbar_init(&sm->v_full[s], 1); mbar_init(&sm->v_empty[s], 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(&sm->s_full[s], 1); mbar_init(&sm->o_done[s], 1);
            mbar_init(&sm->p_ready[s][0], 4); mbar_init(&sm->p_ready[s][1], 4);
        }
        sm->abort = 0;
        fence_barrier_init();
        fence_proxy_async();
        prefetch_tmap(&qmap);
        prefetch_tmap(&kmap);
        prefetch_tmap(&vmap);
    }
    if (warp == 1) tmem_alloc(&sm->tmem_base, kTTmemCols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = sm->tmem_base;
    pdl_enter();

    const int G = a.G, T = a.T, Hkv = a.c.Hkv, pairs = (a.row_tiles + 1) / 2;
    const int pair = blockIdx.x % pairs, part = blockIdx.x / pairs % a.S, hd = blockIdx.x / pairs / a.S;
    const int b = hd / Hkv, g = hd % Hkv, tt = kTT / G;          // drafts a row tile
    const int n = tree_count(a, b), ln = tree_len(a, hd);
    const int ns = ln > 0 ? (ln + kTT - 1) / kTT : 0;
    const int nt = ln < 0 ? 0 : ns + (a.drafts ? (n + kTT - 1) / kTT : 0);
    const int per = (nt + a.S - 1) / a.S, t_lo = min(nt, part * per);
    // my row tiles 2 pair and, where it has rows that are asked for, 2 pair + 1
    const bool any = 2 * pair * tt < n;
    const int split = (2 * pair + 1) * tt >= n;                  // one row tile: its key tiles in turn
    const int nk = any ? min(nt, t_lo + per) - t_lo : 0;         // my key tiles t_lo ..
    const int nk2[2] = {split ? (nk + 1) / 2 : nk, split ? nk / 2 : nk};      // and of either half; its i-th is i, or with one row tile 2 i + u

    if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kTRegsFew));
    if (warp == 0 && nk > 0) {
        // ================= TMA producer: lane 2 x + half copies the x-th page of a tile =================
        if (lane == 0) {
            const int nq = split ? 1 : 2;
            mbar_arrive_expect_tx(&sm->q_full, (uint32_t)(nq * 2 * tt * G * 128));
            for (int u = 0; u < nq; ++u) {
                tma_load_5d(sQ + u * kTTile, &qmap, &sm->q_full, 0, 0, (2 * pair + u) * tt, g, b);
                tma_load_5d(sQ + u * kTTile + kTHalf, &qmap, &sm->q_full, 64, 0, (2 * pair + u) * tt, g, b);
            }
        }
        const int box_rows = a.c.page ? min(a.c.page, kTT) : kTT, boxes = kTT / box_rows;
        const int half = lane & 1, x = lane >> 1;
        // the page of my box of tile t; entries behind the head's length are not read: its last page again
        auto page_of = [&](int t) -> int {
            if (!a.c.page || t >= ns || x >= boxes) return 0;
            const int pg = min(t * kTT + x * box_rows, ln - 1) >> a.c.shift;
            return a.table[(int64_t)hd * a.c.max_pages + pg];
        };
        int id = page_of(t_lo);
        for (int j = 0; j < nk; ++j) {
            const int st = j % kTStages, t = t_lo + j;
            const int id_next = j + 1 < nk ? page_of(t + 1) : 0;   // asked for a tile ahead
            const bool draft = t >= ns;
            int c1 = draft ? (t - ns) * kTT : t * kTT + x * box_rows, c2 = g, c3 = b;
            if (!draft && a.c.page) {
                if (id < 0 || id >= a.c.n_pages) { tree_flag(a, LVLM_DEV_BOUNDS); id = a.c.n_pages; }    // the copy fills zeros there
                c1 &= a.c.page - 1; c2 = id; c3 = 0;
            }
            const bool mine = x < (draft ? 1 : boxes);
            const uint32_t to = st * kTTile + half * kTHalf + (draft ? 0 : x * box_rows * 128);
            if (j >= kTStages && !__all_sync(0xFFFFFFFFu, tree_wait(&sm->k_empty[st], ((j / kTStages) - 1) & 1, sm, a))) break;
            if (lane == 0) mbar_arrive_expect_tx(&sm->k_full[st], kTTile);
            __syncwarp();
            if (mine) tma_load_4d(sK + to, draft ? &kdmap : &kmap, &sm->k_full[st], half * 64, c1, c2, c3);
            if (j >= kTStages && !__all_sync(0xFFFFFFFFu, tree_wait(&sm->v_empty[st], ((j / kTStages) - 1) & 1, sm, a))) break;
            if (lane == 0) mbar_arrive_expect_tx(&sm->v_full[st], kTTile);
            __syncwarp();
            if (mine) tma_load_4d(sV + to, draft ? &vdmap : &vmap, &sm->v_full[st], half * 64, c1, c2, c3);
            id = id_next;
        }
    } else if (warp == 1 && nk > 0) {
        // ================= MMA issuer (the whole warp runs the loop, one elected lane issues) =================
        constexpr uint32_t idesc_qk = idesc_bf16_f32(kTT, kTT);
        constexpr uint32_t idesc_pv = idesc_bf16_f32(kTT, kTT) | (1u << 16);     // B (the V tile) is MN-major
        const uint64_t qd0 = smem_desc_sw128(smem_u32(sQ)), kd0 = smem_desc_sw128(smem_u32(sK));
        const uint64_t vd0 = smem_desc_mn_sw128(smem_u32(sV), kTHalf);
        auto issue_qk = [&](int u, int i) -> bool {
            const int j = split ? 2 * i + u : i, st = j % kTStages;
            if (!__all_sync(0xFFFFFFFFu, tree_wait(&sm->k_full[st], (j / kTStages) & 1, sm, a))) return false;
            tc_fence_after();
            const uint64_t qd = qd0 + (uint32_t)((split ? 0 : u) * (kTTile >> 4)), kd = kd0 + (uint32_t)(st * (kTTile >> 4));
            if (elect_one()) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const uint32_t off = ((k >> 2) * kTHalf + (k & 3) * 32) >> 4;
                    mma_bf16_ss(tmem_base + u * kTT, qd + off, kd + off, idesc_qk, k > 0 ? 1u : 0u);
                }
                mma_commit(&sm->s_full[u]);
                if (split || u == 1) mma_commit(&sm->k_empty[st]);
            }
            __syncwarp();
            return true;
        };
        bool ok = __all_sync(0xFFFFFFFFu, tree_wait(&sm->q_full, 0, sm, a));
        for (int u = 0; u < 2; ++u)
            if (ok && nk2[u] > 0) ok = issue_qk(u, 0);
        for (int i = 0; ok && i < nk2[0]; ++i) {
            for (int u = 0; ok && u < 2; ++u) {
                if (i >= nk2[u]) continue;
                const int j = split ? 2 * i + u : i, st = j % kTStages, t = t_lo + j;
                const uint64_t vd = vd0 + (uint32_t)(st * (kTTile >> 4));
                const uint32_t p_tmem = tmem_base + u * kTT, o_tmem = tmem_base + (2 + u) * kTT;
                ok = __all_sync(0xFFFFFFFFu, tree_wait(&sm->v_full[st], (j / kTStages) & 1, sm, a));
                if (!ok) break;
                if (split || u == 0) {
                    // rows of the tile that hold keys, rows that hold anything (drafts: the copy has zeroed those from T on)
                    const int r_lo = t < ns ? ln - t * kTT : n - (t - ns) * kTT, r_hi = t < ns ? kTT : min(kTT, T - (t - ns) * kTT);
                    if (r_lo < r_hi) {
                        for (int e = lane; e < (r_hi - r_lo) * 16; e += 32)         // (whole rows: their swizzle does not matter)
                            *reinterpret_cast<uint4*>(sV + st * kTTile + ((e >> 3) & 1) * kTHalf + (r_lo + (e >> 4)) * 128 + (e & 7) * 16) =
                                make_uint4(0u, 0u, 0u, 0u);
                        fence_proxy_async();
                        __syncwarp();
                    }
                }
#pragma unroll
                for (int h2 = 0; h2 < 2; ++h2) {
                    ok = __all_sync(0xFFFFFFFFu, ok && tree_wait(&sm->p_ready[u][h2], i & 1, sm, a));
                    if (!ok) break;
                    tc_fence_after();
                    if (elect_one()) {
#pragma unroll
                        for (int k = h2 * 4; k < h2 * 4 + 4; ++k) {       // 16 keys: heads in 8 columns, remainders 16 columns on
                            const uint32_t pa = p_tmem + (k >> 1) * 32 + (k & 1) * 8;
                            mma_bf16_ts(o_tmem, pa, vd + (uint32_t)(k * (2048 >> 4)), idesc_pv, i > 0 || k > 0 ? 1u : 0u);
                            mma_bf16_ts(o_tmem, pa + 16, vd + (uint32_t)(k * (2048 >> 4)), idesc_pv, 1u);
                        }
                        if (h2 == 1) {
                            if (split || u == 1) mma_commit(&sm->v_empty[st]);
                            if (i + 1 == nk2[u]) mma_commit(&sm->o_done[u]);
                        }
                    }
                    __syncwarp();
                }
                if (ok && i + 1 < nk2[u]) ok = issue_qk(u, i + 1);
            }
        }
    }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kTRegsMany));
        // ================= softmax: thread = query row =================
        const int u = (warp - 4) >> 2, quarter = warp & 3;
        const int row = quarter * 32 + lane, tile = 2 * pair + (split ? 0 : u);
        const int t = tile * tt + row / G;                       // my draft
        const bool mine = row < tt * G && t < n;
        const bool work = __any_sync(0xFFFFFFFFu, mine);         // a warp without rows only keeps the barriers going
        const uint32_t s_addr = tmem_base + ((uint32_t)(quarter * 32) << 16) + u * kTT, o_addr = s_addr + 2 * kTT;
        const int n_mine = nk2[u];
        const f32x2 sc = both(a.scale_log2);
        float m_used = -INFINITY;
        f32x2 l_run = both(0.f);
        bool ok = true;
        for (int j = 0; j < n_mine; ++j) {
            ok = __all_sync(0xFFFFFFFFu, tree_wait(&sm->s_full[u], j & 1, sm, a));
            if (!ok) break;
            tc_fence_after();
            if (!work) {
                if (lane == 0) { mbar_arrive(&sm->p_ready[u][0]); mbar_arrive(&sm->p_ready[u][1]); }
                continue;
            }
            float v[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld32(s_addr + c * 32, v[c]);
            tmem_ld_wait();
            const int kt = t_lo + (split ? 2 * j + u : j);       // my key tile
            if (kt < ns) {
                const int lim = ln - kt * kTT;                   // the same for all rows
                if (lim < kTT) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[c][e] = c * 32 + e < lim ? v[c][e] : -INFINITY;
                }
            } else {
                const int w0 = (kt - ns) * (kTT / 32);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const uint32_t bits = mine ? tree_see(a, b, t, n, w0 + c) : 0u;
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[c][e] = (bits >> e) & 1u ? v[c][e] : -INFINITY;
                }
            }
            float t0 = v[0][0], t1 = v[1][0], t2 = v[2][0], t3 = v[3][0];
#pragma unroll
            for (int e = 1; e < 32; ++e) {
                t0 = fmaxf(t0, v[0][e]); t1 = fmaxf(t1, v[1][e]); t2 = fmaxf(t2, v[2][e]); t3 = fmaxf(t3, v[3][e]);
            }
            const float tmax = fmaxf(fmaxf(t0, t1), fmaxf(t2, t3)) * a.scale_log2;       // a positive scale keeps the order
            const bool grow = tmax > -INFINITY && (m_used == -INFINITY || tmax > m_used + kTRescaleStep);
            if (__any_sync(0xFFFFFFFFu, grow)) {
                float corr = 1.f;
                if (grow) { corr = m_used == -INFINITY ? 0.f : ex2_fast(m_used - tmax); m_used = tmax; }
                if (j > 0) {
                    l_run = mul2(l_run, both(corr));
#pragma unroll 1
                    for (int c = 0; c < 4; ++c) {
                        float o[32];
                        tmem_ld32(o_addr + c * 32, o);
                        tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] *= corr;
                        tmem_st32(o_addr + c * 32, o);
                    }
                }
            }
            const f32x2 mneg = both(m_used == -INFINITY ? 0.f : -m_used);
            f32x2 ps0 = both(0.f), ps1 = both(0.f);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t pk[32];
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    float x0, x1;
                    unpack2(fma2(pack2(v[c][2 * e], v[c][2 * e + 1]), sc, mneg), x0, x1);
                    x0 = ex2_fast(x0); x1 = ex2_fast(x1);
                    const f32x2 p = pack2(x0, x1);
                    const uint32_t hi = pack_bf16(x0, x1);
                    float r0, r1;
                    unpack2(add2(p, pack2(-bf16_lo(hi), -bf16_hi(hi))), r0, r1);
                    pk[e] = hi;
                    pk[16 + e] = pack_bf16(r0, r1);
                    if (e & 1) ps1 = add2(ps1, p); else ps0 = add2(ps0, p);
                }
                tmem_st32(s_addr + c * 32, reinterpret_cast<const float*>(pk));
                if (c & 1) {                                     // half of the keys: the product may start on them
                    tmem_st_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sm->p_ready[u][c >> 1]);
                }
            }
            l_run = add2(l_run, add2(ps0, ps1));
        }
        // ---- the rows: 64 channels at a time through shared memory (the Q tiles, which nobody needs any more) ---------------
        float l0, l1;
        unpack2(l_run, l0, l1);
        float l_row = l0 + l1, f0 = 1.f, f1 = 0.f;
        if (split) {
            sm->xm[u][row] = m_used;
            sm->xl[u][row] = l_row;
            asm volatile("bar.sync 1, %0;" ::"n"(2 * kTT) : "memory");
            const float m0 = sm->xm[0][row], m1 = sm->xm[1][row];
            m_used = fmaxf(m0, m1);
            f0 = m0 > -INFINITY ? ex2_fast(m0 - m_used) : 0.f;
            f1 = m1 > -INFINITY ? ex2_fast(m1 - m_used) : 0.f;
            l_row = sm->xl[0][row] * f0 + sm->xl[1][row] * f1;
            for (int x = 0; x < 2; ++x) ok = ok && (nk2[x] == 0 || tree_wait(&sm->o_done[x], 0, sm, a));
        } else if (n_mine > 0) {
            ok = ok && tree_wait(&sm->o_done[u], 0, sm, a);
        }
        ok = __all_sync(0xFFFFFFFFu, ok) && !sm->abort;
        tc_fence_after();
        if (ok && work) {
            const bool last = a.S == 1;
            const float inv = last ? (l_row > 0.f ? 1.0f / l_row : 0.f) : 1.f;
            const uint32_t oa = split ? o_addr - u * kTT : o_addr;       // O of half 0, or of my tile
            const int64_t slot = (((int64_t)hd * a.row_tiles + tile) * a.S + part) * kTT;
            unsigned char* stage = sQ + (warp - 4) * 8192;
            const int rowB = last ? 128 : 256, msk = rowB / 16 - 1;
#pragma unroll 1
            for (int ch0 = split ? 64 * u : 0; ch0 < (split ? 64 * u + 64 : kTT); ch0 += 64) {
#pragma unroll 1
                for (int c = 0; c < 2; ++c) {
                    float o[32];
                    if (nk > 0) {
                        tmem_ld32(oa + ch0 + c * 32, o);
                        tmem_ld_wait();
                    }
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = nk > 0 && f0 > 0.f ? o[e] * f0 : 0.f;
                    if (split && nk2[1] > 0) {
                        float p[32];
                        tmem_ld32(oa + kTT + ch0 + c * 32, p);
                        tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = f1 > 0.f ? fmaf(p[e], f1, o[e]) : o[e];
                    }
                    if (last) {
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            *reinterpret_cast<uint4*>(stage + lane * rowB + (((4 * c + q) ^ (lane & msk)) << 4)) =
                                make_uint4(pack_bf16(o[8 * q] * inv, o[8 * q + 1] * inv), pack_bf16(o[8 * q + 2] * inv, o[8 * q + 3] * inv),
                                           pack_bf16(o[8 * q + 4] * inv, o[8 * q + 5] * inv), pack_bf16(o[8 * q + 6] * inv, o[8 * q + 7] * inv));
                    } else {
#pragma unroll
                        for (int q = 0; q < 8; ++q)
                            *reinterpret_cast<float4*>(stage + lane * rowB + (((8 * c + q) ^ (lane & msk)) << 4)) =
                                make_float4(o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]);
                    }
                }
                __syncwarp();
                const int step = 512 / rowB, ch = lane & msk;
#pragma unroll 4
                for (int r = lane / (rowB / 16); r < 32; r += step) {
                    const uint4 x = *reinterpret_cast<const uint4*>(stage + r * rowB + ((ch ^ (r & msk)) << 4));
                    const int rr = quarter * 32 + r, td = tile * tt + rr / G;
                    if (rr >= tt * G || td >= n) continue;
                    if (last)
                        *reinterpret_cast<uint4*>(a.out + (((int64_t)b * T + td) * a.H + g * G + rr % G) * kHeadDim + ch0 + ch * 8) = x;
                    else
                        *reinterpret_cast<uint4*>(a.part_o + (slot + rr) * kHeadDim + ch0 + ch * 4) = x;
                }
                __syncwarp();
            }
            if (mine && (!split || u == 0)) {
                if (!last) a.part_ml[slot + row] = make_float2(m_used, l_row);
                else if (a.lse) a.lse[((int64_t)b * a.H + g * G + row % G) * T + t] = l_row > 0.f ? (m_used + log2f(l_row)) * kTreeLn2 : -INFINITY;
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (sm->abort) {                              // let copies still in flight land before leaving
#pragma unroll 1
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
    }
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem_base, kTTmemCols);
    }
}

lvlm_status launch_tree_tc(const TreeArgs& a, const TreeMaps& m, cudaStream_t stream) {
    const size_t smem = 1024 + (size_t)kTTile * (2 + 2 * kTStages) + sizeof(TreeTcSmem);
    LVLM_RETURN_IF_CUDA(cudaFuncSetAttribute(tree_tc_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    static const int regs = [] {
        cudaFuncAttributes f;
        return cudaFuncGetAttributes(&f, tree_tc_kernel) == cudaSuccess ? f.numRegs : 0;
    }();
    if (3 * regs < kTRegsFew + 2 * kTRegsMany) return LVLM_ERR_CUDA;       // the split would wait for registers that nobody has
    const int64_t ctas = (int64_t)a.B * a.c.Hkv * a.S * ((a.row_tiles + 1) / 2);
    if (ctas > 0x7FFFFFFFll) return LVLM_ERR_UNSUPPORTED;
    return launch_kernel(tree_tc_kernel, dim3((unsigned)ctas), dim3(kTThreads), smem, stream, 1, m.q, m.k, m.v, m.kd, m.vd, a);
}

}  // namespace lvlm
