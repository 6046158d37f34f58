// lvlm_tree_attn, many query rows or long caches: tcgen05.
//
// The T G query rows of a KV head lie in tiles of up to 128 rows, floor(128 / G) drafts with all heads of the group.  A unit of work is
// two row tiles of a head that take turns at the tensor cores against its key tiles (128 keys: the cache, then the drafts), or one row
// tile, whose key tiles the two halves of a CTA take in turn and whose results they add at the end:
//   S = Q K_j^T      operands by TMA (128-byte swizzle; a box per page where the cache is paged), 128x128 fp32 in tensor memory
//   softmax          thread = query row, running maximum and sum in the log2 domain; probabilities go back as bf16 head + bf16
//                    remainder over the logits they came from (a plain bf16 would cost as much again as the rounding of the result)
//   O += P V_j       A = P from tensor memory, B = V as it lies in memory
// One CTA an SM.  With fewer units than SMs a unit is cut into equal parts, a CTA each.  With more, a unit is a CTA's, in waves; or, where
// long units would leave the last wave half empty (a.runs), the key tiles of all units, weighted by what they take, are laid end to end
// - on the device, which alone knows the lengths - and every CTA takes an equal run of them: a scheduler warp cuts the run into segments,
// a unit each, and the other warps work through them without stopping in between (the keys of the next segment are fetched during
// the epilogue of this one).
// A unit that is cut leaves its parts (max, sum, output) in the workspace, in runs one of them half in `out` (TreeArgs);
// tree_combine_kernel adds them in order.
// What bounds it: long calls the MMAs, 48 of 128x128x16 a turn of both row tiles, a third of them for the remainders of P.  16 sequences of up to
// 244 rows x 1888 keys 53 us (tensor pipe active 0.69 of the time on the busiest SM, which includes start and end), 4 of 1536 rows x 16640
// keys 569 to 602 us from one GPU to another (1050 to 1100 TFLOP/s, remainders counted; pipe active 0.67 on every SM).  Short calls:
// latency; of 16 us (182 rows x 3008 keys) the combining launch is 2.4.  168 registers a thread, the softmax warps' 200 are given later:
// 12 bytes of a thread spill, 48 in the form with runs.
// Rows of V behind the end of the cache or of the drafts are zeroed in shared memory before they are multiplied: they may hold
// anything, and their weight of zero would not stop a NaN.
#include <atomic>

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

constexpr int kTLeast = 4;                   // least work of a CTA that shares, in key tiles of a row tile (2 or more)
constexpr int kTWhole = 24;                  // a unit of no more work is not cut: its epilogue and the addition of its parts take longer
constexpr int kTSegs = 4;                    // segments the scheduler is ahead at most
struct TreeSeg { int hd, tile, t0, nk, split, n, ln, slot; };      // row tile(s) `tile` (and the next), key tiles t0 .. t0 + nk - 1; slot < 0: all of them; hd < 0: the end

struct TreeTcSmem {
    uint64_t seg_full[kTSegs], seg_empty[kTSegs], e_done, x_ready;
    TreeSeg seg[kTSegs];
    long long scan[kTThreads / 32], first_prefix;
    int first_head;
    TreeHead first;
    uint64_t q_full, k_full[kTStages], k_empty[kTStages], v_full[kTStages], v_empty[kTStages], s_full[2], p_ready[2][2], o_done[2];
    uint32_t tmem_base;
    volatile int abort;
    // One row tile: (max, sum) of a row over the key tiles of either half, in two buffers taken in turn: a half without a key tile in the
    // next segment waits for nothing there, and stores its own while the other half may still read these.  It comes to the first
    // buffer again behind the next exchange, which the other half joins only after it has read.
    float xm[2][2][kTT], xl[2][2][kTT];      // [buffer][half][row]
};

// Bounded: a wait that runs out sets the status, and the waits after it give up at once.
__device__ __forceinline__ bool tree_wait(uint64_t* bar, uint32_t parity, TreeTcSmem* sm, const TreeArgs& a) {
    if (mbar_try(bar, parity)) return true;
    if (sm->abort) return false;
    if (mbar_wait(bar, parity)) return true;
    sm->abort = 1;
    tree_flag(a, LVLM_DEV_TIMEOUT);
    return false;
}

// Halves of two words in one: their lower ones (selector 0x5410) or their upper ones (0x7632).
__device__ __forceinline__ uint32_t halves(float x, float y, uint32_t selector) { return __byte_perm(__float_as_uint(x), __float_as_uint(y), selector); }

// Row tiles of a head that are asked for, and what it weighs: a pair of them 2 a key tile, an odd one 1 (at most 2^30: a capacity
// that would give more, in pages that lie in a table many times, is refused); a head without keys one tile, so that its rows are written.
__device__ __forceinline__ int tree_rt(const TreeHead& h, int tt) { return h.n <= tt ? (h.n > 0) : (h.n + tt - 1) / tt; }
__device__ __forceinline__ int tree_weight(const TreeHead& h, int tt) { return max(h.nt, 1) * tree_rt(h, tt); }

// RUNS: the grid shares out the key tiles of all units; else it is (unit, part, head), a CTA has one part of one unit, and no scheduler
template <bool RUNS>
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
        mbar_init(&sm->q_full, 1); mbar_init(&sm->e_done, 8); mbar_init(&sm->x_ready, 8);
        for (int s = 0; s < kTSegs; ++s) { mbar_init(&sm->seg_full[s], 1); mbar_init(&sm->seg_empty[s], 10); }
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
    const uint32_t tmem_base = __shfl_sync(0xFFFFFFFFu, sm->tmem_base, 0);
    pdl_enter();

    const int G = a.G, T = a.T, Hkv = a.c.Hkv, heads = a.B * Hkv, tt = kTT / G;      // tt drafts a row tile
    const int me = RUNS ? blockIdx.x : (blockIdx.z * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x;
    const int pairs = a.units, ut = a.unit_tiles;
    long long total = 0, per = 0, lo = 0, hi = 0;
    if (RUNS) {
    // ---- my run [lo, hi) of the weights of all heads, and the head it begins in ------------------------------------
    const int each = (heads + kTThreads - 1) / kTThreads, h_lo = min(heads, (int)threadIdx.x * each), h_hi = min(heads, h_lo + each);
    long long sum = 0;
    TreeHead head;
#pragma unroll 1
    for (int hd = h_lo; hd < h_hi; ++hd) {
        head = tree_head(a, hd, kTT);
        sum += tree_weight(head, tt);
    }
    long long incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xFFFFFFFFu, incl, o);
        if (lane >= o) incl += x;
    }
    if (lane == 31) sm->scan[warp] = incl;
    __syncthreads();
    long long before = incl - sum;
#pragma unroll
    for (int w = 0; w < kTThreads / 32; ++w) {
        if (w < warp) before += sm->scan[w];
        total += sm->scan[w];
    }
    // equal runs, none so short that it is not worth a CTA's start
    const long long share = total >> 32 ? (total + gridDim.x - 1) / gridDim.x : (long long)(((uint32_t)total + gridDim.x - 1) / gridDim.x);
    per = max((long long)kTLeast, share);
    lo = min(total, per * me);
    hi = min(total, lo + per);
    if (lo < hi && lo >= before && lo < before + sum) {
        long long p = before;
        int hd = h_lo;
        if (each > 1)
            for (;; ++hd) {
                head = tree_head(a, hd, kTT);
                if (lo < p + tree_weight(head, tt)) break;
                p += tree_weight(head, tt);
            }
        sm->first_head = hd;
        sm->first_prefix = p;
        sm->first = head;
    }
    __syncthreads();
    }
    // the s-th segment of my run has been laid out: false where there is none
    auto segment = [&](int s) -> bool {
        if (!__all_sync(0xFFFFFFFFu, tree_wait(&sm->seg_full[s % kTSegs], (s / kTSegs) & 1, sm, a))) return false;
        return sm->seg[s % kTSegs].hd >= 0;
    };
    // and this warp does not read it any more
    auto segment_done = [&](int s) {
        __syncwarp();
        if (RUNS && lane == 0) mbar_arrive(&sm->seg_empty[s % kTSegs]);
    };

    if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kTRegsFew));
    if (warp == 0) {
        // ================= TMA producer: lane 2 x + half copies the x-th page of a tile =================
        const int box_rows = a.c.page ? min(a.c.page, kTT) : kTT, boxes = kTT / box_rows;
        const int half = lane & 1, x = lane >> 1;
        int kc = 0, qc = 0;                                       // tiles and query tiles fetched for the segments before
        auto load_q = [&](int b, int g, int tile, int nq) {
            mbar_arrive_expect_tx(&sm->q_full, (uint32_t)(nq * 2 * tt * G * 128));
            for (int u = 0; u < nq; ++u) {
                tma_load_5d(sQ + u * kTTile, &qmap, &sm->q_full, 0, 0, (tile + u) * tt, g, b);
                tma_load_5d(sQ + u * kTTile + kTHalf, &qmap, &sm->q_full, 64, 0, (tile + u) * tt, g, b);
            }
        };
        bool ok = true;
#pragma unroll 1
        for (int s = 0; ok && (RUNS || s == 0); ++s) {
            TreeSeg w;
            if (RUNS) {
                if (!segment(s)) break;
                w = sm->seg[s % kTSegs];
                segment_done(s);
            } else {
                // a part of a unit a CTA, its one segment, worked out here; the queries do not wait for the length
                const int pair = blockIdx.x, part = blockIdx.y, hd = blockIdx.z;
                if (lane == 0) load_q(hd / Hkv, hd % Hkv, ut * pair, ut);
                const TreeHead h = tree_head(a, hd, kTT);
                const int step = tree_part(h, a.S), t0 = part * step, rt = tree_rt(h, tt);
                w.hd = ut * pair < rt && (t0 < h.nt || part == 0) ? hd : -1;
                w.tile = ut * pair; w.t0 = t0; w.nk = min(h.nt - t0, step); w.split = ut == 1 || ut * pair + 1 == rt; w.n = h.n; w.ln = h.ln;
                w.slot = step >= h.nt ? -1 : me;
                if (lane == 0) {
                    sm->seg[0] = w;
                    mbar_arrive(&sm->seg_full[0]);
                }
                if (w.hd < 0 || w.nk == 0) {                      // nobody else waits for the queries, and no copy outlives its CTA
                    tree_wait(&sm->q_full, 0, sm, a);
                    break;
                }
            }
            const int b = w.hd / Hkv, g = w.hd % Hkv, ns = w.ln > 0 ? (w.ln + kTT - 1) / kTT : 0;
            // the page of my box of tile t; entries behind the head's length are not read: its last page again
            auto page_of = [&](int t) -> int {
                if (!a.c.page || t >= ns || x >= boxes) return 0;
                const int pg = min(t * kTT + x * box_rows, w.ln - 1) >> a.c.shift;
                return a.table[(int64_t)w.hd * a.c.max_pages + pg];
            };
            int id = page_of(w.t0), id_next = w.nk > 1 ? page_of(w.t0 + 1) : 0;      // asked for two tiles ahead
            // the queries: behind the first keys, once the epilogue of the segment before has left their place
            const int q_at = w.nk == 0 || !RUNS ? -1 : qc == 0 ? 0 : min(kTStages, w.nk);
#pragma unroll 1
            for (int j = 0; j <= w.nk && !tree_starved(a); ++j) {
                if (j == q_at) {
                    ok = qc == 0 || __all_sync(0xFFFFFFFFu, tree_wait(&sm->e_done, (qc - 1) & 1, sm, a));
                    if (!ok) break;
                    if (lane == 0) load_q(b, g, w.tile, w.split ? 1 : 2);
                    ++qc;
                }
                if (j == w.nk) break;
                const int i = kc + j, st = i % kTStages, t = w.t0 + j;
                const int id_after = j + 2 < w.nk ? page_of(t + 2) : 0;
                const bool draft = t >= ns;
                int c1 = draft ? (t - ns) * kTT : t * kTT + x * box_rows, c2 = g, c3 = b;
                if (!draft && a.c.page) {
                    if (id < 0 || id >= a.c.n_pages) { tree_flag(a, LVLM_DEV_BOUNDS); id = a.c.n_pages; }    // the copy fills zeros there
                    c1 &= a.c.page - 1; c2 = id; c3 = 0;
                }
                const bool mine = x < (draft ? 1 : boxes);
                const uint32_t to = st * kTTile + half * kTHalf + (draft ? 0 : x * box_rows * 128);
                ok = i < kTStages || __all_sync(0xFFFFFFFFu, tree_wait(&sm->k_empty[st], ((i / kTStages) - 1) & 1, sm, a));
                if (!ok) break;
                if (lane == 0) mbar_arrive_expect_tx(&sm->k_full[st], kTTile);
                __syncwarp();
                if (mine) tma_load_4d(sK + to, draft ? &kdmap : &kmap, &sm->k_full[st], half * 64, c1, c2, c3);
                ok = i < kTStages || __all_sync(0xFFFFFFFFu, tree_wait(&sm->v_empty[st], ((i / kTStages) - 1) & 1, sm, a));
                if (!ok) break;
                if (lane == 0) mbar_arrive_expect_tx(&sm->v_full[st], kTTile);
                __syncwarp();
                if (mine) tma_load_4d(sV + to, draft ? &vdmap : &vmap, &sm->v_full[st], half * 64, c1, c2, c3);
                id = id_next;
                id_next = id_after;
            }
            kc += w.nk;
        }
    } else if (warp == 1) {
        // ================= MMA issuer (the whole warp runs the loop, one elected lane issues) =================
        constexpr uint32_t idesc_qk = idesc_bf16_f32(kTT, kTT);
        constexpr uint32_t idesc_pv = idesc_bf16_f32(kTT, kTT) | (1u << 16);     // B (the V tile) is MN-major
        const uint64_t qd0 = smem_desc_sw128(smem_u32(sQ)), kd0 = smem_desc_sw128(smem_u32(sK));
        const uint64_t vd0 = smem_desc_mn_sw128(smem_u32(sV), kTHalf);
        int kc = 0, qc = 0, pc0 = 0, pc1 = 0;                     // of the segments before: key tiles, query tiles, tiles of either half
        bool ok = true;
#pragma unroll 1
        for (int s = 0; ok && (RUNS || s == 0); ++s) {
            if (!segment(s)) break;
            TreeSeg w = sm->seg[s % kTSegs];
            segment_done(s);
            // (broadcast, so that the compiler knows them to be the same in every lane)
            w.nk = __shfl_sync(0xFFFFFFFFu, w.nk, 0); w.split = __shfl_sync(0xFFFFFFFFu, w.split, 0);
            w.t0 = __shfl_sync(0xFFFFFFFFu, w.t0, 0); w.ln = __shfl_sync(0xFFFFFFFFu, w.ln, 0); w.n = __shfl_sync(0xFFFFFFFFu, w.n, 0);
            if (w.nk == 0) continue;
            const int split = w.split, ns = w.ln > 0 ? (w.ln + kTT - 1) / kTT : 0;
            auto tiles_of = [&](int u) { return split ? (w.nk + 1 - u) / 2 : w.nk; };          // of half u
            auto issue_qk = [&](int u, int i) -> bool {
                const int j = kc + (split ? 2 * i + u : i), st = j % kTStages;
                if ((split || u == 0) && !__all_sync(0xFFFFFFFFu, tree_wait(&sm->k_full[st], (j / kTStages) & 1, sm, a))) return false;
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
            // (the queries come once the epilogue before has read its output, so O may be written as well)
            ok = __all_sync(0xFFFFFFFFu, tree_wait(&sm->q_full, qc & 1, sm, a));
#pragma unroll
            for (int u = 0; u < 2; ++u)
                if (ok && tiles_of(u) > 0) ok = issue_qk(u, 0);
            for (int i = 0; ok && i < tiles_of(0); ++i) {
#pragma unroll
                for (int u = 0; ok && u < 2; ++u) {
                    if (i >= tiles_of(u)) continue;
                    const int jl = split ? 2 * i + u : i, j = kc + jl, st = j % kTStages, t = w.t0 + jl;
                    const uint64_t vd = vd0 + (uint32_t)(st * (kTTile >> 4));
                    const uint32_t p_tmem = tmem_base + u * kTT, o_tmem = tmem_base + (2 + u) * kTT;
                    ok = (!split && u == 1) || __all_sync(0xFFFFFFFFu, tree_wait(&sm->v_full[st], (j / kTStages) & 1, sm, a));
                    if (!ok) break;
                    if (split || u == 0) {
                        // rows of the tile that hold keys, rows that hold anything (drafts: the copy has zeroed those from T on)
                        const int r_lo = t < ns ? w.ln - t * kTT : w.n - (t - ns) * kTT, r_hi = t < ns ? kTT : min(kTT, T - (t - ns) * kTT);
                        if (r_lo < r_hi) {
#pragma unroll 1
                            for (int e = lane; e < (r_hi - r_lo) * 16; e += 32)         // (whole rows: their swizzle does not matter)
                                *reinterpret_cast<uint4*>(sV + st * kTTile + ((e >> 3) & 1) * kTHalf + (r_lo + (e >> 4)) * 128 + (e & 7) * 16) =
                                    make_uint4(0u, 0u, 0u, 0u);
                            fence_proxy_async();
                            __syncwarp();
                        }
                    }
#pragma unroll
                    for (int h2 = 0; h2 < 2; ++h2) {
                        ok = __all_sync(0xFFFFFFFFu, ok && tree_wait(&sm->p_ready[u][h2], ((u ? pc1 : pc0) + i) & 1, sm, a));
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
                                if (i + 1 == tiles_of(u)) mma_commit(&sm->o_done[u]);
                            }
                        }
                        __syncwarp();
                    }
                    if (ok && i + 1 < tiles_of(u)) ok = issue_qk(u, i + 1);
                }
            }
            kc += w.nk; ++qc;
            pc0 += tiles_of(0); pc1 += tiles_of(1);
        }
    } else if (RUNS && warp == 2) {
        // ================= scheduler: cuts my run into segments =================
        long long at = lo, p = lo < hi ? sm->first_prefix : 0;    // how far I am; where head hd begins
        int hd = lo < hi ? sm->first_head : 0, s = 0;
        TreeHead h = sm->first;
        bool ok = true;
        while (ok) {
            TreeSeg w;
            w.hd = -1;
            if (at < hi) {
                const int nt = max(h.nt, 1), rt = tree_rt(h, tt), x = (int)(at - p);
                if (x >= nt * rt) {
                    p += nt * rt;
                    h = tree_head(a, ++hd, kTT);
                    continue;
                }
                const int fp = rt / 2, pair = rt <= 2 ? 0 : min((int)((uint32_t)x / (uint32_t)(2 * nt)), fp), wt = pair < fp ? 2 : 1;
                const long long u0 = p + pair * 2 * nt;           // where the unit begins; a tile weighs wt
                // (a whole unit is the CTA's in whose run it begins)
                const bool whole = wt * nt <= kTWhole;
                const int left = (int)min((long long)(wt * nt), hi - u0);
                const int t0 = whole ? (u0 < lo ? nt : 0) : ((int)(at - u0) + wt - 1) >> (wt - 1), t1 = whole ? nt : (left + wt - 1) >> (wt - 1);
                at = u0 + wt * nt;
                if (t0 >= t1) continue;
                w.hd = hd; w.tile = 2 * pair; w.t0 = t0; w.nk = h.nt > 0 ? t1 - t0 : 0; w.split = wt == 1; w.n = h.n; w.ln = h.ln;
                w.slot = t0 > 0 ? me : t1 < nt ? kTreeTcCtas + me : -1;
                if (t0 == 0 && lane == 0) {
                    // who has the parts of this unit: I, and the CTAs up to the one with its last tile
                    const long long z = u0 + wt * (nt - 1);
                    a.part_of[(int64_t)hd * pairs + pair] = w.slot < 0 ? make_int2(-1, 0) : make_int2(me, (int)((uint32_t)(z - lo) / (uint32_t)per));
                }
            }
            ok = s < kTSegs || __all_sync(0xFFFFFFFFu, tree_wait(&sm->seg_empty[s % kTSegs], ((s / kTSegs) - 1) & 1, sm, a));
            if (!ok) break;
            if (lane == 0) {
                sm->seg[s % kTSegs] = w;
                mbar_arrive(&sm->seg_full[s % kTSegs]);
            }
            ++s;
            if (w.hd < 0) break;
        }
    }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kTRegsMany));
        // ================= softmax: thread = query row =================
        const int u = (warp - 4) >> 2, quarter = warp & 3, row = quarter * 32 + lane;
        const uint32_t s_addr = tmem_base + ((uint32_t)(quarter * 32) << 16) + u * kTT, o_addr = s_addr + 2 * kTT;
        const f32x2 sc = both(a.scale_log2);
        int jc = 0, oc = 0, xc = 0;                              // of the segments before, or their parity: tiles of my half, outputs of half u (bit u), exchanges
#pragma unroll 1
        for (int s = 0; RUNS || s == 0; ++s) {
        if (!segment(s)) break;
        const TreeSeg& w = sm->seg[s % kTSegs];                   // (read where it is needed: registers are short)
        const int split = w.split, n_mine = split ? (w.nk + 1 - u) / 2 : w.nk;
        // a warp without rows only keeps the barriers going
        const bool work = (quarter * 32 < tt * G) && (w.tile + (split ? 0 : u)) * tt + quarter * 32 / G < w.n;
        int lim = w.ln - (w.t0 + (split ? u : 0)) * kTT;         // rows of the key tile that hold keys, 0 or less: it is one of the drafts
        const int lim_step = split ? 2 * kTT : kTT;
        float m_used = -INFINITY;
        f32x2 l_run = both(0.f);
        bool ok = true;
#pragma unroll 1
        for (int j = 0; j < n_mine; ++j, lim -= lim_step) {
            ok = __all_sync(0xFFFFFFFFu, tree_wait(&sm->s_full[u], (jc + j) & 1, sm, a));
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
            if (lim < kTT) {
                const int ns = w.ln > 0 ? (w.ln + kTT - 1) / kTT : 0, t = (w.tile + (split ? 0 : u)) * tt + row / G, b = w.hd / Hkv;
                const int w0 = (w.t0 + (split ? 2 * j + u : j) - ns) * (kTT / 32);       // the tile's first mask word
                const bool mine = row < tt * G && t < w.n;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t bits;
                    if (lim > 0) bits = lim >= c * 32 + 32 ? 0xFFFFFFFFu : lim <= c * 32 ? 0u : (1u << (lim - c * 32)) - 1u;
                    else bits = mine ? tree_see(a, b, t, w.n, w0 + c) : 0u;
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
        // ---- the rows ------------------------------------------------------------------------------------------------------
        const int n = w.n, tile = w.tile + (split ? 0 : u), b = w.hd / Hkv, g = w.hd % Hkv;
        const int t = tile * tt + row / G;                       // my draft
        const bool mine = row < tt * G && t < n;
        float l0, l1;
        unpack2(l_run, l0, l1);
        float l_row = l0 + l1, f0 = 1.f, f1 = 0.f;
        if (w.nk == 0) {                                         // no key at all: zeros (such a unit is never cut)
#pragma unroll 1
            for (int r = 0; r < 32; ++r) {
                const int rr = quarter * 32 + r, td = tile * tt + rr / G;
                if ((split && u == 1) || rr >= tt * G || td >= n) continue;
                *reinterpret_cast<uint2*>(a.out + (((int64_t)b * T + td) * a.H + g * G + rr % G) * kHeadDim + lane * 4) = make_uint2(0u, 0u);
            }
            if (mine && a.lse && (!split || u == 0)) a.lse[((int64_t)b * a.H + g * G + row % G) * T + t] = -INFINITY;
            segment_done(s);
            continue;
        }
        if (split) {
            sm->xm[xc][u][row] = m_used;
            sm->xl[xc][u][row] = l_row;
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm->x_ready);
            ok = ok && tree_wait(&sm->x_ready, xc, sm, a);
            tree_stall(a, u);
            const float m0 = sm->xm[xc][0][row], m1 = sm->xm[xc][1][row];
            m_used = fmaxf(m0, m1);
            f0 = m0 > -INFINITY ? ex2_fast(m0 - m_used) : 0.f;
            f1 = m1 > -INFINITY ? ex2_fast(m1 - m_used) : 0.f;
            l_row = sm->xl[xc][0][row] * f0 + sm->xl[xc][1][row] * f1;
            xc ^= 1;
            ok = ok && (n_mine == 0 || tree_wait(&sm->o_done[u], (oc >> u) & 1, sm, a));
            ok = ok && ((w.nk + u) / 2 == 0 || tree_wait(&sm->o_done[u ^ 1], (oc >> (u ^ 1)) & 1, sm, a));
        } else {
            ok = ok && tree_wait(&sm->o_done[u], (oc >> u) & 1, sm, a);
        }
        ok = __all_sync(0xFFFFFFFFu, ok) && !sm->abort;
        tc_fence_after();
        if (ok && work) {
            const uint32_t oa = split ? o_addr - u * kTT : o_addr;       // O of half 0, or of my tile
            const int c_lo = split ? 64 * u : 0, c_hi = split ? c_lo + 64 : kTT;     // one row tile: a half finishes half of the channels
            const int place = split ? row : u * kTT + row;
            const bool begins = RUNS && w.slot >= kTreeTcCtas;           // (then w.slot is the place of its (max, sum) alone)
            const float inv = w.slot >= 0 ? 1.f : l_row > 0.f ? 1.0f / l_row : 0.f;
            f0 *= inv; f1 *= inv;
            const int my_at = mine ? t * a.H + row % G : -1;             // my row of the sequence's output
            __nv_bfloat16* out = a.out + ((int64_t)b * T * a.H + g * G) * kHeadDim + (lane & 3) * 8;
            float4* part = reinterpret_cast<float4*>(a.part_o) + (int64_t)w.slot * (kHeadDim / 4) * a.pitch + place;
            unsigned char* stage = sQ + (warp - 4) * 2048;
#pragma unroll 1
            for (int c0 = c_lo; c0 < c_hi; c0 += 32) {                   // 32 channels at a time
                float o[32];
                tmem_ld32(oa + c0, o);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 32; ++e) o[e] = f0 > 0.f ? o[e] * f0 : 0.f;
                if (split && w.nk > 1) {
                    float p[32];
                    tmem_ld32(oa + kTT + c0, p);
                    tmem_ld_wait();
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = f1 > 0.f ? fmaf(p[e], f1, o[e]) : o[e];
                }
                if (w.slot >= 0 && !begins) {
                    // a part: groups of four channels of all rows side by side, so that the threads' stores are
#pragma unroll
                    for (int q = 0; q < 8; ++q) part[(c0 / 4 + q) * a.pitch] = make_float4(o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]);
                } else {
                    // the rows themselves, through shared memory (the Q tile, which nobody needs any more); of a part that begins a unit
                    // the upper halves of its words
                    if (begins) {
                        uint2* low = a.part_lo + (int64_t)me * (kHeadDim / 4) * a.pitch + place;
#pragma unroll
                        for (int q = 0; q < 8; ++q) low[(c0 / 4 + q) * a.pitch] = make_uint2(halves(o[4 * q], o[4 * q + 1], 0x5410), halves(o[4 * q + 2], o[4 * q + 3], 0x5410));
                    }
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        uint32_t x[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[i] = begins ? halves(o[8 * q + 2 * i], o[8 * q + 2 * i + 1], 0x7632) : pack_bf16(o[8 * q + 2 * i], o[8 * q + 2 * i + 1]);
                        *reinterpret_cast<uint4*>(stage + lane * 64 + ((q ^ (lane >> 1 & 3)) << 4)) = make_uint4(x[0], x[1], x[2], x[3]);
                    }
                    __syncwarp();
#pragma unroll
                    for (int r0 = 0; r0 < 32; r0 += 8) {
                        const int r = r0 + (lane >> 2), at = __shfl_sync(0xFFFFFFFFu, my_at, r);
                        const uint4 x = *reinterpret_cast<const uint4*>(stage + r * 64 + (((lane & 3) ^ (r >> 1 & 3)) << 4));
                        if (at >= 0) *reinterpret_cast<uint4*>(out + (int64_t)at * kHeadDim + c0) = x;
                    }
                    __syncwarp();
                }
            }
            if (!split || u == 0) {
                if (w.slot >= 0) a.part_ml[(int64_t)w.slot * a.pitch + place] = make_float2(m_used, l_row);
                else if (mine && a.lse) a.lse[((int64_t)b * a.H + g * G + row % G) * T + t] = l_row > 0.f ? (m_used + log2f(l_row)) * kTreeLn2 : -INFINITY;
            }
        }
        oc ^= split && w.nk == 1 ? 1 : 3;
        jc += n_mine;
        // the next queries may come, the next output may be written
        fence_proxy_async();
        tc_fence_before();
        __syncwarp();
        segment_done(s);
        if (lane == 0) mbar_arrive(&sm->e_done);
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

template <bool RUNS>
static lvlm_status launch_tree_tc(const TreeArgs& a, const TreeMaps& m, dim3 ctas, cudaStream_t stream) {
    const size_t smem = 1024 + (size_t)kTTile * (2 + 2 * kTStages) + sizeof(TreeTcSmem);
    LVLM_RETURN_IF_CUDA(cudaFuncSetAttribute(tree_tc_kernel<RUNS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    static std::atomic<int> looked_up{0};                                  // (once; any thread finds the same)
    int regs = looked_up.load(std::memory_order_relaxed);
    if (regs == 0) {
        cudaFuncAttributes f;
        LVLM_RETURN_IF_CUDA(cudaFuncGetAttributes(&f, tree_tc_kernel<RUNS>));
        regs = f.numRegs;
        looked_up.store(regs, std::memory_order_relaxed);
    }
    if (3 * regs < kTRegsFew + 2 * kTRegsMany) return LVLM_ERR_CUDA;       // the split would wait for registers that nobody has
    return launch_kernel(tree_tc_kernel<RUNS>, ctas, dim3(kTThreads), smem, stream, 1, m.q, m.k, m.v, m.kd, m.vd, a);
}

lvlm_status launch_tree_tc(const TreeArgs& a, const TreeMaps& m, cudaStream_t stream) {
    if (a.runs) return launch_tree_tc<true>(a, m, dim3(kTreeTcCtas), stream);
    return launch_tree_tc<false>(a, m, dim3((unsigned)a.units, (unsigned)a.S, (unsigned)(a.B * a.c.Hkv)), stream);
}

}  // namespace lvlm
