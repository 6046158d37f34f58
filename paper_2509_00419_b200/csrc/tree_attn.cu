// lvlm_tree_attn: the drafted tokens of a sequence attend to its cache (contiguous or paged, ragged per KV head) and to one
// another through a mask.
//
// For every (sequence, KV head) the T G query rows of the group (row r = draft r / G, head r % G of the group) meet the
// same keys: len cache rows, then the count drafts.  An online softmax runs over the keys.
//
// Few rows (tree_mma_kernel, here): mma.sync, one or two groups of 16 query rows a CTA.  A CTA is a producer warp and four compute
// warps a group around a ring of stages of 64 keys, fetched by TMA tile copies (a box per page and 64 channels); a warp takes 16
// keys of a stage.  The keys of a head are cut into runs for the CTAs of a cluster; the warps are added in shared memory, the CTAs through
// distributed shared memory: one launch, no workspace.
// Many rows, or few heads with many keys: tree_tc.cu, on tcgen05; parts of a unit that it cut are added by tree_combine_kernel, here.
#include "exp2.cuh"
#include "sm100.cuh"
#include "tree_attn.cuh"

namespace lvlm {

using namespace sm100;

constexpr int kTreeRows = 16;                        // query rows of a group
constexpr int kTreeStageKeys = 64;
constexpr int kTreeBox = kTreeStageKeys * 128;       // 64 keys x 64 channels
constexpr int kTreeStageBytes = 4 * kTreeBox;        // K low, K high, V low, V high channels
constexpr int kTreeMaxCluster = 8;
static_assert(2 * kTreeRows <= 32, "at most 32 rows, so at most 32 drafts: a mask word a row");
constexpr int kTreePitch = kHeadDim + 4;             // of a row of the results in shared memory

// R groups: two CTAs an SM with a ring of 96 KB each, or one with 192 KB.
template <int R> struct TreeMma {
    static constexpr int kWarps = 4 * R, kThreads = (kWarps + 1) * 32, kStages = R == 1 ? 3 : 6;
    static constexpr size_t kSmem = 1024 + (size_t)kStages * kTreeStageBytes;
    static_assert(kSmem <= kMaxDynSmem && kWarps * kTreeRows * kTreePitch * 4 <= kStages * kTreeStageBytes, "");
};

__device__ __forceinline__ void tree_ldmatrix(uint32_t addr, uint32_t* r) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];\n"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void tree_ldmatrix_trans(uint32_t addr, uint32_t* r) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];\n"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
// D (16x8 fp32) += A (16x16 bf16, row) * B (16x8 bf16, col)
__device__ __forceinline__ void tree_mma(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};\n"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Offset inside a stage of the 16-byte chunk `ch` (0..15) of key row `r`: half boxes of 64 channels, rows of 128 bytes,
// chunks XOR-swizzled with the row as the TMA copy wrote them.
__device__ __forceinline__ uint32_t tree_off(int r, int ch) {
    return (uint32_t)((ch >> 3) * kTreeBox + r * 128 + (((ch & 7) ^ (r & 7)) << 4));
}

// grid.x = (head, rank), clusters of S CTAs: all rows of a head are a CTA's
template <int R>
__global__ void __launch_bounds__(TreeMma<R>::kThreads, R == 1 ? 2 : 1)
tree_mma_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
                const __grid_constant__ CUtensorMap kdmap, const __grid_constant__ CUtensorMap vdmap, const TreeArgs a) {
    constexpr int kWarps = TreeMma<R>::kWarps, kThreads = TreeMma<R>::kThreads, kStages = TreeMma<R>::kStages, kRows = R * kTreeRows;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    __shared__ uint64_t s_full[kStages], s_empty[kStages];
    __shared__ float2 s_ml[kWarps][kTreeRows], s_ML[kRows];
    __shared__ int s_abort;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) { mbar_init(&s_full[s], 1); mbar_init(&s_empty[s], kWarps); }
        s_abort = 0;
        fence_barrier_init();
    }
    if (tid == 32) { prefetch_tmap(&kmap); prefetch_tmap(&vmap); prefetch_tmap(&kdmap); prefetch_tmap(&vdmap); }
    __syncthreads();
    pdl_enter();
    const int S = a.S, T = a.T, G = a.G, Hkv = a.c.Hkv;
    const int part = (int)cluster_ctarank(), hd = blockIdx.x / S, b = hd / Hkv, g = hd % Hkv;
    const TreeHead h = tree_head(a, hd, kTreeStageKeys);
    const int n = h.n, ln = h.ln, ns = h.ns, rows = n * G;      // rows behind `rows` are not asked for
    if (rows == 0) return;
    // a head whose length is bad has no keys and gives zeros
    const int per = (h.nt + S - 1) / S, t_lo = min(h.nt, part * per), nstage = min(h.nt, t_lo + per) - t_lo;

    const int row = lane >> 2, qd = lane & 3, kq = warp & 3, gr0 = (warp >> 2) * kTreeRows;          // my group's rows; mine are row and row + 8 of them
    float o[16][4], m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    volatile int* abort_flag = &s_abort;
    auto wait_on = [&](uint64_t* bar, uint32_t parity) -> bool {
        if (*abort_flag) return false;
        if (mbar_wait(bar, parity)) return true;
        *abort_flag = 1;
        tree_flag(a, LVLM_DEV_TIMEOUT);
        return false;
    };
    if (warp == kWarps) {
        // ---- producer: lane i copies the i-th box of K and V halves of a stage ----------------------------------
        const int box_rows = a.c.page ? min(a.c.page, kTreeStageKeys) : kTreeStageKeys, boxes = kTreeStageKeys / box_rows;    // 1, 2 or 4
        const int quarter = lane & 3, bx = lane >> 2;
        // the page of my box of stage st; entries behind the head's length are not read: its last page again
        auto page_of = [&](int st) -> int {
            if (!a.c.page || st >= ns || bx >= boxes) return 0;
            return a.table[(int64_t)hd * a.c.max_pages + (min(st * kTreeStageKeys + bx * box_rows, ln - 1) >> a.c.shift)];
        };
        int id = page_of(t_lo);
        for (int i = 0; i < nstage && !tree_starved(a); ++i) {
            const int s = i % kStages, st = t_lo + i;
            const int id_next = i + 1 < nstage ? page_of(st + 1) : 0;      // asked for a stage ahead
            if (i >= kStages && !__all_sync(0xFFFFFFFFu, wait_on(&s_empty[s], (uint32_t)(i / kStages - 1) & 1u))) break;
            if (lane == 0) mbar_arrive_expect_tx(&s_full[s], kTreeStageBytes);
            __syncwarp();
            unsigned char* to = smem + s * kTreeStageBytes + quarter * kTreeBox;
            if (st >= ns) {
                if (lane < 4) tma_load_4d(to, quarter < 2 ? &kdmap : &vdmap, &s_full[s], (quarter & 1) * 64, (st - ns) * kTreeStageKeys, g, b);
            } else if (bx < boxes) {
                int c1 = st * kTreeStageKeys + bx * box_rows, c2 = g, c3 = b;
                if (a.c.page) {
                    if (id < 0 || id >= a.c.n_pages) { tree_flag(a, LVLM_DEV_BOUNDS); id = a.c.n_pages; }   // the copy fills zeros there
                    c1 &= a.c.page - 1; c2 = id; c3 = 0;
                }
                tma_load_4d(to + bx * box_rows * 128, quarter < 2 ? &kmap : &vmap, &s_full[s], (quarter & 1) * 64, c1, c2, c3);
            }
            id = id_next;
        }
    } else {
        uint32_t qa[8][4];
        const uint32_t* qp[2];
        uint32_t see[2];                                        // draft mask of my two rows
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int r = gr0 + row + 8 * u, t = r / G, hh = r % G;
            qp[u] = r < rows ? reinterpret_cast<const uint32_t*>(a.q + (int64_t)b * a.q_sb + (int64_t)t * a.q_sn + (int64_t)(g * G + hh) * a.q_sh) : nullptr;
            see[u] = r < rows ? tree_see(a, b, t, n, 0) : 0u;
        }
#pragma unroll
        for (int ks = 0; ks < 8; ++ks)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                qa[ks][u] = qp[u] ? *(qp[u] + ks * 8 + qd) : 0u;
                qa[ks][2 + u] = qp[u] ? *(qp[u] + ks * 8 + 4 + qd) : 0u;
            }
        for (int i = 0; i < nstage; ++i) {
            const int s = i % kStages, st = t_lo + i;
            const bool draft = st >= ns;
            const int k0 = (draft ? st - ns : st) * kTreeStageKeys + kq * 16, kend = draft ? n : ln;   // my keys, of how many
            const bool ok = __all_sync(0xFFFFFFFFu, wait_on(&s_full[s], (uint32_t)(i / kStages) & 1u));
            if (ok && k0 < kend && gr0 < rows) {
                const uint32_t at = smem_u32(smem) + s * kTreeStageBytes;
                const int rr = kq * 16;
                // rows behind the end hold anything: their weight is zero, so must be V (every group's warp writes the zeros that it reads)
                if (k0 + 16 > kend) {
                    for (int e = lane; e < (k0 + 16 - kend) * 16; e += 32)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};"
                                     ::"r"(at + 2 * kTreeBox + tree_off(rr + (kend - k0) + (e >> 4), e & 15)), "r"(0u) : "memory");
                    fence_proxy_async();
                    __syncwarp();
                }
                float sc[2][4];
#pragma unroll
                for (int x = 0; x < 2; ++x) sc[x][0] = sc[x][1] = sc[x][2] = sc[x][3] = 0.f;
                const int mi = lane >> 3, r8 = lane & 7;
#pragma unroll
                for (int ks = 0; ks < 8; ++ks) {
                    uint32_t kb[4];
                    tree_ldmatrix(at + tree_off(rr + (mi >> 1) * 8 + r8, 2 * ks + (mi & 1)), kb);
                    tree_mma(sc[0], qa[ks], kb[0], kb[1]);
                    tree_mma(sc[1], qa[ks], kb[2], kb[3]);
                }
                // entry (x, e): row + 8 (e >> 1), key k0 + 8 x + 2 qd + (e & 1)
                float tmax[2] = {-INFINITY, -INFINITY};
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int j = k0 + 8 * x + 2 * qd + (e & 1), u = e >> 1;
                        bool vis = j < kend;
                        if (draft) vis = vis && ((see[u] >> (j & 31)) & 1u);       // (j < kend <= 32 where it counts)
                        sc[x][e] = vis ? sc[x][e] * a.scale_log2 : -INFINITY;
                        tmax[u] = fmaxf(tmax[u], sc[x][e]);
                    }
                float corr[2], mu[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    tmax[u] = fmaxf(tmax[u], __shfl_xor_sync(0xFFFFFFFFu, tmax[u], 1));
                    tmax[u] = fmaxf(tmax[u], __shfl_xor_sync(0xFFFFFFFFu, tmax[u], 2));
                    const float m_new = fmaxf(m_run[u], tmax[u]);
                    corr[u] = m_run[u] == -INFINITY ? 0.f : ex2_fast(m_run[u] - m_new);
                    m_run[u] = m_new;
                    mu[u] = m_new == -INFINITY ? 0.f : m_new;    // nothing seen yet: every probability is 2^-inf
                }
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sc[x][e] = ex2_fast(sc[x][e] - mu[e >> 1]);
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    l_run[u] = l_run[u] * corr[u] + (sc[0][2 * u] + sc[0][2 * u + 1]) + (sc[1][2 * u] + sc[1][2 * u + 1]);
#pragma unroll
                for (int c = 0; c < 16; ++c) { o[c][0] *= corr[0]; o[c][1] *= corr[0]; o[c][2] *= corr[1]; o[c][3] *= corr[1]; }
                // P as a bf16 head and a bf16 remainder: the product keeps 16 bits of it
                uint32_t hi[4], lo[4];
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const float p0 = sc[x][2 * u], p1 = sc[x][2 * u + 1];
                        const uint32_t w = pack_bf16(p0, p1);
                        hi[2 * x + u] = w;
                        lo[2 * x + u] = pack_bf16(p0 - bf16_lo(w), p1 - bf16_hi(w));
                    }
#pragma unroll
                for (int dp = 0; dp < 8; ++dp) {
                    uint32_t vb[4];
                    tree_ldmatrix_trans(at + 2 * kTreeBox + tree_off(rr + (mi & 1) * 8 + r8, 2 * dp + (mi >> 1)), vb);
                    tree_mma(o[2 * dp], hi, vb[0], vb[1]);
                    tree_mma(o[2 * dp + 1], hi, vb[2], vb[3]);
                    tree_mma(o[2 * dp], lo, vb[0], vb[1]);
                    tree_mma(o[2 * dp + 1], lo, vb[2], vb[3]);
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&s_empty[s]);
        }
    }
    // ---- the four warps' results, in warp order, through the ring ---------------------------------------------------
    __syncthreads();
    if (s_abort) {                                              // copies may still be in flight: let them land
#pragma unroll 1
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
        __syncthreads();
    }
    float* so = reinterpret_cast<float*>(smem);                 // [warps][16][132]
    if (warp < kWarps) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            l_run[u] += __shfl_xor_sync(0xFFFFFFFFu, l_run[u], 1);
            l_run[u] += __shfl_xor_sync(0xFFFFFFFFu, l_run[u], 2);
            if (qd == 0) s_ml[warp][row + 8 * u] = make_float2(m_run[u], l_run[u]);
#pragma unroll
            for (int c = 0; c < 16; ++c)
                *reinterpret_cast<float2*>(so + (warp * kTreeRows + row + 8 * u) * kTreePitch + c * 8 + qd * 2) = make_float2(o[c][2 * u], o[c][2 * u + 1]);
        }
    }
    __syncthreads();
    for (int idx = tid; idx < kRows * (kHeadDim / 4); idx += kThreads) {
        const int rr = idx / (kHeadDim / 4), c4 = idx % (kHeadDim / 4);
        const int w0 = rr / kTreeRows * 4, rg = rr % kTreeRows;
        float M = -INFINITY, Ls = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < 4; ++w) M = fmaxf(M, s_ml[w0 + w][rg].x);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float2 ml = s_ml[w0 + w][rg];
            const float f = ml.x > -INFINITY ? ex2_fast(ml.x - M) : 0.f;
            const float4 x = *reinterpret_cast<const float4*>(so + ((w0 + w) * kTreeRows + rg) * kTreePitch + c4 * 4);
            v.x += x.x * f; v.y += x.y * f; v.z += x.z * f; v.w += x.w * f;
            Ls += ml.y * f;
        }
        // (over the group's first warp's, which only this thread reads)
        *reinterpret_cast<float4*>(so + (w0 * kTreeRows + rg) * kTreePitch + c4 * 4) = v;
        if (c4 == 0) s_ML[rr] = make_float2(M, Ls);
    }
    // ---- the CTAs of the cluster, in rank order; a CTA finishes a slice of the rows and channels ---------------------------
    cluster_barrier();
    for (int idx = part * kThreads + tid; idx < kRows * (kHeadDim / 4); idx += S * kThreads) {
        const int rr = idx / (kHeadDim / 4), c4 = idx % (kHeadDim / 4);
        if (rr >= rows) continue;
        const float* mine = so + (rr / kTreeRows * 4 * kTreeRows + rr % kTreeRows) * kTreePitch + c4 * 4;
        float2 ml[kTreeMaxCluster];
        float4 x[kTreeMaxCluster];
#pragma unroll
        for (int c = 0; c < kTreeMaxCluster; ++c) {
            ml[c] = make_float2(-INFINITY, 0.f);
            x[c] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (c < S) {
                ml[c] = cluster_ld(&s_ML[rr], c);
                x[c] = cluster_ld(reinterpret_cast<const float4*>(mine), c);
            }
        }
        float M = -INFINITY, Ls = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int c = 0; c < kTreeMaxCluster; ++c) M = fmaxf(M, ml[c].x);
#pragma unroll
        for (int c = 0; c < kTreeMaxCluster; ++c) {
            const float f = ml[c].x > -INFINITY ? ex2_fast(ml[c].x - M) : 0.f;
            v.x += x[c].x * f; v.y += x[c].y * f; v.z += x[c].z * f; v.w += x[c].w * f;
            Ls += ml[c].y * f;
        }
        const int t = rr / G, hq = g * G + rr % G;
        const float inv = Ls > 0.f ? 1.0f / Ls : 0.f;
        *reinterpret_cast<uint2*>(a.out + (((int64_t)b * T + t) * a.H + hq) * kHeadDim + c4 * 4) =
            make_uint2(pack_bf16(v.x * inv, v.y * inv), pack_bf16(v.z * inv, v.w * inv));
        if (a.lse && c4 == 0) a.lse[((int64_t)b * a.H + hq) * T + t] = Ls > 0.f ? (M + log2f(Ls)) * kTreeLn2 : -INFINITY;
    }
    cluster_arrive_exec();                                      // my reads of the other CTAs' shared memory are done
    cluster_wait();                                             // and nobody leaves while its own is still read
}

// Adds the parts of a unit that was cut.  Lane = row, a warp CH groups of four channels of 32 rows: the loads are the lines that the parts
// were stored in.  SL warps share the same channels: each takes every SL-th part, and they are added in their order.  grid (units, row
// blocks, channel blocks).  Bound by latency where parts are many and units few: lengths are read before the wait for the kernel ahead
// (it has waited for whatever wrote them), the first outputs are on their way while the weights are worked out, which the warps share.
// 4 units of 37 parts: 9.5 us with a warp going through all parts, 4.8 with four.
constexpr int kTreeCombineWarps = 8;
constexpr int kTreeMostParts = kTreeTcCtas;
template <int CH, int SL, bool RUNS>
__global__ void __launch_bounds__(kTreeCombineWarps * 32) tree_combine_kernel(const TreeArgs a) {
    __shared__ float s_m[kTreeMostParts][32], s_l[kTreeMostParts][32];
    __shared__ float4 s_v[SL > 1 ? kTreeCombineWarps : 1][32];
    __shared__ float s_ls[SL > 1 ? kTreeCombineWarps : 1][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, slice = warp % SL;
    const int hd = blockIdx.x / a.units, unit = blockIdx.x % a.units, b = hd / a.c.Hkv, g = hd % a.c.Hkv;
    const int place = blockIdx.y * 32 + lane, row = place % kTreeTcRows, tile = unit * a.unit_tiles + place / kTreeTcRows;
    const TreeHead h = tree_head(a, hd, kTreeTcRows);
    pdl_enter();
    if (unit * a.unit_tiles * a.tile_rows >= h.n * a.G) return; // nothing asked for
    int2 of;                                                    // first slot and how many more parts
    if (RUNS) {
        of = a.part_of[blockIdx.x];
        if (of.x >= 0 && !tree_record(of.x, of.y)) {            // (uniform over the block, like all that ends it here)
            if (threadIdx.x == 0) tree_flag(a, LVLM_DEV_TIMEOUT);
            return;
        }
    } else {
        const int step = tree_part(h, a.S);
        of = make_int2(step >= h.nt ? -1 : hd * a.S * a.units + unit, (h.nt - 1) / step);
    }
    if (of.x < 0) return;                                       // not cut
    const int r = tile * a.tile_rows + row, t = r / a.G;
    const bool mine = row < a.tile_rows && t < h.n;
    const int c0 = (blockIdx.z * (kTreeCombineWarps / SL) + warp / SL) * CH, parts = min(of.y + 1, kTreeMostParts);
    auto slot = [&](int p) -> int64_t { return RUNS ? (p == 0 ? kTreeTcCtas + of.x : of.x + p) : of.x + a.units * p; };
    const int head = g * a.G + r % a.G;
    uint2* to = reinterpret_cast<uint2*>(a.out + (((int64_t)b * a.T + t) * a.H + head) * kHeadDim) + c0;
    constexpr int kAhead = 16 / CH;
    static_assert(!RUNS || SL == 1, "the thread that reads what lies in a row of out writes it");
    float4 x[kAhead][CH];
    auto fetch = [&](int p0) {                                  // parts p0, p0 + SL, ...
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (RUNS && p0 + u == 0) {                          // in two halves: see TreeArgs
                const uint2* low = a.part_lo + (int64_t)of.x * (kHeadDim / 4) * a.pitch + place;
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    const uint2 up = mine ? to[c] : make_uint2(0u, 0u), lo = low[(c0 + c) * a.pitch];
                    x[u][c] = make_float4(__uint_as_float(__byte_perm(lo.x, up.x, 0x5410)), __uint_as_float(__byte_perm(lo.x, up.x, 0x7632)),
                                          __uint_as_float(__byte_perm(lo.y, up.y, 0x5410)), __uint_as_float(__byte_perm(lo.y, up.y, 0x7632)));
                }
            } else if (p0 + u * SL < parts) {
                const float4* from = reinterpret_cast<const float4*>(a.part_o + slot(p0 + u * SL) * a.pitch * kHeadDim) + place;
#pragma unroll
                for (int c = 0; c < CH; ++c) x[u][c] = from[(c0 + c) * a.pitch];
            }
    };
    fetch(slice);
    for (int p = warp; p < parts; p += kTreeCombineWarps) {
        const float2 ml = a.part_ml[slot(p) * a.pitch + place];
        s_m[p][lane] = ml.x;
        s_l[p][lane] = ml.y;
    }
    __syncthreads();
    float M = -INFINITY, Ls = 0.f;
#pragma unroll 8
    for (int p = 0; p < parts; ++p) M = fmaxf(M, s_m[p][lane]);
    float4 v[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) v[c] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int p0 = slice; p0 < parts;) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int p = p0 + u * SL;
            if (p >= parts) break;
            const float m = s_m[p][lane];
            if (m == -INFINITY) continue;                       // (without weight)
            const float w = ex2_fast(m - M);
            Ls += s_l[p][lane] * w;
#pragma unroll
            for (int c = 0; c < CH; ++c) { v[c].x += x[u][c].x * w; v[c].y += x[u][c].y * w; v[c].z += x[u][c].z * w; v[c].w += x[u][c].w * w; }
        }
        p0 += kAhead * SL;
        if (p0 < parts) fetch(p0);
    }
    if (SL > 1) {
        s_v[warp][lane] = v[0];
        s_ls[warp][lane] = Ls;
        __syncthreads();
        if (slice > 0) return;
#pragma unroll
        for (int w = 1; w < SL; ++w) {
            const float4 y = s_v[warp + w][lane];
            v[0].x += y.x; v[0].y += y.y; v[0].z += y.z; v[0].w += y.w;
            Ls += s_ls[warp + w][lane];
        }
    }
    if (!mine) return;
    const float inv = Ls > 0.f ? 1.0f / Ls : 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) to[c] = make_uint2(pack_bf16(v[c].x * inv, v[c].y * inv), pack_bf16(v[c].z * inv, v[c].w * inv));
    if (a.lse && c0 == 0) a.lse[((int64_t)b * a.H + head) * a.T + t] = Ls > 0.f ? (M + log2f(Ls)) * kTreeLn2 : -INFINITY;
}

// Row tiles of a unit of the tcgen05 kernel.  Two share the keys that they read; one makes twice as many units, which fill the SMs
// better and end sooner.  us, one / two: 4 heads of 4 tiles x 216 keys 11.3 / 16.8, 64 of 2 x 3008 47 / 54, 8 of 2 x 33000 56 / 58,
// 16 of 2 x 9000 42 / 40, 16 of 2 x 33000 118 / 95, 8 of 6 x 33000 150 / 135.
static int tree_unit_tiles(int64_t heads, int tiles, int64_t keys) {
    return tiles > 1 && (heads * tiles > kTreeTcCtas || (keys > 16000 && heads * tiles >= 32)) ? 2 : 1;
}

// How a call is carried out.  `need` is what this form uses, `total` what a caller is told: at least what any problem that is no larger
// uses, so that it never shrinks as a problem grows.
struct TreeLayout {
    int tc, R, runs, S, tiles, unit_tiles, units, pitch;
    int64_t ctas;
    size_t off_o, off_lo, off_of, need, total;
};

// Bytes of the parts of units, and of runs: rows of (max, sum), of outputs, of the lower halves of those that begin a unit, and who has them.
static size_t parts_bytes(int64_t places) { return align_up((size_t)places * 8, 256) + (size_t)places * kHeadDim * 4; }
static size_t runs_bytes(int64_t pitch, int64_t units) {
    return (size_t)kTreeTcCtas * pitch * (2 * 8 + kHeadDim * 4 + kHeadDim * 2) + align_up((size_t)units * 8, 256);
}
static void tree_workspace(TreeLayout* L, int64_t heads) {
    const size_t places = (size_t)kTreeTcCtas * L->pitch;                    // a slot a CTA (a multiple of 256 bytes of anything)
    if (L->runs) {
        L->off_o = 2 * places * 8;
        L->off_lo = L->off_o + places * kHeadDim * 4;
        L->off_of = L->off_lo + places * kHeadDim * 2;
        L->need = runs_bytes(L->pitch, heads * L->units);
    } else {
        const int64_t used = L->tc && L->S > 1 ? heads * L->units * L->S * L->pitch : 0;
        L->off_o = align_up((size_t)used * 8, 256);
        L->off_lo = L->off_of = 0;
        L->need = used ? parts_bytes(used) : 0;
    }
}

static bool tree_layout(const lvlm_dims* d, int64_t cap, TreeLayout* L) {
    if (d->B <= 0 || d->H <= 0 || d->Hkv <= 0 || d->H % d->Hkv || d->T <= 0 || d->T > kTreeMaxT || d->H / d->Hkv > kTreeMaxGroup || cap <= 0) return false;
    const int G = d->H / d->Hkv, rows = d->T * G;
    const int64_t heads = (int64_t)d->B * d->Hkv;
    const int64_t keys = d->N > 0 && d->N < cap ? d->N : cap;
    const int drafts = d->draft_cap > 0 ? d->T : 0;
    // tcgen05: units in as many parts as fill the SMs
    const int tc_rows = kTreeTcRows / G * G, tiles = (rows + tc_rows - 1) / tc_rows;
    const int64_t tc_steps = (keys + kTreeTcRows - 1) / kTreeTcRows + (drafts + kTreeTcRows - 1) / kTreeTcRows;
    const int unit_tiles = tree_unit_tiles(heads, tiles, keys), tc_units = (tiles + unit_tiles - 1) / unit_tiles;
    const int64_t units = heads * tc_units;
    int64_t parts = units < kTreeTcCtas ? kTreeTcCtas / units : 1;
    const int64_t most = (tc_steps + 1) / 2;                 // (two key tiles a part: one, and more parts, is no faster)
    parts = parts > most ? most : parts;
    // More units than SMs: a CTA each, in waves, or runs.  Estimates of either in us, for equal lengths (us measured, waves / runs): 256 units of
    // two row tiles, 216 keys 40 / 52, 1100 72 / 85, 3008 153 / 164, 9000 440 / 479; 160 of one, 1100 keys 46 / 53, 9000 232 / 151; 224
    // of two, 3008 keys 150 / 143, 16640 700 / 577.
    const double turn = unit_tiles == 2 ? 2.85 : 1.45, waves_us = (double)((units + kTreeTcCtas - 1) / kTreeTcCtas) * ((double)(tc_steps + parts - 1) / parts * turn + 7);
    const double runs_us = 30 + 1.15 * 1.43 * (double)heads * tiles * tc_steps / kTreeTcCtas;
    L->runs = (units > kTreeTcCtas && runs_us < waves_us) || heads > 65535;
    // mma.sync
    const int R = (rows + kTreeRows - 1) / kTreeRows, room = R == 1 ? 2 * kTreeTcCtas : kTreeTcCtas;       // CTAs that run at a time
    const int64_t stages = (keys + kTreeStageKeys - 1) / kTreeStageKeys + (drafts + kTreeStageKeys - 1) / kTreeStageKeys;
    int S = 1;
    while (S < kTreeMaxCluster && heads * 2 * S <= room && stages >= 2 * S) S *= 2;

    // Estimates in us, fitted to caches of 100 to 33000 keys of 4 to 256 heads (10 % off), from a stage a CTA.  Measured, mma.sync / tcgen05:
    // 16 rows or less, 4 heads x 3008 keys 10.8 / 13.0, x 9000 22 / 17; 16 heads x 9000 26 / 26; 64 heads x 9000 51 / 68; 17 to 32 rows,
    // 8 heads x 1100 10.2 / 11.5, x 9000 27 / 20, 64 heads x 3008 35 / 33.  The rule is wrong by up to 12 % at 17 to 32 rows of many heads with
    // short caches: 128 heads x 100 11.7 / 10.6, x 300 15.2 / 13.7, 256 heads x 100 22.4 / 20.1, x 300 29.8 / 26.8 go to mma.sync.
    const int64_t waves = (heads * S + room - 1) / room, run = (stages + S - 1) / S;
    const double mma_us = R == 1 ? 5 + (heads * S <= kTreeTcCtas ? 1.0 : 1.2) * waves * run : 7 + 1.13 * waves * run;
    const double tc_us = units <= kTreeTcCtas ? 12 + 1.55 * (double)((tc_steps + parts - 1) / parts) * unit_tiles : L->runs ? runs_us : waves_us;
    L->tc = R > 2 || tc_us < mma_us;
    L->R = R;
    L->S = L->tc ? (int)parts : S;
    L->tiles = tiles;
    L->unit_tiles = unit_tiles;
    L->units = tc_units;
    L->pitch = unit_tiles * kTreeTcRows;
    L->ctas = !L->tc ? heads * S : L->runs ? kTreeTcCtas : units * parts;
    if (!L->tc) L->runs = 0;
    tree_workspace(L, heads);
    // The largest problem's: parts are no more than the CTAs, nor than half the key tiles of a cache of any length up to its capacity.
    const int64_t cap_steps = (cap + kTreeTcRows - 1) / kTreeTcRows + (drafts + kTreeTcRows - 1) / kTreeTcRows;
    const int64_t pitch = (tiles > 1 ? 2 : 1) * kTreeTcRows, slots = heads * tiles * ((cap_steps + 1) / 2);
    const size_t parted = parts_bytes((slots < kTreeTcCtas ? slots : kTreeTcCtas) * pitch), in_runs = runs_bytes(pitch, heads * tiles);
    L->total = heads * tiles > kTreeTcCtas && in_runs > parted ? in_runs : parted;
    return true;
}

template <int R>
static lvlm_status launch_tree_mma(const TreeArgs& a, const TreeMaps& m, const TreeLayout& L, cudaStream_t stream) {
    LVLM_RETURN_IF_CUDA(cudaFuncSetAttribute(tree_mma_kernel<R>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxDynSmem));
    return launch_kernel(tree_mma_kernel<R>, dim3((unsigned)L.ctas), dim3(TreeMma<R>::kThreads), TreeMma<R>::kSmem, stream, L.S, m.k, m.v, m.kd, m.vd, a);
}

size_t tree_attn_workspace(const lvlm_dims* d) {
    TreeLayout L;
    const int64_t cap = d->page > 0 ? (int64_t)d->page * d->max_pages : d->cap;
    return tree_layout(d, cap, &L) ? L.total : 0;
}

#ifdef LVLM_TEST_HOOKS
static int g_tree_starve = 0, g_tree_stall = 0;
#endif

}  // namespace lvlm

#ifdef LVLM_TEST_HOOKS
extern "C" void lvlm_debug_starve_tree(int on) { lvlm::g_tree_starve = on ? 1 : 0; }
extern "C" int lvlm_debug_tree_record(int first, int more) { return lvlm::tree_record(first, more); }
extern "C" void lvlm_debug_stall_tree(int us) { lvlm::g_tree_stall = us; }
#endif

extern "C" lvlm_status lvlm_tree_attn(const void* q, const void* Kc, const void* Vc, const int32_t* table, const int32_t* len,
                                       const void* Kd, const void* Vd, const uint32_t* mask, const int32_t* count,
                                       const lvlm_dims* d, float scale, void* out, float* lse,
                                       void* ws, size_t ws_bytes, int32_t* dev_status, void* stream_) {
    using namespace lvlm;
    cudaStream_t stream = (cudaStream_t)stream_;
    if (!q || !Kc || !Vc || !len || !out || !d || d->B <= 0 || d->H <= 0 || d->Hkv <= 0 || d->H % d->Hkv || d->T <= 0 || !(scale > 0.f))
        return LVLM_ERR_INVALID_ARG;
    if ((Kd == nullptr) != (Vd == nullptr) || (mask && !Kd) || (Kd && d->draft_cap < d->T)) return LVLM_ERR_INVALID_ARG;
    if (d->D != kHeadDim || d->T > kTreeMaxT || d->H / d->Hkv > kTreeMaxGroup) return LVLM_ERR_UNSUPPORTED;
    TreeArgs a;
    const lvlm_status gs = cache_geom(d, table, &a.c);
    if (gs != LVLM_OK) return gs;
    a.q_sh = d->q_stride_h ? d->q_stride_h : d->D;
    a.q_sn = d->q_stride_n ? d->q_stride_n : (int64_t)d->H * d->D;
    a.q_sb = d->q_stride_b ? d->q_stride_b : (int64_t)d->T * a.q_sn;
    const int64_t d_sh = d->draft_stride_h ? d->draft_stride_h : (int64_t)d->draft_cap * d->D;
    const int64_t d_sb = d->draft_stride_b ? d->draft_stride_b : (int64_t)d->Hkv * d_sh;
    if (!aligned16(q) || !aligned16(Kc) || !aligned16(Vc) || !aligned16(Kd) || !aligned16(Vd) || !aligned16(out) || a.q_sh % 8 ||
        a.q_sn % 8 || a.q_sb % 8 || d_sh % 8 || d_sb % 8)
        return LVLM_ERR_ALIGNMENT;
    // Queries may be overwritten where a row's result takes its own query's place; anywhere else CTAs may still have to read them.
    const int64_t packed_n = (int64_t)d->H * d->D, packed_b = d->T * packed_n;
    if (out == q ? (d->H > 1 && a.q_sh != d->D) || (d->T > 1 && a.q_sn != packed_n) || (d->B > 1 && a.q_sb != packed_b)
                 : overlap(q, 2 * ((d->B - 1) * a.q_sb + (d->T - 1) * a.q_sn + (d->H - 1) * a.q_sh + kHeadDim), out, 2 * (int64_t)d->B * packed_b))
        return LVLM_ERR_INVALID_ARG;
    TreeLayout L;
    if (!tree_layout(d, a.c.cap, &L)) return LVLM_ERR_INVALID_ARG;
    if (((int64_t)a.c.cap / kTreeTcRows + 3) * L.tiles > 0x3FFFFFFF) return LVLM_ERR_UNSUPPORTED;     // (tree_weight)
    // In runs a part lies in `out` while other CTAs may still fetch the queries of its unit: where out is q, units go in waves.
    if (L.runs && out == q) {
        if ((int64_t)d->B * d->Hkv > 65535) return LVLM_ERR_INVALID_ARG;
        L.runs = 0;
        L.S = 1;
        L.ctas = (int64_t)d->B * d->Hkv * L.units;
        tree_workspace(&L, (int64_t)d->B * d->Hkv);
    }
    if (L.need && (!ws || !aligned256(ws) || ws_bytes < L.need)) return LVLM_ERR_WORKSPACE;
    char* wsb = static_cast<char*>(ws);
    TreeMaps m;
    {
        const bool paged = a.c.page > 0;
        const int box_rows = L.tc ? kTreeTcRows : kTreeStageKeys;
        const uint64_t dims[4] = {(uint64_t)kHeadDim, (uint64_t)(paged ? a.c.page : a.c.cap), (uint64_t)(paged ? a.c.n_pages : d->Hkv), (uint64_t)(paged ? 1 : d->B)};
        const uint64_t strides[3] = {(uint64_t)kHeadDim * 2, (uint64_t)a.c.sh * 2, (uint64_t)(paged ? a.c.sh : a.c.sb) * 2};
        const uint32_t box[4] = {64, (uint32_t)(paged && a.c.page < box_rows ? a.c.page : box_rows), 1, 1};
        if (!make_tmap_bf16(&m.k, Kc, 4, dims, strides, box) || !make_tmap_bf16(&m.v, Vc, 4, dims, strides, box)) return LVLM_ERR_CUDA;
        m.kd = m.k; m.vd = m.v;                                 // without drafts: not read
        if (Kd) {
            const uint64_t ddims[4] = {(uint64_t)kHeadDim, (uint64_t)d->T, (uint64_t)d->Hkv, (uint64_t)d->B};
            const uint64_t dstr[3] = {(uint64_t)kHeadDim * 2, (uint64_t)d_sh * 2, (uint64_t)d_sb * 2};
            const uint32_t dbox[4] = {64, (uint32_t)box_rows, 1, 1};
            if (!make_tmap_bf16(&m.kd, Kd, 4, ddims, dstr, dbox) || !make_tmap_bf16(&m.vd, Vd, 4, ddims, dstr, dbox)) return LVLM_ERR_CUDA;
        }
    }
    a.q = static_cast<const __nv_bfloat16*>(q);
    a.table = table; a.len = len; a.mask = mask; a.count = count;
    a.out = static_cast<__nv_bfloat16*>(out); a.lse = lse;
    a.B = d->B; a.H = d->H; a.G = d->H / d->Hkv; a.T = d->T; a.W = (d->T + 31) / 32; a.drafts = Kd != nullptr; a.mask_shared = d->mask_shared != 0;
    a.S = L.S; a.runs = L.runs; a.tile_rows = kTreeTcRows / a.G * a.G; a.unit_tiles = L.unit_tiles; a.units = L.units; a.pitch = L.pitch;
    a.scale_log2 = scale * kTreeLog2e;
    a.part_ml = reinterpret_cast<float2*>(wsb);
    a.part_o = reinterpret_cast<float*>(wsb + L.off_o);
    a.part_lo = reinterpret_cast<uint2*>(wsb + L.off_lo);
    a.part_of = reinterpret_cast<int2*>(wsb + L.off_of);
    a.dev_status = dev_status;
#ifdef LVLM_TEST_HOOKS
    a.starve = g_tree_starve;
    a.stall = g_tree_stall;
#endif
    if (L.ctas > 0x7FFFFFFFll) return LVLM_ERR_UNSUPPORTED;
    lvlm_status st;
    if (L.tc) {
        const uint64_t dims[5] = {(uint64_t)kHeadDim, (uint64_t)a.G, (uint64_t)d->T, (uint64_t)d->Hkv, (uint64_t)d->B};
        const uint64_t strides[4] = {(uint64_t)a.q_sh * 2, (uint64_t)a.q_sn * 2, (uint64_t)a.G * a.q_sh * 2, (uint64_t)a.q_sb * 2};
        const uint32_t box[5] = {64, (uint32_t)a.G, (uint32_t)(kTreeTcRows / a.G), 1, 1};
        if (!make_tmap_bf16(&m.q, q, 5, dims, strides, box)) return LVLM_ERR_CUDA;
        st = launch_tree_tc(a, m, stream);
    } else {
        return L.R == 1 ? launch_tree_mma<1>(a, m, L, stream) : launch_tree_mma<2>(a, m, L, stream);
    }
    if (st != LVLM_OK || (L.S == 1 && !L.runs)) return st;
    // the fewer units, the finer.  us of the whole call with <1, 4> / <1, 1> / <4, 1>: 4 units of 37 parts 26.7 / 31.4 / 50, 8 of 12 18.8 /
    // 16.1 / 16.9, 16 of 9 - / 23.5 / 22.4, 32 of 2 29.5 / 16.9 / 14.1
    const int64_t units = (int64_t)d->B * d->Hkv * L.units;
    const unsigned blocks = (unsigned)(L.pitch / 32);
    const dim3 threads(kTreeCombineWarps * 32);
    if (L.runs) return launch_kernel(tree_combine_kernel<4, 1, true>, dim3((unsigned)units, blocks, 1), threads, 0, stream, 1, a);
    if (units * blocks * 16 <= 2 * kTreeTcCtas) return launch_kernel(tree_combine_kernel<1, 4, false>, dim3((unsigned)units, blocks, 16), threads, 0, stream, 1, a);
    if (units * blocks * 4 <= kTreeTcCtas) return launch_kernel(tree_combine_kernel<1, 1, false>, dim3((unsigned)units, blocks, 4), threads, 0, stream, 1, a);
    return launch_kernel(tree_combine_kernel<4, 1, false>, dim3((unsigned)units, blocks, 1), threads, 0, stream, 1, a);
}
