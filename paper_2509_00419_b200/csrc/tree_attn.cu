// lvlm_tree_attn: the drafted tokens of a sequence attend to its cache (contiguous or paged, ragged per KV head) and to one
// another through a mask.
//
// For every (sequence, KV head) the T G query rows of the group (row r = token r / G, head r % G of the group) meet the
// same keys: len cache rows, then the count drafts.  An online softmax runs over the keys; the keys of a head are cut into S runs
// whose partial (max, sum, output) a second small launch adds in order.
//
// This kernel: tiles of 16 query rows on mma.sync.  A CTA is a producer warp and four compute warps around a ring of
// stages of 64 keys, fetched by TMA tile copies (a box per page and 64 channels); a compute warp takes 16 keys of a stage.
#include "exp2.cuh"
#include "sm100.cuh"
#include "tree_attn.cuh"

namespace lvlm {

using namespace sm100;

constexpr int kTreeWarps = 4;
constexpr int kTreeThreads = (kTreeWarps + 1) * 32;
constexpr int kTreeRows = 16;                        // query rows a CTA
constexpr int kTreeStageKeys = 64;
constexpr int kTreeBox = kTreeStageKeys * 128;       // 64 keys x 64 channels
constexpr int kTreeStageBytes = 4 * kTreeBox;        // K low, K high, V low, V high channels
constexpr int kTreeStages = 3;
constexpr int kTreeTargetCtas = 2 * 148;             // CTAs wanted in flight: two an SM,
constexpr int kTreeTcCtas = 148;                     // and one of the tcgen05 kernel
constexpr int64_t kTreeMostSlots = 2 * kTreeTcCtas * kTreeTcRows;       // rows of partial results: two row tiles a CTA at most
static_assert(kTreeMostSlots >= kTreeTargetCtas * kTreeRows, "");

// Which kernel.
static bool tree_uses_tc(int64_t rows, int64_t) { return rows > kTreeRows; }

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

// grid.x = heads * row_tiles * S
__global__ void __launch_bounds__(kTreeThreads, 2)
tree_mma_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
                const __grid_constant__ CUtensorMap kdmap, const __grid_constant__ CUtensorMap vdmap, const TreeArgs a) {
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    __shared__ uint64_t s_full[kTreeStages], s_empty[kTreeStages];
    __shared__ float2 s_ml[kTreeWarps][kTreeRows];
    __shared__ int s_abort;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int s = 0; s < kTreeStages; ++s) { mbar_init(&s_full[s], 1); mbar_init(&s_empty[s], kTreeWarps); }
        s_abort = 0;
        fence_barrier_init();
    }
    __syncthreads();
    pdl_enter();
    const int S = a.S, T = a.T, G = a.G, Hkv = a.c.Hkv;
    const int part = blockIdx.x % S, tile = blockIdx.x / S % a.row_tiles, hd = blockIdx.x / S / a.row_tiles;
    const int b = hd / Hkv, g = hd % Hkv, r0 = tile * kTreeRows;
    const int n = tree_count(a, b), rows = n * G;               // rows behind `rows` are not asked for
    if (r0 >= rows) return;
    const int ln = tree_len(a, hd);
    // stages of the cache, then of the drafts; a head whose length is bad has none and gives zeros
    const int ns = ln > 0 ? (ln + kTreeStageKeys - 1) / kTreeStageKeys : 0;
    const int nt = ln < 0 ? 0 : ns + (a.drafts ? (n + kTreeStageKeys - 1) / kTreeStageKeys : 0);
    const int per = (nt + S - 1) / S, t_lo = min(nt, part * per), nstage = min(nt, t_lo + per) - t_lo;

    const int row = lane >> 2, qd = lane & 3;                   // my rows row and row + 8 of the tile
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
    if (warp == kTreeWarps) {
        // ---- producer: lane i copies the i-th box of K and V halves of a stage ----------------------------------
        const int box_rows = a.c.page ? min(a.c.page, kTreeStageKeys) : kTreeStageKeys;
        for (int i = 0; i < nstage; ++i) {
            const int s = i % kTreeStages, st = t_lo + i;
            if (i >= kTreeStages && !__all_sync(0xFFFFFFFFu, wait_on(&s_empty[s], (uint32_t)(i / kTreeStages - 1) & 1u))) break;
            if (lane == 0) mbar_arrive_expect_tx(&s_full[s], kTreeStageBytes);
            __syncwarp();
            unsigned char* to = smem + s * kTreeStageBytes;
            if (st >= ns) {
                if (lane < 4) tma_load_4d(to + lane * kTreeBox, lane < 2 ? &kdmap : &vdmap, &s_full[s], (lane & 1) * 64, (st - ns) * kTreeStageKeys, g, b);
            } else {
                const int boxes = kTreeStageKeys / box_rows;    // 1, 2 or 4
                if (lane < 4 * boxes) {
                    const int part4 = lane & 3, bx = lane >> 2, j = st * kTreeStageKeys + bx * box_rows;
                    int c1 = j, c2 = g, c3 = b;
                    if (a.c.page) {
                        // entries behind the head's length are not read: the last page of the head again
                        const int pg = min(j, ln - 1) >> a.c.shift;
                        int id = *(a.table + (int64_t)hd * a.c.max_pages + pg);
                        if (id < 0 || id >= a.c.n_pages) { tree_flag(a, LVLM_DEV_BOUNDS); id = a.c.n_pages; }   // the copy fills zeros there
                        c1 = j & (a.c.page - 1); c2 = id; c3 = 0;
                    }
                    tma_load_4d(to + part4 * kTreeBox + bx * box_rows * 128, part4 < 2 ? &kmap : &vmap, &s_full[s], (part4 & 1) * 64, c1, c2, c3);
                }
            }
        }
    } else {
        uint32_t qa[8][4];
        const uint32_t* qp[2];
        uint32_t see[2][kTreeMaxT / 32];                        // draft mask of my two rows
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int r = r0 + row + 8 * u, t = r / G, hh = r % G;
            qp[u] = r < rows ? reinterpret_cast<const uint32_t*>(a.q + (int64_t)b * a.q_sb + (int64_t)t * a.q_sn + (int64_t)(g * G + hh) * a.q_sh) : nullptr;
#pragma unroll
            for (int w = 0; w < kTreeMaxT / 32; ++w) see[u][w] = r < rows ? tree_see(a, b, t, n, w) : 0u;
        }
#pragma unroll
        for (int ks = 0; ks < 8; ++ks)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                qa[ks][u] = qp[u] ? *(qp[u] + ks * 8 + qd) : 0u;
                qa[ks][2 + u] = qp[u] ? *(qp[u] + ks * 8 + 4 + qd) : 0u;
            }
        for (int i = 0; i < nstage; ++i) {
            const int s = i % kTreeStages, st = t_lo + i;
            const bool draft = st >= ns;
            const int k0 = (draft ? st - ns : st) * kTreeStageKeys + warp * 16, kend = draft ? n : ln;   // my keys, of how many
            const bool ok = __all_sync(0xFFFFFFFFu, wait_on(&s_full[s], (uint32_t)(i / kTreeStages) & 1u));
            if (ok && k0 < kend) {
                const uint32_t at = smem_u32(smem) + s * kTreeStageBytes;
                const int rr = warp * 16;
                if (k0 + 16 > kend) {                           // rows behind the end hold anything: their weight is zero, so must be V
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
                        if (draft) {
                            uint32_t word = 0;
#pragma unroll
                            for (int w = 0; w < kTreeMaxT / 32; ++w) word = w == (j >> 5) ? see[u][w] : word;
                            vis = vis && ((word >> (j & 31)) & 1u);
                        }
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
    float* so = reinterpret_cast<float*>(smem);                 // [4][16][132]
    constexpr int kPitch = kHeadDim + 4;
    if (warp < kTreeWarps) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            l_run[u] += __shfl_xor_sync(0xFFFFFFFFu, l_run[u], 1);
            l_run[u] += __shfl_xor_sync(0xFFFFFFFFu, l_run[u], 2);
            if (qd == 0) s_ml[warp][row + 8 * u] = make_float2(m_run[u], l_run[u]);
#pragma unroll
            for (int c = 0; c < 16; ++c)
                *reinterpret_cast<float2*>(so + (warp * kTreeRows + row + 8 * u) * kPitch + c * 8 + qd * 2) = make_float2(o[c][2 * u], o[c][2 * u + 1]);
        }
    }
    __syncthreads();
    for (int idx = tid; idx < kTreeRows * (kHeadDim / 4); idx += kTreeThreads) {
        const int rr = idx / (kHeadDim / 4), c4 = idx % (kHeadDim / 4), r = r0 + rr;
        if (r >= rows) continue;
        float M = -INFINITY, Ls = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kTreeWarps; ++w) M = fmaxf(M, s_ml[w][rr].x);
#pragma unroll
        for (int w = 0; w < kTreeWarps; ++w) {
            const float2 ml = s_ml[w][rr];
            const float f = ml.x > -INFINITY ? ex2_fast(ml.x - M) : 0.f;
            const float4 x = *reinterpret_cast<const float4*>(so + (w * kTreeRows + rr) * kPitch + c4 * 4);
            v.x += x.x * f; v.y += x.y * f; v.z += x.z * f; v.w += x.w * f;
            Ls += ml.y * f;
        }
        if (S > 1) {
            const int64_t at = (int64_t)blockIdx.x * kTreeRows + rr;
            reinterpret_cast<float4*>(a.part_o + at * kHeadDim)[c4] = v;
            if (c4 == 0) a.part_ml[at] = make_float2(M, Ls);
        } else {
            const int t = r / G, h = g * G + r % G;
            const float inv = Ls > 0.f ? 1.0f / Ls : 0.f;
            *reinterpret_cast<uint2*>(a.out + (((int64_t)b * T + t) * a.H + h) * kHeadDim + c4 * 4) =
                make_uint2(pack_bf16(v.x * inv, v.y * inv), pack_bf16(v.z * inv, v.w * inv));
            if (a.lse && c4 == 0) a.lse[((int64_t)b * a.H + h) * T + t] = Ls > 0.f ? (M + log2f(Ls)) * kTreeLn2 : -INFINITY;
        }
    }
}

// Adds the S parts of a row in order.  A warp a row: a lane has four channels.
constexpr int kTreeCombineThreads = 128;
__global__ void __launch_bounds__(kTreeCombineThreads) tree_combine_kernel(const TreeArgs a) {
    pdl_enter();
    const int lane = threadIdx.x & 31, hd = blockIdx.y, b = hd / a.c.Hkv, g = hd % a.c.Hkv;
    const int r = blockIdx.x * (kTreeCombineThreads / 32) + (threadIdx.x >> 5);
    if (r >= tree_count(a, b) * a.G) return;
    const int64_t rows = a.pitch, at = ((int64_t)hd * a.row_tiles + r / a.tile_rows) * a.S * a.pitch + r % a.tile_rows;
    float M = -INFINITY, Ls = 0.f;
    for (int p = lane; p < a.S; p += 32) M = fmaxf(M, a.part_ml[at + p * rows].x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xFFFFFFFFu, M, o));
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int p = 0; p < a.S; ++p) {
        const float2 ml = a.part_ml[at + p * rows];
        if (ml.x == -INFINITY) continue;
        const float f = ex2_fast(ml.x - M);
        const float4 x = reinterpret_cast<const float4*>(a.part_o + (at + p * rows) * kHeadDim)[lane];
        v.x += x.x * f; v.y += x.y * f; v.z += x.z * f; v.w += x.w * f;
        Ls += ml.y * f;
    }
    const int t = r / a.G, h = g * a.G + r % a.G;
    const float inv = Ls > 0.f ? 1.0f / Ls : 0.f;
    *reinterpret_cast<uint2*>(a.out + (((int64_t)b * a.T + t) * a.H + h) * kHeadDim + lane * 4) =
        make_uint2(pack_bf16(v.x * inv, v.y * inv), pack_bf16(v.z * inv, v.w * inv));
    if (a.lse && lane == 0) a.lse[((int64_t)b * a.H + h) * a.T + t] = Ls > 0.f ? (M + log2f(Ls)) * kTreeLn2 : -INFINITY;
}

// tc: the tcgen05 kernel.  `used`: bytes of workspace this call touches; `total` is what a caller is told: room for as many parts as any
// problem of no more heads, rows and keys is cut into.
struct TreeLayout { int tc, S, row_tiles, tile_rows, pitch; size_t off_o, used, total; };

static bool tree_layout(const lvlm_dims* d, int64_t cap, TreeLayout* L) {
    if (d->B <= 0 || d->H <= 0 || d->Hkv <= 0 || d->H % d->Hkv || d->T <= 0 || d->T > kTreeMaxT || d->H / d->Hkv > kTreeMaxGroup || cap <= 0) return false;
    const int G = d->H / d->Hkv;
    const int64_t heads = (int64_t)d->B * d->Hkv, rows = (int64_t)d->T * G;
    const int64_t keys = (d->N > 0 && d->N < cap ? d->N : cap) + (d->draft_cap > 0 ? d->T : 0);
    L->tc = tree_uses_tc(rows, keys);
    L->pitch = L->tc ? kTreeTcRows : kTreeRows;
    L->tile_rows = L->tc ? kTreeTcRows / G * G : kTreeRows;
    L->row_tiles = (int)((rows + L->tile_rows - 1) / L->tile_rows);
    const int64_t units = heads * (L->tc ? (L->row_tiles + 1) / 2 : L->row_tiles);       // CTAs where nothing is cut
    const int64_t steps = (keys + (L->tc ? kTreeTcRows : kTreeStageKeys) - 1) / (L->tc ? kTreeTcRows : kTreeStageKeys);
    int64_t S = (L->tc ? kTreeTcCtas : kTreeTargetCtas) / units;
    S = S < 1 ? 1 : S > steps ? steps : S;
    L->S = (int)S;
    const int64_t slots = S > 1 ? heads * L->row_tiles * S * L->pitch : 0;
    L->off_o = align_up((size_t)slots * 8, 256);
    L->used = L->off_o + (size_t)slots * kHeadDim * 4;
    const int64_t tc_tile = kTreeTcRows / G * G, stages = (keys + kTreeStageKeys - 1) / kTreeStageKeys;
    const int64_t tc_rows = (rows + tc_tile - 1) / tc_tile * kTreeTcRows, mma_rows = (rows + kTreeRows - 1) / kTreeRows * kTreeRows;
    const int64_t most = heads * (tc_rows > mma_rows ? tc_rows : mma_rows) * stages;
    L->total = align_up((size_t)(most < kTreeMostSlots ? most : kTreeMostSlots) * (8 + kHeadDim * 4) + 256, 256);
    return true;
}

size_t tree_attn_workspace(const lvlm_dims* d) {
    TreeLayout L;
    const int64_t cap = d->page > 0 ? (int64_t)d->page * d->max_pages : d->cap;
    return tree_layout(d, cap, &L) ? L.total : 0;
}

}  // namespace lvlm

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
    TreeLayout L;
    if (!tree_layout(d, a.c.cap, &L)) return LVLM_ERR_INVALID_ARG;
    if (L.S > 1 && (!ws || !aligned256(ws) || ws_bytes < L.total)) return LVLM_ERR_WORKSPACE;
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
    a.S = L.S; a.row_tiles = L.row_tiles; a.tile_rows = L.tile_rows; a.pitch = L.pitch;
    a.scale_log2 = scale * kTreeLog2e;
    a.part_ml = reinterpret_cast<float2*>(wsb);
    a.part_o = reinterpret_cast<float*>(wsb + L.off_o);
    a.dev_status = dev_status;
    const int64_t heads = (int64_t)d->B * d->Hkv, ctas = heads * L.row_tiles * L.S;
    if (ctas > 0x7FFFFFFFll) return LVLM_ERR_UNSUPPORTED;
    lvlm_status st;
    if (L.tc) {
        const uint64_t dims[5] = {(uint64_t)kHeadDim, (uint64_t)a.G, (uint64_t)d->T, (uint64_t)d->Hkv, (uint64_t)d->B};
        const uint64_t strides[4] = {(uint64_t)a.q_sh * 2, (uint64_t)a.q_sn * 2, (uint64_t)a.G * a.q_sh * 2, (uint64_t)a.q_sb * 2};
        const uint32_t box[5] = {64, (uint32_t)a.G, (uint32_t)(kTreeTcRows / a.G), 1, 1};
        if (!make_tmap_bf16(&m.q, q, 5, dims, strides, box)) return LVLM_ERR_CUDA;
        st = launch_tree_tc(a, m, stream);
    } else {
        const size_t smem = 1024 + (size_t)kTreeStages * kTreeStageBytes;
        LVLM_RETURN_IF_CUDA(cudaFuncSetAttribute(tree_mma_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxDynSmem));
        st = launch_kernel(tree_mma_kernel, dim3((unsigned)ctas), dim3(kTreeThreads), smem, stream, 1, m.k, m.v, m.kd, m.vd, a);
    }
    if (st != LVLM_OK || L.S == 1) return st;
    const int rows = d->T * a.G, per = kTreeCombineThreads / 32;
    return launch_kernel(tree_combine_kernel, dim3((unsigned)((rows + per - 1) / per), (unsigned)heads), dim3(kTreeCombineThreads), 0, stream, 1, a);
}
