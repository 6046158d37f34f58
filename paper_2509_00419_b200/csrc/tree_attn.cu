// lvlm_tree_attn: the drafted tokens of a sequence attend to its cache (contiguous or paged, ragged per KV head) and to one
// another through a mask.
//
// For every (sequence, KV head) the T G query rows of the group (row r = draft r / G, head r % G of the group) meet the
// same keys: len cache rows, then the count drafts.  An online softmax runs over the keys.
//
// Few rows (tree_mma_kernel, here): a tile of 16 query rows on mma.sync.  The keys of a head are cut into runs for the CTAs of a
// cluster.  A CTA is a producer warp and four compute warps around a ring of stages of 64 keys, fetched by TMA tile copies (a box per
// page and 64 channels); a compute warp takes 16 keys of a stage.  The warps are added in shared memory, the CTAs of the cluster
// through distributed shared memory: one launch, no workspace.
// Many rows or keys: tree_tc.cu, on tcgen05; parts of a unit that it cut are added by tree_combine_kernel, here.
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
constexpr int kTreeTargetCtas = 2 * 148;             // CTAs wanted in flight, two an SM
constexpr int kTreeMaxCluster = 8;
constexpr int kTreeMmaWords = 2;                     // mask words of a row: T <= 64

// Which kernel.
static bool tree_uses_tc(int T, int64_t rows, int64_t) { return rows > kTreeRows || T > 32 * kTreeMmaWords; }

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

// grid.x = heads * row_tiles * S, clusters of S CTAs
__global__ void __launch_bounds__(kTreeThreads, 2)
tree_mma_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
                const __grid_constant__ CUtensorMap kdmap, const __grid_constant__ CUtensorMap vdmap, const TreeArgs a) {
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    __shared__ uint64_t s_full[kTreeStages], s_empty[kTreeStages];
    __shared__ float2 s_ml[kTreeWarps][kTreeRows], s_ML[kTreeRows];
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
    const int part = (int)cluster_ctarank(), tile = blockIdx.x / S % a.row_tiles, hd = blockIdx.x / S / a.row_tiles;
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
        const int box_rows = a.c.page ? min(a.c.page, kTreeStageKeys) : kTreeStageKeys, boxes = kTreeStageKeys / box_rows;    // 1, 2 or 4
        const int quarter = lane & 3, bx = lane >> 2;
        // the page of my box of stage st; entries behind the head's length are not read: its last page again
        auto page_of = [&](int st) -> int {
            if (!a.c.page || st >= ns || bx >= boxes) return 0;
            return a.table[(int64_t)hd * a.c.max_pages + (min(st * kTreeStageKeys + bx * box_rows, ln - 1) >> a.c.shift)];
        };
        int id = page_of(t_lo);
        for (int i = 0; i < nstage; ++i) {
            const int s = i % kTreeStages, st = t_lo + i;
            const int id_next = i + 1 < nstage ? page_of(st + 1) : 0;      // asked for a stage ahead
            if (i >= kTreeStages && !__all_sync(0xFFFFFFFFu, wait_on(&s_empty[s], (uint32_t)(i / kTreeStages - 1) & 1u))) break;
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
        uint32_t see[2][kTreeMmaWords];                         // draft mask of my two rows
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int r = r0 + row + 8 * u, t = r / G, hh = r % G;
            qp[u] = r < rows ? reinterpret_cast<const uint32_t*>(a.q + (int64_t)b * a.q_sb + (int64_t)t * a.q_sn + (int64_t)(g * G + hh) * a.q_sh) : nullptr;
#pragma unroll
            for (int w = 0; w < kTreeMmaWords; ++w) see[u][w] = r < rows ? tree_see(a, b, t, n, w) : 0u;
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
                            for (int w = 0; w < kTreeMmaWords; ++w) word = w == (j >> 5) ? see[u][w] : word;
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
        const int rr = idx / (kHeadDim / 4), c4 = idx % (kHeadDim / 4);
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
        *reinterpret_cast<float4*>(so + rr * kPitch + c4 * 4) = v;      // (over the first warp's, which only this thread reads)
        if (c4 == 0) s_ML[rr] = make_float2(M, Ls);
    }
    // ---- the CTAs of the cluster, in rank order; a CTA finishes a slice of the rows and channels ---------------------------
    cluster_barrier();
    for (int idx = part * kTreeThreads + tid; idx < kTreeRows * (kHeadDim / 4); idx += S * kTreeThreads) {
        const int rr = idx / (kHeadDim / 4), c4 = idx % (kHeadDim / 4), r = r0 + rr;
        if (r >= rows) continue;
        float2 ml[kTreeMaxCluster];
        float4 x[kTreeMaxCluster];
#pragma unroll
        for (int c = 0; c < kTreeMaxCluster; ++c) {
            ml[c] = make_float2(-INFINITY, 0.f);
            x[c] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (c < S) {
                ml[c] = cluster_ld(&s_ML[rr], c);
                x[c] = cluster_ld(reinterpret_cast<const float4*>(so + rr * kPitch + c4 * 4), c);
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
        const int t = r / G, h = g * G + r % G;
        const float inv = Ls > 0.f ? 1.0f / Ls : 0.f;
        *reinterpret_cast<uint2*>(a.out + (((int64_t)b * T + t) * a.H + h) * kHeadDim + c4 * 4) =
            make_uint2(pack_bf16(v.x * inv, v.y * inv), pack_bf16(v.z * inv, v.w * inv));
        if (a.lse && c4 == 0) a.lse[((int64_t)b * a.H + h) * T + t] = Ls > 0.f ? (M + log2f(Ls)) * kTreeLn2 : -INFINITY;
    }
    cluster_arrive_exec();                                      // my reads of the other CTAs' shared memory are done
    cluster_wait();                                             // and nobody leaves while its own is still read
}

// Adds the parts of a unit (a pair of row tiles of a head) that the tcgen05 kernel cut, in order.  Lane = row, a warp CH groups of four
// channels of 32 rows: the loads are the lines that the parts were stored in.  grid (units, row blocks, channel blocks).
constexpr int kTreeCombineWarps = 8;
template <int CH>
__global__ void __launch_bounds__(kTreeCombineWarps * 32) tree_combine_kernel(const TreeArgs a) {
    pdl_enter();
    const int pairs = (a.row_tiles + 1) / 2, lane = threadIdx.x & 31;
    const int2 of = a.part_of[blockIdx.x];
    const int hd = blockIdx.x / pairs, pair = blockIdx.x % pairs, b = hd / a.c.Hkv, g = hd % a.c.Hkv, tt = a.tile_rows / a.G;
    const int place = blockIdx.y * 32 + lane, row = place % kTreeTcRows, tile = 2 * pair + place / kTreeTcRows;
    const int n = tree_count(a, b);
    if (2 * pair * tt >= n || of.x < 0) return;                 // nothing asked for, or not cut (of is only written where something is)
    const int t = tile * tt + row / a.G;
    const bool mine = row < a.tile_rows && t < n;
    const int c0 = (blockIdx.z * kTreeCombineWarps + (threadIdx.x >> 5)) * CH, parts = of.y + 1;
    // part p >= 1 lies in the first slot of its CTA
    const int64_t rest = (int64_t)(of.x & ~1);
    auto slot = [&](int p) -> int64_t { return p == 0 ? of.x : rest + 2 * p; };
    float M = -INFINITY;
#pragma unroll 4
    for (int p = 0; p < parts; ++p) M = fmaxf(M, a.part_ml[slot(p) * a.pitch + place].x);
    float4 v[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) v[c] = make_float4(0.f, 0.f, 0.f, 0.f);
    float Ls = 0.f;
    constexpr int kAhead = 8 / CH;
    for (int p0 = 0; p0 < parts; p0 += kAhead) {
        float4 x[kAhead][CH];
        float2 ml[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            ml[u] = make_float2(-INFINITY, 0.f);
            if (p0 + u < parts) {
                const int64_t s = slot(p0 + u);
                ml[u] = a.part_ml[s * a.pitch + place];
#pragma unroll
                for (int c = 0; c < CH; ++c) x[u][c] = reinterpret_cast<const float4*>(a.part_o + s * a.pitch * kHeadDim)[(int64_t)(c0 + c) * a.pitch + place];
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (ml[u].x == -INFINITY) continue;
            const float w = ex2_fast(ml[u].x - M);
            Ls += ml[u].y * w;
#pragma unroll
            for (int c = 0; c < CH; ++c) { v[c].x += x[u][c].x * w; v[c].y += x[u][c].y * w; v[c].z += x[u][c].z * w; v[c].w += x[u][c].w * w; }
        }
    }
    if (!mine) return;
    const int h = g * a.G + row % a.G;
    const float inv = Ls > 0.f ? 1.0f / Ls : 0.f;
    uint2* to = reinterpret_cast<uint2*>(a.out + (((int64_t)b * a.T + t) * a.H + h) * kHeadDim) + c0;
#pragma unroll
    for (int c = 0; c < CH; ++c) to[c] = make_uint2(pack_bf16(v[c].x * inv, v[c].y * inv), pack_bf16(v[c].z * inv, v[c].w * inv));
    if (a.lse && c0 == 0) a.lse[((int64_t)b * a.H + h) * a.T + t] = Ls > 0.f ? (M + log2f(Ls)) * kTreeLn2 : -INFINITY;
}

// tc: the tcgen05 kernel.  `total` is what a caller is told, whichever kernel it is, so that it never shrinks as a problem grows.
struct TreeLayout { int tc, S, row_tiles, tile_rows, pitch; size_t off_o, off_of, total; };

static bool tree_layout(const lvlm_dims* d, int64_t cap, TreeLayout* L) {
    if (d->B <= 0 || d->H <= 0 || d->Hkv <= 0 || d->H % d->Hkv || d->T <= 0 || d->T > kTreeMaxT || d->H / d->Hkv > kTreeMaxGroup || cap <= 0) return false;
    const int G = d->H / d->Hkv;
    const int64_t heads = (int64_t)d->B * d->Hkv, rows = (int64_t)d->T * G;
    const int64_t keys = (d->N > 0 && d->N < cap ? d->N : cap) + (d->draft_cap > 0 ? d->T : 0);
    const int64_t mma_tiles = heads * ((rows + kTreeRows - 1) / kTreeRows);
    L->tc = tree_uses_tc(d->T, rows, keys);
    // the tcgen05 kernel: CTAs by the work there is at most, two slots each
    const int64_t tc_tile = kTreeTcRows / G * G, tc_tiles = (rows + tc_tile - 1) / tc_tile;
    const int64_t work = heads * tc_tiles * ((keys + kTreeTcRows - 1) / kTreeTcRows + 1) / kTreeTcLeast;
    const int64_t tc_S = work < 1 ? 1 : work > kTreeTcCtas ? kTreeTcCtas : work;
    L->pitch = (tc_tiles > 1 ? 2 : 1) * kTreeTcRows;
    const int64_t places = tc_S > 1 ? 2 * tc_S * L->pitch : 0;
    L->off_o = align_up((size_t)places * 8, 256);
    L->off_of = L->off_o + (size_t)places * kHeadDim * 4;
    L->total = align_up(L->off_of + (size_t)(heads * ((tc_tiles + 1) / 2)) * 8, 256);
    // the other: clusters as large as the GPU has room for, a CTA with a stage of keys at least
    int S = 1;
    while (S < kTreeMaxCluster && mma_tiles * 2 * S <= kTreeTargetCtas && keys >= 2 * S * kTreeStageKeys) S *= 2;
    L->S = L->tc ? (int)tc_S : S;
    L->tile_rows = L->tc ? (int)tc_tile : kTreeRows;
    L->row_tiles = (int)((rows + L->tile_rows - 1) / L->tile_rows);
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
    if (!ws || !aligned256(ws) || ws_bytes < L.total) return LVLM_ERR_WORKSPACE;
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
    a.part_of = reinterpret_cast<int2*>(wsb + L.off_of);
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
        return launch_kernel(tree_mma_kernel, dim3((unsigned)ctas), dim3(kTreeThreads), smem, stream, L.S, m.k, m.v, m.kd, m.vd, a);
    }
    if (st != LVLM_OK || L.S == 1) return st;
    // a warp takes one group of channels where few units leave the GPU idle otherwise
    const int64_t units = heads * ((L.row_tiles + 1) / 2);
    const unsigned blocks = (unsigned)(L.pitch / 32);
    if (units * blocks < 148)
        return launch_kernel(tree_combine_kernel<1>, dim3((unsigned)units, blocks, 4), dim3(kTreeCombineWarps * 32), 0, stream, 1, a);
    return launch_kernel(tree_combine_kernel<4>, dim3((unsigned)units, blocks, 1), dim3(kTreeCombineWarps * 32), 0, stream, 1, a);
}
