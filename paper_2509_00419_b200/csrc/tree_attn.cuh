// What the kernels of lvlm_tree_attn share.
#pragma once
#include <cuda.h>

#include "cache.cuh"

namespace lvlm {

constexpr int kTreeMaxT = 256;                       // drafts a sequence: eight mask words a row
constexpr int kTreeMaxGroup = 64;
constexpr int kTreeTcRows = 128;                     // rows of a tile of the tcgen05 kernel
constexpr int kTreeTcCtas = 148;                     // its CTAs, one an SM
constexpr float kTreeLog2e = 1.4426950408889634f, kTreeLn2 = 0.6931471805599453f;

struct TreeArgs {
    const __nv_bfloat16* q; const int32_t* table; const int32_t* len; const uint32_t* mask; const int32_t* count;
    __nv_bfloat16* out; float* lse;
    int B, H, G, T, W, drafts, mask_shared;          // W mask words a row; drafts = 0: no Kd
    int S;                   // CTAs of a cluster; tcgen05 kernel: parts that the keys of a unit are cut into
    // tcgen05 kernel:
    int runs;                // the grid shares out the key tiles of all units instead
    int tile_rows;           // query rows of a tile (row r = draft r / G, head r % G of the group)
    int unit_tiles, units;   // row tiles of a unit of work (1 or 2); units of a head
    int pitch;               // places for the rows of a unit in a slot of the workspace
    int64_t q_sb, q_sn, q_sh;
    float scale_log2;
    // Partial results.  A slot holds `pitch` rows, groups of four channels of all rows side by side.  Slot (head, part, unit).  With runs a
    // CTA has at most one part that goes on with a unit, in slot `CTA`, and one that begins a unit, in slot kTreeTcCtas + CTA: of its fp32
    // outputs the upper 16 bits lie in the rows of `out` that the unit ends in, only the lower ones in part_lo, so that the workspace
    // stays below 32 MB.  part_of [head, unit]: the CTA that begins it, -1 = it was not cut, and how many more have a part of it.
    float2* part_ml;         // (max in the log2 domain, sum)
    float* part_o;           // output relative to that max
    uint2* part_lo;          // lower 16 bits of four channels
    int2* part_of;
    CacheGeom c;
    int32_t* dev_status;
#ifdef LVLM_TEST_HOOKS
    int starve, stall;
#endif
};

// The test build can keep the producers from fetching keys, so that waits run out, and hold up the warps of half 0 of a tcgen05 CTA
// for some microseconds before they read what the halves exchange.
#ifdef LVLM_TEST_HOOKS
__device__ __forceinline__ bool tree_starved(const TreeArgs& a) { return a.starve != 0; }
__device__ __forceinline__ void tree_stall(const TreeArgs& a, int half) {
    for (int i = 0; half == 0 && i < a.stall; ++i) __nanosleep(1000);
}
#else
__device__ __forceinline__ bool tree_starved(const TreeArgs&) { return false; }
__device__ __forceinline__ void tree_stall(const TreeArgs&, int) {}
#endif

__device__ __forceinline__ void tree_flag(const TreeArgs& a, int bit) {
    if (a.dev_status) atomicOr(a.dev_status, bit);
}
// The drafts and the cache rows of a head (-1: its length is no length), and its steps of `keys` keys: of the cache, and in all.
struct TreeHead { int n, ln, ns, nt; };
__device__ __forceinline__ TreeHead tree_head(const TreeArgs& a, int hd, int keys) {
    const int ln = __ldcg(a.len + hd), n = a.count ? __ldcg(a.count + hd / a.c.Hkv) : a.T;      // (both on their way before either is looked at)
    TreeHead h;
    h.n = n < 0 || n > a.T ? 0 : n;
    h.ln = ln < 0 || ln > a.c.cap ? -1 : ln;
    if (h.n != n || h.ln < 0) tree_flag(a, LVLM_DEV_BOUNDS);
    h.ns = h.ln > 0 ? (h.ln + keys - 1) / keys : 0;
    h.nt = h.ln < 0 ? 0 : h.ns + (a.drafts ? (h.n + keys - 1) / keys : 0);
    return h;
}
// Steps in a part of a unit.
__device__ __forceinline__ int tree_part(const TreeHead& h, int S) { return S == 1 ? max(h.nt, 1) : max(1, (h.nt + S - 1) / S); }

// Whether a record of part_of names CTAs that there are: the one that begins the unit, and at least one that goes on with it.  A scheduler
// that gave up on a wait leaves the records behind it as the workspace held them.
__host__ __device__ inline bool tree_record(int first, int more) { return first >= 0 && more > 0 && more < kTreeTcCtas - first; }

// Word w of what draft t sees, limited to the n drafts there are.
__device__ __forceinline__ uint32_t tree_see(const TreeArgs& a, int b, int t, int n, int w) {
    const int u0 = w * 32;
    if (!a.drafts || u0 >= n) return 0u;
    uint32_t bits;
    if (a.mask) bits = a.mask[((int64_t)(a.mask_shared ? 0 : b) * a.T + t) * a.W + w];
    else bits = t >= u0 + 31 ? 0xFFFFFFFFu : t < u0 ? 0u : (2u << (t - u0)) - 1u;
    return n < u0 + 32 ? bits & ((1u << (n - u0)) - 1u) : bits;
}

struct TreeMaps { CUtensorMap q, k, v, kd, vd; };
lvlm_status launch_tree_tc(const TreeArgs& a, const TreeMaps& m, cudaStream_t stream);

}  // namespace lvlm
