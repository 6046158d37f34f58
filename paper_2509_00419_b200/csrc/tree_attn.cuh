// What the kernels of lvlm_tree_attn share.
#pragma once
#include <cuda.h>

#include "cache.cuh"

namespace lvlm {

constexpr int kTreeMaxT = 256;                       // drafts a sequence: eight mask words a row
constexpr int kTreeMaxGroup = 64;
constexpr int kTreeTcRows = 128;                     // rows of a tile of the tcgen05 kernel
constexpr int kTreeTcCtas = 148;                     // its CTAs, one an SM
constexpr int kTreeTcLeast = 4;                      // least work of one, in key tiles of a row tile (2 or more)
constexpr float kTreeLog2e = 1.4426950408889634f, kTreeLn2 = 0.6931471805599453f;

struct TreeArgs {
    const __nv_bfloat16* q; const int32_t* table; const int32_t* len; const uint32_t* mask; const int32_t* count;
    __nv_bfloat16* out; float* lse;
    int B, H, G, T, W, drafts, mask_shared;          // W mask words a row; drafts = 0: no Kd
    int S, row_tiles;        // CTAs of a cluster (tcgen05 kernel: of the grid); tiles of its T G query rows
    int tile_rows, pitch;    // query rows in a tile, and places for rows in a slot of the workspace
    int64_t q_sb, q_sn, q_sh;
    float scale_log2;
    // Partial results of the tcgen05 kernel.  A slot holds `pitch` rows, groups of four channels of all rows side by side; a CTA has two slots,
    // for its first segment and its last; part_of [head, pair of row tiles]: the first slot of a unit, -1 = it was not cut, and how
    // many more CTAs have a part of it, in their first slots.
    float2* part_ml;         // (max in the log2 domain, sum)
    float* part_o;           // output relative to that max
    int2* part_of;
    CacheGeom c;
    int32_t* dev_status;
};

__device__ __forceinline__ void tree_flag(const TreeArgs& a, int bit) {
    if (a.dev_status) atomicOr(a.dev_status, bit);
}
__device__ __forceinline__ int tree_count(const TreeArgs& a, int b) {
    if (!a.count) return a.T;
    const int n = *(a.count + b);
    if (n < 0 || n > a.T) { tree_flag(a, LVLM_DEV_BOUNDS); return 0; }
    return n;
}
// The cache rows of a head, -1: its length is no length.
__device__ __forceinline__ int tree_len(const TreeArgs& a, int hd) {
    const int ln = *(a.len + hd);
    if (ln < 0 || ln > a.c.cap) { tree_flag(a, LVLM_DEV_BOUNDS); return -1; }
    return ln;
}

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
