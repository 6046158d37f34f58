// lvlm_rope_append and lvlm_commit_rows: new rows enter a cache, contiguous or paged, behind what every head holds.
//
// Both are copies bound by HBM: every byte is read once and written once (rope_append also reads 4 rot bytes of angles a token,
// shared by all its heads).  Rotation: a pair (x, y) of channels turns by the angle of its frequency, (x c - y s, y c + x s),
// in fp32, rounded once to bf16.  The cosines come from a table because an fp32 angle of a far position is off by
// position x 2^-24 radians.
#include "cache.cuh"

namespace lvlm {

constexpr int kRowLanes = 8;                       // lanes of a 256-byte row: two 16-byte chunks each
// Threads of a CTA, a token.  Many tokens: two warps, each with many rows after one wait for the positions, and 18 CTAs an SM; a token
// or a few: all rows at once.  us with 64 / 256 threads: 26200 tokens of 48 rows 100 / 164 (the bytes at the copy rate: 96), 16640 of
// 64 rows 87 / 115 (84); one token 3.6 / 2.7, 208 tokens of 48 rows 4.4 / 3.3.
constexpr int kRopeMany = 64, kRopeFew = 256, kRopeFewTokens = 2 * 148;
constexpr int kCommitThreads = 256;
// Rows of K and of V a CTA moves.  A CTA waits for three loads, one behind the other (length, page, row), so it is many CTAs that keep
// HBM busy: 8 an SM.  570 MB: 107 us with 64 rows a CTA, 95 with 32, 90.6 with their registers cut to fit 8 (the copy rate: 86).
constexpr int kCommitRows = 32;

struct RopeArgs {
    const __nv_bfloat16* q; const __nv_bfloat16* k_new; const __nv_bfloat16* v_new;
    const int32_t* pos; const float* cos_sin; const int32_t* count;
    __nv_bfloat16* q_out; __nv_bfloat16* Kc; __nv_bfloat16* Vc;
    const int32_t* table; const int32_t* len; int32_t* len_out;
    float* acc_score; int32_t* pos_cache;
    int B, H, T, rot, interleaved, n_pos, axes, sect0, sect1;
    int bump;                                      // 1: len_out is written (it is not len), 2: at the end (a sequence has one CTA)
    int64_t q_sb, q_sn, q_sh, qo_sb, qo_sn, qo_sh, n_sb, n_sn, n_sh;
    CacheGeom c;
    int32_t* dev_status;
};

__device__ __forceinline__ void flag_bounds(int32_t* dev_status) {
    if (dev_status) atomicOr(dev_status, LVLM_DEV_BOUNDS);
}

// The new rows of a sequence or head: n of them, 0 where the number given is none.
__device__ __forceinline__ int checked_count(const int32_t* count, int64_t at, int T, int32_t* dev_status) {
    if (!count) return T;
    const int n = *(count + at);
    if (n < 0 || n > T) { flag_bounds(dev_status); return 0; }
    return n;
}
// Where the n new rows of a head begin, or -1: they do not fit.
__device__ __forceinline__ int checked_start(const int32_t* len, int64_t hd, int n, int cap, int32_t* dev_status) {
    const int ln = len ? len[hd] : 0;
    if (ln < 0 || ln > cap || n > cap - ln) { flag_bounds(dev_status); return -1; }
    return ln;
}

// Eight channels (x) and their partners (y), turned.
__device__ __forceinline__ void turn(uint4& x, uint4& y, const float* cs, const float* sn) {
    uint32_t* a = reinterpret_cast<uint32_t*>(&x);
    uint32_t* b = reinterpret_cast<uint32_t*>(&y);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float a0 = bf16_lo(a[i]), a1 = bf16_hi(a[i]), b0 = bf16_lo(b[i]), b1 = bf16_hi(b[i]);
        a[i] = pack_bf16(a0 * cs[2 * i] - b0 * sn[2 * i], a1 * cs[2 * i + 1] - b1 * sn[2 * i + 1]);
        b[i] = pack_bf16(b0 * cs[2 * i] + a0 * sn[2 * i], b1 * cs[2 * i + 1] + a1 * sn[2 * i + 1]);
    }
}
// The same for neighbours: the pairs are the halves of a word.
__device__ __forceinline__ void turn_neighbours(uint4& x, uint4& y, const float* cs, const float* sn) {
    uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float a = bf16_lo(w[i]), b = bf16_hi(w[i]);
        w[i] = pack_bf16(a * cs[i] - b * sn[i], b * cs[i] + a * sn[i]);
    }
    x = make_uint4(w[0], w[1], w[2], w[3]);
    y = make_uint4(w[4], w[5], w[6], w[7]);
}

// grid.x = B * T tokens.  A token's rows are its H queries, Hkv keys and Hkv values, shared out to groups of 8 lanes; a group takes two
// at a time, so that their loads overlap, with its eight frequencies' cosines and sines in registers for all of them.
template <int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == kRopeMany ? 18 : 1) rope_append_kernel(const RopeArgs a) {
    constexpr int kGroups = THREADS / kRowLanes;
    pdl_enter();
    const int lane8 = threadIdx.x & (kRowLanes - 1), group = threadIdx.x / kRowLanes;
    const int b = blockIdx.x / a.T, t = blockIdx.x % a.T, Hkv = a.c.Hkv, rows = a.H + 2 * Hkv;
    const int n = checked_count(a.count, b, a.T, a.dev_status);
    const bool live = t < n;
    if (!live && !(a.bump && t == 0)) return;

    // chunks of 16 bytes: c0 and c1 are a rotated pair of chunks, or two that stay
    const int half = a.rot / 16;                   // chunks of the first half of the rotated channels
    const bool turned = lane8 < half;
    int c0 = 2 * lane8, c1 = 2 * lane8 + 1;
    if (!a.interleaved && turned) { c0 = lane8; c1 = lane8 + half; }
    float cs[8], sn[8];
    if (turned && live) {
        const int f0 = lane8 * 8;                  // my frequencies f0 .. f0 + 7
        auto axis_of = [&](int f) -> int { return a.axes == 3 ? (f >= a.sect0) + (f >= a.sect0 + a.sect1) : 0; };
        auto position = [&](int axis) -> int {
            const int p = a.pos[((int64_t)axis * a.B + b) * a.T + t];
            if (p >= 0 && p < a.n_pos) return p;
            flag_bounds(a.dev_status);
            return -1;
        };
        if (axis_of(f0) == axis_of(f0 + 7)) {
            const int p = position(axis_of(f0));
            const float4* c4 = reinterpret_cast<const float4*>(a.cos_sin + (int64_t)(p < 0 ? 0 : p) * a.rot + f0);
            const float4* s4 = c4 + a.rot / 8;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float4 c = p < 0 ? make_float4(1.f, 1.f, 1.f, 1.f) : c4[i], s = p < 0 ? make_float4(0.f, 0.f, 0.f, 0.f) : s4[i];
                cs[4 * i] = c.x; cs[4 * i + 1] = c.y; cs[4 * i + 2] = c.z; cs[4 * i + 3] = c.w;
                sn[4 * i] = s.x; sn[4 * i + 1] = s.y; sn[4 * i + 2] = s.z; sn[4 * i + 3] = s.w;
            }
        } else {                                   // a section ends among them
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int p = position(axis_of(f0 + i));
                const float* row = a.cos_sin + (int64_t)(p < 0 ? 0 : p) * a.rot + f0 + i;
                cs[i] = p < 0 ? 1.f : row[0];
                sn[i] = p < 0 ? 0.f : row[a.rot / 2];
            }
        }
    }
    for (int r0 = group; r0 < rows; r0 += 2 * kGroups) {
        uint4 x[2], y[2];
        __nv_bfloat16* to[2];
        bool turns[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int r = r0 + u * kGroups;
            to[u] = nullptr;
            if (r >= rows) continue;
            const __nv_bfloat16* from;
            turns[u] = turned;
            if (r < a.H) {
                if (!live) continue;
                from = a.q + (int64_t)b * a.q_sb + (int64_t)t * a.q_sn + (int64_t)r * a.q_sh;
                to[u] = a.q_out + (int64_t)b * a.qo_sb + (int64_t)t * a.qo_sn + (int64_t)r * a.qo_sh;
            } else {
                const bool key = r < a.H + Hkv;
                const int g = r - a.H - (key ? 0 : Hkv);
                const int64_t hd = (int64_t)b * Hkv + g;
                const int ln = checked_start(a.len, hd, n, a.c.cap, a.dev_status);
                if (a.bump == 1 && key && t == 0 && lane8 == 0) a.len_out[hd] = ln >= 0 ? ln + n : a.len ? a.len[hd] : 0;
                if (ln < 0 || !live) continue;
                const int64_t off = cache_row(a.c, a.table, b, g, ln + t);
                if (off < 0) { flag_bounds(a.dev_status); continue; }
                if (key && lane8 == 0) {
                    if (a.acc_score) a.acc_score[hd * a.c.cap + ln + t] = 0.f;
                    if (a.pos_cache) a.pos_cache[hd * a.c.cap + ln + t] = a.pos[(int64_t)b * a.T + t];
                }
                from = (key ? a.k_new : a.v_new) + (int64_t)b * a.n_sb + (int64_t)t * a.n_sn + (int64_t)g * a.n_sh;
                to[u] = (key ? a.Kc : a.Vc) + off;
                turns[u] = turned && key;
            }
            x[u] = reinterpret_cast<const uint4*>(from)[c0];
            y[u] = reinterpret_cast<const uint4*>(from)[c1];
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if (!to[u]) continue;
            if (turns[u]) {
                if (a.interleaved) turn_neighbours(x[u], y[u], cs, sn);
                else turn(x[u], y[u], cs, sn);
            }
            reinterpret_cast<uint4*>(to[u])[c0] = x[u];
            reinterpret_cast<uint4*>(to[u])[c1] = y[u];
        }
    }
    if (a.bump == 2) {                             // len_out is len, which every thread has read by now
        __syncthreads();
        for (int g = threadIdx.x; g < Hkv; g += THREADS) {
            const int64_t hd = (int64_t)b * Hkv + g;
            const int ln = checked_start(a.len, hd, n, a.c.cap, nullptr);
            if (ln >= 0) a.len_out[hd] = ln + n;
        }
    }
}

// len += count where the launch before it still read len from many CTAs.
__global__ void __launch_bounds__(256) grow_len_kernel(int32_t* len, const int32_t* count, int count_heads, int heads, int Hkv, int T, int cap) {
    pdl_enter();
    const int hd = blockIdx.x * 256 + threadIdx.x;
    if (hd >= heads) return;
    const int n = checked_count(count, count_heads ? hd : hd / Hkv, T, nullptr);
    const int ln = checked_start(len, hd, n, cap, nullptr);
    if (ln >= 0) len[hd] = ln + n;
}

struct CommitArgs {
    const __nv_bfloat16* Kd; const __nv_bfloat16* Vd;
    const int32_t* index; const int32_t* count; const int32_t* pos;
    __nv_bfloat16* Kc; __nv_bfloat16* Vc;
    const int32_t* table; const int32_t* len; int32_t* len_out;
    float* acc_score; int32_t* pos_cache;
    int T, draft_cap, count_heads, bump;
    int64_t d_sb, d_sh;
    CacheGeom c;
    int32_t* dev_status;
};

// grid (heads, runs of kCommitRows rows): 16 lanes move a row of K and the row of V of the same number.
__global__ void __launch_bounds__(kCommitThreads, 8) commit_rows_kernel(const CommitArgs a) {
    pdl_enter();
    const int Hkv = a.c.Hkv, hd = blockIdx.x, b = hd / Hkv, g = hd % Hkv;
    const int n = checked_count(a.count, a.count_heads ? hd : b, a.T, a.dev_status);
    const int ln = checked_start(a.len, hd, n, a.c.cap, a.dev_status);
    if (a.bump) {
        if (a.len_out == a.len) __syncthreads();   // (one CTA a head then)
        if (blockIdx.y == 0 && threadIdx.x == 0 && (ln >= 0 || a.len_out != a.len)) a.len_out[hd] = ln >= 0 ? ln + n : a.len ? a.len[hd] : 0;
    }
    if (ln < 0) return;
    const int ch = threadIdx.x & 15;
    const int i0 = blockIdx.y * kCommitRows;
    constexpr int kStep = kCommitThreads / 16;
    const int64_t src0 = (int64_t)b * a.d_sb + (int64_t)g * a.d_sh;
    uint4 x[kCommitRows / kStep], y[kCommitRows / kStep];
    int64_t off[kCommitRows / kStep];
#pragma unroll
    for (int u = 0; u < kCommitRows / kStep; ++u) {
        const int i = i0 + u * kStep + threadIdx.x / 16;
        off[u] = -1;
        if (i >= n) continue;
        const int j = a.index ? *(a.index + (int64_t)b * a.T + i) : i;
        if (j < 0 || j >= a.draft_cap) { flag_bounds(a.dev_status); continue; }
        off[u] = cache_row(a.c, a.table, b, g, ln + i);
        if (off[u] < 0) { flag_bounds(a.dev_status); continue; }
        if (ch == 0) {
            if (a.acc_score) a.acc_score[(int64_t)hd * a.c.cap + ln + i] = 0.f;
            if (a.pos_cache) a.pos_cache[(int64_t)hd * a.c.cap + ln + i] = a.pos[(int64_t)b * a.draft_cap + j];
        }
        x[u] = reinterpret_cast<const uint4*>(a.Kd + src0 + (int64_t)j * kHeadDim)[ch];
        y[u] = reinterpret_cast<const uint4*>(a.Vd + src0 + (int64_t)j * kHeadDim)[ch];
    }
#pragma unroll
    for (int u = 0; u < kCommitRows / kStep; ++u) {
        if (off[u] < 0) continue;
        reinterpret_cast<uint4*>(a.Kc + off[u])[ch] = x[u];
        reinterpret_cast<uint4*>(a.Vc + off[u])[ch] = y[u];
    }
}

// Whether len_out [heads] lies over lengths or counts that other threads may still have to read: over len or count [counts] other than
// place for place (count only where len_out is len: the thread that writes such a length has read both).
static bool lengths_clash(const int32_t* len, const int32_t* len_out, int64_t heads, const int32_t* count, int64_t counts) {
    if (!len_out) return false;
    if (len && len != len_out && overlap(len, heads * 4, len_out, heads * 4)) return true;
    return count && overlap(count, counts * 4, len_out, heads * 4) && !(len == len_out && count == len_out && counts == heads);
}

static lvlm_status grow_len(int32_t* len, const int32_t* count, int count_heads, int heads, const CacheGeom& c, int T, cudaStream_t stream) {
    return launch_kernel(grow_len_kernel, dim3((unsigned)((heads + 255) / 256)), dim3(256), 0, stream, 1, len, count, count_heads, heads,
                         c.Hkv, T, c.cap);
}

}  // namespace lvlm

extern "C" lvlm_status lvlm_rope_append(const void* q, const void* k_new, const void* v_new, const int32_t* pos,
                                         const float* cos_sin, const int32_t* count, void* q_out, void* Kc, void* Vc,
                                         const int32_t* table, const int32_t* len, int32_t* len_out, float* acc_score,
                                         int32_t* pos_cache, const lvlm_dims* d, int32_t* dev_status, void* stream_) {
    using namespace lvlm;
    cudaStream_t stream = (cudaStream_t)stream_;
    if (!k_new || !v_new || !Kc || !Vc || !d || d->B <= 0 || d->Hkv <= 0 || d->T <= 0) return LVLM_ERR_INVALID_ARG;
    if ((q == nullptr) != (q_out == nullptr) || (q && (d->H <= 0 || d->H % d->Hkv))) return LVLM_ERR_INVALID_ARG;
    if (d->rot < 0 || d->rot > kHeadDim || (d->rot > 0 && (!pos || !cos_sin || d->n_pos <= 0)) || (pos_cache && !pos)) return LVLM_ERR_INVALID_ARG;
    const int axes = d->axes ? d->axes : 1;
    if ((axes != 1 && axes != 3) || (axes == 3 && (d->sect0 < 0 || d->sect1 < 0 || (int64_t)d->sect0 + d->sect1 > d->rot / 2))) return LVLM_ERR_INVALID_ARG;
    if (d->D != kHeadDim || d->rot % 16) return LVLM_ERR_UNSUPPORTED;
    RopeArgs a;
    const lvlm_status g = cache_geom(d, table, &a.c);
    if (g != LVLM_OK) return g;
    a.B = d->B; a.H = q ? d->H : 0; a.T = d->T;
    a.q_sh = d->q_stride_h ? d->q_stride_h : d->D;
    a.q_sn = d->q_stride_n ? d->q_stride_n : (int64_t)d->H * d->D;
    a.q_sb = d->q_stride_b ? d->q_stride_b : (int64_t)d->T * a.q_sn;
    a.qo_sh = d->D; a.qo_sn = (int64_t)d->H * d->D; a.qo_sb = (int64_t)d->T * a.qo_sn;
    if (q_out == q) { a.qo_sh = a.q_sh; a.qo_sn = a.q_sn; a.qo_sb = a.q_sb; }
    a.n_sh = d->new_stride_h ? d->new_stride_h : d->D;
    a.n_sn = d->new_stride_n ? d->new_stride_n : (int64_t)d->Hkv * d->D;
    a.n_sb = d->new_stride_b ? d->new_stride_b : (int64_t)d->T * a.n_sn;
    if (!aligned16(cos_sin) || !aligned16(q) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(q_out) || !aligned16(Kc) || !aligned16(Vc) ||
        a.q_sh % 8 || a.q_sn % 8 || a.q_sb % 8 || a.n_sh % 8 || a.n_sn % 8 || a.n_sb % 8)
        return LVLM_ERR_ALIGNMENT;
    if (q && q_out != q &&
        overlap(q, 2 * ((d->B - 1) * a.q_sb + (d->T - 1) * a.q_sn + (d->H - 1) * a.q_sh + kHeadDim), q_out, 2 * (int64_t)d->B * a.qo_sb))
        return LVLM_ERR_INVALID_ARG;
    const int64_t tokens = (int64_t)d->B * d->T, heads = (int64_t)d->B * d->Hkv;
    if (tokens > 0x7FFFFFFFll || heads > 0x7FFFFFFFll) return LVLM_ERR_UNSUPPORTED;
    if (lengths_clash(len, len_out, heads, count, d->B)) return LVLM_ERR_INVALID_ARG;
    a.q = static_cast<const __nv_bfloat16*>(q);
    a.k_new = static_cast<const __nv_bfloat16*>(k_new);
    a.v_new = static_cast<const __nv_bfloat16*>(v_new);
    a.pos = pos; a.cos_sin = cos_sin; a.count = count;
    a.q_out = static_cast<__nv_bfloat16*>(q_out);
    a.Kc = static_cast<__nv_bfloat16*>(Kc);
    a.Vc = static_cast<__nv_bfloat16*>(Vc);
    a.table = table; a.len = len; a.len_out = len_out; a.acc_score = acc_score; a.pos_cache = pos_cache;
    a.rot = d->rot; a.interleaved = d->interleaved != 0; a.n_pos = d->n_pos; a.axes = axes; a.sect0 = d->sect0; a.sect1 = d->sect1;
    const bool in_place = len_out != nullptr && len_out == len;
    a.bump = !len_out ? 0 : !in_place ? 1 : d->T == 1 ? 2 : 0;
    a.dev_status = dev_status;
    const lvlm_status st = tokens <= kRopeFewTokens ? launch_kernel(rope_append_kernel<kRopeFew>, dim3((unsigned)tokens), dim3(kRopeFew), 0, stream, 1, a)
                                                    : launch_kernel(rope_append_kernel<kRopeMany>, dim3((unsigned)tokens), dim3(kRopeMany), 0, stream, 1, a);
    if (st != LVLM_OK || !in_place || d->T == 1) return st;
    return grow_len(len_out, count, 0, (int)heads, a.c, d->T, stream);
}

extern "C" lvlm_status lvlm_commit_rows(const void* Kd, const void* Vd, const int32_t* index, const int32_t* count,
                                         const int32_t* pos, void* Kc, void* Vc, const int32_t* table, const int32_t* len,
                                         int32_t* len_out, float* acc_score, int32_t* pos_cache, const lvlm_dims* d,
                                         int32_t* dev_status, void* stream_) {
    using namespace lvlm;
    cudaStream_t stream = (cudaStream_t)stream_;
    if (!Kd || !Vd || !Kc || !Vc || !d || d->B <= 0 || d->Hkv <= 0 || d->T <= 0 || d->draft_cap <= 0 || (!index && d->T > d->draft_cap) ||
        Kd == Kc || Vd == Vc || Kd == Vc || Vd == Kc || (pos == nullptr) != (pos_cache == nullptr))
        return LVLM_ERR_INVALID_ARG;
    if (d->D != kHeadDim) return LVLM_ERR_UNSUPPORTED;
    CommitArgs a;
    const lvlm_status g = cache_geom(d, table, &a.c);
    if (g != LVLM_OK) return g;
    a.d_sh = d->draft_stride_h ? d->draft_stride_h : (int64_t)d->draft_cap * d->D;
    a.d_sb = d->draft_stride_b ? d->draft_stride_b : (int64_t)d->Hkv * a.d_sh;
    if (!aligned16(Kd) || !aligned16(Vd) || !aligned16(Kc) || !aligned16(Vc) || a.d_sh % 8 || a.d_sb % 8) return LVLM_ERR_ALIGNMENT;
    const int64_t heads = (int64_t)d->B * d->Hkv, runs = ((int64_t)d->T + kCommitRows - 1) / kCommitRows;
    if (heads > 0x7FFFFFFFll || runs > 65535) return LVLM_ERR_UNSUPPORTED;
    if (lengths_clash(len, len_out, heads, count, d->count_heads ? heads : d->B)) return LVLM_ERR_INVALID_ARG;
    a.Kd = static_cast<const __nv_bfloat16*>(Kd);
    a.Vd = static_cast<const __nv_bfloat16*>(Vd);
    a.index = index; a.count = count; a.pos = pos;
    a.Kc = static_cast<__nv_bfloat16*>(Kc);
    a.Vc = static_cast<__nv_bfloat16*>(Vc);
    a.table = table; a.len = len; a.len_out = len_out; a.acc_score = acc_score; a.pos_cache = pos_cache;
    a.T = d->T; a.draft_cap = d->draft_cap; a.count_heads = d->count_heads != 0;
    const bool later = len_out != nullptr && len_out == len && runs > 1;
    a.bump = len_out != nullptr && !later;
    a.dev_status = dev_status;
    const lvlm_status st = launch_kernel(commit_rows_kernel, dim3((unsigned)heads, (unsigned)runs), dim3(kCommitThreads), 0, stream, 1, a);
    if (st != LVLM_OK || !later) return st;
    return grow_len(len_out, count, a.count_heads, (int)heads, a.c, d->T, stream);
}
