// d3tom_attend_cache: attention of each sample's newest rows over its cache in pages.
//
// The keys of a long cache are cut into runs of equal length; each run gives, for every row and head, the maximum m of its logits, the sum
// l of their exponentials relative to it and the values O added up with them, all float32; runs are joined by
//   o = sum_s O_s 2^(m_s - m) / sum_s l_s 2^(m_s - m),  m = max_s m_s    (logits in units of log 2).
// What the slots got (weight_out) is formed from the joined sums behind that: p = 2^(logit - lse).
#include "cache.hpp"
#include "direct_load.hpp"

namespace d3tom {

struct AttendCacheArgs {
    CacheView cache;
    const void *q, *k_pages, *v_pages;
    size_t q_stride;
    const int32_t* q_off;
    int nB, rows, max_q, max_len, H, G, causal; // G: query heads of a key head
    float scale2;                               // scale * log2(e)
    float per_G, per_heads, per_Hkv;            // 1 / G, 1 / (nB Hkv), 1 / Hkv
    int S, run;                                 // runs of a cache, slots of a run
    void* o;
    float *lse, *lse2;                          // natural logarithm (the caller's), base 2 (for the weights)
    float *part_o, *part_ml;                    // [rows, H, S, dh], [rows, H, S, 2]
    float* logits;                              // [rows, H, lpad], units of log 2, or none
    int last_slot;                              // that a sample's part of the page table has a place for
    int lpad, tiles;                            // tiles: of 64 or 128 rows, of a sample and key head
    const float* weight_in;
    float* weight_out;
    int weight_stride;
};

// A sample's rows: first one, how many.  Offsets that do not fit are cut to what there is.
__device__ __forceinline__ int sample_rows(const AttendCacheArgs& a, int b, int& r0) {
    r0 = min(max(a.q_off[b], 0), a.rows);
    return min(max(min(a.q_off[b + 1], a.rows) - r0, 0), a.max_q);
}
// slots that row i of nq sees
__device__ __forceinline__ int row_limit(const AttendCacheArgs& a, int n, int nq, int i) { return a.causal ? max(n - nq + i + 1, 0) : n; }

// What a row's sum gives.  It is 0 where the row saw nothing (no slot, or logits of -infinity alone); NaN among its logits makes it NaN, which output, lse and weights then show.
__device__ __forceinline__ float row_factor(float z) { return z == 0.f ? 0.f : 1.0f / z; }
// (units of log 2; for the weights: whatever the logit of a row that saw nothing, 2^(logit - lse) is 0)
__device__ __forceinline__ float weights_lse2(float m, float z) { return z == 0.f ? INFINITY : m + log2f(z); }
__device__ __forceinline__ void store_lse(const AttendCacheArgs& a, size_t at, float m, float z) {
    if (a.lse) a.lse[at] = (m + log2f(z)) * 0.6931471805599453f;
    if (a.lse2) a.lse2[at] = weights_lse2(m, z);
}

// Any head size.  One workgroup per row, head and run: 256 slots at a time, 16 lanes to a key; for the output a thread takes one 16-byte chunk
// of the channels and every (256 / chunks)-th slot.  Far from memory's bound, since every query head reads its keys for itself and products are vector instructions: a row each of 16
// samples of 900 .. 2688 slots, bf16, 32 heads over 8 of 80 and of 96 channels, 16 over 4 of 256: 90, 116 and 116 us for 77, 93 and 124 MB.
template <typename T>
__global__ __launch_bounds__(256) void attend_cache_generic_kernel(AttendCacheArgs a) {
    constexpr int EPC = 16 / sizeof(T);
    __shared__ float prob[256];
    __shared__ uint32_t page_row[256];                 // page of the slot
    __shared__ float red[8];
    __shared__ __attribute__((aligned(16))) float sums[256 * EPC];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int dh = a.cache.dh, nch = dh / EPC;
    int id = blockIdx.x;
    const int s = id % a.S; id /= a.S;
    const int h = id % a.H; id /= a.H;
    const int i = id % a.max_q, b = id / a.max_q;
    int r0;
    const int nq = sample_rows(a, b, r0);
    if (i >= nq) return;
    const int n = a.cache.length(b, a.max_len);
    const int limit = row_limit(a, n, nq, i);
    const int j0 = s * a.run, j1 = min(limit, j0 + a.run);
    const size_t row = (size_t)(r0 + i);
    const uint4* q = reinterpret_cast<const uint4*>(static_cast<const T*>(a.q) + row * a.q_stride + (size_t)h * dh);
    const size_t kvh = (size_t)(h / a.G) * dh, rs = a.cache.row_elems();
    const T *kp = static_cast<const T*>(a.k_pages) + kvh, *vp = static_cast<const T*>(a.v_pages) + kvh;

    const int l = lane & 15, g = lane >> 4;
    uint4 qr[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) qr[t] = q[min(l + 16 * t, nch - 1)];
    const int ch = tid % nch, grp = tid / nch, ngrp = 256 / nch;
    float acc[EPC];
#pragma unroll
    for (int e = 0; e < EPC; ++e) acc[e] = 0.f;
    float m = -INFINITY, z = 0.f;
    for (int c0 = j0; c0 < j1; c0 += 256) {
        const int cnt = min(256, j1 - c0);
        __syncthreads();
        if (tid < cnt) page_row[tid] = a.cache.readable(a.cache.page_of(b, c0 + tid));
        prob[tid] = -INFINITY;
        __syncthreads();
        for (int u = 0; u < 16; ++u) {
            const int x = wave * 64 + u * 4 + g;
            const int xc = min(x, cnt - 1);
            const uint4* k = reinterpret_cast<const uint4*>(kp + a.cache.row(page_row[xc], c0 + xc) * rs);
            float d = 0.f;
#pragma unroll
            for (int t = 0; t < 4; ++t)
                if (l + 16 * t < nch) d = chunk_dot<T>(qr[t], k[l + 16 * t], d);
            d = row16_sum(d);
            if (l == 0 && x < cnt) prob[x] = d * a.scale2;
        }
        __syncthreads();
        const float mine = prob[tid];
        float mx = wave_max(mine);
        if (lane == 0) red[wave] = mx;
        __syncthreads();
        const float mn = fmaxf(m, fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
        const float p = mine == -INFINITY ? 0.f : exp2f(mine - mn);
        prob[tid] = p;
        const float zs = wave_sum(p);
        if (lane == 0) red[4 + wave] = zs;
        __syncthreads();
        const float alpha = m == -INFINITY ? 0.f : exp2f(m - mn);
        z = z * alpha + ((red[4] + red[5]) + (red[6] + red[7]));
        m = mn;
#pragma unroll
        for (int e = 0; e < EPC; ++e) acc[e] *= alpha;
        if (grp < ngrp)
            for (int x = grp; x < cnt; x += ngrp) {
                const uint4 w = reinterpret_cast<const uint4*>(vp + a.cache.row(page_row[x], c0 + x) * rs)[ch];
                const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
                const float px = prob[x];
#pragma unroll
                for (int e = 0; e < EPC; ++e) {
                    float v;
                    if constexpr (EPC == 8) v = (e & 1) ? bf16_hi(ww[e >> 1]) : bf16_lo(ww[e >> 1]);
                    else v = __uint_as_float(ww[e]);
                    acc[e] = __builtin_fmaf(px, v, acc[e]);
                }
            }
    }
#pragma unroll
    for (int e = 0; e < EPC; ++e) sums[tid * EPC + e] = grp < ngrp ? acc[e] : 0.f;
    __syncthreads();
    const size_t at = (row * a.H + h) * a.S + s;
    if (tid < dh) {
        const int c = tid / EPC, e = tid % EPC;
        float t = 0.f;
        for (int x = 0; x < ngrp; ++x) t += sums[(x * nch + c) * EPC + e];
        if (a.S > 1) a.part_o[at * dh + tid] = t;
        else Elem<T>::store(static_cast<T*>(a.o) + at * dh + tid, z == 0.f ? 0.f : t / z);
    }
    if (tid == 0) {
        if (a.S > 1) { a.part_ml[at * 2] = m; a.part_ml[at * 2 + 1] = z; }
        else store_lse(a, at, m, z);
    }
}


// ---- heads of 64 and 128 on the matrix instructions ----------------------------------------------------------------------
// The rows of a sample that share a key head (G heads of every new row) are the columns of
//     S^T = K Q^T     A = K (LDS), B = Q^T (registers)
//     O^T += V^T P^T  A = V^T (LDS; bf16: the transposing read), B = P^T as the accumulators of the first product hold it
// sixteen of them, MFMA 16x16x32 (bf16) or four 16x16x4 (float32), whose lanes take four neighbouring channels each: the order of a contraction is free.
// Lane (r, g) = (lane % 16, lane / 16) has column r and, of every 16 keys, keys 4g .. 4g + 3.
//
// Bound by memory: a key's row is read for 16 columns at most.  What keeps it busy is bytes in flight, so every wave is on its own, with a ring of two stages (K and V of
// 8 KB each) that direct loads fill: while one stage is used the other and the next are on their way, and no wave waits for another one before
// the end, when the four waves of a workgroup join what they have through LDS.  One row each of two samples of 131071 slots, 32 heads over 8 of 128, bf16:
// 185 us, 5.8 TB/s.  One row of 3709 slots, 32 key heads: 13.4 us, 4.5 TB/s.
template <typename T, int DH> struct AcTile {
    static constexpr int ROWB = DH * (int)sizeof(T), NCHK = ROWB / 16;      // bytes and 16-byte chunks of a row of a head
    static constexpr int TILE = 8192, KEYS = TILE / ROWB, KB = KEYS / 16;   // of K or V: keys, blocks of 16
    static constexpr int LD = 8, LDB = LD / KB, RPI = 64 / NCHK;            // direct loads of a tile, of a block; rows of one
    static constexpr int KS = NCHK / 4, DB = DH / 16;                       // steps of the first product, 16-channel blocks of O^T
    static constexpr int STAGE = 2 * TILE, WAVE_LDS = 2 * STAGE, PITCH = DH + 4;
    // what the position of a chunk in a row is turned by, so that the 16 rows of a fragment lie in different banks
    static __device__ __forceinline__ int k_turn(int row) { return row & (NCHK - 1) & 15; }
    static __device__ __forceinline__ int v_turn(int row) {
        if constexpr (sizeof(T) == 4) return ((row >> 2) & 3) * 4;
        else return NCHK == 16 ? (row & 3) * 4 : ((row >> 1) & 1) * 2;
    }
};
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short ac_short4;
typedef __attribute__((__vector_size__(8 * sizeof(short)))) short ac_short8;

#if defined(__HIP_DEVICE_COMPILE__)
__device__ __forceinline__ f32x4 ac_mma(const uint4& a, const uint4& b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// Float32 logits as four sums side by side.  One after the other, dh / 4 roundings deep, they were most of the output's error where a sample has few slots: over 600
// calls of all lengths, its ratio to the error of the same attention in elementary float32 operations was 1.08 in the middle and 3.6 at most, and is 0.63 and 1.5.  5 rows over
// 213 slots 6.9 -> 6.5 us, a row each over 16 samples of 1000 slots (32 heads over 8 of 64) 18.1 -> 17.3; 32 rows each over 4 of 1500 (8 over 2 of 128) 20.9 -> 21.1.
template <int KS>
__device__ __forceinline__ f32x4 ac_logits_f32(const uint4 (&k)[KS], const uint4 (&q)[KS]) {
    f32x4 sum[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
        const f32x4 x = __builtin_bit_cast(f32x4, k[kk]), y = __builtin_bit_cast(f32x4, q[kk]);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], sum[e], 0, 0, 0);
    }
    f32x4 all;
#pragma unroll
    for (int e = 0; e < 4; ++e) all[e] = (sum[0][e] + sum[1][e]) + (sum[2][e] + sum[3][e]);
    return all;
}
__device__ __forceinline__ float quad_max(float v) { return quad_combine(v, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float quad_sum(float v) { return quad_combine(v, [](float a, float b) { return a + b; }); }
#endif

// A tile's logits of one block of rows, in units of log 2, to probabilities relative to the running maximum; O and the sum are scaled where that has moved.
// It moves only where a logit is AC_SLACK above it: the probabilities are then at most 2^AC_SLACK, which costs no precision in float32 sums and none in bf16 (its
// steps are relative), and the scaling, 4 DB multiplications, is rare behind the first tiles: with sixteen rows to a wave one of them has a new maximum in most tiles.
// `left`: keys in front of the lane's first one that are still seen, where the tile has any that are not.
constexpr float AC_SLACK = 6.f;
template <int KB, int DB>
__device__ __forceinline__ void ac_softmax(f32x4 (&st)[KB], f32x4 (&o)[DB], float& m, float& l, float scale2, bool masked, int left) {
#if defined(__HIP_DEVICE_COMPILE__)
    if (masked) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int e = 0; e < 4; ++e) st[kb][e] = kb * 16 + e < left ? st[kb][e] : -INFINITY;
    }
    float top = -INFINITY;                                 // (the median of two values and infinity is the larger one, without an instruction that quiets NaN first)
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int e = 0; e < 4; ++e) top = __builtin_amdgcn_fmed3f(top, st[kb][e], INFINITY);
    top *= scale2;
    if (__builtin_amdgcn_ballot_w64(top > m + AC_SLACK) != 0) {
        const float mn = fmaxf(m, quad_max(top));
        const float alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        l *= alpha;
#pragma unroll
        for (int t = 0; t < DB; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[t][e] *= alpha;
    }
    const float ref = m == -INFINITY ? 0.f : m;            // a column that has seen nothing yet: all its p are 0
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(st[kb][e], scale2, -ref));
            st[kb][e] = p;
            sum[e] += p;
        }
    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
#endif
}

// The matrix instructions multiply values that a column does not see by its probability of 0, which NaN and infinities survive.  In tiles that not all columns see (of causal rows
// alone, one or two of a run) such values of those slots are taken for 0, and where there were any, the columns that do see them get them behind the last tile: 0 + v is
// what p v makes of a value that is not finite.  (Kernels of their own for such rows: others would be up to 1 % slower.  The looking itself: 32 rows each of 4 samples, 32 heads over 8 of
// 128, bf16, and 2048 rows as before; 5 rows over 213 slots of float32 heads of 64 6.34 -> 6.48 us; 4 rows each of 8 samples of 1500 slots, bf16, 128 and 64 channels, 13.9 -> 14.1 and
// 11.35 -> 11.56; 32 rows each of 2 of 1500, float32, 29.9 -> 30.8.)
// A word of values of keys k0 and, bf16, k1 (its upper half): those that are not finite and not among the first `seen` keys to 0.
template <typename T>
__device__ __forceinline__ bool ac_clean(uint32_t& w, int k0, int k1, int seen) {
    const uint32_t before = w;
    if constexpr (sizeof(T) == 2) {
        if (k0 >= seen && (w & 0x7F80u) == 0x7F80u) w &= 0xFFFF0000u;
        if (k1 >= seen && (w & 0x7F800000u) == 0x7F800000u) w &= 0xFFFFu;
    } else {
        if (k0 >= seen && (w & 0x7F800000u) == 0x7F800000u) w = 0u;
    }
    return w != before;
}
// the larger magnitudes of two words, as unsigned numbers; whether one of them belongs to a value that is not finite
template <typename T>
__device__ __forceinline__ uint32_t ac_magnitudes(uint32_t most, uint32_t w) {
    if constexpr (sizeof(T) == 2) {
        typedef unsigned short us2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(us2, most), __builtin_bit_cast(us2, w & 0x7FFF7FFFu)));
    } else {
        return max(most, w & 0x7FFFFFFFu);
    }
}
template <typename T>
__device__ __forceinline__ bool ac_not_finite(uint32_t most) { return most >= 0x7F800000u || (sizeof(T) == 2 && (most & 0xFFFFu) >= 0x7F80u); }
// The values of one head in slots [from, to) that are not finite, to the columns that see them.  `mine(slot)`: whether the slot was in a tile of this wave.
template <typename T, int DH, int QB, int DB, typename F>
__device__ __forceinline__ void ac_add_not_finite(const AttendCacheArgs& a, int b, int kvh, int from, int to, F&& mine, f32x4 (&o)[QB][DB], const int (&limit)[QB]) {
    const int g = (threadIdx.x & 63) >> 4;
#pragma nounroll
    for (int j = from; j < to; ++j) {
        if (!mine(j)) continue;
        const T* v = static_cast<const T*>(a.v_pages) + a.cache.row(a.cache.readable(a.cache.page_of(b, j)), j) * a.cache.row_elems() + (size_t)kvh * DH + 4 * g;
#pragma unroll
        for (int t = 0; t < DB; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float x = Elem<T>::load(v + t * 16 + e);
                const bool odd = (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u;
#pragma unroll
                for (int qb = 0; qb < QB; ++qb)
                    if (odd && j < limit[qb]) o[qb][t][e] += x;
            }
    }
}

// UNEVEN: rows of a sample may see different numbers of slots.
constexpr int WAVES = 4;
template <typename T, int DH, bool UNEVEN>
__global__ __launch_bounds__(64 * WAVES, 2) void attend_cache_kernel(AttendCacheArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    using C = AcTile<T, DH>;
    constexpr int ROWB = C::ROWB, NCHK = C::NCHK, KEYS = C::KEYS, KB = C::KB, LDB = C::LDB, RPI = C::RPI, KS = C::KS, DB = C::DB;
    extern __shared__ __attribute__((aligned(16))) char ring[];
    __shared__ float part_m[WAVES][16], part_l[WAVES][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
    // First runs first, so that the XCDs (every eighth workgroup) have samples of all lengths, and first runs, which every sample has, do not meet on some of them.
    int unit = blockIdx.x;
    const int heads = a.nB * a.cache.Hkv, s = __builtin_amdgcn_readfirstlane(div_by(unit, heads, a.per_heads));
    unit -= s * heads;
    const int b = __builtin_amdgcn_readfirstlane(div_by(unit, a.cache.Hkv, a.per_Hkv)), kvh = unit - b * a.cache.Hkv;
    // Pages of this wave's blocks of 16 slots: lane i has that of block i % KB of its tile i / KB.  Requested with the sample's sizes, not behind them: what lies
    // behind its last page is never used.
    const int j0 = s * a.run, my_slot = j0 + ((lane / KB) * WAVES + wave) * KEYS + (lane % KB) * 16;
    const int my_page = a.cache.page_of(b, min(my_slot, a.last_slot));
    int r0;
    const int nq = sample_rows(a, b, r0);
    const int R = nq * a.G;                            // 16 at most
    if (R <= 0) return;
    const int n = a.cache.length(b, a.max_len);
    const int j1 = min(row_limit(a, n, nq, nq - 1), j0 + a.run);
    if (j0 >= j1 && s > 0) return;
    const int x = min(r, R - 1), xi = div_by(x, a.G, a.per_G), xh = kvh * a.G + (x - xi * a.G);          // this lane's column
    const size_t row = (size_t)(r0 + xi);
    const int limit = min(row_limit(a, n, nq, xi), j1);
    const int limit0 = min(row_limit(a, n, nq, 0), j1);                                                        // slots that all columns see

    const int ntile = j1 > j0 ? (j1 - j0 + KEYS - 1) / KEYS : 0;
    const int mine = (ntile - wave + WAVES - 1) / WAVES;                                       // tiles wave, wave + WAVES, ...
    const uint32_t ids = a.cache.readable(my_page);

    const uint32_t row_bytes = (uint32_t)a.cache.row_elems() * sizeof(T);
    const int ld_pos = lane % NCHK, ld_row = lane / NCHK;
    int k_off[LDB], v_off[LDB];
#pragma unroll
    for (int i = 0; i < LDB; ++i) {
        const int x2 = i * RPI + ld_row;
        k_off[i] = x2 * row_bytes + ((ld_pos ^ C::k_turn(x2)) << 4);
        v_off[i] = x2 * row_bytes + ((ld_pos ^ C::v_turn(x2)) << 4);
    }
    const uint32_t ring0 = (uint32_t)(size_t)(lds_ptr_t)ring + wave * C::WAVE_LDS;
    const char* kbase = static_cast<const char*>(a.k_pages) + (size_t)kvh * ROWB;
    const char* vbase = static_cast<const char*>(a.v_pages) + (size_t)kvh * ROWB;
    // tile t of this wave; rows past j1 load as zeros without touching memory
    auto issue = [&](const char* base, const int (&off)[LDB], int t, uint32_t lds) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            const int slot = j0 + (t * WAVES + wave) * KEYS + kb * 16;
            const uint32_t page = __builtin_amdgcn_readlane(ids, (t * KB + kb) & 63);
            const int there = min(max(j1 - slot, 0), 16);
            const __amdgpu_buffer_rsrc_t rs = make_uniform_rsrc(base + a.cache.row(page, slot) * row_bytes, there ? (uint32_t)(there - 1) * row_bytes + ROWB : 0u);
#pragma unroll
            for (int i = 0; i < LDB; ++i) direct_load_16(rs, off[i], lds + (kb * LDB + i) * 1024);
        }
    };
    auto issue_k = [&](int t) { issue(kbase, k_off, t, ring0 + (t & 1) * C::STAGE); };
    auto issue_v = [&](int t) { issue(vbase, v_off, t, ring0 + (t & 1) * C::STAGE + C::TILE); };
    // The queries in front of them, on the same way: sixteen rows whose place in LDS all waves share, behind the rings.  (Loaded as fragments into registers, 64
    // bytes of a row at a time, they are slower than the keys, and these waited for them: 1 us.)
    const uint32_t q_lds = (uint32_t)(size_t)(lds_ptr_t)ring + WAVES * C::WAVE_LDS;
    constexpr int QLD = 16 / RPI;
    const __amdgpu_buffer_rsrc_t rq = make_uniform_rsrc(static_cast<const char*>(a.q) + ((size_t)r0 * a.q_stride + (size_t)kvh * a.G * DH) * sizeof(T), ~0u);
#pragma unroll
    for (int i = 0; i < (QLD + WAVES - 1) / WAVES; ++i) {
        const int li = i * WAVES + wave;
        if (QLD % WAVES == 0 || li < QLD) {
            const int x2 = li * RPI + ld_row, X = min(x2, R - 1), Xi = div_by(X, a.G, a.per_G);
            direct_load_16(rq, (uint32_t)(Xi * (int)a.q_stride + (X - Xi * a.G) * DH) * sizeof(T) + ((ld_pos ^ C::k_turn(x2)) << 4), q_lds + li * 1024);
        }
    }
    if (mine > 0) { issue_k(0); issue_v(0); }
    if (mine > 1) { issue_k(1); issue_v(1); }

    int k_addr[KS], v_addr[DB];
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) k_addr[kk] = r * ROWB + (((kk * 4 + g) ^ C::k_turn(r)) << 4);
#pragma unroll
    for (int t = 0; t < DB; ++t) {
        if constexpr (sizeof(T) == 2) {
            const int vr = 4 * g + (r >> 2), chunk = t * 2 + ((r & 3) >> 1);
            v_addr[t] = C::TILE + vr * ROWB + ((chunk ^ C::v_turn(vr)) << 4) + (r & 1) * 8;
        } else {
            v_addr[t] = C::TILE + 4 * g * ROWB + (((t * 4 + (r >> 2)) ^ C::v_turn(4 * g)) << 4) + (r & 3) * 4;
        }
    }
    f32x4 os[1][DB], (&o)[DB] = os[0];
#pragma unroll
    for (int t = 0; t < DB; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    const int clean_from = limit0 < j1 ? limit0 : INT_MAX;     // (ac_clean)
    bool cleaned = false;
    if (mine > 1) wait_loads<4 * C::LD>();             // the queries are there
    else if (mine > 0) wait_loads<2 * C::LD>();
    else wait_loads<0>();
    wait_loads_and_barrier<63>();
    uint4 qf[KS];
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) qf[kk] = *reinterpret_cast<const uint4*>(ring + WAVES * C::WAVE_LDS + k_addr[kk]);
    float* kept = a.logits ? a.logits + (row * a.H + xh) * a.lpad : nullptr;
    const bool real = r < R;

    for (int t = 0; t < mine; ++t) {
        const char* w = ring + wave * C::WAVE_LDS + (t & 1) * C::STAGE;
        const int key0 = j0 + (t * WAVES + wave) * KEYS;
        if (t + 1 < mine) wait_loads<3 * C::LD>();         // K of this tile is there
        else wait_loads<C::LD>();
        f32x4 st[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            if constexpr (sizeof(T) == 2) {
                st[kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < KS; ++kk) st[kb] = ac_mma(*reinterpret_cast<const uint4*>(w + k_addr[kk] + kb * 16 * ROWB), qf[kk], st[kb]);
            } else {
                uint4 kf[KS];
#pragma unroll
                for (int kk = 0; kk < KS; ++kk) kf[kk] = *reinterpret_cast<const uint4*>(w + k_addr[kk] + kb * 16 * ROWB);
                st[kb] = ac_logits_f32(kf, qf);
            }
        }
        wait_lds();
        if (t + 2 < mine) issue_k(t + 2);
        if (kept && real) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
                if (key0 + kb * 16 < j1) *reinterpret_cast<f32x4*>(kept + key0 + kb * 16 + 4 * g) = f32x4{st[kb][0] * a.scale2, st[kb][1] * a.scale2, st[kb][2] * a.scale2, st[kb][3] * a.scale2};
        }
        ac_softmax<KB, DB>(st, o, m, l, a.scale2, key0 + KEYS > limit0, limit - key0 - 4 * g);
        if (t + 2 < mine) wait_loads<3 * C::LD>();         // V of this tile
        else if (t + 1 < mine) wait_loads<2 * C::LD>();
        else wait_loads<0>();
        if (UNEVEN && key0 + KEYS > clean_from) {
#pragma nounroll
            for (int c = max(clean_from - key0, 0) * NCHK + lane; c < min(j1 - key0, KEYS) * NCHK; c += 64) {
                uint4* chunk = reinterpret_cast<uint4*>(ring + wave * C::WAVE_LDS + (t & 1) * C::STAGE + C::TILE + c * 16);
                uint32_t x[4] = {chunk->x, chunk->y, chunk->z, chunk->w};
                bool changed = false;
#pragma unroll
                for (int i = 0; i < 4; ++i) changed |= ac_clean<T>(x[i], 0, 0, 0);
                if (changed) *chunk = make_uint4(x[0], x[1], x[2], x[3]);
                cleaned |= changed;
            }
        }
        // Probabilities as two bf16 parts, their upper bits and what is left (2^-15 of them goes): rounded to one part they were a quarter of the output's error (relative to the
        // same in 64 bits 2.2e-3, now 1.65e-3, the output's own rounding), and matrix instructions are not what bounds few rows: a row each of 16 samples of 900 .. 2688 slots
        // (weighed) 36.8 -> 37.1 us, one of 3709 slots and 32 key heads 15.4 -> 15.6, of 8 samples of 400 slots 7.5 -> 7.8, of 512 slots and 8 key heads 6.9 -> 7.2, 4 rows each of 8 samples of 1500
        // slots and 64 channels 11.3 -> 11.0.  (The second part's product behind the request of the tile after the next, its values in registers: in front of it 0 .. 0.1 us more.  The
        // second parts in the place of columns that there are not: no faster.)
        constexpr int PAIRS = sizeof(T) == 2 ? KB / 2 : 1;
        bf16x8 v8[PAIRS][DB];
        if constexpr (sizeof(T) == 2) {
            typedef __attribute__((address_space(3))) ac_short4* tr_ptr;
#pragma unroll
            for (int kp = 0; kp < PAIRS; ++kp) {
                uint32_t upper[4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    upper[i] = __builtin_amdgcn_perm(__float_as_uint(st[2 * kp + i / 2][(i & 1) * 2 + 1]), __float_as_uint(st[2 * kp + i / 2][(i & 1) * 2]), 0x07060302u);
#pragma unroll
                for (int t2 = 0; t2 < DB; ++t2) {
                    const char* p = w + v_addr[t2] + kp * 32 * ROWB;
                    const ac_short4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)p), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)(p + 16 * ROWB));
                    v8[kp][t2] = __builtin_bit_cast(bf16x8, ac_short8(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7)));
                    o[t2] = ac_mma(__builtin_bit_cast(uint4, v8[kp][t2]), make_uint4(upper[0], upper[1], upper[2], upper[3]), o[t2]);
                }
            }
        } else {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int t2 = 0; t2 < DB; ++t2)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[t2] = __builtin_amdgcn_mfma_f32_16x16x4f32(*reinterpret_cast<const float*>(w + v_addr[t2] + (kb * 16 + e) * ROWB), st[kb][e], o[t2], 0, 0, 0);
        }
        wait_lds();
        if (t + 2 < mine) issue_v(t + 2);
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int kp = 0; kp < PAIRS; ++kp) {
                bf16x8 lower;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float p = st[2 * kp + e / 4][e % 4];
                    lower[e] = (__bf16)(p - __uint_as_float(__float_as_uint(p) & 0xFFFF0000u));
                }
#pragma unroll
                for (int t2 = 0; t2 < DB; ++t2) o[t2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8[kp][t2], lower, o[t2], 0, 0, 0);
            }
        }
    }
    if (UNEVEN && __builtin_amdgcn_ballot_w64(cleaned) != 0) {
        const int limits[1] = {limit};
        ac_add_not_finite<T, DH>(a, b, kvh, max(limit0, j0), j1, [&](int j) { return ((j - j0) / KEYS) % WAVES == wave; }, os, limits);
    }
    wait_loads_and_barrier<0>();                           // nothing is on its way into the rings any more
    // the waves' parts, rows of queries
    float* part = reinterpret_cast<float*>(ring);
    l = quad_sum(l);
    float* to = part + (wave * 16 + r) * C::PITCH + 4 * g;
#pragma unroll
    for (int t = 0; t < DB; ++t) *reinterpret_cast<f32x4*>(to + t * 16) = o[t];
    if (g == 0) { part_m[wave][r] = m; part_l[wave][r] = l; }
    __syncthreads();
    // four threads of every wave to a row
    constexpr int TPR = 4 * WAVES, CH = DH / TPR;
    const int y = tid / TPR;
    if (y >= R) return;
    const int yi = div_by(y, a.G, a.per_G), yh = kvh * a.G + (y - yi * a.G);
    float mt = -INFINITY;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) mt = fmaxf(mt, part_m[w][y]);
    float f[WAVES], z = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        f[w] = part_m[w][y] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(part_m[w][y] - mt);
        z += part_l[w][y] * f[w];
    }
    const size_t at = ((size_t)(r0 + yi) * a.H + yh) * a.S + s;
    const float inv = a.S > 1 ? 1.f : row_factor(z);
    const int c0 = (tid % TPR) * CH;
    float acc[CH];
#pragma unroll
    for (int e = 0; e < CH; ++e) acc[e] = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w)
#pragma unroll
        for (int e = 0; e < CH; ++e) acc[e] = __builtin_fmaf(part[(w * 16 + y) * C::PITCH + c0 + e], f[w], acc[e]);
#pragma unroll
    for (int e = 0; e < CH; ++e) acc[e] *= inv;
    if (a.S > 1) {
#pragma unroll
        for (int e = 0; e < CH; e += 4) *reinterpret_cast<f32x4*>(a.part_o + at * DH + c0 + e) = f32x4{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
        if (c0 == 0) { a.part_ml[at * 2] = mt; a.part_ml[at * 2 + 1] = z; }
    } else {
        T* out = static_cast<T*>(a.o) + at * DH + c0;
        if constexpr (sizeof(T) == 2) store_bf16<CH>(out, acc);
        else {
#pragma unroll
            for (int e = 0; e < CH; e += 4) *reinterpret_cast<f32x4*>(out + e) = f32x4{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
        }
        if (c0 == 0) store_lse(a, at, mt, z);
    }
#endif
}

// More than 16 rows to a key head: eight waves share the tiles.  Wave (kg, rg) has QB blocks of 16 rows (of four such groups rg) and half of every tile's keys, so that a
// key's row is read from LDS four times and from memory once for 64 QB rows, and two waves of a SIMD alternate between matrix instructions and
// exponentials.  Tiles of 16 KB of K and of V, of which every wave loads an eighth, in a ring of four stages; one barrier a tile: behind it this tile is there for everybody, and
// everybody is done with the last but one, whose place is loaded again.  At the end the two waves of the same rows exchange halves of the channels.
template <typename T, int DH> struct AcShared {
    using C = AcTile<T, DH>;
    static constexpr int TILE = 16384, KEYS = TILE / C::ROWB, KB = KEYS / 16, LD = 2, STAGE = 2 * TILE, STAGES = 4, LDS = STAGES * STAGE;
    static constexpr int KW = KB / 2;                  // blocks of 16 keys of a wave
    static constexpr int PAGES = 256;                  // blocks of 16 slots of a run whose pages lie in LDS
};
template <typename T, int DH, int QB, bool UNEVEN>
__global__ __launch_bounds__(512, 2) void attend_cache_rows_kernel(AttendCacheArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    using C = AcTile<T, DH>;
    using W = AcShared<T, DH>;
    constexpr int ROWB = C::ROWB, NCHK = C::NCHK, KEYS = W::KEYS, KB = W::KB, KW = W::KW, LD = W::LD, RPI = C::RPI, KS = C::KS, DB = C::DB;
    extern __shared__ __attribute__((aligned(16))) char ring[];
    __shared__ uint32_t pages[W::PAGES];
    __shared__ float other_m[2][4][QB * 16], other_l[2][4][QB * 16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
    const int kg = wave >> 2, rg = wave & 3;
    // Tiles of rows of the same keys run on one XCD, one after the other; first runs first (see above).
    int id = blockIdx.x;
    const int xcd = id & 7;
    id >>= 3;
    int tile = 0;
    if (a.tiles > 1) { tile = id % a.tiles; id /= a.tiles; }
    int unit = id * 8 + xcd;
    const int heads = a.nB * a.cache.Hkv, s = __builtin_amdgcn_readfirstlane(div_by(unit, heads, a.per_heads));
    unit -= s * heads;
    const int b = __builtin_amdgcn_readfirstlane(div_by(unit, a.cache.Hkv, a.per_Hkv)), kvh = unit - b * a.cache.Hkv;
    if (s >= a.S) return;
    const int j0 = s * a.run, my_page = a.cache.page_of(b, min(j0 + (tid & (W::PAGES - 1)) * 16, a.last_slot));         // (see above)
    int r0;
    const int nq = sample_rows(a, b, r0);
    constexpr int ROWS = 64 * QB;
    const int R = nq * a.G, R0 = tile * ROWS;
    if (R0 >= R) return;
    const int n = a.cache.length(b, a.max_len);
    const int j1 = min(row_limit(a, n, nq, div_by(min(R0 + ROWS, R) - 1, a.G, a.per_G)), j0 + a.run);
    if (j0 >= j1 && s > 0) return;
    const int W0 = R0 + rg * 16 * QB;                  // this wave's first row
    const bool works = W0 < R;
    size_t row[QB];
    int xh[QB], limit[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int x = min(W0 + qb * 16 + r, R - 1), xi = div_by(x, a.G, a.per_G);
        xh[qb] = kvh * a.G + (x - xi * a.G);
        row[qb] = (size_t)(r0 + xi);
        limit[qb] = min(row_limit(a, n, nq, xi), j1);
    }
    const int limit0 = min(row_limit(a, n, nq, div_by(min(W0, R - 1), a.G, a.per_G)), j1);
    const int ntile = j1 > j0 ? (j1 - j0 + KEYS - 1) / KEYS : 0;
    if (tid < W::PAGES) pages[tid] = a.cache.readable(my_page);
    const uint32_t row_bytes = (uint32_t)a.cache.row_elems() * sizeof(T);
    const int ld_pos = lane % NCHK, ld_row = lane / NCHK;
    const uint32_t ring0 = (uint32_t)(size_t)(lds_ptr_t)ring;
    const char* kbase = static_cast<const char*>(a.k_pages) + (size_t)kvh * ROWB;
    const char* vbase = static_cast<const char*>(a.v_pages) + (size_t)kvh * ROWB;
    int k_off[LD], v_off[LD];                          // of the row inside its block of 16
#pragma unroll
    for (int i = 0; i < LD; ++i) {
        const int x = ((wave * LD + i) * RPI + ld_row) & 15;
        k_off[i] = x * row_bytes + ((ld_pos ^ C::k_turn(x)) << 4);
        v_off[i] = x * row_bytes + ((ld_pos ^ C::v_turn(x)) << 4);
    }
    // this wave's loads of tile t; `ids`: lane i has the page of the tile's block i
    auto issue = [&](int t, uint32_t ids) {
        const uint32_t lds = ring0 + (t & (W::STAGES - 1)) * W::STAGE + wave * LD * 1024;
#pragma unroll
        for (int i = 0; i < LD; ++i) {
            const int kb = (wave * LD + i) * RPI / 16, slot = j0 + t * KEYS + kb * 16;
            const uint32_t page = __builtin_amdgcn_readlane(ids, kb);
            const int there = min(max(j1 - slot, 0), 16);
            const uint32_t bytes = there ? (uint32_t)(there - 1) * row_bytes + ROWB : 0u;
            const size_t at = a.cache.row(page, slot) * row_bytes;
            direct_load_16(make_uniform_rsrc(kbase + at, bytes), k_off[i], lds + i * 1024);
            direct_load_16(make_uniform_rsrc(vbase + at, bytes), v_off[i], lds + W::TILE + i * 1024);
        }
    };
    auto pages_of = [&](int t) { return pages[min(t * KB + (lane & (KB - 1)), W::PAGES - 1)]; };
    // the queries lie where tiles 2 and 3 will
    constexpr int QLD = ROWS / RPI / 8;
    {
        const __amdgpu_buffer_rsrc_t rq = make_uniform_rsrc(static_cast<const char*>(a.q) + ((size_t)(r0 + div_by(R0, a.G, a.per_G)) * a.q_stride + (size_t)kvh * a.G * DH) * sizeof(T), ~0u);
#pragma unroll
        for (int i = 0; i < QLD; ++i) {
            const int x = (wave * QLD + i) * RPI + ld_row, X = min(R0 + x, R - 1), Xi = div_by(X, a.G, a.per_G);
            direct_load_16(rq, (uint32_t)((Xi - div_by(R0, a.G, a.per_G)) * (int)a.q_stride + (X - Xi * a.G) * DH) * sizeof(T) + ((ld_pos ^ C::k_turn(x & 15)) << 4),
                           ring0 + 2 * W::STAGE + (wave * QLD + i) * 1024);
        }
    }
    __syncthreads();
    if (ntile > 0) issue(0, pages_of(0));
    if (ntile > 1) issue(1, pages_of(1));
    if (ntile > 1) wait_loads_and_barrier<2 * 2 * LD>();       // the queries are there
    else if (ntile > 0) wait_loads_and_barrier<2 * LD>();
    else wait_loads_and_barrier<0>();
    uint4 qf[QB][KS];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
        for (int kk = 0; kk < KS; ++kk)
            qf[qb][kk] = *reinterpret_cast<const uint4*>(ring + 2 * W::STAGE + ((rg * QB + qb) * 16 + r) * ROWB + (((kk * 4 + g) ^ C::k_turn(r)) << 4));

    int k_addr[KS], v_addr[DB];
    const int half = kg * KW * 16 * ROWB;              // this wave's keys of a tile
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) k_addr[kk] = half + r * ROWB + (((kk * 4 + g) ^ C::k_turn(r)) << 4);
#pragma unroll
    for (int t = 0; t < DB; ++t) {
        if constexpr (sizeof(T) == 2) {
            const int vr = 4 * g + (r >> 2), chunk = t * 2 + ((r & 3) >> 1);
            v_addr[t] = W::TILE + half + vr * ROWB + ((chunk ^ C::v_turn(vr)) << 4) + (r & 1) * 8;
        } else {
            v_addr[t] = W::TILE + half + 4 * g * ROWB + (((t * 4 + (r >> 2)) ^ C::v_turn(4 * g)) << 4) + (r & 3) * 4;
        }
    }
    f32x4 o[QB][DB];
    float m[QB], l[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        m[qb] = -INFINITY; l[qb] = 0.f;
#pragma unroll
        for (int t = 0; t < DB; ++t) o[qb][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    f32x4 st[QB][KW];
    uint4 kf[KW][KS];
    constexpr int VN = sizeof(T) == 2 ? KW / 2 : KW;
    f32x4 vf[VN][DB];                                  // bf16: the 8 keys of a lane; float32: its 4
    auto read_k = [&](int t) {
        const char* w = ring + (t & (W::STAGES - 1)) * W::STAGE;
#pragma unroll
        for (int kb = 0; kb < KW; ++kb)
#pragma unroll
            for (int kk = 0; kk < KS; ++kk) kf[kb][kk] = *reinterpret_cast<const uint4*>(w + k_addr[kk] + kb * 16 * ROWB);
        __builtin_amdgcn_sched_barrier(0);
    };
    auto read_v = [&](int t) {
        const char* w = ring + (t & (W::STAGES - 1)) * W::STAGE;
#pragma unroll
        for (int i = 0; i < VN; ++i)
#pragma unroll
            for (int t2 = 0; t2 < DB; ++t2) {
                if constexpr (sizeof(T) == 2) {
                    typedef __attribute__((address_space(3))) ac_short4* tr_ptr;
                    const char* p = w + v_addr[t2] + i * 32 * ROWB;
                    const ac_short4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)p), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)(p + 16 * ROWB));
                    vf[i][t2] = __builtin_bit_cast(f32x4, ac_short8(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7)));
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) vf[i][t2][e] = *reinterpret_cast<const float*>(w + v_addr[t2] + (i * 16 + e) * ROWB);
                }
            }
        __builtin_amdgcn_sched_barrier(0);
    };
    const int clean_from = limit0 < j1 ? limit0 : INT_MAX;
    bool cleaned = false;
    auto clean_v = [&](int t) {                        // (see above; in registers: the tile is other rows' too)
        const int seen = clean_from - (j0 + t * KEYS + kg * KW * 16);
        if (seen >= KW * 16) return;
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < VN; ++i)
#pragma unroll
            for (int t2 = 0; t2 < DB; ++t2)
#pragma unroll
                for (int e = 0; e < 4; ++e) most = ac_magnitudes<T>(most, __float_as_uint(vf[i][t2][e]));
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(ac_not_finite<T>(most)) == 0, 1)) return;
#pragma unroll
        for (int i = 0; i < VN; ++i)
#pragma unroll
            for (int t2 = 0; t2 < DB; ++t2)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    uint32_t x = __float_as_uint(vf[i][t2][e]);
                    const int at = sizeof(T) == 2 ? i * 32 + (e >> 1) * 16 + 4 * g + (e & 1) * 2 : i * 16 + 4 * g + e;
                    cleaned |= ac_clean<T>(x, at, at + 1, seen);
                    vf[i][t2][e] = __uint_as_float(x);
                }
    };
    auto scores = [&]() {                              // S = K Q^T
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int kb = 0; kb < KW; ++kb)
#pragma unroll
                for (int qb = 0; qb < QB; ++qb) st[qb][kb] = ac_logits_f32(kf[kb], qf[qb]);
        } else {
#pragma unroll
            for (int kb = 0; kb < KW; ++kb)
#pragma unroll
                for (int qb = 0; qb < QB; ++qb) st[qb][kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kk = 0; kk < KS; ++kk)
#pragma unroll
                for (int kb = 0; kb < KW; ++kb)
#pragma unroll
                    for (int qb = 0; qb < QB; ++qb) st[qb][kb] = ac_mma(kf[kb][kk], qf[qb][kk], st[qb][kb]);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto softmax = [&](int t) {
        const int key0 = j0 + t * KEYS + kg * KW * 16;
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) ac_softmax<KW, DB>(st[qb], o[qb], m[qb], l[qb], a.scale2, key0 + KW * 16 > limit0, limit[qb] - key0 - 4 * g);
        __builtin_amdgcn_sched_barrier(0);
    };
    // O += V P.  bf16: probabilities are rounded, relative to the running maximum, as their rows share the matrix instructions' time: in two parts, as above, 2048 rows over 2048 slots would take 116 us
    // instead of 92, 32 rows each of 4 samples of 1951 .. 3773 slots 28.0 instead of 25.2.
    auto values = [&]() {
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int kp = 0; kp < VN; ++kp) {
                bf16x8 pf[QB];
#pragma unroll
                for (int qb = 0; qb < QB; ++qb)
#pragma unroll
                    for (int e = 0; e < 4; ++e) { pf[qb][e] = (__bf16)st[qb][2 * kp][e]; pf[qb][4 + e] = (__bf16)st[qb][2 * kp + 1][e]; }
#pragma unroll
                for (int t2 = 0; t2 < DB; ++t2)
#pragma unroll
                    for (int qb = 0; qb < QB; ++qb) o[qb][t2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf[kp][t2]), pf[qb], o[qb][t2], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int kb = 0; kb < VN; ++kb)
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int t2 = 0; t2 < DB; ++t2)
#pragma unroll
                        for (int qb = 0; qb < QB; ++qb) o[qb][t2] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[kb][t2][e], st[qb][kb][e], o[qb][t2], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // Waves of half 1 are half a tile behind: they meet the others for the next tile between their two products, so that a SIMD's two waves want its vector
    // and matrix units in turn.  (The tile before is then still read: two are on their way.)  Every wave comes to every barrier.
    uint32_t ids = pages_of(2);
    auto meet = [&](int t) {                           // tile t is there, tile t - 2 is done with
        if (t + 1 < ntile) wait_loads_and_barrier<2 * LD>();
        else wait_loads_and_barrier<0>();
        if (t + 2 < ntile) issue(t + 2, ids);
        ids = pages_of(t + 3);
    };
    if (ntile > 0) meet(0);
    for (int t = 0; t < ntile; ++t) {
        if (kg == 0 && t > 0) meet(t);
        if (works) {
            read_k(t);
            scores();
        }
        if (kg == 1 && t + 1 < ntile) meet(t + 1);
        if (works) {
            read_v(t);
            softmax(t);
            if (UNEVEN) clean_v(t);
            values();
        }
    }
    if (UNEVEN && __builtin_amdgcn_ballot_w64(cleaned) != 0)
        ac_add_not_finite<T, DH>(a, b, kvh, max(limit0, j0), j1, [&](int j) { return (((j - j0) % KEYS) / (KW * 16)) == kg; }, o, limit);
    wait_loads_and_barrier<0>();                       // nothing is on its way into LDS any more, and nobody reads the ring
    // wave kg keeps the channels of half kg and gives the others away
    f32x4* swap = reinterpret_cast<f32x4*>(ring);
    constexpr int HD = DB / 2;
    if (works) {
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            l[qb] = quad_sum(l[qb]);
            if (g == 0) { other_m[kg][rg][qb * 16 + r] = m[qb]; other_l[kg][rg][qb * 16 + r] = l[qb]; }
#pragma unroll
            for (int t = 0; t < HD; ++t) swap[(((rg * QB + qb) * 2 + kg) * HD + t) * 64 + lane] = kg ? o[qb][t] : o[qb][HD + t];
        }
    }
    __syncthreads();
    if (!works) return;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        if (W0 + qb * 16 + r >= R) continue;
        const float m2 = other_m[kg ^ 1][rg][qb * 16 + r], l2 = other_l[kg ^ 1][rg][qb * 16 + r];
        const float mt = fmaxf(m[qb], m2);
        const float f1 = m[qb] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[qb] - mt), f2 = m2 == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m2 - mt);
        // (in the same order in both waves)
        const float z = kg ? __builtin_fmaf(l2, f2, l[qb] * f1) : __builtin_fmaf(l[qb], f1, l2 * f2);
        const size_t at = (row[qb] * a.H + xh[qb]) * a.S + s;
        const float inv = a.S > 1 ? 1.f : row_factor(z);
#pragma unroll
        for (int t = 0; t < HD; ++t) {
            const f32x4 x = kg ? o[qb][HD + t] : o[qb][t], y = swap[(((rg * QB + qb) * 2 + (kg ^ 1)) * HD + t) * 64 + lane];
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = __builtin_fmaf(x[e], f1, y[e] * f2) * inv;
            const size_t to = at * DH + (kg * HD + t) * 16 + 4 * g;
            if (a.S > 1) *reinterpret_cast<f32x4*>(a.part_o + to) = f32x4{v[0], v[1], v[2], v[3]};
            else if constexpr (sizeof(T) == 2) store_bf16<4>(static_cast<T*>(a.o) + to, v);
            else *reinterpret_cast<f32x4*>(static_cast<T*>(a.o) + to) = f32x4{v[0], v[1], v[2], v[3]};
        }
        if (g == 0 && kg == 0) {
            if (a.S > 1) { a.part_ml[at * 2] = mt; a.part_ml[at * 2 + 1] = z; }
            else store_lse(a, at, mt, z);
        }
    }
#endif
}

// The runs of the rows joined: dh / 4 threads to a row and head, and `groups` such groups of threads that have every groups-th run, JW_UNROLL of them requested
// together, so that few runs are one trip to memory; the groups meet in LDS.
constexpr int JW_UNROLL = 4;
__device__ __forceinline__ int runs_of(const AttendCacheArgs& a, int limit) { return max(1, (limit + a.run - 1) / a.run); }

// (a group of threads may be a single one: float32 heads of 4 channels)
template <int NT> struct JoinLds { f32x4 t[NT]; float m[NT], z[NT]; };
template <typename T, int NT>
__device__ __forceinline__ void join_rows(const AttendCacheArgs& a, int b, int block, int groups, JoinLds<NT>& lds) {
    const int tid = threadIdx.x, dh = a.cache.dh;
    int r0;
    const int nq = sample_rows(a, b, r0);
    const int n = a.cache.length(b, a.max_len);
    const int tpr = dh >> 2, per = NT / tpr / groups, y = tid / tpr, c = tid - y * tpr;
    const int which = y / groups, g = y - which * groups, item = block * per + which;
    const bool there = which < per && item < nq * a.H;
    const size_t at = (size_t)r0 * a.H + item;
    float m = -INFINITY, z = 0.f;
    f32x4 t = {0.f, 0.f, 0.f, 0.f};
    if (there) {
        const int S = runs_of(a, row_limit(a, n, nq, item / a.H));
        const float2* ml = reinterpret_cast<const float2*>(a.part_ml) + at * a.S;
        const f32x4* part = reinterpret_cast<const f32x4*>(a.part_o + at * a.S * dh) + c;
        for (int s = g; s < S; s += groups * JW_UNROLL) {
            float2 v[JW_UNROLL];
            f32x4 p[JW_UNROLL];
#pragma unroll
            for (int u = 0; u < JW_UNROLL; ++u) {
                const int su = min(s + u * groups, S - 1);
                v[u] = ml[su];
                p[u] = part[(size_t)su * tpr];
            }
            float mn = m;
#pragma unroll
            for (int u = 0; u < JW_UNROLL; ++u) mn = fmaxf(mn, v[u].x);             // (a run that comes twice does not change it)
            const float ref = mn == -INFINITY ? 0.f : mn, f0 = exp2f(m - ref);
            m = mn;
            z *= f0;
#pragma unroll
            for (int e = 0; e < 4; ++e) t[e] *= f0;
#pragma unroll
            for (int u = 0; u < JW_UNROLL; ++u) {
                const float f = s + u * groups < S ? exp2f(v[u].x - ref) : 0.f;
                z = __builtin_fmaf(v[u].y, f, z);
#pragma unroll
                for (int e = 0; e < 4; ++e) t[e] = __builtin_fmaf(p[u][e], f, t[e]);
            }
        }
    }
    if (groups > 1) {
        lds.t[tid] = t;
        if (c == 0) { lds.m[y] = m; lds.z[y] = z; }
        __syncthreads();
        if (there && g == 0) {
            float mt = m;
            for (int i = 1; i < groups; ++i) mt = fmaxf(mt, lds.m[y + i]);
            const float ref = mt == -INFINITY ? 0.f : mt, f0 = exp2f(m - ref);
            z *= f0;
#pragma unroll
            for (int e = 0; e < 4; ++e) t[e] *= f0;
            for (int i = 1; i < groups; ++i) {
                const float f = exp2f(lds.m[y + i] - ref);
                const f32x4 p = lds.t[tid + i * tpr];
                z = __builtin_fmaf(lds.z[y + i], f, z);
#pragma unroll
                for (int e = 0; e < 4; ++e) t[e] = __builtin_fmaf(p[e], f, t[e]);
            }
            m = mt;
        }
    }
    if (!there || g != 0) return;
    const float inv = row_factor(z);
    T* o = static_cast<T*>(a.o) + at * dh + c * 4;
    const float w[4] = {t[0] * inv, t[1] * inv, t[2] * inv, t[3] * inv};
    if constexpr (sizeof(T) == 2) store_bf16<4>(o, w);
    else *reinterpret_cast<f32x4*>(o) = f32x4{w[0], w[1], w[2], w[3]};
    if (c == 0) store_lse(a, at, m, z);
}

// log-sum-exp (weights_lse2) of `cnt` rows and heads from item c0 on, into LDS: from their runs, by TPI threads to a row and head, or as it stands in a.lse2
template <int NT, int TPI>
__device__ __forceinline__ void runs_lse2(const AttendCacheArgs& a, int r0, int nq, int n, int c0, int cnt, float* lse2) {
    constexpr int AT_ONCE = 8;                         // runs requested together
    const int sub = threadIdx.x % TPI;
    for (int u0 = 0; u0 < cnt; u0 += NT / TPI) {       // (all lanes together: they exchange what they have)
        const int u = u0 + threadIdx.x / TPI, uc = min(u, cnt - 1), S = runs_of(a, row_limit(a, n, nq, (c0 + uc) / a.H));
        const float2* ml = reinterpret_cast<const float2*>(a.part_ml) + ((size_t)r0 * a.H + c0 + uc) * a.S;
        float m = -INFINITY, z = 0.f;
        for (int s = sub; s < S; s += TPI * AT_ONCE) {
            float2 v[AT_ONCE];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) v[i] = ml[min(s + i * TPI, S - 1)];
            float mn = m;
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) mn = fmaxf(mn, v[i].x);
            const float ref = mn == -INFINITY ? 0.f : mn;
            z *= __builtin_amdgcn_exp2f(m - ref);
            m = mn;
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) z += s + i * TPI < S ? v[i].y * __builtin_amdgcn_exp2f(v[i].x - ref) : 0.f;
        }
#pragma unroll
        for (int o = 1; o < TPI; o <<= 1) {             // (a sum of NaN beside a maximum of -infinity stays NaN)
            const float m2 = __shfl_xor(m, o), z2 = __shfl_xor(z, o), mn = fmaxf(m, m2), ref = mn == -INFINITY ? 0.f : mn;
            z = z * __builtin_amdgcn_exp2f(m - ref) + z2 * __builtin_amdgcn_exp2f(m2 - ref);
            m = mn;
        }
        if (sub == 0 && u < cnt) lse2[u] = weights_lse2(m, z);
    }
}
template <int NT>
__device__ __forceinline__ void rows_lse2(const AttendCacheArgs& a, int r0, int nq, int n, int c0, int cnt, float* lse2) {
    if (a.S == 1) {
        for (int u = threadIdx.x; u < cnt; u += NT) lse2[u] = a.lse2[(size_t)r0 * a.H + c0 + u];
    } else if (cnt * 8 <= NT) {
        runs_lse2<NT, 8>(a, r0, nq, n, c0, cnt, lse2);
    } else {
        runs_lse2<NT, 1>(a, r0, nq, n, c0, cnt, lse2);
    }
}

// What the slots got where the logits are not kept: they are formed again, K Q^T once more (the keys' rows a third time through memory is less than
// 4 bytes a logit there and back).  A workgroup has a tile of a sample's slots and goes over all heads and rows, wave w over key heads w, w + 8, ...
// (or parts of a head's rows where there are fewer), each wave on its own.  The keys of a head come through LDS into its registers, then the queries, 16 rows at a time with
// their lse, through a ring in the same place.  (Loaded as fragments, 64 bytes of a row at a time, the keys took 6700 clocks and every block of queries 2000.)
// In the end bound by vector instructions: an fma, an exp2 and an addition a logit.  Four samples of 1951 .. 3773 slots and 32 rows, 32 heads over 8 of 128: 15.9 us; of a
// workgroup's 32000 clocks the keys' way into LDS takes 9500 (23 MB), the first queries 3000, the blocks of rows 13000; the first wave
// then waits up to 6000 for the others and the sums.  (The rows' lse come from the joining launch in front: formed by every
// workgroup for itself in one launch with the joining, four samples of 128 rows to a key head took 27 us instead of 21.)
constexpr int CW_WAVES = 8;
template <typename T, int DH> struct CwTile {
    using C = AcTile<T, DH>;
    static constexpr int KB = C::KS > 4 ? 2 : 4, KEYS = KB * 16;                            // of a wave's registers
    static constexpr int QROWS = 16 * C::ROWB, SLOT = QROWS + 256, SLOTS = C::KS > 4 ? 2 : 4;       // queries of a block, and 64 words of lse
    static constexpr int WAVE_LDS = SLOTS * SLOT > KEYS * C::ROWB ? SLOTS * SLOT : KEYS * C::ROWB, LDS = CW_WAVES * WAVE_LDS;
};
template <typename T, int DH>
__global__ __launch_bounds__(CW_WAVES * 64, 2) void cache_weigh_kernel(AttendCacheArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    using C = AcTile<T, DH>;
    using W = CwTile<T, DH>;
    constexpr int KS = C::KS, KB = W::KB, KEYS = W::KEYS, ROWB = C::ROWB, NCHK = C::NCHK, RPI = C::RPI, LDB = C::LDB, SLOTS = W::SLOTS;
    extern __shared__ __attribute__((aligned(16))) char ring[];
    __shared__ float sums[CW_WAVES][KEYS];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
    const int b = blockIdx.y, key0 = blockIdx.x * KEYS;
    int page[KB];                                       // of the tile's blocks, requested with the sample's sizes
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) page[kb] = a.cache.page_of(b, min(key0 + kb * 16, a.last_slot));
    const int n = a.cache.length(b, a.max_len);
    if (key0 >= n) return;
    int r0;
    const int nq = sample_rows(a, b, r0), R = nq * a.G;
    const int jt = key0 + tid;
    const size_t to = (size_t)b * a.weight_stride + jt;
    const float before = tid < KEYS && jt < n && a.weight_in ? a.weight_in[to] : 0.f;
    const uint32_t row_bytes = (uint32_t)a.cache.row_elems() * sizeof(T);
    const int ld_pos = lane % NCHK, ld_row = lane / NCHK;
    const uint32_t mine = (uint32_t)(size_t)(lds_ptr_t)ring + wave * W::WAVE_LDS;
    const char* at = ring + wave * W::WAVE_LDS;
    int k_off[LDB], q_addr[KS];
#pragma unroll
    for (int i = 0; i < LDB; ++i) {
        const int x = i * RPI + ld_row;
        k_off[i] = x * row_bytes + ((ld_pos ^ C::k_turn(x)) << 4);
    }
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) q_addr[kk] = r * ROWB + (((kk * 4 + g) ^ C::k_turn(r)) << 4);
    f32x4 acc[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) acc[kb] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int parts = a.cache.Hkv >= CW_WAVES ? 1 : (CW_WAVES + a.cache.Hkv - 1) / a.cache.Hkv, step = parts * 16;
    const int step_i = step / a.G, step_x = step - step_i * a.G;                            // rows and heads from one block to the next
    for (int it = wave; it < a.cache.Hkv * parts; it += CW_WAVES) {
        const int kvh = it / parts, first = (it - kvh * parts) * 16;
        if (first >= R) continue;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            const int slot = key0 + kb * 16, there = min(max(n - slot, 0), 16);
            const uint32_t p = a.cache.readable(__builtin_amdgcn_readfirstlane(page[kb]));
            const __amdgpu_buffer_rsrc_t rk = make_uniform_rsrc(static_cast<const char*>(a.k_pages) + a.cache.row(p, slot) * row_bytes + (size_t)kvh * ROWB,
                                                                there ? (uint32_t)(there - 1) * row_bytes + ROWB : 0u);
#pragma unroll
            for (int i = 0; i < LDB; ++i) direct_load_16(rk, k_off[i], mine + (kb * LDB + i) * 1024);
        }
        wait_loads<0>();
        uint4 kf[KB][KS];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int kk = 0; kk < KS; ++kk) kf[kb][kk] = *reinterpret_cast<const uint4*>(at + kb * 16 * ROWB + q_addr[kk]);
        wait_lds();
        // The block that is requested next: its first row, and (row, head) of this lane's rows in the loads and of its column, all moving on together.
        int x0 = first, i0 = div_by(first, a.G, a.per_G), li[LDB], lx[LDB], ci, cx;
#pragma unroll
        for (int i = 0; i < LDB; ++i) {
            const int x = first + i * RPI + ld_row;
            li[i] = div_by(x, a.G, a.per_G);
            lx[i] = x - li[i] * a.G;
        }
        ci = div_by(first + r, a.G, a.per_G);
        cx = first + r - ci * a.G;
        int rest = first - i0 * a.G;
        int seen_i = ci;                                // row of this lane's column in the block that is used next
        auto request = [&](int s) {
            const size_t row = (size_t)(r0 + i0);
            const uint32_t all = x0 < R ? ~0u : 0u;     // (a block that there is not: no memory is touched, the loads are counted)
            const __amdgpu_buffer_rsrc_t rq = make_uniform_rsrc(static_cast<const char*>(a.q) + (row * a.q_stride + (size_t)kvh * a.G * DH) * sizeof(T), all);
            const __amdgpu_buffer_rsrc_t rl = make_uniform_rsrc(a.lse2 + row * a.H + (size_t)kvh * a.G, all);
#pragma unroll
            for (int i = 0; i < LDB; ++i) {
                const uint32_t off = (uint32_t)((min(li[i], nq - 1) - i0) * (int)a.q_stride + lx[i] * DH) * sizeof(T);
                const int x = i * RPI + ld_row;
                direct_load_16(rq, off + ((ld_pos ^ C::k_turn(x)) << 4), mine + s * W::SLOT + i * 1024);
                li[i] += step_i; lx[i] += step_x;
                if (lx[i] >= a.G) { lx[i] -= a.G; ++li[i]; }
            }
            direct_load_4(rl, (uint32_t)((min(ci, nq - 1) - i0) * a.H + cx) * 4u, mine + s * W::SLOT + W::QROWS);
            ci += step_i; cx += step_x;
            if (cx >= a.G) { cx -= a.G; ++ci; }
            x0 += step; i0 += step_i; rest += step_x;
            if (rest >= a.G) { rest -= a.G; ++i0; }
        };
        int seen_x = cx;
#pragma unroll
        for (int s = 0; s < SLOTS - 1; ++s) request(s);
        int s = 0;
        for (int x = first; x < R; x += step) {
            wait_loads<(SLOTS - 2) * (LDB + 1)>();      // this block is there
            request(s == 0 ? SLOTS - 1 : s - 1);
            const char* w = at + s * W::SLOT;
            uint4 qf[KS];
#pragma unroll
            for (int kk = 0; kk < KS; ++kk) qf[kk] = *reinterpret_cast<const uint4*>(w + q_addr[kk]);
            const float ref = *reinterpret_cast<const float*>(w + W::QROWS + lane * 4);
            const int limit = seen_i < nq ? row_limit(a, n, nq, seen_i) : 0, seen = limit - key0 - 4 * g;
            seen_i += step_i; seen_x += step_x;
            if (seen_x >= a.G) { seen_x -= a.G; ++seen_i; }
            const bool masked = __builtin_amdgcn_ballot_w64(limit < key0 + KEYS) != 0;
            f32x4 st[KB];
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) st[kb] = ac_logits_f32(kf[kb], qf);
            } else {
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) st[kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < KS; ++kk)
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb) st[kb] = ac_mma(kf[kb][kk], qf[kk], st[kb]);
            }
            if (masked) {
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(st[kb][e], a.scale2, -ref));
                        acc[kb][e] += kb * 16 + e < seen ? p : 0.f;
                    }
            } else {
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[kb][e] += __builtin_amdgcn_exp2f(__builtin_fmaf(st[kb][e], a.scale2, -ref));
            }
            wait_lds();
            s = s + 1 == SLOTS ? 0 : s + 1;
        }
        wait_loads<0>();                                // nothing is on its way where the next head's keys will lie
    }
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float v = row16_sum(acc[kb][e]);
            if (r == 0) sums[wave][kb * 16 + 4 * g + e] = v;
        }
    __syncthreads();
    if (tid < KEYS && jt < n) {
        float total = 0.f;
#pragma unroll
        for (int w = 0; w < CW_WAVES; ++w) total += sums[w][tid];
        a.weight_out[to] = before + total / (float)a.H;
    }
#endif
}

// Joins, and what the slots got where the logits were kept: p = 2^(logit - lse), with the rows' lse formed from the runs' sums by every workgroup for itself (a launch
// of its own for that would cost more).
constexpr int JW_ROWS = 1024;                  // rows and heads whose lse a workgroup holds at a time
constexpr int JW_BATCH = 8;                    // rows of logits requested at once
template <typename T>
__global__ __launch_bounds__(256) void attend_cache_join_kernel(AttendCacheArgs a, int join_wgs, int groups) {
    __shared__ float lse2[JW_ROWS];
    __shared__ __attribute__((aligned(16))) JoinLds<256> lds;
    const int tid = threadIdx.x, b = blockIdx.y;
    if ((int)blockIdx.x < join_wgs) {
        join_rows<T, 256>(a, b, blockIdx.x, groups, lds);
        return;
    }
    int r0;
    const int nq = sample_rows(a, b, r0);
    const int n = a.cache.length(b, a.max_len);
    // 64 slots to a workgroup, every wave has a quarter of the rows, JW_BATCH of them requested together, the first ones in front of the rows' lse
    const int slot0 = ((int)blockIdx.x - join_wgs) * 64, j = slot0 + (tid & 63), wave = tid >> 6;
    if (slot0 >= n) return;
    const int items = nq * a.H;
    const size_t to = (size_t)b * a.weight_stride + j;
    const float before = a.weight_in && wave == 0 && j < n ? a.weight_in[to] : 0.f;
    float total = 0.f;
    for (int c0 = 0; c0 < items; c0 += JW_ROWS) {
        const int cnt = min(items - c0, JW_ROWS);
        const float* x = a.logits + ((size_t)r0 * a.H + c0) * a.lpad + min(j, n - 1);
        float v[JW_BATCH];
        auto request = [&](int u0) {
#pragma unroll
            for (int i = 0; i < JW_BATCH; ++i) v[i] = x[(size_t)min(u0 + wave + 4 * i, cnt - 1) * a.lpad];
        };
        request(0);
        __syncthreads();
        rows_lse2<256>(a, r0, nq, n, c0, cnt, lse2);
        __syncthreads();
        for (int u0 = 0; u0 < cnt; u0 += 4 * JW_BATCH) {
            if (u0 > 0) request(u0);
#pragma unroll
            for (int i = 0; i < JW_BATCH; ++i) {
                const int u = u0 + wave + 4 * i;
                const bool seen = u < cnt && j < row_limit(a, n, nq, (c0 + u) / a.H);
                total += seen ? exp2f(v[i] - lse2[min(u, cnt - 1)]) : 0.f;
            }
        }
    }
    lds.t[tid][0] = total;
    __syncthreads();
    if (wave == 0 && j < n) a.weight_out[to] = before + ((lds.t[tid][0] + lds.t[tid + 64][0]) + (lds.t[tid + 128][0] + lds.t[tid + 192][0])) / (float)a.H;
}

// What the slots got: a workgroup has 64 slots of a sample, 16 lanes a slot, and goes over all heads and rows.
template <typename T>
__global__ __launch_bounds__(256) void cache_weigh_generic_kernel(AttendCacheArgs a) {
    constexpr int EPC = 16 / sizeof(T);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & 15, g = lane >> 4;
    const int b = blockIdx.y, dh = a.cache.dh, nch = dh / EPC;
    const int n = a.cache.length(b, a.max_len);
    int r0;
    const int nq = sample_rows(a, b, r0);
    if ((int)blockIdx.x * 64 >= n) return;
    const size_t rs = a.cache.row_elems();
    for (int u = 0; u < 4; ++u) {
        const int j = blockIdx.x * 64 + wave * 16 + u * 4 + g, jc = min(j, n - 1);
        const T* kp = static_cast<const T*>(a.k_pages) + a.cache.row(a.cache.readable(a.cache.page_of(b, jc)), jc) * rs;
        float total = 0.f;
        for (int hk = 0; hk < a.cache.Hkv; ++hk) {
            uint4 kr[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) kr[t] = reinterpret_cast<const uint4*>(kp + (size_t)hk * dh)[min(l + 16 * t, nch - 1)];
            for (int i = 0; i < nq; ++i) {
                const int limit = row_limit(a, n, nq, i);
                for (int x = 0; x < a.G; ++x) {
                    const int h = hk * a.G + x;
                    const uint4* q = reinterpret_cast<const uint4*>(static_cast<const T*>(a.q) + (size_t)(r0 + i) * a.q_stride + (size_t)h * dh);
                    float d = 0.f;
#pragma unroll
                    for (int t = 0; t < 4; ++t)
                        if (l + 16 * t < nch) d = chunk_dot<T>(q[l + 16 * t], kr[t], d);
                    d = row16_sum(d) * a.scale2 - a.lse2[(size_t)(r0 + i) * a.H + h];
                    if (j < limit) total += exp2f(d);
                }
            }
        }
        if (l == 0 && j < n && j < a.weight_stride) {
            const size_t at = (size_t)b * a.weight_stride + j;
            a.weight_out[at] = (a.weight_in ? a.weight_in[at] : 0.f) + total / (float)a.H;
        }
    }
}

// How a call goes: a rule on host-known sizes only.
//   heads of 64 and 128   up to 16 rows to a key head: waves on their own; more: 64 or 128 rows that share tiles.  A run for every compute unit: more runs cost a round of
//                         workgroups each (32 samples of 2048 slots, 8 key heads of 128 in one, two, four rounds 49, 54, 57 us), fewer leave units idle (8 samples 17.3
//                         and 16.2 us with 128 and 256).  One run, without the joining, where a head's K is short, at most 128 KB (bf16) or 96 KB: one sample,
//                         8 heads of 128, 512 and 768 slots 7.3 and 9.1 us in one run, 8.1 and 7.9 in several; heads of 64, 1024 and 1280 slots 7.7 and 8.8, 8.2 and 8.2; float32 heads
//                         of 128, 192 slots 8.7, 9.9; of 64, 384 and 512 slots 8.2 and 9.8, 8.0 and 8.1.  (4 samples: the same.)
//   others                a workgroup per row, head and run
enum { AC_GENERIC = 0, AC_WAVES, AC_ROWS64, AC_ROWS128 };
struct AttendCachePlan {
    int kernel;
    bool keep;                                  // logits are kept for the weights
    int S, run, tiles, lpad;
    size_t lse2, part_o, part_ml, logits, bytes;        // places in the workspace
};
constexpr int AC_MAX_RUN = 4096;                // the pages of a run: in a wave's 64 lanes for each quarter, or 256 words of LDS
static AttendCachePlan attend_cache_plan(const d3tom_paged_cache& c, int rows, int max_q, int max_len, int H, int weighed) {
    AttendCachePlan p;
    const long long R = (long long)max_q * (H / c.Hkv);
    p.kernel = c.dh != 64 && c.dh != 128 ? AC_GENERIC : R <= 16 ? AC_WAVES : R <= 64 || (c.dt == D3TOM_F32 && c.dh == 128) ? AC_ROWS64 : AC_ROWS128;
    const int tile_rows[] = {1, 16, 64, 128}, want[] = {1024, 256, 256, 256};
    p.tiles = (int)((R + tile_rows[p.kernel] - 1) / tile_rows[p.kernel]);
    const long long groups = (long long)c.B * (p.kernel == AC_GENERIC ? (long long)max_q * H : (long long)c.Hkv * p.tiles), step = p.kernel == AC_GENERIC ? 256 : 128;
    long long S = groups >= want[p.kernel] ? 1 : want[p.kernel] / groups;
    const long long most = (max_len + step - 1) / step;
    S = S > most ? most : S;
    if (p.kernel == AC_WAVES && (size_t)max_len * c.dh * elem_bytes(c.dt) <= (c.dt == D3TOM_BF16 ? 128u : 96u) * 1024) S = 1;
    p.run = (int)((most + S - 1) / S * step);
    if (p.kernel != AC_GENERIC && p.run > AC_MAX_RUN) p.run = AC_MAX_RUN;
    p.S = (max_len + p.run - 1) / p.run;
    p.keep = weighed && p.kernel == AC_WAVES;
    p.lpad = (max_len + 15) / 16 * 16;
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o += align_up(bytes, 256); return at; };
    const size_t rh = (size_t)rows * H;
    p.lse2 = take(weighed ? rh * 4 : 0);
    p.part_o = take(p.S > 1 ? rh * p.S * c.dh * 4 : 0);
    p.part_ml = take(p.S > 1 ? rh * p.S * 8 : 0);
    p.logits = take(p.keep ? rh * p.lpad * 4 : 0);
    p.bytes = o;
    return p;
}
// What a workspace needs that is to serve every call of at most these sizes (fewer rows may mean more runs, or logits that are kept): a plan has at most want * tile rows
// times runs where the units ask for runs, and a run for every AC_MAX_RUN slots otherwise.
static size_t attend_cache_ws_bytes(const d3tom_paged_cache& c, int rows, int max_q, int max_len, int H, int weighed) {
    const size_t rh = (size_t)rows * H, most = rh * ((max_len + 127) / 128), some = 128 * 512 + rh * ((max_len + AC_MAX_RUN - 1) / AC_MAX_RUN);
    const size_t parts = most < some ? most : some, kept = rh < (size_t)c.B * c.Hkv * 16 ? rh : (size_t)c.B * c.Hkv * 16;
    size_t bytes = 4 * 256 + parts * (c.dh * 4 + 8);
    if (weighed) bytes += rh * 4 + kept * ((max_len + 15) / 16 * 16) * 4;
    const size_t plan = attend_cache_plan(c, rows, max_q, max_len, H, weighed).bytes;          // more only for more rows than B * max_q
    return bytes > plan ? bytes : plan;
}
// What the launches of a plan hold: workgroups of the attention (512 threads where rows share tiles), and the rows and heads that the joining goes over, which also bound a row's number.
static bool attend_cache_fits(const d3tom_paged_cache& c, const AttendCachePlan& p, int max_q, int H) {
    const double items = (double)c.B * max_q * H;
    const double groups = p.kernel == AC_GENERIC ? items * p.S : (double)c.B * c.Hkv * p.S * p.tiles;
    return items <= CACHE_MOST_GROUPS && groups <= (p.kernel == AC_GENERIC || p.kernel == AC_WAVES ? CACHE_MOST_GROUPS : CACHE_MOST_GROUPS / 2);
}
template <typename T, int DH, bool UNEVEN>
static int attend_cache_launch(const AttendCacheArgs& a, int kernel, hipStream_t st) {
    static PerDeviceOnce once;
    using C = AcTile<T, DH>;
    constexpr int WAVES_LDS = WAVES * C::WAVE_LDS + 16 * C::ROWB, ROWS_LDS = AcShared<T, DH>::LDS;
    constexpr int WIDE = C::KS > 4 ? 1 : 2;     // (float32 heads of 128 have no registers for 128 rows: the plan gives them 64)
    if (!once.run([] {
            return raise_dynamic_lds(attend_cache_kernel<T, DH, UNEVEN>, WAVES_LDS) && raise_dynamic_lds(attend_cache_rows_kernel<T, DH, 1, UNEVEN>, ROWS_LDS) &&
                   raise_dynamic_lds(attend_cache_rows_kernel<T, DH, WIDE, UNEVEN>, ROWS_LDS);
        })) return D3TOM_ERR_DEVICE;
    const int units = a.nB * a.cache.Hkv * a.S, wgs = (units + 7) / 8 * 8 * a.tiles;
    if (kernel == AC_WAVES) D3TOM_LAUNCH(CACHE_ATTEND, st, (attend_cache_kernel<T, DH, UNEVEN><<<units, 64 * WAVES, WAVES_LDS, st>>>(a)));
    else if (kernel == AC_ROWS64) D3TOM_LAUNCH(CACHE_ATTEND, st, (attend_cache_rows_kernel<T, DH, 1, UNEVEN><<<wgs, 512, ROWS_LDS, st>>>(a)));
    else D3TOM_LAUNCH(CACHE_ATTEND, st, (attend_cache_rows_kernel<T, DH, WIDE, UNEVEN><<<wgs, 512, ROWS_LDS, st>>>(a)));
    return D3TOM_OK;
}
// threads that share a row's runs when `threads` join rows of dh channels
static int join_groups(int S, int dh, int threads) {
    int groups = 1;
    while (groups * JW_UNROLL < S && groups * 2 <= threads / (dh / 4)) groups *= 2;
    return groups;
}
template <typename T, int DH>
static int cache_weigh_launch(const AttendCacheArgs& a, hipStream_t st) {
    static PerDeviceOnce once;
    using W = CwTile<T, DH>;
    if (!once.run([] { return raise_dynamic_lds(cache_weigh_kernel<T, DH>, W::LDS); })) return D3TOM_ERR_DEVICE;
    const dim3 grid((a.max_len + W::KEYS - 1) / W::KEYS, a.nB);
    D3TOM_LAUNCH(CACHE_WEIGH, st, (cache_weigh_kernel<T, DH><<<grid, CW_WAVES * 64, W::LDS, st>>>(a)));
    return D3TOM_OK;
}
static int attend_cache_check(const d3tom_paged_cache* c, int rows, int max_q, int max_len, int H) {
    const int rc = cache_check(c);
    if (rc != D3TOM_OK) return rc;
    if (rows < 1 || max_q < 1 || max_q > rows || max_len < 1 || H < 1 || H % c->Hkv) return D3TOM_ERR_INVALID_ARG;
    if ((int64_t)max_len > (int64_t)c->table_stride * c->page_size) return D3TOM_ERR_INVALID_ARG;
    if (max_len > D3TOM_MAX_CACHE_LEN) return D3TOM_ERR_UNSUPPORTED;                // 512 threads for every 32 slots: fewer than 2^32
    return D3TOM_OK;
}

}  // namespace d3tom

using namespace d3tom;

extern "C" size_t d3tom_attend_cache_workspace_bytes(const d3tom_paged_cache* cache, int rows, int max_q, int max_len, int H, int weighed) {
    if (attend_cache_check(cache, rows, max_q, max_len, H) != D3TOM_OK) return 0;
    return attend_cache_ws_bytes(*cache, rows, max_q, max_len, H, weighed);
}

extern "C" int d3tom_attend_cache(const void* q, int64_t q_stride, const d3tom_paged_cache* cache, const int32_t* q_off, int rows, int max_q,
                                  int max_len, int H, float scale, int causal, void* o, float* lse, const float* weight_in, float* weight_out,
                                  int weight_stride, void* ws, size_t ws_bytes, void* stream) {
    hipStream_t st = (hipStream_t)stream;
    int rc = attend_cache_check(cache, rows, max_q, max_len, H);
    if (rc != D3TOM_OK) return rc;
    const int dt = cache->dt, dh = cache->dh;
    if ((rc = rows_check(q, q_stride, H, dh, dt)) != D3TOM_OK || (rc = rows_check(o, (int64_t)H * dh, H, dh, dt)) != D3TOM_OK) return rc;
    if (q_stride * elem_bytes(dt) > (1 << 24)) return D3TOM_ERR_UNSUPPORTED;        // 128 rows apart is a 32-bit offset
    if (!q_off || !ws || !(scale > 0.f) || !(scale < 3.0e38f)) return D3TOM_ERR_INVALID_ARG;
    if ((weight_in && !weight_out) || (weight_out && weight_stride < max_len)) return D3TOM_ERR_INVALID_ARG;
    const AttendCachePlan p = attend_cache_plan(*cache, rows, max_q, max_len, H, weight_out != nullptr);
    if (!attend_cache_fits(*cache, p, max_q, H)) return D3TOM_ERR_UNSUPPORTED;
    if (ws_bytes < attend_cache_ws_bytes(*cache, rows, max_q, max_len, H, weight_out != nullptr) || (((uintptr_t)ws) & 255u)) return D3TOM_ERR_WORKSPACE_TOO_SMALL;
    AttendCacheArgs a{};
    a.cache = cache_view(*cache);
    a.q = q; a.k_pages = cache->k_pages; a.v_pages = cache->v_pages; a.q_stride = q_stride; a.q_off = q_off;
    a.nB = cache->B; a.rows = rows; a.max_q = max_q; a.max_len = max_len; a.H = H; a.G = H / cache->Hkv; a.causal = causal != 0;
    a.scale2 = scale * LOG2E;
    a.per_G = 1.0f / (float)a.G; a.per_Hkv = 1.0f / (float)cache->Hkv; a.per_heads = 1.0f / ((float)cache->Hkv * (float)cache->B);
    a.last_slot = max_len - 1;                  // (the table has all of max_len)
    a.S = p.S; a.run = p.run; a.o = o; a.lse = lse; a.lpad = p.lpad; a.tiles = p.tiles;
    a.lse2 = weight_out ? (float*)((char*)ws + p.lse2) : nullptr;
    a.part_o = (float*)((char*)ws + p.part_o); a.part_ml = (float*)((char*)ws + p.part_ml);
    a.logits = p.keep ? (float*)((char*)ws + p.logits) : nullptr;
    a.weight_in = weight_in; a.weight_out = weight_out; a.weight_stride = weight_stride;
    const bool bf16 = dt == D3TOM_BF16;
    if (p.kernel != AC_GENERIC) {
        const bool uneven = causal && max_q > 1;
        if (bf16) rc = dh == 128 ? (uneven ? attend_cache_launch<uint16_t, 128, true>(a, p.kernel, st) : attend_cache_launch<uint16_t, 128, false>(a, p.kernel, st))
                                 : (uneven ? attend_cache_launch<uint16_t, 64, true>(a, p.kernel, st) : attend_cache_launch<uint16_t, 64, false>(a, p.kernel, st));
        else rc = dh == 128 ? (uneven ? attend_cache_launch<float, 128, true>(a, p.kernel, st) : attend_cache_launch<float, 128, false>(a, p.kernel, st))
                            : (uneven ? attend_cache_launch<float, 64, true>(a, p.kernel, st) : attend_cache_launch<float, 64, false>(a, p.kernel, st));
        if (rc != D3TOM_OK) return rc;
    } else {
        const int wgs = cache->B * max_q * H * p.S;
        if (bf16) D3TOM_LAUNCH(CACHE_ATTEND, st, (attend_cache_generic_kernel<uint16_t><<<wgs, 256, 0, st>>>(a)));
        else D3TOM_LAUNCH(CACHE_ATTEND, st, (attend_cache_generic_kernel<float><<<wgs, 256, 0, st>>>(a)));
    }
    const int groups = join_groups(p.S, dh, 256);
    const int per = 256 / (dh / 4) / groups, join_wgs = p.S > 1 ? (max_q * H + per - 1) / per : 0, weigh_wgs = p.keep ? (max_len + 63) / 64 : 0;
    if (join_wgs + weigh_wgs > 0) {
        const dim3 grid(join_wgs + weigh_wgs, cache->B);
        if (bf16) D3TOM_LAUNCH(CACHE_JOIN, st, (attend_cache_join_kernel<uint16_t><<<grid, 256, 0, st>>>(a, join_wgs, groups)));
        else D3TOM_LAUNCH(CACHE_JOIN, st, (attend_cache_join_kernel<float><<<grid, 256, 0, st>>>(a, join_wgs, groups)));
    }
    if (weight_out && !p.keep && p.kernel != AC_GENERIC) {
        return bf16 ? (dh == 128 ? cache_weigh_launch<uint16_t, 128>(a, st) : cache_weigh_launch<uint16_t, 64>(a, st))
                    : (dh == 128 ? cache_weigh_launch<float, 128>(a, st) : cache_weigh_launch<float, 64>(a, st));
    } else if (weight_out && !p.keep) {
        const dim3 wgrid((max_len + 63) / 64, cache->B);
        if (bf16) D3TOM_LAUNCH(CACHE_WEIGH, st, (cache_weigh_generic_kernel<uint16_t><<<wgrid, 256, 0, st>>>(a)));
        else D3TOM_LAUNCH(CACHE_WEIGH, st, (cache_weigh_generic_kernel<float><<<wgrid, 256, 0, st>>>(a)));
    }
    return D3TOM_OK;
}
