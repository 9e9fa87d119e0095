// d3tom_attend_cache: attention of each sample's newest rows over its cache in pages.
//
// The keys of a long cache are cut into runs of equal length; each run gives, for every row and head, the maximum m of its logits, the sum
// l of their exponentials relative to it and the values O added up with them, all float32; runs are joined by
//   o = sum_s O_s 2^(m_s - m) / sum_s l_s 2^(m_s - m),  m = max_s m_s    (logits in units of log 2).
// What the slots got (weight_out) is formed from the joined sums behind that: p = 2^(logit - lse).
#include "cache.hpp"

namespace d3tom {

struct AttendCacheArgs {
    CacheView cache;
    const void *q, *k_pages, *v_pages;
    size_t q_stride;
    const int32_t* q_off;
    int rows, max_q, max_len, H, G, causal;     // G: query heads of a key head
    float scale2;                               // scale * log2(e)
    int S, run;                                 // runs of a cache, slots of a run
    void* o;
    float *lse, *lse2;                          // natural logarithm (the caller's), base 2 (for the weights)
    float *part_o, *part_ml;                    // [rows, H, S, dh], [rows, H, S, 2]
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

template <typename T>
__device__ __forceinline__ void store_out(T* p, const float* v, int n) {
    for (int e = 0; e < n; ++e) Elem<T>::store(p + e, v[e]);
}

// Any head size.  One workgroup per row, head and run: 256 slots at a time, 16 lanes to a key; for the output a thread takes one 16-byte chunk
// of the channels and every (256 / chunks)-th slot.
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
        else Elem<T>::store(static_cast<T*>(a.o) + at * dh + tid, z > 0.f ? t / z : 0.f);
    }
    if (tid == 0) {
        if (a.S > 1) { a.part_ml[at * 2] = m; a.part_ml[at * 2 + 1] = z; }
        else {
            const float l2 = z > 0.f ? m + log2f(z) : -INFINITY;
            if (a.lse) a.lse[at] = l2 * 0.6931471805599453f;
            if (a.lse2) a.lse2[at] = l2;
        }
    }
}

// the runs of a row and head joined: one workgroup for each
template <typename T>
__global__ __launch_bounds__(256) void attend_cache_join_kernel(AttendCacheArgs a) {
    const int tid = threadIdx.x, dh = a.cache.dh;
    const size_t at = blockIdx.x;
    const float* ml = a.part_ml + at * a.S * 2;
    float m = -INFINITY;
    for (int s = 0; s < a.S; ++s) m = fmaxf(m, ml[2 * s]);
    float z = 0.f, t = 0.f;
    for (int s = 0; s < a.S; ++s) {
        if (ml[2 * s] == -INFINITY) continue;
        const float f = exp2f(ml[2 * s] - m);
        z += ml[2 * s + 1] * f;
        if (tid < dh) t += a.part_o[(at * a.S + s) * dh + tid] * f;
    }
    if (tid < dh) Elem<T>::store(static_cast<T*>(a.o) + at * dh + tid, z > 0.f ? t / z : 0.f);
    if (tid == 0) {
        const float l2 = z > 0.f ? m + log2f(z) : -INFINITY;
        if (a.lse) a.lse[at] = l2 * 0.6931471805599453f;
        if (a.lse2) a.lse2[at] = l2;
    }
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

struct AttendCachePlan {
    int S, run;
    size_t lse2, part_o, part_ml, bytes;        // places in the workspace
};
static AttendCachePlan attend_cache_plan(const d3tom_paged_cache& c, int rows, int max_q, int max_len, int H, int weighed) {
    AttendCachePlan p;
    const long long groups = (long long)c.B * max_q * H;
    long long S = groups >= 1024 ? 1 : 1024 / groups;
    const long long most = (max_len + 255) / 256;
    S = S > most ? most : S;
    p.run = (int)((most + S - 1) / S) * 256;
    p.S = (max_len + p.run - 1) / p.run;
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o += align_up(bytes, 256); return at; };
    const size_t rh = (size_t)rows * H;
    p.lse2 = take(weighed ? rh * 4 : 0);
    p.part_o = take(p.S > 1 ? rh * p.S * c.dh * 4 : 0);
    p.part_ml = take(p.S > 1 ? rh * p.S * 8 : 0);
    p.bytes = o > 256 ? o : 256;
    return p;
}
static int attend_cache_check(const d3tom_paged_cache* c, int rows, int max_q, int max_len, int H) {
    const int rc = cache_check(c);
    if (rc != D3TOM_OK) return rc;
    if (rows < 1 || max_q < 1 || max_q > rows || max_len < 1 || H < 1 || H % c->Hkv) return D3TOM_ERR_INVALID_ARG;
    if ((int64_t)max_len > (int64_t)c->table_stride * c->page_size) return D3TOM_ERR_INVALID_ARG;
    return D3TOM_OK;
}

}  // namespace d3tom

using namespace d3tom;

extern "C" size_t d3tom_attend_cache_workspace_bytes(const d3tom_paged_cache* cache, int rows, int max_q, int max_len, int H, int weighed) {
    if (attend_cache_check(cache, rows, max_q, max_len, H) != D3TOM_OK) return 0;
    return attend_cache_plan(*cache, rows, max_q, max_len, H, weighed).bytes;
}

extern "C" int d3tom_attend_cache(const void* q, int64_t q_stride, const d3tom_paged_cache* cache, const int32_t* q_off, int rows, int max_q,
                                  int max_len, int H, float scale, int causal, void* o, float* lse, const float* weight_in, float* weight_out,
                                  int weight_stride, void* ws, size_t ws_bytes, void* stream) {
    hipStream_t st = (hipStream_t)stream;
    int rc = attend_cache_check(cache, rows, max_q, max_len, H);
    if (rc != D3TOM_OK) return rc;
    const int dt = cache->dt, dh = cache->dh;
    if ((rc = rows_check(q, q_stride, H, dh, dt)) != D3TOM_OK || (rc = rows_check(o, (int64_t)H * dh, H, dh, dt)) != D3TOM_OK) return rc;
    if (!q_off || !ws || !(scale > 0.f) || !(scale < 3.0e38f)) return D3TOM_ERR_INVALID_ARG;
    if ((weight_in && !weight_out) || (weight_out && weight_stride < max_len)) return D3TOM_ERR_INVALID_ARG;
    const AttendCachePlan p = attend_cache_plan(*cache, rows, max_q, max_len, H, weight_out != nullptr);
    if (ws_bytes < p.bytes || (((uintptr_t)ws) & 255u)) return D3TOM_ERR_WORKSPACE_TOO_SMALL;
    const double most = 16777215.0;             // workgroups of 256 threads in a launch
    if ((double)cache->B * max_q * H * p.S > most || (double)rows * H > most) return D3TOM_ERR_UNSUPPORTED;
    AttendCacheArgs a{};
    a.cache = cache_view(*cache);
    a.q = q; a.k_pages = cache->k_pages; a.v_pages = cache->v_pages; a.q_stride = q_stride; a.q_off = q_off;
    a.rows = rows; a.max_q = max_q; a.max_len = max_len; a.H = H; a.G = H / cache->Hkv; a.causal = causal != 0;
    a.scale2 = scale * LOG2E;
    a.S = p.S; a.run = p.run; a.o = o; a.lse = lse;
    a.lse2 = weight_out ? (float*)((char*)ws + p.lse2) : nullptr;
    a.part_o = (float*)((char*)ws + p.part_o); a.part_ml = (float*)((char*)ws + p.part_ml);
    a.weight_in = weight_in; a.weight_out = weight_out; a.weight_stride = weight_stride;
    const int wgs = cache->B * max_q * H * p.S;
    const dim3 wgrid((max_len + 63) / 64, cache->B);
#define D3TOM_ATTEND_CACHE(T)                                                                                              \
    do {                                                                                                                   \
        D3TOM_LAUNCH(CACHE_ATTEND, st, (attend_cache_generic_kernel<T><<<wgs, 256, 0, st>>>(a)));                          \
        if (p.S > 1) D3TOM_LAUNCH(CACHE_JOIN, st, (attend_cache_join_kernel<T><<<rows * H, 256, 0, st>>>(a)));             \
        if (weight_out) D3TOM_LAUNCH(CACHE_WEIGH, st, (cache_weigh_generic_kernel<T><<<wgrid, 256, 0, st>>>(a)));          \
    } while (0)
    if (dt == D3TOM_BF16) D3TOM_ATTEND_CACHE(uint16_t);
    else D3TOM_ATTEND_CACHE(float);
#undef D3TOM_ATTEND_CACHE
    return D3TOM_OK;
}
