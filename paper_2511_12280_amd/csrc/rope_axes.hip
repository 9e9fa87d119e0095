// d3tom_rope_axes and d3tom_cache_append: rotary positions with several axes, and new rows on their way into the pages of a cache.
// Both are pure HBM streaming: every row is read once and written once, in 16-byte accesses, float32 arithmetic, one rounding.
//
// Pair (c, c + dh/2) of a head turns by the angle pos[row, axis(c)] * frequency(c).  The dh/2 angles of a row serve all its heads, of q and k:
// a workgroup has a row, its first dh/2 threads evaluate the angles into LDS, the workgroup then streams the row.  (Positions are any
// int32: an angle of 131071 radians has no correct digit behind the second in float32's product and reduction, so that both are in double precision.)  14580 rows of
// 32 + 8 heads of 128, bf16: 56 us, 5.3 TB/s, where a large copy reaches 5.1 on this card.  A single row: 2.8 us.
#include "cache.hpp"

namespace d3tom {

constexpr int RX_MAX_HALF = 128;        // pairs of a head

struct AxesArgs {
    const int32_t* pos;
    int axes, ladder;
    int end[D3TOM_MAX_AXES];            // first pair behind each section
    double log2_theta;
};

// (cos, sin) of pair c's angle in a row
__device__ __forceinline__ float2 axes_cos_sin(const AxesArgs& ax, size_t row, int c, int dh) {
    int a = 0, start = 0, stop = ax.end[0];
#pragma unroll
    for (int i = 1; i < D3TOM_MAX_AXES; ++i)
        if (i < ax.axes && c >= ax.end[i - 1]) { a = i; start = ax.end[i - 1]; stop = ax.end[i]; }
    if (c >= stop) return make_float2(1.f, 0.f);
    const double e = ax.ladder == D3TOM_AXES_OWN ? (double)(c - start) / (double)(stop - start) : 2.0 * (double)c / (double)dh;
    double s, co;
    sincos((double)ax.pos[row * ax.axes + a] * exp2(-e * ax.log2_theta), &s, &co);
    return make_float2((float)co, (float)s);
}

// what a launch moves: queries and keys turned, values as they are
struct RowJob {
    const void *q, *k, *v;
    size_t q_stride, k_stride, v_stride;
    int H, Hkv, dh;
    void *q_out, *k_out;                // contiguous; k_out: not for a cache
    // into the pages (APPEND)
    CacheView cache;
    void *k_pages, *v_pages;
    const int32_t* new_off;
    const int32_t* tokens;
    int32_t* slot_token;
    float* slot_weight;
    int slot_stride, rows;
};

template <typename T>
__device__ __forceinline__ void turn_chunk(const T* a, const T* b, T* oa, T* ob, const float2* cs) {
    constexpr int EPC = 16 / sizeof(T);
    const uint4 A = *reinterpret_cast<const uint4*>(a), Bv = *reinterpret_cast<const uint4*>(b);
    const uint32_t aw[4] = {A.x, A.y, A.z, A.w}, bw[4] = {Bv.x, Bv.y, Bv.z, Bv.w};
    uint32_t ao[4], bo[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (EPC == 8) {
            float a0, b0, a1, b1;
            rope_rotate(bf16_lo(aw[e]), bf16_lo(bw[e]), cs[2 * e].x, cs[2 * e].y, a0, b0);
            rope_rotate(bf16_hi(aw[e]), bf16_hi(bw[e]), cs[2 * e + 1].x, cs[2 * e + 1].y, a1, b1);
            ao[e] = pack_bf16x2(a0, a1);
            bo[e] = pack_bf16x2(b0, b1);
        } else {
            float a0, b0;
            rope_rotate(__uint_as_float(aw[e]), __uint_as_float(bw[e]), cs[e].x, cs[e].y, a0, b0);
            ao[e] = __float_as_uint(a0);
            bo[e] = __float_as_uint(b0);
        }
    }
    *reinterpret_cast<uint4*>(oa) = make_uint4(ao[0], ao[1], ao[2], ao[3]);
    *reinterpret_cast<uint4*>(ob) = make_uint4(bo[0], bo[1], bo[2], bo[3]);
}

template <typename T, bool TURN, bool APPEND>
__global__ __launch_bounds__(256) void rope_rows_kernel(RowJob job, AxesArgs ax) {
    constexpr int EPC = 16 / sizeof(T);
    __shared__ __attribute__((aligned(16))) float2 cs[RX_MAX_HALF];
    const int tid = threadIdx.x;
    const int half = job.dh >> 1;
    size_t row = blockIdx.x;
    T *k_to = nullptr, *v_to = nullptr;
    if constexpr (APPEND) {
        const int b = blockIdx.y;
        int r0 = job.new_off[b], r1 = job.new_off[b + 1], n = job.cache.len[b];
        r0 = max(r0, 0);
        r1 = min(max(r1, 0), job.rows);
        if ((int)blockIdx.x >= r1 - r0) return;
        row += r0;
        const int slot = n - (r1 - r0) + (int)blockIdx.x;
        if (slot >= 0 && (slot >> job.cache.shift) < job.cache.table_stride) {
            const int page = job.cache.page_of(b, slot);
            if (job.cache.writable(page)) {
                const size_t at = job.cache.row((uint32_t)page, slot) * job.cache.row_elems();
                k_to = static_cast<T*>(job.k_pages) + at;
                v_to = static_cast<T*>(job.v_pages) + at;
            }
            if (tid == 0 && slot < job.slot_stride) {
                if (job.slot_token) job.slot_token[(size_t)b * job.slot_stride + slot] = job.tokens[row];
                if (job.slot_weight) job.slot_weight[(size_t)b * job.slot_stride + slot] = 0.f;
            }
        }
    } else if (job.k) {
        k_to = static_cast<T*>(job.k_out) + row * job.Hkv * job.dh;
    }
    if constexpr (TURN) {
        if (tid < half) cs[tid] = axes_cos_sin(ax, row, tid, job.dh);
        __syncthreads();
        const int cpp = half / EPC;                      // 16-byte chunks of half a head
        const int nq = job.q ? job.H * cpp : 0, nk = k_to ? job.Hkv * cpp : 0;
        const T* q = static_cast<const T*>(job.q) + row * job.q_stride;
        const T* k = static_cast<const T*>(job.k) + row * job.k_stride;
        T* q_to = static_cast<T*>(job.q_out) + row * job.H * job.dh;
        for (int u = tid; u < nq + nk; u += 256) {
            const int w = u < nq ? u : u - nq, h = w / cpp, c = (w - h * cpp) * EPC, at = h * job.dh + c;
            const T* from = (u < nq ? q : k) + at;
            T* to = (u < nq ? q_to : k_to) + at;
            turn_chunk<T>(from, from + half, to, to + half, cs + c);
        }
    } else if (k_to) {
        const uint4* k = reinterpret_cast<const uint4*>(static_cast<const T*>(job.k) + row * job.k_stride);
        for (int u = tid; u < job.Hkv * job.dh / EPC; u += 256) reinterpret_cast<uint4*>(k_to)[u] = k[u];
    }
    if constexpr (APPEND) {
        if (v_to) {
            const uint4* v = reinterpret_cast<const uint4*>(static_cast<const T*>(job.v) + row * job.v_stride);
            for (int u = tid; u < job.Hkv * job.dh / EPC; u += 256) reinterpret_cast<uint4*>(v_to)[u] = v[u];
        }
    }
}

static int axes_check(const d3tom_axes* axes, int dh, int dt, AxesArgs* out) {
    if (!axes || !axes->pos) return D3TOM_ERR_INVALID_ARG;
    if (axes->axes < 1 || axes->axes > D3TOM_MAX_AXES) return D3TOM_ERR_INVALID_ARG;
    if (axes->ladder != D3TOM_AXES_SHARED && axes->ladder != D3TOM_AXES_OWN) return D3TOM_ERR_INVALID_ARG;
    if (!(axes->theta > 1.f) || !(axes->theta < 3.0e38f)) return D3TOM_ERR_INVALID_ARG;
    if (dh > 2 * RX_MAX_HALF || dh % (32 / elem_bytes(dt))) return D3TOM_ERR_UNSUPPORTED;
    int64_t sum = 0;
    for (int a = 0; a < D3TOM_MAX_AXES; ++a) {
        if (a < axes->axes) {
            if (axes->pairs[a] < 1) return D3TOM_ERR_INVALID_ARG;
            sum += axes->pairs[a];
            if (sum > dh / 2) return D3TOM_ERR_INVALID_ARG;
        }
        out->end[a] = (int)sum;
    }
    out->pos = axes->pos; out->axes = axes->axes; out->ladder = axes->ladder;
    out->log2_theta = log2((double)axes->theta);
    return D3TOM_OK;
}

}  // namespace d3tom

using namespace d3tom;

extern "C" int d3tom_rope_axes(const void* q, int64_t q_stride, const void* k, int64_t k_stride, int dt, int rows, int H, int Hkv, int dh,
                               const d3tom_axes* axes, void* q_out, void* k_out, void* stream) {
    hipStream_t st = (hipStream_t)stream;
    if ((!q && !k) || rows < 1 || dh < 1 || (dt != D3TOM_F32 && dt != D3TOM_BF16)) return D3TOM_ERR_INVALID_ARG;
    RowJob job{};
    AxesArgs ax;
    int rc = axes_check(axes, dh, dt, &ax);
    if (rc != D3TOM_OK) return rc;
    if (q && ((rc = rows_check(q, q_stride, H, dh, dt)) != D3TOM_OK || (rc = rows_check(q_out, (int64_t)H * dh, H, dh, dt)) != D3TOM_OK)) return rc;
    if (k && ((rc = rows_check(k, k_stride, Hkv, dh, dt)) != D3TOM_OK || (rc = rows_check(k_out, (int64_t)Hkv * dh, Hkv, dh, dt)) != D3TOM_OK)) return rc;
    if ((q && H > 65535) || (k && Hkv > 65535) || rows > CACHE_MOST_GROUPS) return D3TOM_ERR_UNSUPPORTED;
    job.q = q; job.k = k; job.q_stride = q_stride; job.k_stride = k_stride;
    job.H = H; job.Hkv = Hkv; job.dh = dh; job.q_out = q_out; job.k_out = k_out; job.rows = rows;
    if (dt == D3TOM_BF16) D3TOM_LAUNCH(ROPE, st, (rope_rows_kernel<uint16_t, true, false><<<rows, 256, 0, st>>>(job, ax)));
    else D3TOM_LAUNCH(ROPE, st, (rope_rows_kernel<float, true, false><<<rows, 256, 0, st>>>(job, ax)));
    return D3TOM_OK;
}

extern "C" int d3tom_cache_append(const d3tom_paged_cache* cache, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                                  const int32_t* new_off, int rows, int max_new, const d3tom_axes* axes, const void* q, int64_t q_stride,
                                  int H, void* q_out, const int32_t* tokens, int32_t* slot_token, float* slot_weight, int slot_stride,
                                  void* stream) {
    hipStream_t st = (hipStream_t)stream;
    int rc = cache_check(cache);
    if (rc != D3TOM_OK) return rc;
    const int dt = cache->dt, dh = cache->dh;
    if (!new_off || rows < 1 || max_new < 1 || max_new > rows) return D3TOM_ERR_INVALID_ARG;
    if ((rc = rows_check(k, k_stride, cache->Hkv, dh, dt)) != D3TOM_OK || (rc = rows_check(v, v_stride, cache->Hkv, dh, dt)) != D3TOM_OK) return rc;
    if ((slot_token && !tokens) || ((slot_token || slot_weight) && slot_stride < 1) || (q && !axes)) return D3TOM_ERR_INVALID_ARG;
    AxesArgs ax{};
    if (axes && (rc = axes_check(axes, dh, dt, &ax)) != D3TOM_OK) return rc;
    if (q && ((rc = rows_check(q, q_stride, H, dh, dt)) != D3TOM_OK || (rc = rows_check(q_out, (int64_t)H * dh, H, dh, dt)) != D3TOM_OK)) return rc;
    if ((q && H > 65535) || (double)max_new * cache->B > CACHE_MOST_GROUPS) return D3TOM_ERR_UNSUPPORTED;
    RowJob job{};
    job.q = q; job.k = k; job.v = v; job.q_stride = q_stride; job.k_stride = k_stride; job.v_stride = v_stride;
    job.H = H; job.Hkv = cache->Hkv; job.dh = dh; job.q_out = q_out;
    job.cache = cache_view(*cache);
    job.k_pages = cache->k_pages; job.v_pages = cache->v_pages;
    job.new_off = new_off; job.tokens = tokens; job.slot_token = slot_token; job.slot_weight = slot_weight;
    job.slot_stride = slot_stride; job.rows = rows;
    const dim3 grid(max_new, cache->B);
#define D3TOM_APPEND(T, TURN) D3TOM_LAUNCH(CACHE_APPEND, st, (rope_rows_kernel<T, TURN, true><<<grid, 256, 0, st>>>(job, ax)))
    if (dt == D3TOM_BF16) { if (axes) D3TOM_APPEND(uint16_t, true); else D3TOM_APPEND(uint16_t, false); }
    else { if (axes) D3TOM_APPEND(float, true); else D3TOM_APPEND(float, false); }
#undef D3TOM_APPEND
    return D3TOM_OK;
}
