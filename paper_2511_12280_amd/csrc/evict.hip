// d3tom_cache_evict: a cache shortened by the attention weight that its slots have got.
//
// Order of the slots: an unsigned key per slot, all ones for a protected one, else the order-preserving image of its weight; larger
// first, equal keys by the slot.  One workgroup per sample finds the k-th largest key eight bits at a time (counts of integers: the
// order of the additions does not show), then goes over the slots in ascending order and numbers the holes (slots below k that do
// not stay) and the movers (slots from k on that do): there are as many of either.  A second launch moves the rows: every mover
// lies at k or above and every hole below it, so that the moves need no order among themselves.
#include "cache.hpp"

namespace d3tom {

constexpr int EV_THREADS = 1024;

struct EvictArgs {
    CacheView cache;
    int max_len;
    const int32_t* keep;
    int first, recent;
    const float* weight_in;
    const int32_t* token_in;
    float* weight_out;
    int32_t* token_out;
    int stride;
    int32_t *len_out, *src;
    int32_t *moves, *holes, *movers;            // [B], [B, max_len / 2] twice
    int room;                                   // max_len / 2
    char *k_pages, *v_pages;
    int row_bytes;
};

__device__ __forceinline__ uint32_t evict_key(float w, int token, int first, long long newest) {
    if (token < first || (long long)token > newest) return 0xFFFFFFFFu;
    const uint32_t u = __float_as_uint(w + 0.f);        // -0 is 0
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__global__ __launch_bounds__(EV_THREADS) void evict_select_kernel(EvictArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    __shared__ int hist[256];
    __shared__ int wave_a[EV_THREADS / 64], wave_b[EV_THREADS / 64];
    __shared__ int s_digit, s_above;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, b = blockIdx.x;
    const int n = a.cache.length(b, a.max_len);
    const int k = min(max(a.keep[b], 0), n);
    const float* w = a.weight_in + (size_t)b * a.stride;
    const int32_t* tok = a.token_in + (size_t)b * a.stride;
    float* w_out = a.weight_out + (size_t)b * a.stride;
    int32_t* t_out = a.token_out + (size_t)b * a.stride;
    int32_t* src = a.src ? a.src + (size_t)b * a.stride : nullptr;
    int32_t *holes = a.holes + (size_t)b * a.room, *movers = a.movers + (size_t)b * a.room;

    // the last number that is not protected as recent
    int top = INT32_MIN;
    for (int j = tid; j < n; j += EV_THREADS) top = max(top, tok[j]);
    for (int o = 32; o > 0; o >>= 1) top = max(top, __shfl_xor(top, o));
    if (lane == 0) wave_a[wave] = top;
    __syncthreads();
    for (int i = 0; i < EV_THREADS / 64; ++i) top = max(top, wave_a[i]);
    const long long newest = (long long)top - a.recent;

    // the k-th largest key, and how many larger ones there are
    uint32_t prefix = 0;
    int need = k;                               // of the keys that agree with the prefix so far
    for (int shift = 24; shift >= 0 && k < n && k > 0; shift -= 8) {
        __syncthreads();
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        for (int j = tid; j < n; j += EV_THREADS) {
            const uint32_t key = evict_key(w[j], tok[j], a.first, newest);
            if (shift == 24 || (key >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(key >> shift) & 255], 1);
        }
        __syncthreads();
        if (tid == 0) {
            int d = 255, above = 0;
            while (d > 0 && above + hist[d] < need) above += hist[d--];
            s_digit = d; s_above = above;
        }
        __syncthreads();
        prefix |= (uint32_t)s_digit << shift;
        need -= s_above;
    }
    // slots in ascending order: whether each stays, holes and movers numbered
    int ties = 0, nh = 0, nm = 0;               // of the slots in front
    for (int j0 = 0; j0 < n; j0 += EV_THREADS) {
        const int j = j0 + tid;
        const bool live = j < n;
        float wj = 0.f;
        int tj = 0;
        uint32_t key = 0;
        if (live) { wj = w[j]; tj = tok[j]; key = evict_key(wj, tj, a.first, newest); }
        const bool tie = live && k < n && k > 0 && key == prefix;
        int sc = wave_incl_scan(tie ? 1 : 0);
        __syncthreads();
        if (lane == 63) wave_a[wave] = sc;
        __syncthreads();
        int before = 0, all = 0;
        for (int i = 0; i < EV_THREADS / 64; ++i) { before += i < wave ? wave_a[i] : 0; all += wave_a[i]; }
        const int rank = ties + before + sc - 1;
        ties += all;
        const bool stays = live && (k == n || (k > 0 && (key > prefix || (tie && rank < need))));
        const bool hole = live && j < k && !stays, mover = j >= k && stays;
        const int hs = wave_incl_scan(hole ? 1 : 0), ms = wave_incl_scan(mover ? 1 : 0);
        __syncthreads();
        if (lane == 63) { wave_a[wave] = hs; wave_b[wave] = ms; }
        __syncthreads();
        int hb = 0, ha = 0, mb = 0, ma = 0;
        for (int i = 0; i < EV_THREADS / 64; ++i) {
            hb += i < wave ? wave_a[i] : 0; ha += wave_a[i];
            mb += i < wave ? wave_b[i] : 0; ma += wave_b[i];
        }
        if (hole) holes[nh + hb + hs - 1] = j;
        if (mover) movers[nm + mb + ms - 1] = j;
        nh += ha; nm += ma;
        if (stays && j < k) {
            w_out[j] = wj; t_out[j] = tj;
            if (src) src[j] = j;
        }
    }
    __syncthreads();                            // the lists, and everything that is read, are there
    for (int i = tid; i < nh; i += EV_THREADS) {
        const int to = holes[i], from = movers[i];
        w_out[to] = w[from]; t_out[to] = tok[from];
        if (src) src[to] = from;
    }
    if (tid == 0) { a.moves[b] = nh; a.len_out[b] = k; }
#endif
}

// 16 bytes to a thread, 256 threads along the rows of the sample's moves
__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a) {
    const int b = blockIdx.y, chunks = a.row_bytes / 16;
    const long long total = (long long)a.moves[b] * chunks;
    const int32_t *holes = a.holes + (size_t)b * a.room, *movers = a.movers + (size_t)b * a.room;
    for (long long u = (long long)blockIdx.x * 256 + threadIdx.x; u < total; u += (long long)gridDim.x * 256) {
        const int i = (int)(u / chunks), c = (int)(u - (long long)i * chunks);
        const int to = holes[i], from = movers[i];
        const int pt = a.cache.page_of(b, to);
        if (!a.cache.writable(pt)) continue;
        const size_t at = a.cache.row((uint32_t)pt, to) * a.row_bytes + (size_t)c * 16;
        const size_t of = a.cache.row(a.cache.readable(a.cache.page_of(b, from)), from) * a.row_bytes + (size_t)c * 16;
        *reinterpret_cast<uint4*>(a.k_pages + at) = *reinterpret_cast<const uint4*>(a.k_pages + of);
        *reinterpret_cast<uint4*>(a.v_pages + at) = *reinterpret_cast<const uint4*>(a.v_pages + of);
    }
}

struct EvictWs { size_t moves, holes, movers, bytes; };
static EvictWs evict_ws(int B, int max_len) {
    EvictWs w;
    const size_t list = align_up((size_t)B * (max_len / 2) * 4, 256);
    w.moves = 0;
    w.holes = align_up((size_t)B * 4, 256);
    w.movers = w.holes + list;
    w.bytes = w.movers + list;
    return w;
}
static int evict_check(const d3tom_paged_cache* c, int max_len) {
    const int rc = cache_check(c);
    if (rc != D3TOM_OK) return rc;
    if (max_len < 1 || (int64_t)max_len > (int64_t)c->table_stride * c->page_size) return D3TOM_ERR_INVALID_ARG;
    if (max_len > D3TOM_MAX_EVICT_LEN) return D3TOM_ERR_UNSUPPORTED;
    return D3TOM_OK;
}

}  // namespace d3tom

using namespace d3tom;

extern "C" size_t d3tom_cache_evict_workspace_bytes(const d3tom_paged_cache* cache, int max_len) {
    return evict_check(cache, max_len) == D3TOM_OK ? evict_ws(cache->B, max_len).bytes : 0;
}

extern "C" int d3tom_cache_evict(const d3tom_paged_cache* cache, int max_len, const int32_t* keep, int first, int recent,
                                 const float* weight_in, const int32_t* token_in, float* weight_out, int32_t* token_out, int slot_stride,
                                 int32_t* len_out, int32_t* src, void* ws, size_t ws_bytes, void* stream) {
    hipStream_t st = (hipStream_t)stream;
    const int rc = evict_check(cache, max_len);
    if (rc != D3TOM_OK) return rc;
    if (!keep || !weight_in || !token_in || !weight_out || !token_out || !len_out || !ws) return D3TOM_ERR_INVALID_ARG;
    if (slot_stride < max_len || first < 0 || recent < 0) return D3TOM_ERR_INVALID_ARG;
    const EvictWs w = evict_ws(cache->B, max_len);
    if (ws_bytes < w.bytes || (((uintptr_t)ws) & 255u)) return D3TOM_ERR_WORKSPACE_TOO_SMALL;
    EvictArgs a{};
    a.cache = cache_view(*cache);
    a.max_len = max_len; a.keep = keep; a.first = first; a.recent = recent;
    a.weight_in = weight_in; a.token_in = token_in; a.weight_out = weight_out; a.token_out = token_out; a.stride = slot_stride;
    a.len_out = len_out; a.src = src;
    a.moves = (int32_t*)((char*)ws + w.moves); a.holes = (int32_t*)((char*)ws + w.holes); a.movers = (int32_t*)((char*)ws + w.movers);
    a.room = max_len / 2;
    a.k_pages = (char*)cache->k_pages; a.v_pages = (char*)cache->v_pages;
    a.row_bytes = cache->Hkv * cache->dh * elem_bytes(cache->dt);
    D3TOM_LAUNCH(EVICT_SELECT, st, (evict_select_kernel<<<cache->B, EV_THREADS, 0, st>>>(a)));
    if (a.room > 0) {
        const long long units = ((long long)a.room * (a.row_bytes / 16) + 255) / 256;
        const long long each = 4096 / cache->B + 1;
        const dim3 grid((unsigned)(units < each ? units : each), cache->B);
        D3TOM_LAUNCH(EVICT_MOVE, st, (evict_move_kernel<<<grid, 256, 0, st>>>(a)));
    }
    return D3TOM_OK;
}
