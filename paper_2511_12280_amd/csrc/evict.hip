// d3tom_cache_evict: a cache shortened by the attention weight that its slots have got.
//
// Order of the slots: an unsigned key per slot, all ones for a protected one, else the order-preserving image of its weight; larger
// first, equal keys by the slot.  One workgroup per sample finds the k-th largest key by counting: 2048 bins over the range that the keys
// have (weights are spread over many octaves, and the image is nearly their logarithm, so that the counts do not meet in few bins as they would in bins of a
// fixed number of leading bits), then over the bin that the key lies in, at most three times.  Counts of integers: the order of the additions does not
// show.  It leaves a bit for every slot that stays, and for each word of 64 how many holes (slots below k that do not stay) and movers (slots
// from k on that do) lie in front of it: there are as many of either.
//
// A second launch has a workgroup for every word below k: it pairs the word's holes with the movers of the same numbers and moves their rows.
// Every mover lies at k or above and every hole below it, so that the moves need no order among themselves.
//
// The selection has one compute unit per sample; its keys stay in registers up to 16384 slots and are formed again in every turn beyond that.
// The moves are bound by memory.
#include "cache.hpp"

namespace d3tom {

constexpr int EV_THREADS = 1024, EV_WAVES = EV_THREADS / 64, EV_BINS = 2048;

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
    // workspace: (slots, those that stay) [B]; [B, words]: a bit per slot that stays, holes and movers in front
    int2* sizes;
    unsigned long long* stays;
    int32_t *holes, *movers;
    int words;
    char *k_pages, *v_pages;
    int row_bytes;
};

constexpr uint32_t EV_PROTECTED = 0xFFFFFFFFu;
__device__ __forceinline__ uint32_t evict_image(float w) {
    const uint32_t u = __float_as_uint(w + 0.f);        // -0 is 0
    return min((u & 0x80000000u) ? ~u : (u | 0x80000000u), EV_PROTECTED - 1u);
}

// all lanes' extreme
template <int O>
__device__ __forceinline__ int ev_across(int v) { return __builtin_amdgcn_update_dpp(0, v, O, 0xF, 0xF, true); }
template <typename F>
__device__ __forceinline__ int ev_reduce(int v, F&& f) {
#if defined(__HIP_DEVICE_COMPILE__)
    v = f(v, ev_across<0xB1>(v));
    v = f(v, ev_across<0x4E>(v));
    v = f(v, ev_across<0x141>(v));
    v = f(v, ev_across<0x140>(v));
    typedef unsigned u2 __attribute__((ext_vector_type(2)));
    u2 r = __builtin_amdgcn_permlane16_swap((unsigned)v, (unsigned)v, false, false);
    v = f((int)r[0], (int)r[1]);
    r = __builtin_amdgcn_permlane32_swap((unsigned)v, (unsigned)v, false, false);
    return f((int)r[0], (int)r[1]);
#else
    return v;
#endif
}

// P: keys of a thread in registers, 64 slots to a wave and turn; 0: any number, formed again each time, EV_BATCH turns requested together
constexpr int EV_BATCH = 8;
template <int P>
__global__ __launch_bounds__(EV_THREADS) void evict_select_kernel(EvictArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    __shared__ int hist[EV_BINS];
    __shared__ int wave_a[EV_WAVES], wave_b[EV_WAVES], wave_c[EV_WAVES];
    __shared__ uint32_t wave_lo[EV_WAVES], wave_hi[EV_WAVES];
    __shared__ int s_digit, s_above, s_equal;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), b = blockIdx.x;
    const int n = a.cache.length(b, a.max_len);
    const int k = min(max(a.keep[b], 0), n);
    if (n == 0) {
        if (tid == 0) a.sizes[b] = make_int2(0, 0);
        return;
    }
    const float* w = a.weight_in + (size_t)b * a.stride;
    const int32_t* tok = a.token_in + (size_t)b * a.stride;
    // A wave has consecutive slots.  Every turn is taken, live or not: loads behind a branch would wait for each other.
    const int turns = P > 0 ? P : (n + EV_THREADS - 1) / EV_THREADS, first_slot = wave * turns * 64;
    uint32_t image[P > 0 ? P : 1];                      // of the weight, then the key
    int32_t token[P > 0 ? P : 1];
    if constexpr (P > 0) {
#pragma unroll
        for (int u = 0; u < P; ++u) {
            const int j = min(first_slot + u * 64 + lane, n - 1);
            image[u] = evict_image(w[j]);
            token[u] = tok[j];
        }
    }
    // f(turn, image of the weight, token) for every turn
    auto each = [&](auto&& f) {
        if constexpr (P > 0) {
#pragma unroll
            for (int u = 0; u < P; ++u) f(u, image[u], token[u]);
        } else {
            for (int u0 = 0; u0 < turns; u0 += EV_BATCH) {
                float wv[EV_BATCH];
                int32_t tv[EV_BATCH];
#pragma unroll
                for (int u = 0; u < EV_BATCH; ++u) {
                    const int j = min(first_slot + (u0 + u) * 64 + lane, n - 1);
                    wv[u] = w[j];
                    tv[u] = tok[j];
                }
#pragma unroll
                for (int u = 0; u < EV_BATCH; ++u)
                    if (u0 + u < turns) f(u0 + u, evict_image(wv[u]), tv[u]);
            }
        }
    };
    auto live_of = [&](int u) {                         // the turn's live slots
        const int at = first_slot + u * 64;
        return at >= n ? 0ull : n - at >= 64 ? ~0ull : (1ull << (n - at)) - 1;
    };
    // the last number, and the range of the images
    int top = INT32_MIN;
    uint32_t lo = ~0u, hi = 0;
    each([&](int, uint32_t im, int32_t t) { top = max(top, t); lo = min(lo, im); hi = max(hi, im); });
    top = ev_reduce(top, [](int x, int y) { return max(x, y); });
    lo = (uint32_t)ev_reduce((int)lo, [](int x, int y) { return (int)min((uint32_t)x, (uint32_t)y); });
    hi = (uint32_t)ev_reduce((int)hi, [](int x, int y) { return (int)max((uint32_t)x, (uint32_t)y); });
    if (lane == 0) { wave_a[wave] = top; wave_lo[wave] = lo; wave_hi[wave] = hi; }
    hist[tid] = 0;
    hist[tid + EV_THREADS] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < EV_WAVES; ++i) { top = max(top, wave_a[i]); lo = min(lo, wave_lo[i]); hi = max(hi, wave_hi[i]); }
    const long long newest = (long long)top - a.recent;
    auto key_of = [&](uint32_t im, int32_t t) { return t < a.first || (long long)t > newest ? EV_PROTECTED : im; };

    // the k-th largest key, and how many of the keys equal to it stay
    uint32_t limit = 0;
    int need = 0, equal = 0;
    if (k > 0 && k < n) {
        int shift = 0;
        while (((hi - lo) >> shift) > EV_BINS - 2) ++shift;
        need = k;
        bool first = true;
        uint32_t span = 0;                              // of the keys that are left, behind the first time
        while (true) {
            each([&](int u, uint32_t im, int32_t t) {
                const uint32_t key = key_of(im, t), at = key - lo;
                const int bin = first && key == EV_PROTECTED ? EV_BINS - 1 : (int)(at >> shift);
                if (((live_of(u) >> lane) & 1) && (first || (key != EV_PROTECTED && key >= lo && at <= span))) atomicAdd(&hist[bin], 1);
            });
            __syncthreads();
            // counts from the last bin down: a thread has two
            const int h1 = hist[EV_BINS - 1 - 2 * tid], h0 = hist[EV_BINS - 2 - 2 * tid];
            const int sum = wave_incl_scan(h1 + h0);
            if (lane == 63) wave_a[wave] = sum;
            __syncthreads();
            hist[tid] = 0;
            hist[tid + EV_THREADS] = 0;
            int above = sum - h1 - h0;
#pragma unroll
            for (int i = 0; i < EV_WAVES; ++i) above += i < wave ? wave_a[i] : 0;
            if (above < need && need <= above + h1) { s_digit = EV_BINS - 1 - 2 * tid; s_above = above; s_equal = h1; }
            else if (above + h1 < need && need <= above + h1 + h0) { s_digit = EV_BINS - 2 - 2 * tid; s_above = above + h1; s_equal = h0; }
            __syncthreads();
            const int digit = s_digit;
            need -= s_above;
            equal = s_equal;
            if (first && digit == EV_BINS - 1) { limit = EV_PROTECTED; break; }
            lo += (uint32_t)digit << shift;
            if (shift == 0) { limit = lo; break; }
            span = (1u << shift) - 1;
            shift = max(shift - 11, 0);
            first = false;
        }
    } else {
        limit = k > 0 ? 0u : EV_PROTECTED;              // all stay, or none
        equal = k > 0 ? 0 : n + 1;
    }
    // The words, in ascending order.  Of the keys equal to the k-th the first `need` stay: where that is not all of them, those in front are counted.
    const bool count_ties = need < equal;
    int tied = 0;
    if (count_ties) {
        each([&](int u, uint32_t im, int32_t t) { tied += __popcll(__builtin_amdgcn_ballot_w64(key_of(im, t) == limit) & live_of(u)); });
        if (lane == 0) wave_b[wave] = tied;
        __syncthreads();
        tied = 0;
#pragma unroll
        for (int i = 0; i < EV_WAVES; ++i) tied += i < wave ? wave_b[i] : 0;
        __syncthreads();
    }
    const size_t row = (size_t)b * a.words + wave * turns;
    const int words = min((n + 63) / 64 - wave * turns, turns);        // of this wave
    const bool at_end = P > 0 || turns <= 64;
    unsigned long long my_word = 0;
    int my_h = 0, my_m = 0, nh = 0, nm = 0;             // lane u % 64 keeps what belongs to turn u, 64 turns are stored together
    each([&](int u, uint32_t im, int32_t t) {
        const uint32_t key = key_of(im, t);
        const unsigned long long live = live_of(u);
        unsigned long long word = __builtin_amdgcn_ballot_w64(key >= limit) & live;
        if (count_ties) {
            unsigned long long same = __builtin_amdgcn_ballot_w64(key == limit) & live;
            const int there = __popcll(same), allowed = min(max(need - tied, 0), there);
            tied += there;
            word &= ~same;
            for (int i = there; i > allowed; --i) same &= ~(1ull << (63 - __clzll((long long)same)));
            word |= same;
        }
        const int at = first_slot + u * 64;
        const unsigned long long low = at >= k ? 0ull : k - at >= 64 ? ~0ull : (1ull << (k - at)) - 1;
        const bool mine = lane == (u & 63);
        my_word = mine ? word : my_word;
        my_h = mine ? nh : my_h;
        my_m = mine ? nm : my_m;
        nh += __popcll(low & ~word);
        nm += __popcll(word & ~low);
        if (!at_end && ((u & 63) == 63 || u == turns - 1)) {
            const int to = (u & ~63) + lane;
            if (to <= u && to < words) { a.stays[row + to] = my_word; a.holes[row + to] = my_h; a.movers[row + to] = my_m; }
        }
    });
    if (lane == 0) { wave_b[wave] = nh; wave_c[wave] = nm; }
    __syncthreads();
    nh = nm = 0;
#pragma unroll
    for (int i = 0; i < EV_WAVES; ++i) { nh += i < wave ? wave_b[i] : 0; nm += i < wave ? wave_c[i] : 0; }
    // with the counts of the waves in front
    for (int at = lane; at < words; at += 64) {
        if (at_end) a.stays[row + at] = my_word;
        a.holes[row + at] = (at_end ? my_h : a.holes[row + at]) + nh;
        a.movers[row + at] = (at_end ? my_m : a.movers[row + at]) + nm;
    }
    if (tid == 0) a.sizes[b] = make_int2(n, k);
#endif
}

// The word's moves: 2^lanes lanes have the 16-byte chunks of one (a row of k and the one of v behind it), EV_AT_ONCE of them to a lane at once.  And
// what the word's slots keep of numbers.  len_out may be the cache's lengths: nothing reads them any more.
constexpr int EV_AT_ONCE = 4;
typedef uint32_t ev_u32x4 __attribute__((ext_vector_type(4)));
__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a, int lanes) {
    __shared__ int from_s[64], to_s[64], s_start;
    const int b = blockIdx.y, tid = threadIdx.x;
    const int2 size = a.sizes[b];
    const int n = size.x, k = size.y, word = blockIdx.x, slot0 = word * 64;
    if (word == 0 && tid == 0) a.len_out[b] = k;
    if (slot0 >= k) return;
    const size_t row = (size_t)b * a.words, at = (size_t)b * a.stride;
    const unsigned long long low = k - slot0 >= 64 ? ~0ull : (1ull << (k - slot0)) - 1, stay = a.stays[row + word] & low, hole = low & ~stay;
    const int h0 = a.holes[row + word], count = __popcll(hole);
    // the word that has mover h0: the last one with at most h0 movers in front (words without any in between have none to give)
    const int w0 = k >> 6, w1 = (n - 1) >> 6;
    if (count > 0) {
        for (int w = w0 + tid; w <= w1; w += 256) {
            const int mine = a.movers[row + w];
            if (mine <= h0 && (w == w1 || a.movers[row + w + 1] > h0)) s_start = w;
        }
    }
    if (tid < 64) {
        const int j = slot0 + tid;
        const unsigned long long in_front = (1ull << tid) - 1;
        if ((stay >> tid) & 1) {
            a.weight_out[at + j] = a.weight_in[at + j];
            a.token_out[at + j] = a.token_in[at + j];
            if (a.src) a.src[at + j] = j;
        }
        if ((hole >> tid) & 1) to_s[__popcll(hole & in_front)] = j;
    }
    if (count == 0) return;
    __syncthreads();
    if (tid < 64) {
        const unsigned long long in_front = (1ull << tid) - 1;
        for (int w = s_start, got = a.movers[row + w] - h0; got < count && w <= w1; ++w) {
            const unsigned long long low_w = k - w * 64 >= 64 ? ~0ull : k <= w * 64 ? 0ull : (1ull << (k - w * 64)) - 1;
            const unsigned long long movers = a.stays[row + w] & ~low_w;
            const int rank = got + __popcll(movers & in_front);
            if (((movers >> tid) & 1) && rank >= 0 && rank < count) from_s[rank] = w * 64 + tid;
            got += __popcll(movers);
        }
    }
    __syncthreads();
    if (tid < count) {
        const int to = to_s[tid], from = from_s[tid];
        a.weight_out[at + to] = a.weight_in[at + from];
        a.token_out[at + to] = a.token_in[at + from];
        if (a.src) a.src[at + to] = from;
    }
    const int half = a.row_bytes / 16, chunks = 2 * half, step = 1 << lanes, c0 = tid & (step - 1);
    for (int i = tid >> lanes; i < count; i += 256 >> lanes) {
        const int to = to_s[i], from = from_s[i];
        const int pt = a.cache.page_of(b, to), pf = a.cache.page_of(b, from);
        if (!a.cache.writable(pt)) continue;
        const size_t dst = a.cache.row((uint32_t)pt, to) * a.row_bytes, of = a.cache.row(a.cache.readable(pf), from) * a.row_bytes;
        for (int c = c0; c < chunks; c += step * EV_AT_ONCE) {
            ev_u32x4 v[EV_AT_ONCE];
#pragma unroll
            for (int u = 0; u < EV_AT_ONCE; ++u) {
                const int x = min(c + u * step, chunks - 1);
                v[u] = *reinterpret_cast<const ev_u32x4*>((x < half ? a.k_pages : a.v_pages) + of + (size_t)(x < half ? x : x - half) * 16);
            }
#pragma unroll
            for (int u = 0; u < EV_AT_ONCE; ++u) {
                const int x = c + u * step;
                if (x < chunks) *reinterpret_cast<ev_u32x4*>((x < half ? a.k_pages : a.v_pages) + dst + (size_t)(x < half ? x : x - half) * 16) = v[u];
            }
        }
    }
}

struct EvictWs { size_t sizes, stays, holes, movers, bytes; int words; };
static EvictWs evict_ws(int B, int max_len) {
    EvictWs w;
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o += align_up(bytes, 256); return at; };
    w.words = (max_len + 63) / 64;
    w.sizes = take((size_t)B * 8);
    w.stays = take((size_t)B * w.words * 8);
    w.holes = take((size_t)B * w.words * 4);
    w.movers = take((size_t)B * w.words * 4);
    w.bytes = o;
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
    a.sizes = (int2*)((char*)ws + w.sizes);
    a.stays = (unsigned long long*)((char*)ws + w.stays);
    a.holes = (int32_t*)((char*)ws + w.holes); a.movers = (int32_t*)((char*)ws + w.movers);
    a.words = w.words;
    a.k_pages = (char*)cache->k_pages; a.v_pages = (char*)cache->v_pages;
    a.row_bytes = cache->Hkv * cache->dh * elem_bytes(cache->dt);
#define D3TOM_SELECT(P) D3TOM_LAUNCH(EVICT_SELECT, st, (evict_select_kernel<P><<<cache->B, EV_THREADS, 0, st>>>(a)))
    if (max_len <= 4 * EV_THREADS) D3TOM_SELECT(4);
    else if (max_len <= 16 * EV_THREADS) D3TOM_SELECT(16);
    else D3TOM_SELECT(0);
#undef D3TOM_SELECT
    int lanes = 0;                                      // log2 of the lanes of a move: one for each 16 bytes, a wave at most
    while (lanes < 6 && (16 << lanes) < 2 * a.row_bytes) ++lanes;
    const dim3 grid(w.words, cache->B);
    D3TOM_LAUNCH(EVICT_MOVE, st, (evict_move_kernel<<<grid, 256, 0, st>>>(a, lanes)));
    return D3TOM_OK;
}
