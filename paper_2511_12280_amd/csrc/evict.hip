// d3tom_cache_evict: a cache shortened by the attention weight that its slots have got.
//
// Order of the slots: an unsigned key per slot, all ones for a protected one, else the order-preserving image of its weight; larger
// first, equal keys by the slot.  The k-th largest key is found by counting: 2048 bins over the range that the keys have (weights are spread over
// many octaves, and the image is nearly their logarithm, so that the counts do not meet in few bins as they would in bins of a fixed number of leading
// bits), then twice over the bin that the key lies in.  Counts of integers: the order of the additions does not show.  What is left of it is a
// bit for every slot that stays, and for each word of 64 how many holes (slots below k that do not stay) and movers (slots from k on that do) lie in front
// of it: there are as many of either.
//
// A sample of up to 16384 slots is a single workgroup's, its keys in registers.  Longer caches are cut into slices with a workgroup each, in a launch for every step:
// what a step needs of all slices is small and read by every workgroup.  (One workgroup for 65521 slots took 72 us at best: a compute unit waits 2 us for a batch of
// 64 KB, four times eight batches.)
//
// The last launch has a workgroup for every word below k: it pairs the word's holes with the movers of the same numbers and moves their rows.
// Every mover lies at k or above and every hole below it, so that the moves need no order among themselves.  Bound by memory where rows are many:
// 65521 slots halved, rows of 2 KB: the moves 34 us of 63 (3.9 TB/s there and back), the selection's six launches the rest; 16 samples of 900 .. 2688 slots cut to nine
// tenths: selection 9.7 us (a workgroup to a sample, step behind step), moves 8.0.
#include "cache.hpp"

namespace d3tom {

constexpr int EV_THREADS = 1024, EV_WAVES = EV_THREADS / 64, EV_BINS = 2048, EV_LEVELS = 3;
constexpr int EV_TURNS = 4, EV_SLICE = EV_THREADS * EV_TURNS, EV_ALONE_TURNS = 16;        // of 64 slots, of a wave: in slices; of a workgroup alone, at most

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
    // of several slices: (largest number, range of the images) and (larger and equal keys below k, from k on) [B, slices]; counts [B, levels, bins]
    int slices;
    int4 *ranges, *counts;
    int32_t* bins;
    struct EvictSearch* searches;               // [B, steps]: the search behind each level
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

// the search: keys lo + (bin << shift) ..., `need` of them still to be found from the top
struct EvictSearch {
    uint32_t lo, limit, span;
    int shift, need, equal;
    int first, found;
    __device__ __forceinline__ void start(uint32_t low, uint32_t high, int k) {
        lo = low; need = k; equal = 0; limit = 0; span = 0; first = true; found = false;
        shift = high > low ? max(21 - __clz((int)(high - low)), 0) : 0;
        if (((high - low) >> shift) > EV_BINS - 2) ++shift;            // the last bin is the protected ones'
    }
    // the bin of a key, -1 for one that is out already
    __device__ __forceinline__ int bin(uint32_t key) const {
        if (first) return key == EV_PROTECTED ? EV_BINS - 1 : (int)((key - lo) >> shift);
        return key != EV_PROTECTED && key >= lo && key - lo <= span ? (int)((key - lo) >> shift) : -1;
    }
};
#if defined(__HIP_DEVICE_COMPILE__)
// What a workgroup has of its slice: turn u of wave w is slots base + (w * EV_TURNS + u) * 64 ...
template <int TURNS> struct EvictSlice {
    int base, n, k, wave, lane;
    uint32_t image[TURNS];
    int32_t token[TURNS];
    __device__ __forceinline__ int at(int u) const { return base + (wave * TURNS + u) * 64; }
    __device__ __forceinline__ unsigned long long live(int u) const { const int j = at(u); return j >= n ? 0ull : n - j >= 64 ? ~0ull : (1ull << (n - j)) - 1; }
    __device__ __forceinline__ unsigned long long low(int u) const { const int j = at(u); return j >= k ? 0ull : k - j >= 64 ? ~0ull : (1ull << (k - j)) - 1; }
    // (every slot, live or not: loads behind a branch would wait for each other)
    __device__ __forceinline__ void load(const float* w, const int32_t* tok) {
#pragma unroll
        for (int u = 0; u < TURNS; ++u) {
            const int j = min(at(u) + lane, n - 1);
            image[u] = evict_image(w[j]);
            token[u] = tok[j];
        }
    }
    __device__ __forceinline__ uint32_t key(int u, int first, long long newest) const { return token[u] < first || (long long)token[u] > newest ? EV_PROTECTED : image[u]; }
};
struct EvictLds {
    int hist[EV_BINS];
    int a[EV_WAVES], b[EV_WAVES], c[EV_WAVES];
    uint32_t lo[EV_WAVES], hi[EV_WAVES];
    int digit, above, equal;
    uint32_t list[64];
    int listed;
};
// largest number, smallest and largest image of the workgroup's lanes
__device__ __forceinline__ void evict_extremes(int& top, uint32_t& lo, uint32_t& hi, int wave, int lane, EvictLds& lds) {
    top = ev_reduce(top, [](int x, int y) { return max(x, y); });
    lo = (uint32_t)ev_reduce((int)lo, [](int x, int y) { return (int)min((uint32_t)x, (uint32_t)y); });
    hi = (uint32_t)ev_reduce((int)hi, [](int x, int y) { return (int)max((uint32_t)x, (uint32_t)y); });
    if (lane == 0) { lds.a[wave] = top; lds.lo[wave] = lo; lds.hi[wave] = hi; }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < EV_WAVES; ++i) { top = max(top, lds.a[i]); lo = min(lo, lds.lo[i]); hi = max(hi, lds.hi[i]); }
}
// One step of the search: counts h1, h0 of this thread's two bins, from the last one down.  A barrier in front of it separates it from the use of lds.a before.
__device__ __forceinline__ void evict_step(EvictSearch& s, int h1, int h0, int tid, EvictLds& lds) {
    const int wave = tid >> 6, sum = wave_incl_scan(h1 + h0);
    if ((tid & 63) == 63) lds.a[wave] = sum;
    __syncthreads();
    int above = sum - h1 - h0;
#pragma unroll
    for (int i = 0; i < EV_WAVES; ++i) above += i < wave ? lds.a[i] : 0;
    if (above < s.need && s.need <= above + h1) { lds.digit = EV_BINS - 1 - 2 * tid; lds.above = above; lds.equal = h1; }
    else if (above + h1 < s.need && s.need <= above + h1 + h0) { lds.digit = EV_BINS - 2 - 2 * tid; lds.above = above + h1; lds.equal = h0; }
    __syncthreads();
    const int digit = lds.digit;
    s.need -= lds.above;
    s.equal = lds.equal;
    if (s.first && digit == EV_BINS - 1) { s.limit = EV_PROTECTED; s.found = true; return; }
    s.lo += (uint32_t)digit << s.shift;
    if (s.shift == 0) { s.limit = s.lo; s.found = true; return; }
    s.span = (1u << s.shift) - 1;
    s.shift = max(s.shift - 11, 0);
    s.first = false;
}
// The slice's words.  tied: keys equal to the limit in front of the slice, of which the first `need` stay; nh, nm: holes and movers in front of it.
template <int TURNS>
__device__ __forceinline__ void evict_words(const EvictArgs& a, const EvictSlice<TURNS>& sl, int b, uint32_t limit, int need, int equal, long long newest, int tied, int nh, int nm, EvictLds& lds) {
    const int wave = sl.wave, lane = sl.lane;
    const bool count_ties = need < equal;
    if (count_ties) {
        int mine = 0;
#pragma unroll
        for (int u = 0; u < TURNS; ++u) mine += __popcll(__builtin_amdgcn_ballot_w64(sl.key(u, a.first, newest) == limit) & sl.live(u));
        __syncthreads();
        if (lane == 0) lds.a[wave] = mine;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < EV_WAVES; ++i) tied += i < wave ? lds.a[i] : 0;
    }
    unsigned long long my_word = 0;
    int h = 0, m = 0, my_h = 0, my_m = 0;
#pragma unroll
    for (int u = 0; u < TURNS; ++u) {
        const uint32_t key = sl.key(u, a.first, newest);
        const unsigned long long live = sl.live(u), low = sl.low(u);
        unsigned long long word = __builtin_amdgcn_ballot_w64(key >= limit) & live;
        if (count_ties) {
            unsigned long long same = __builtin_amdgcn_ballot_w64(key == limit) & live;
            const int there = __popcll(same), allowed = min(max(need - tied, 0), there);
            tied += there;
            word &= ~same;
            for (int i = there; i > allowed; --i) same &= ~(1ull << (63 - __clzll((long long)same)));
            word |= same;
        }
        if (lane == u) { my_word = word; my_h = h; my_m = m; }      // lane u keeps what belongs to turn u
        h += __popcll(low & ~word);
        m += __popcll(word & ~low);
    }
    if (lane == 0) { lds.b[wave] = h; lds.c[wave] = m; }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < EV_WAVES; ++i) { nh += i < wave ? lds.b[i] : 0; nm += i < wave ? lds.c[i] : 0; }
    if (lane < TURNS && sl.at(lane) < sl.n) {
        const size_t to = (size_t)b * a.words + sl.at(lane) / 64;
        a.stays[to] = my_word;
        a.holes[to] = my_h + nh;
        a.movers[to] = my_m + nm;
    }
}
#endif

// everything in one workgroup, 1024 TURNS slots at most
template <int TURNS>
__global__ __launch_bounds__(EV_THREADS) void evict_select_kernel(EvictArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    __shared__ EvictLds lds;
    const int tid = threadIdx.x, b = blockIdx.x;
    EvictSlice<TURNS> sl;
    sl.base = 0; sl.wave = __builtin_amdgcn_readfirstlane(tid >> 6); sl.lane = tid & 63;
    sl.n = a.cache.length(b, a.max_len);
    sl.k = min(max(a.keep[b], 0), sl.n);
    if (tid == 0) a.sizes[b] = make_int2(sl.n, sl.k);
    if (sl.n == 0) return;
    sl.load(a.weight_in + (size_t)b * a.stride, a.token_in + (size_t)b * a.stride);
    int top = sl.token[0];
    uint32_t lo = sl.image[0], hi = sl.image[0];
#pragma unroll
    for (int u = 1; u < TURNS; ++u) { top = max(top, sl.token[u]); lo = min(lo, sl.image[u]); hi = max(hi, sl.image[u]); }
    lds.hist[tid] = 0;
    lds.hist[tid + EV_THREADS] = 0;
    evict_extremes(top, lo, hi, sl.wave, sl.lane, lds);
    const long long newest = (long long)top - a.recent;
    // all stay, or none, unless the k-th key says which
    uint32_t limit = sl.k > 0 ? 0u : EV_PROTECTED;
    int need = 0, equal = sl.k > 0 ? 0 : sl.n + 1;
    if (sl.k > 0 && sl.k < sl.n) {
        EvictSearch s;
        s.start(lo, hi, sl.k);
        while (!s.found) {
#pragma unroll
            for (int u = 0; u < TURNS; ++u) {
                const int bin = s.bin(sl.key(u, a.first, newest));
                if (((sl.live(u) >> sl.lane) & 1) && bin >= 0) atomicAdd(&lds.hist[bin], 1);
            }
            __syncthreads();
            const int h1 = lds.hist[EV_BINS - 1 - 2 * tid], h0 = lds.hist[EV_BINS - 2 - 2 * tid];
            lds.hist[EV_BINS - 1 - 2 * tid] = 0;        // (its own two, for the next time)
            lds.hist[EV_BINS - 2 - 2 * tid] = 0;
            evict_step(s, h1, h0, tid, lds);
            if (TURNS > EV_TURNS && !s.found && s.equal <= 64) {
                // The bin's keys, in no order, one to a lane of every wave: bit by bit, those with the bit are in front.  Instead of further passes over all slots:
                // a call for one sample of 4200, 8192 and 16384 slots 22.9, 27.7 and 24.6 us with the passes, 21.1, 26.2 and 23.2 with this.  With 4 turns a pass is
                // short and this the longer way (selection in 16 samples of 900 .. 2688 slots: 9.7 us with the passes, 10.2 with this).
                if (tid == 0) lds.listed = 0;
                __syncthreads();
#pragma unroll
                for (int u = 0; u < TURNS; ++u) {
                    const uint32_t key = sl.key(u, a.first, newest);
                    if (((sl.live(u) >> sl.lane) & 1) && s.bin(key) >= 0) lds.list[atomicAdd(&lds.listed, 1)] = key;
                }
                __syncthreads();
                const uint32_t rest = lds.list[sl.lane] - s.lo;
                unsigned long long left = s.equal == 64 ? ~0ull : (1ull << s.equal) - 1;
                uint32_t found = 0;
                for (int bit = 31 - __clz((int)s.span); bit >= 0; --bit) {
                    const unsigned long long ones = __builtin_amdgcn_ballot_w64((rest >> bit) & 1) & left;
                    const int count = __popcll(ones);
                    if (count >= s.need) { left = ones; found |= 1u << bit; }
                    else { s.need -= count; left &= ~ones; }
                }
                s.limit = s.lo + found;
                s.equal = __popcll(left);
                s.found = 1;
            }
        }
        limit = s.limit; need = s.need; equal = s.equal;
    }
    evict_words(a, sl, b, limit, need, equal, newest, 0, 0, 0, lds);
#endif
}

// Several slices.  STEP 0: the slice's extremes, and the sample's counts cleared.  1 .. EV_LEVELS: the bins of that level counted, behind the search through the levels before.
// EV_LEVELS + 1: larger and equal keys of the slice.  EV_LEVELS + 2: its words.
template <int STEP>
__global__ __launch_bounds__(EV_THREADS) void evict_slices_kernel(EvictArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    __shared__ EvictLds lds;
    const int tid = threadIdx.x, slice = blockIdx.x, b = blockIdx.y;
    EvictSlice<EV_TURNS> sl;
    sl.base = slice * EV_SLICE; sl.wave = __builtin_amdgcn_readfirstlane(tid >> 6); sl.lane = tid & 63;
    sl.n = a.cache.length(b, a.max_len);
    sl.k = min(max(a.keep[b], 0), sl.n);
    int32_t* bins = a.bins + (size_t)b * EV_LEVELS * EV_BINS;
    if (STEP == 0) {
        for (int i = slice * EV_THREADS + tid; i < EV_LEVELS * EV_BINS; i += a.slices * EV_THREADS) bins[i] = 0;
        if (slice == 0 && tid == 0) a.sizes[b] = make_int2(sl.n, sl.k);
    }
    const int slices = (sl.n + EV_SLICE - 1) / EV_SLICE;               // that the sample has
    if (slice >= slices) return;
    sl.load(a.weight_in + (size_t)b * a.stride, a.token_in + (size_t)b * a.stride);
    int4* ranges = a.ranges + (size_t)b * a.slices;
    int top;
    uint32_t lo, hi;
    if (STEP == 0) {
        top = sl.token[0];
        lo = hi = sl.image[0];
#pragma unroll
        for (int u = 1; u < EV_TURNS; ++u) { top = max(top, sl.token[u]); lo = min(lo, sl.image[u]); hi = max(hi, sl.image[u]); }
    } else {
        const int4 r = ranges[min(tid, slices - 1)];                   // (256 slices at most)
        top = r.x; lo = (uint32_t)r.y; hi = (uint32_t)r.z;
    }
    evict_extremes(top, lo, hi, sl.wave, sl.lane, lds);
    if (STEP == 0) {
        if (tid == 0) ranges[slice] = make_int4(top, (int)lo, (int)hi, 0);
        return;
    }
    const long long newest = (long long)top - a.recent;
    uint32_t limit = sl.k > 0 ? 0u : EV_PROTECTED;
    int need = 0, equal = sl.k > 0 ? 0 : sl.n + 1;
    EvictSearch s;
    s.start(lo, hi, sl.k);
    s.found = !(sl.k > 0 && sl.k < sl.n);
    if (!s.found) {
        // the search as the launch before left it, and through the level that it counted
        constexpr int LEVEL = STEP - 2;
        EvictSearch* saved = a.searches + (size_t)b * EV_LEVELS;
        if (LEVEL >= 0 && LEVEL < EV_LEVELS) {
            const int h1 = bins[LEVEL * EV_BINS + EV_BINS - 1 - 2 * tid], h0 = bins[LEVEL * EV_BINS + EV_BINS - 2 - 2 * tid];
            if (LEVEL > 0) s = saved[LEVEL > 0 ? LEVEL - 1 : 0];
            if (!s.found) {
                __syncthreads();
                evict_step(s, h1, h0, tid, lds);
            }
            if (slice == 0 && tid == 0) saved[LEVEL < EV_LEVELS ? LEVEL : 0] = s;
        } else if (LEVEL >= EV_LEVELS) {
            s = saved[EV_LEVELS - 1];
        }
        limit = s.limit; need = s.need; equal = s.equal;
    }
    if (STEP <= EV_LEVELS) {
        if (s.found) return;
        lds.hist[tid] = 0;
        lds.hist[tid + EV_THREADS] = 0;
        __syncthreads();
#pragma unroll
        for (int u = 0; u < EV_TURNS; ++u) {
            const int bin = s.bin(sl.key(u, a.first, newest));
            if (((sl.live(u) >> sl.lane) & 1) && bin >= 0) atomicAdd(&lds.hist[bin], 1);
        }
        __syncthreads();
        for (int i = tid; i < EV_BINS; i += EV_THREADS)
            if (lds.hist[i]) atomicAdd(&bins[(STEP - 1) * EV_BINS + i], lds.hist[i]);
        return;
    }
    int4* counts = a.counts + (size_t)b * a.slices;
    if (STEP == EV_LEVELS + 1) {
        int more = 0, same = 0, more_high = 0, same_high = 0;
#pragma unroll
        for (int u = 0; u < EV_TURNS; ++u) {
            const uint32_t key = sl.key(u, a.first, newest);
            const unsigned long long live = sl.live(u), low = sl.low(u);
            const unsigned long long m = __builtin_amdgcn_ballot_w64(key > limit) & live, t = __builtin_amdgcn_ballot_w64(key == limit) & live;
            more += __popcll(m & low); more_high += __popcll(m & ~low);
            same += __popcll(t & low); same_high += __popcll(t & ~low);
        }
        __syncthreads();
        if (sl.lane == 0) { lds.a[sl.wave] = more; lds.b[sl.wave] = same; lds.c[sl.wave] = more_high; lds.lo[sl.wave] = (uint32_t)same_high; }
        __syncthreads();
        if (tid == 0) {
            int4 c = make_int4(0, 0, 0, 0);
            for (int i = 0; i < EV_WAVES; ++i) { c.x += lds.a[i]; c.y += lds.b[i]; c.z += lds.c[i]; c.w += (int)lds.lo[i]; }
            counts[slice] = c;
        }
        return;
    }
    // Larger and equal keys in front of the slice; of the equal ones the first `need` stay, so that holes and movers follow from them.
    const int4 c = tid < slice ? counts[tid] : make_int4(0, 0, 0, 0);
    int more = c.x, same = c.y, more_high = c.z, same_high = c.w;
    auto add = [](int x, int y) { return x + y; };
    more = ev_reduce(more, add); same = ev_reduce(same, add); more_high = ev_reduce(more_high, add); same_high = ev_reduce(same_high, add);
    __syncthreads();
    if (sl.lane == 0) { lds.a[sl.wave] = more; lds.b[sl.wave] = same; lds.c[sl.wave] = more_high; lds.lo[sl.wave] = (uint32_t)same_high; }
    __syncthreads();
    more = same = more_high = same_high = 0;
#pragma unroll
    for (int i = 0; i < EV_WAVES; ++i) { more += lds.a[i]; same += lds.b[i]; more_high += lds.c[i]; same_high += (int)lds.lo[i]; }
    const bool all = sl.k == sl.n, none = sl.k == 0;
    const int before = min(sl.base, sl.k), kept = all ? before : none ? 0 : more + min(need, same);              // slots below k in front, those that stay
    const int moved = all || none ? 0 : more_high + min(need, same + same_high) - min(need, same);
    __syncthreads();
    evict_words(a, sl, b, limit, need, equal, newest, same + same_high, before - kept, moved, lds);
#endif
}

// The word's moves, as one sequence of 16-byte chunks (a row of k and the one of v behind it, move after move): EV_AT_ONCE of them to a thread at once.  And
// what the word's slots keep of numbers.  len_out may be the cache's lengths: nothing reads them any more.
constexpr int EV_AT_ONCE = 4, EV_MOVE_THREADS = 512;
typedef uint32_t ev_u32x4 __attribute__((ext_vector_type(4)));
__global__ __launch_bounds__(EV_MOVE_THREADS) void evict_move_kernel(EvictArgs a, float per_chunks) {
    __shared__ int from_s[64], to_s[64], found_w[64], found_m[64], s_found;
    __shared__ unsigned long long found_bits[64];
    __shared__ size_t from_at[64], to_at[64];
    const int b = blockIdx.y, tid = threadIdx.x;
    const int2 size = a.sizes[b];
    const int n = size.x, k = size.y, word = blockIdx.x, slot0 = word * 64;
    if (word == 0 && tid == 0) a.len_out[b] = k;
    if (slot0 >= k) return;
    const size_t row = (size_t)b * a.words, at = (size_t)b * a.stride;
    const unsigned long long low = k - slot0 >= 64 ? ~0ull : (1ull << (k - slot0)) - 1, stay = a.stays[row + word] & low, hole = low & ~stay;
    const int h0 = a.holes[row + word], count = __popcll(hole);
    // Words that have some of movers h0 .. h0 + count - 1 (each has at least one: 64 at most), a thread to a word from k on.  The last ones' movers end with the holes.
    const int w0 = k >> 6, w1 = (n - 1) >> 6;
    if (tid == 0) s_found = 0;
    __syncthreads();
    for (int w = w0 + tid; w <= w1; w += EV_MOVE_THREADS) {
        const unsigned long long low_w = k - w * 64 >= 64 ? ~0ull : k <= w * 64 ? 0ull : (1ull << (k - w * 64)) - 1;
        const int m = a.movers[row + w];
        const unsigned long long movers = a.stays[row + w] & ~low_w;
        if (movers && m < h0 + count && m + __popcll(movers) > h0) {
            const int i = atomicAdd(&s_found, 1);       // (in no order: every mover has its own place)
            found_w[i] = w; found_m[i] = m; found_bits[i] = movers;
        }
    }
    if (tid < 64) {
        const int j = slot0 + tid;
        if ((stay >> tid) & 1) {
            a.weight_out[at + j] = a.weight_in[at + j];
            a.token_out[at + j] = a.token_in[at + j];
            if (a.src) a.src[at + j] = j;
        }
        if ((hole >> tid) & 1) to_s[__popcll(hole & ((1ull << tid) - 1))] = j;
    }
    __syncthreads();
    const int lane = tid & 63;
    for (int i = tid >> 6; i < s_found; i += EV_MOVE_THREADS / 64) {       // a wave to a word
        const unsigned long long movers = found_bits[i];
        const int rank = found_m[i] - h0 + __popcll(movers & ((1ull << lane) - 1));
        if (((movers >> lane) & 1) && rank >= 0 && rank < count) from_s[rank] = found_w[i] * 64 + lane;
    }
    __syncthreads();
    if (tid < count) {
        const int to = to_s[tid], from = from_s[tid], pt = a.cache.page_of(b, to), pf = a.cache.page_of(b, from);
        to_at[tid] = a.cache.writable(pt) ? a.cache.row((uint32_t)pt, to) * a.row_bytes : ~(size_t)0;
        from_at[tid] = a.cache.row(a.cache.readable(pf), from) * a.row_bytes;
        a.weight_out[at + to] = a.weight_in[at + from];
        a.token_out[at + to] = a.token_in[at + from];
        if (a.src) a.src[at + to] = from;
    }
    __syncthreads();
    const int half = a.row_bytes / 16, chunks = 2 * half;
    // (64 moves of rows of 64 MB at most: groups of moves whose chunks are below 2^24)
    const int group = max(1, min(count, (1 << 24) / chunks - 1));
    for (int i0 = 0; i0 < count; i0 += group) {
        const int total = min(group, count - i0) * chunks;
        for (int x0 = tid; x0 < total; x0 += EV_MOVE_THREADS * EV_AT_ONCE) {
            ev_u32x4 v[EV_AT_ONCE];
            char* dst[EV_AT_ONCE];
#pragma unroll
            for (int u = 0; u < EV_AT_ONCE; ++u) {
                const int x = min(x0 + u * EV_MOVE_THREADS, total - 1), i = div_by(x, chunks, per_chunks), c = x - i * chunks;
                char* pages = (c < half ? a.k_pages : a.v_pages) + (size_t)(c < half ? c : c - half) * 16;
                const size_t to = to_at[i0 + i];
                dst[u] = to == ~(size_t)0 || x0 + u * EV_MOVE_THREADS >= total ? nullptr : pages + to;
                v[u] = *reinterpret_cast<const ev_u32x4*>(pages + from_at[i0 + i]);
            }
#pragma unroll
            for (int u = 0; u < EV_AT_ONCE; ++u)
                if (dst[u]) *reinterpret_cast<ev_u32x4*>(dst[u]) = v[u];
        }
    }
}

struct EvictWs { size_t sizes, stays, holes, movers, ranges, counts, bins, searches, bytes; int words, slices; };
static EvictWs evict_ws(int B, int max_len) {
    EvictWs w;
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o += align_up(bytes, 256); return at; };
    w.words = (max_len + 63) / 64;
    w.slices = max_len <= EV_ALONE_TURNS * EV_THREADS ? 1 : (max_len + EV_SLICE - 1) / EV_SLICE;
    const size_t more = w.slices > 1 ? (size_t)B : 0;
    w.sizes = take((size_t)B * 8);
    w.stays = take((size_t)B * w.words * 8);
    w.holes = take((size_t)B * w.words * 4);
    w.movers = take((size_t)B * w.words * 4);
    w.ranges = take(more * w.slices * 16);
    w.counts = take(more * w.slices * 16);
    w.bins = take(more * EV_LEVELS * EV_BINS * 4);
    w.searches = take(more * EV_LEVELS * sizeof(EvictSearch));
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
    a.slices = w.slices;
    a.ranges = (int4*)((char*)ws + w.ranges); a.counts = (int4*)((char*)ws + w.counts); a.bins = (int32_t*)((char*)ws + w.bins);
    a.searches = (EvictSearch*)((char*)ws + w.searches);
    a.k_pages = (char*)cache->k_pages; a.v_pages = (char*)cache->v_pages;
    a.row_bytes = cache->Hkv * cache->dh * elem_bytes(cache->dt);
    if (max_len <= EV_SLICE) {
        D3TOM_LAUNCH(EVICT_SELECT, st, (evict_select_kernel<EV_TURNS><<<cache->B, EV_THREADS, 0, st>>>(a)));
    } else if (w.slices == 1) {
        D3TOM_LAUNCH(EVICT_SELECT, st, (evict_select_kernel<EV_ALONE_TURNS><<<cache->B, EV_THREADS, 0, st>>>(a)));
    } else {
        static_assert(EV_LEVELS == 3 && D3TOM_MAX_EVICT_LEN <= EV_THREADS * EV_SLICE, "the launches below; a thread for every slice");
        const dim3 grid(w.slices, cache->B);
#define D3TOM_STEP(N) D3TOM_LAUNCH(EVICT_SELECT, st, (evict_slices_kernel<N><<<grid, EV_THREADS, 0, st>>>(a)))
        D3TOM_STEP(0); D3TOM_STEP(1); D3TOM_STEP(2); D3TOM_STEP(3); D3TOM_STEP(4); D3TOM_STEP(5);
#undef D3TOM_STEP
    }
    const dim3 grid(w.words, cache->B);
    D3TOM_LAUNCH(EVICT_MOVE, st, (evict_move_kernel<<<grid, EV_MOVE_THREADS, 0, st>>>(a, 8.0f / (float)a.row_bytes)));
    return D3TOM_OK;
}
