// d3tom_cache_evict: a cache shortened by the attention weight that its slots have got.
//
// Order of the slots: an unsigned key per slot, all ones for a protected one, else the order-preserving image of its weight; larger
// first, equal keys by the slot.  One workgroup per sample finds the k-th largest key by counting: 2048 bins over the range that the keys
// have (weights are spread over many octaves, and the image is nearly their logarithm, so that the counts do not meet in few bins as they would in bins of a
// fixed number of leading bits), then over the bin that the key lies in, at most three times.  Counts of integers: the order of the additions does not
// show.  Slots in ascending order, the holes (slots below k that do not stay) and the movers (slots from k on that do) are then numbered:
// there are as many of either.  A second launch moves the rows and their numbers: every mover lies at k or above and every hole below it, so
// that the moves need no order among themselves.
//
// The selection has one compute unit per sample; its keys stay in registers up to 65536 slots and are formed again in every turn beyond that.
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
    // workspace: moves and kept counts [B], whether each slot stays, 64 to a word [B, words], holes and movers [B, room]
    int32_t *moves, *kept;
    unsigned long long* stays;
    int32_t *holes, *movers;
    int words, room;
    char *k_pages, *v_pages;
    int row_bytes;
};

constexpr uint32_t EV_PROTECTED = 0xFFFFFFFFu;
__device__ __forceinline__ uint32_t evict_key(float w, int token, int first, long long newest) {
    if (token < first || (long long)token > newest) return EV_PROTECTED;
    const uint32_t u = __float_as_uint(w + 0.f);        // -0 is 0
    return min((u & 0x80000000u) ? ~u : (u | 0x80000000u), EV_PROTECTED - 1u);
}

// P: keys of a thread in registers, 64 slots to a wave and turn; 0: any number, formed again each time
template <int P>
__global__ __launch_bounds__(EV_THREADS) void evict_select_kernel(EvictArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    __shared__ int hist[EV_BINS];
    __shared__ int wave_a[EV_WAVES], wave_b[EV_WAVES];
    __shared__ uint32_t wave_lo[EV_WAVES], wave_hi[EV_WAVES];
    __shared__ int s_digit, s_above;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), b = blockIdx.x;
    const int n = a.cache.length(b, a.max_len);
    const int k = min(max(a.keep[b], 0), n);
    const float* w = a.weight_in + (size_t)b * a.stride;
    const int32_t* tok = a.token_in + (size_t)b * a.stride;
    const int turns = (n + EV_THREADS - 1) / EV_THREADS, j0 = wave * turns * 64 + lane;       // a wave has consecutive slots
    auto each = [&](auto&& f) {
        if constexpr (P > 0) {
#pragma unroll
            for (int u = 0; u < P; ++u)
                if (u < turns) f(u);
        } else {
            for (int u = 0; u < turns; ++u) f(u);
        }
    };
    // the last number that is not protected as recent
    int top = INT32_MIN;
    each([&](int u) { const int j = j0 + u * 64; top = max(top, j < n ? tok[j] : INT32_MIN); });
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = max(top, __shfl_xor(top, o));
    if (lane == 0) wave_a[wave] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < EV_WAVES; ++i) top = max(top, wave_a[i]);
    const long long newest = (long long)top - a.recent;

    uint32_t keys[P > 0 ? P : 1];
    if constexpr (P > 0) each([&](int u) { const int j = min(j0 + u * 64, n - 1); keys[u] = evict_key(w[j], tok[j], a.first, newest); });
    auto key_of = [&](int u) {
        if constexpr (P > 0) return keys[u];
        else { const int j = min(j0 + u * 64, n - 1); return evict_key(w[j], tok[j], a.first, newest); }
    };
    // the k-th largest key, and how many of the keys equal to it stay
    uint32_t limit = 0;
    int need = 0;
    if (k > 0 && k < n) {
        uint32_t lo = EV_PROTECTED, hi = 0;             // of the unprotected keys
        each([&](int u) {
            const uint32_t key = key_of(u);
            if (key != EV_PROTECTED) { lo = min(lo, key); hi = max(hi, key); }
        });
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) { lo = min(lo, (uint32_t)__shfl_xor((int)lo, o)); hi = max(hi, (uint32_t)__shfl_xor((int)hi, o)); }
        if (lane == 0) { wave_lo[wave] = lo; wave_hi[wave] = hi; }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < EV_WAVES; ++i) { lo = min(lo, wave_lo[i]); hi = max(hi, wave_hi[i]); }
        if (lo > hi) lo = hi = 0;                       // all are protected
        int shift = 0;
        while (((hi - lo) >> shift) > EV_BINS - 2) ++shift;
        bool first = true;
        need = k;
        uint32_t span = 0;                              // of the keys that are left, behind the first turn
        while (true) {
            hist[tid] = 0;
            hist[tid + EV_THREADS] = 0;
            __syncthreads();
            each([&](int u) {
                const uint32_t key = key_of(u), at = key - lo;
                const int bin = first && key == EV_PROTECTED ? EV_BINS - 1 : (int)(at >> shift);
                if (j0 + u * 64 < n && (first || (key != EV_PROTECTED && key >= lo && at <= span))) atomicAdd(&hist[bin], 1);
            });
            __syncthreads();
            // counts from the last bin down: a thread has two
            const int h1 = hist[EV_BINS - 1 - 2 * tid], h0 = hist[EV_BINS - 2 - 2 * tid];
            const int sum = wave_incl_scan(h1 + h0);
            if (lane == 63) wave_a[wave] = sum;
            __syncthreads();
            int above = sum - h1 - h0;
#pragma unroll
            for (int i = 0; i < EV_WAVES; ++i) above += i < wave ? wave_a[i] : 0;
            if (above < need && need <= above + h1) { s_digit = EV_BINS - 1 - 2 * tid; s_above = above; }
            else if (above + h1 < need && need <= above + h1 + h0) { s_digit = EV_BINS - 2 - 2 * tid; s_above = above + h1; }
            __syncthreads();
            const int digit = s_digit;
            need -= s_above;
            if (first && digit == EV_BINS - 1) { limit = EV_PROTECTED; break; }
            lo += (uint32_t)digit << shift;
            if (shift == 0) { limit = lo; break; }
            span = (1u << shift) - 1;
            shift = max(shift - 11, 0);
            first = false;
        }
    }
    // slots that stay, holes and movers, in ascending order
    const bool all = k == n, none = k == 0;
    int ties = 0;
    if (!all && !none) {
        each([&](int u) { ties += __popcll(__builtin_amdgcn_ballot_w64(j0 + u * 64 < n && key_of(u) == limit)); });
        __syncthreads();
        if (lane == 0) wave_a[wave] = ties;
        __syncthreads();
        ties = 0;
#pragma unroll
        for (int i = 0; i < EV_WAVES; ++i) ties += i < wave ? wave_a[i] : 0;
    }
    const unsigned long long below = (1ull << lane) - 1;
    auto stays = [&](int u, int& tied) {                // whether this lane's slot of turn u stays; tied: equal keys in front of the turn
        const int j = j0 + u * 64;
        if (all) return j < n;
        if (none) return false;
        const uint32_t key = key_of(u);
        const bool tie = j < n && key == limit;
        const unsigned long long t = __builtin_amdgcn_ballot_w64(tie);
        const int rank = tied + __popcll(t & below);
        tied += __popcll(t);
        return j < n && (key > limit || (tie && rank < need));
    };
    int nh = 0, nm = 0, tied = ties;
    unsigned long long* bits = a.stays + (size_t)b * a.words + wave * turns;
    each([&](int u) {
        const int j = j0 + u * 64;
        const bool st = stays(u, tied);
        const unsigned long long word = __builtin_amdgcn_ballot_w64(st);
        if (lane == 0 && j < n) bits[u] = word;
        nh += __popcll(__builtin_amdgcn_ballot_w64(j < k && !st));
        nm += __popcll(__builtin_amdgcn_ballot_w64(j >= k && st));
    });
    __syncthreads();
    if (lane == 0) { wave_a[wave] = nh; wave_b[wave] = nm; }
    __syncthreads();
    int moves = 0;
    nh = nm = 0;
#pragma unroll
    for (int i = 0; i < EV_WAVES; ++i) { nh += i < wave ? wave_a[i] : 0; nm += i < wave ? wave_b[i] : 0; moves += wave_a[i]; }
    int32_t *holes = a.holes + (size_t)b * a.room, *movers = a.movers + (size_t)b * a.room;
    tied = ties;
    each([&](int u) {
        const int j = j0 + u * 64;
        const bool st = stays(u, tied), hole = j < k && !st, mover = j >= k && st;
        const unsigned long long h = __builtin_amdgcn_ballot_w64(hole), m = __builtin_amdgcn_ballot_w64(mover);
        if (hole) holes[nh + __popcll(h & below)] = j;
        if (mover) movers[nm + __popcll(m & below)] = j;
        nh += __popcll(h);
        nm += __popcll(m);
    });
    if (tid == 0) { a.moves[b] = moves; a.kept[b] = k; }
#endif
}

// The moves: EV_AT_ONCE of them (or of as many as a workgroup has threads for) are requested together.  And what the staying slots below the
// new end keep.  len_out may be the cache's lengths: nothing reads them any more.
constexpr int EV_AT_ONCE = 4;
__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a) {
    const int b = blockIdx.y, tid = threadIdx.x, moves = a.moves[b], k = a.kept[b];
    const float* w = a.weight_in + (size_t)b * a.stride;
    const int32_t* tok = a.token_in + (size_t)b * a.stride;
    float* w_out = a.weight_out + (size_t)b * a.stride;
    int32_t* t_out = a.token_out + (size_t)b * a.stride;
    int32_t* src = a.src ? a.src + (size_t)b * a.stride : nullptr;
    const unsigned long long* bits = a.stays + (size_t)b * a.words;
    const int32_t *holes = a.holes + (size_t)b * a.room, *movers = a.movers + (size_t)b * a.room;
    if (blockIdx.x == 0 && tid == 0) a.len_out[b] = k;
    for (int j = blockIdx.x * 256 + tid; j < k; j += gridDim.x * 256)
        if ((bits[j >> 6] >> (j & 63)) & 1) {
            w_out[j] = w[j];
            t_out[j] = tok[j];
            if (src) src[j] = j;
        }
    for (int i = blockIdx.x * 256 + tid; i < moves; i += gridDim.x * 256) {
        const int to = holes[i], from = movers[i];
        w_out[to] = w[from];
        t_out[to] = tok[from];
        if (src) src[to] = from;
    }
    // a row of k and the one of v behind it: `chunks` of 16 bytes
    const int half = a.row_bytes / 16, chunks = 2 * half;
    const int per = chunks >= 256 ? 1 : 256 / chunks, mine = chunks >= 256 ? 0 : tid / chunks, c0 = chunks >= 256 ? tid : tid - mine * chunks;
    if (mine >= per) return;
    for (int i0 = blockIdx.x * per * EV_AT_ONCE; i0 < moves; i0 += gridDim.x * per * EV_AT_ONCE) {
        size_t to[EV_AT_ONCE], from[EV_AT_ONCE];
        bool there[EV_AT_ONCE];
#pragma unroll
        for (int u = 0; u < EV_AT_ONCE; ++u) {
            const int i = i0 + u * per + mine, ic = min(i, moves - 1);
            const int h = holes[ic], m = movers[ic];
            const int pt = a.cache.page_of(b, h), pf = a.cache.page_of(b, m);
            there[u] = i < moves && a.cache.writable(pt);
            to[u] = a.cache.row(a.cache.readable(pt), h) * a.row_bytes;
            from[u] = a.cache.row(a.cache.readable(pf), m) * a.row_bytes;
        }
        for (int c = c0; c < chunks; c += 256) {
            char* pages = c < half ? a.k_pages : a.v_pages;
            const int at = (c < half ? c : c - half) * 16;
            uint4 v[EV_AT_ONCE];
#pragma unroll
            for (int u = 0; u < EV_AT_ONCE; ++u) v[u] = *reinterpret_cast<const uint4*>(pages + from[u] + at);
#pragma unroll
            for (int u = 0; u < EV_AT_ONCE; ++u)
                if (there[u]) *reinterpret_cast<uint4*>(pages + to[u] + at) = v[u];
        }
    }
}

struct EvictWs { size_t moves, kept, stays, holes, movers, bytes; int words, room; };
static EvictWs evict_ws(int B, int max_len) {
    EvictWs w;
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o += align_up(bytes, 256); return at; };
    w.words = (max_len + EV_THREADS - 1) / EV_THREADS * EV_WAVES;
    w.room = max_len / 2 > 1 ? max_len / 2 : 1;
    w.moves = take((size_t)B * 4);
    w.kept = take((size_t)B * 4);
    w.stays = take((size_t)B * w.words * 8);
    w.holes = take((size_t)B * w.room * 4);
    w.movers = take((size_t)B * w.room * 4);
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
    a.moves = (int32_t*)((char*)ws + w.moves); a.kept = (int32_t*)((char*)ws + w.kept);
    a.stays = (unsigned long long*)((char*)ws + w.stays);
    a.holes = (int32_t*)((char*)ws + w.holes); a.movers = (int32_t*)((char*)ws + w.movers);
    a.words = w.words; a.room = w.room;
    a.k_pages = (char*)cache->k_pages; a.v_pages = (char*)cache->v_pages;
    a.row_bytes = cache->Hkv * cache->dh * elem_bytes(cache->dt);
#define D3TOM_SELECT(P) D3TOM_LAUNCH(EVICT_SELECT, st, (evict_select_kernel<P><<<cache->B, EV_THREADS, 0, st>>>(a)))
    if (max_len <= 4 * EV_THREADS) D3TOM_SELECT(4);
    else if (max_len <= 16 * EV_THREADS) D3TOM_SELECT(16);
    else if (max_len <= 64 * EV_THREADS) D3TOM_SELECT(64);
    else D3TOM_SELECT(0);
#undef D3TOM_SELECT
    const int chunks = a.row_bytes / 8, at_once = EV_AT_ONCE * (chunks >= 256 ? 1 : 256 / chunks);
    const int units = (max_len + 255) / 256 > (w.room + at_once - 1) / at_once ? (max_len + 255) / 256 : (w.room + at_once - 1) / at_once;
    const int each = 4096 / cache->B + 1;
    const dim3 grid(units < each ? units : each, cache->B);
    D3TOM_LAUNCH(EVICT_MOVE, st, (evict_move_kernel<<<grid, 256, 0, st>>>(a)));
    return D3TOM_OK;
}
