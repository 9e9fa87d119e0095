// The key/value cache in pages: what its kernels share.  Internal, not part of the C ABI.
#pragma once
#include "common.hpp"

namespace d3tom {

// The cache as a kernel takes it.
struct CacheView {
    const int32_t* table;
    const int32_t* len;
    int num_pages, shift, table_stride, Hkv, dh;

    __device__ __forceinline__ int page_of(int b, int slot) const { return table[(size_t)b * table_stride + (slot >> shift)]; }
    // a page that is read: one that there is not counts as the last one
    __device__ __forceinline__ uint32_t readable(int page) const { return min((uint32_t)page, (uint32_t)num_pages - 1u); }
    __device__ __forceinline__ bool writable(int page) const { return (uint32_t)page < (uint32_t)num_pages; }
    // rows (of Hkv * dh elements) in front of the slot's: 64 bits, a cache may be larger than 4 GB
    __device__ __forceinline__ size_t row(uint32_t page, int slot) const { return ((size_t)page << shift) + (uint32_t)(slot & ((1 << shift) - 1)); }
    __device__ __forceinline__ size_t row_elems() const { return (size_t)Hkv * dh; }
    __device__ __forceinline__ int length(int b, int max_len) const { return min(max(len[b], 0), max_len); }
};

// x / d of numbers below 2^24, `per` = 1 / d: the float quotient is less than one off.  (The integer division is 40 instructions, and a kernel has a handful of
// them in front of its first load.)
__device__ __forceinline__ int div_by(int x, int d, float per) {
    int q = (int)((float)x * per);
    q -= q * d > x ? 1 : 0;
    q += (q + 1) * d <= x ? 1 : 0;
    return q;
}

inline CacheView cache_view(const d3tom_paged_cache& c) {
    CacheView v;
    v.table = c.page_table; v.len = c.kv_len;
    v.num_pages = c.num_pages; v.table_stride = c.table_stride; v.Hkv = c.Hkv; v.dh = c.dh;
    v.shift = 0;
    while ((1 << v.shift) < c.page_size) ++v.shift;
    return v;
}

inline int elem_bytes(int dt) { return dt == D3TOM_BF16 ? 2 : 4; }

inline int cache_check(const d3tom_paged_cache* c) {
    if (!c || !c->k_pages || !c->v_pages || !c->page_table || !c->kv_len) return D3TOM_ERR_INVALID_ARG;
    if (!aligned16(c->k_pages) || !aligned16(c->v_pages)) return D3TOM_ERR_INVALID_ARG;
    if (c->dt != D3TOM_F32 && c->dt != D3TOM_BF16) return D3TOM_ERR_INVALID_ARG;
    if (c->num_pages < 1 || c->page_size < 1 || c->table_stride < 1 || c->B < 1 || c->Hkv < 1 || c->dh < 1) return D3TOM_ERR_INVALID_ARG;
    if (c->page_size < 16 || c->page_size > 4096 || (c->page_size & (c->page_size - 1))) return D3TOM_ERR_UNSUPPORTED;
    if (c->dh > 256 || (c->dh * elem_bytes(c->dt)) % 16 || c->B > 65535 || c->Hkv > 65535) return D3TOM_ERR_UNSUPPORTED;
    return D3TOM_OK;
}

// Workgroups of a launch: a dimension of a grid has fewer than 2^32 threads, and a workgroup 256 of them.
constexpr double CACHE_MOST_GROUPS = 16000000.0;

// rows of heads * dh elements, `stride` elements apart
inline int rows_check(const void* p, int64_t stride, int heads, int dh, int dt) {
    if (!p || !aligned16(p) || heads < 1) return D3TOM_ERR_INVALID_ARG;
    if (stride < (int64_t)heads * dh || (stride * elem_bytes(dt)) % 16) return D3TOM_ERR_INVALID_ARG;
    return D3TOM_OK;
}

}  // namespace d3tom
