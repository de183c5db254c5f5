// What the kernels over the 8-bit paged cache share: its view on the device and the checks of what its tables hold.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "flat_internal.cuh"

namespace flat {
namespace cache {

constexpr int MIN_EXP = -117;                            // (the least e4m3 number times 2^-117 is the least normal bf16 number)

struct CacheView {
    uint8_t *k, *v, *k_exp, *v_exp;
    const int32_t *table, *cu, *lens;
    int num_pages, Hkv, page, page_shift, num_seqs, max_pages;
    int32_t* status;
};
inline CacheView cache_view(const flat_attn_cache_t& c) {
    int shift = 0;
    while ((1 << shift) < c.page) ++shift;
    return CacheView{static_cast<uint8_t*>(c.k_cache), static_cast<uint8_t*>(c.v_cache), c.k_exp, c.v_exp, c.page_table, c.cu_seqlens, c.seq_lens,
                     c.num_pages, c.Hkv, c.page, shift, c.num_seqs, c.max_pages, c.status};
}

// A sequence's new tokens q0 .. q0 + n - 1 and its length.
struct Span {
    int q0, n, len;
};
__device__ __forceinline__ bool read_span(const CacheView& c, int s, int64_t total, int max_new, Span& sp) {
    const int q0 = c.cu[s], q1 = c.cu[s + 1], len = c.lens[s];
    const int64_t n = static_cast<int64_t>(q1) - q0;
    sp = Span{q0, static_cast<int>(n), len};
    if (q0 >= 0 && n >= 0 && q1 <= total && n <= max_new && n <= len && len <= static_cast<int64_t>(c.max_pages) * c.page) return true;
    if (c.status) atomicExch(c.status, FLAT_CACHE_BAD_LENGTH);
    sp = Span{0, 0, 0};
    return false;
}
// The page at place `index` of sequence s (an index below the sequence's page count).
__device__ __forceinline__ bool read_page(const CacheView& c, int s, int index, int& id) {
    id = c.table[static_cast<int64_t>(s) * c.max_pages + index];
    if (id >= 0 && id < c.num_pages) return true;
    if (c.status) atomicExch(c.status, FLAT_CACHE_BAD_PAGE);
    id = 0;
    return false;
}

// The NaN among four e4m3 (0x7f and 0xff), as whole bytes.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return (((w & 0x7f7f7f7fu) + 0x01010101u) >> 7 & 0x01010101u) * 255u; }

}  // namespace cache
}  // namespace flat
