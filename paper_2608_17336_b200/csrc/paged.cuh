// What the kernels of the paged key/value cache share: the checked description of the cache and where a token lies in it.
// Not part of the public ABI.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "tilemix.h"

namespace tilemix {

struct PagedCache {
    int B, Hk, d, page_shift, n_pages, max_pages, capacity;   // capacity: tokens that a table row can name
    int64_t ks[3], vs[3], table_stride;                       // strides in elements: (page, head, token)
    uint8_t* k_pool;
    uint8_t* v_pool;
    float* k_scale;
    float* v_scale;
    const int32_t* table;
    const int32_t* cache_len;
};

// Checks the description (no pointer but the struct's own is followed); returns TILEMIX_OK or a negative error.
int resolve_paged(const tilemix_paged_t* p, PagedCache* c);

#ifdef __CUDACC__
__device__ __forceinline__ int paged_len(const PagedCache& c, int b) { return min(max(c.cache_len[b], 0), c.capacity); }

// Page of token `pos` (0 <= pos < capacity) of sequence b; -1: a hole.
__device__ __forceinline__ int paged_page(const PagedCache& c, int b, int pos) {
    const int page = c.table[b * c.table_stride + (pos >> c.page_shift)];
    return static_cast<unsigned>(page) < static_cast<unsigned>(c.n_pages) ? page : -1;
}

// Two values of the activation type as floats, and back.
__device__ __forceinline__ float2 act_to_float2(uint32_t v, __half) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }
__device__ __forceinline__ float2 act_to_float2(uint32_t v, __nv_bfloat16) {
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}
__device__ __forceinline__ uint32_t act_pack2(float a, float b, __half) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t act_pack2(float a, float b, __nv_bfloat16) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
#endif

}  // namespace tilemix
