// Shared by the paged-cache kernels: the pool's description, address arithmetic and the host's checks.
#pragma once

#include "chai_common.cuh"

namespace chai {

// n / d for 0 <= n < 2^31 by a multiplication: with s = ceil(log2 d) and m = floor(2^32 (2^s - d) / d) + 1 the
// quotient is (hi32(m n) + n) >> s (Granlund and Montgomery, "Division by invariant integers using multiplication", 1994).
// (A division by a kernel argument costs about twenty instructions; the copy kernels
// would need one for every 16 bytes.)
struct FastDiv {
    unsigned d, m, s;
    FastDiv() = default;
    explicit FastDiv(unsigned div) : d(div), m(0), s(0) {
        while ((1ull << s) < d) ++s;
        m = (unsigned)(((1ull << 32) * ((1ull << s) - d)) / d + 1);
    }
    __device__ __forceinline__ unsigned div(unsigned n) const { return (__umulhi(m, n) + n) >> s; }
};

// The pool as every paged call describes it.  Page strides are in elements (e4m3: bytes).
struct PagePool {
    const int32_t* block_table;  // [B, max_pages]
    size_t k_page_stride, v_page_stride;
    int n_pages, page_size, max_pages;
    FastDiv by_page;
    int capacity;  // positions a block-table row can address
};

constexpr int kPagedMaxHeads = 1024;

// Checks what the three calls have in common and fills the pool's description.  es: bytes of a cached element.
inline int make_pool(const char* fn, const int32_t* block_table, int B, int H, int k, int n_pages, int page_size,
                     int max_pages, int D, size_t k_page_stride, size_t v_page_stride, size_t es, PagePool* pool) {
    CHAI_REQUIRE(B > 0 && H > 0 && k >= 1 && k <= H, CHAI_ERR_INVALID_ARG, "%s: need B, H > 0 and 1 <= k <= H", fn);
    CHAI_REQUIRE(n_pages > 0 && max_pages > 0 && page_size > 0, CHAI_ERR_INVALID_ARG,
                 "%s: need n_pages, max_pages, page_size > 0", fn);
    CHAI_REQUIRE(page_size % 8 == 0 && page_size <= 65536, CHAI_ERR_UNSUPPORTED,
                 "%s: page_size %d (a multiple of 8 up to 65536 supported)", fn, page_size);
    CHAI_REQUIRE(D == 64 || D == 128, CHAI_ERR_UNSUPPORTED, "%s: head_dim %d (64 or 128 supported)", fn, D);
    CHAI_REQUIRE(H <= kPagedMaxHeads && B <= 65535, CHAI_ERR_UNSUPPORTED, "%s: H must be <= %d and B <= 65535", fn,
                 kPagedMaxHeads);
    CHAI_REQUIRE((long long)max_pages * page_size < (1ll << 30), CHAI_ERR_UNSUPPORTED,
                 "%s: max_pages * page_size must be below 2^30", fn);
    const size_t k_dense = (size_t)k * page_size * D, v_dense = (size_t)H * page_size * D;
    if (k_page_stride == 0) k_page_stride = k_dense;
    if (v_page_stride == 0) v_page_stride = v_dense;
    CHAI_REQUIRE(k_page_stride >= k_dense && v_page_stride >= v_dense && k_page_stride * es % 16 == 0 &&
                     v_page_stride * es % 16 == 0,
                 CHAI_ERR_INVALID_ARG,
                 "%s: page strides %zu and %zu must be at least k*page_size*D=%zu and H*page_size*D=%zu elements and "
                 "multiples of 16 bytes",
                 fn, k_page_stride, v_page_stride, k_dense, v_dense);
    pool->block_table = block_table;
    pool->k_page_stride = k_page_stride;
    pool->v_page_stride = v_page_stride;
    pool->n_pages = n_pages;
    pool->page_size = page_size;
    pool->max_pages = max_pages;
    pool->by_page = FastDiv((unsigned)page_size);
    pool->capacity = max_pages * page_size;
    return CHAI_OK;
}

inline bool aligned32(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 31u) == 0; }

// Records a status that a kernel met first (nothing without a workspace).
__device__ __forceinline__ void flag_status(WsHeader* hdr, int status, int b) {
    if (hdr != nullptr && atomicCAS(&hdr->status, CHAI_OK, status) == CHAI_OK) {
        hdr->bad_b = b;
        hdr->bad_h = -1;
    }
}

}  // namespace chai
