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

// ---- rows on their way into the pages ---------------------------------------------------------------------------

// What a thread moves at once on the dense side: 16 bytes, or 32 where the other side is e4m3 (8 or 16 bytes there).
template <bool FP8>
struct Dense;
template <>
struct Dense<false> {
    static constexpr int BYTES = 16;
    uint4 a;
    __device__ __forceinline__ void zero() { a = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void load(const void* p, bool) { a = ld_stream16(p); }
    __device__ __forceinline__ void store(void* p, bool) const { __stcs(static_cast<uint4*>(p), a); }
};
template <>
struct Dense<true> {
    static constexpr int BYTES = 32;
    uint4 a, b;
    __device__ __forceinline__ void zero() { a = b = make_uint4(0, 0, 0, 0); }
    // (wide: the array starts on a 32-byte boundary; 16 are what callers owe)
    __device__ __forceinline__ void load(const void* p, bool wide) {
        if (!wide) {
            a = ld_stream16(p);
            b = ld_stream16(static_cast<const uint4*>(p) + 1);
            return;
        }
        asm volatile("ld.global.nc.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w), "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w)
                     : "l"(p));
    }
    __device__ __forceinline__ void store(void* p, bool wide) const {
        if (!wide) {
            __stcs(static_cast<uint4*>(p), a);
            __stcs(static_cast<uint4*>(p) + 1, b);
            return;
        }
        asm volatile("st.global.L1::no_allocate.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(a.x), "r"(a.y), "r"(a.z),
                     "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w)
                     : "memory");
    }
};

// Bits of |x| if x is finite, else 0: positive floats order like their bits, so an integer maximum finds the largest.
__device__ __forceinline__ unsigned finite_magnitude(float x) {
    const unsigned a = __float_as_uint(x) & 0x7fffffffu;
    return a < 0x7f800000u ? a : 0u;
}
// Bits of the largest finite |x| of a row whose LPR lanes hold 32 bytes each.  Infinities and NaN are met last: their
// bits are larger than any finite number's, so only a row that has some is looked at element by element.
template <typename TS, int LPR>
__device__ __forceinline__ unsigned row_max(const unsigned* w, const float* f) {
    unsigned m = 0;
    if constexpr (sizeof(TS) == 2) {  // two numbers at a time
#pragma unroll
        for (int i = 0; i < 8; ++i) m = __vmaxu2(m, w[i] & 0x7fff7fffu);
#pragma unroll
        for (int o = LPR / 2; o > 0; o >>= 1) m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, o));
        m = max(m << 16, m & 0xffff0000u);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, w[i] & 0x7fffffffu);
#pragma unroll
        for (int o = LPR / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    }
    if (__any_sync(0xffffffffu, m >= 0x7f800000u)) {
        m = 0;
#pragma unroll
        for (int e = 0; e < 32 / (int)sizeof(TS); ++e) m = max(m, finite_magnitude(f[e]));
#pragma unroll
        for (int o = LPR / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    }
    return m;
}
// The smallest e >= -126 with amax <= 448 * 2^e.  448 = 1.75 * 2^8: with amax = 1.m * 2^x, e is x - 8, and one more if
// 1.m > 1.75; adding 0x1fffff to the bits carries into the exponent exactly then.
__device__ __forceinline__ int scale_exponent(unsigned amax_bits) {
    const int x = (int)((amax_bits + 0x1fffffu) >> 23) - 127;
    return max(x - 8, -126);
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }

template <int N>
__device__ __forceinline__ void quantize(const float* f, float inv, unsigned* words) {  // N floats -> N bytes
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        const unsigned lo = __nv_cvt_float2_to_fp8x2(make_float2(f[4 * i] * inv, f[4 * i + 1] * inv), __NV_SATFINITE, __NV_E4M3);
        const unsigned hi = __nv_cvt_float2_to_fp8x2(make_float2(f[4 * i + 2] * inv, f[4 * i + 3] * inv), __NV_SATFINITE, __NV_E4M3);
        words[i] = lo | (hi << 16);
    }
}

}  // namespace chai
