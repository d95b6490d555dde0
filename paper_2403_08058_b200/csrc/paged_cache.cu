// What writes a paged cache and what reads it back (Section 3.5: after clustering only the representatives' keys are
// cached; Section 4.3: every head keeps its values).
//
//   chai_append_kv_paged, _fp8   N new tokens per request -> rows of the request's pages, as they are or as e4m3
//   chai_read_kv_paged, _fp8     the cached rows of every request -> dense arrays
//
// Both are copies, bound by HBM.  A block takes a run of tokens of one plane; a thread moves several 16-byte vectors of
// the dense side, all loads issued before the first store.  (One sequence of vectors over planes and tokens alike, with
// a division to find the plane of each, was bound by its instructions instead: append to e4m3 65 us where this takes
// 31, read-back from e4m3 69 us and 49; of the 6566 GB/s that a copy reaches those are 88 % and 92 %.)  A decode step's
// few rows go to one block per request that also advances the request's length.
#include <type_traits>

#include "paged.cuh"

namespace chai {
namespace {

constexpr int kStepThreads = 256, kStepUnroll = 4;  // threads a block, vectors a thread: a decode step's append
constexpr int kRowThreads = 128, kRowUnroll = 4;    // ... a prompt's, and read-back
// Blocks of a plane of a request for `runs` runs of tokens.  A grid is made for the width of the dense arrays (N, T_out), for
// the host does not know the lengths, and blocks behind them cost half a nanosecond each: 16 ragged requests of up to 2048
// tokens were read into arrays for 32768 in 339 us, with at most so many blocks that go on from run to run (LOOP) in 63;
// e4m3 172 and 50; appends from such arrays 340 and 102.  Where nothing is empty one run a block is a little faster: 16 of
// up to 8192 read in 240.4 us, 242.1 with LOOP; e4m3 append of 4 x 2043 31.2 us, 32.5.  So 64 blocks (2048 to 4096 tokens) or,
// with few planes, as many as make 256 an SM: one request of 65536 read in 203.5 us, with 64 an SM in 207.4.
constexpr int kRowBlocks = 64, kRowFill = 148 * 256;
inline int row_blocks(int runs, int planes, int B) {
    const long long fill = (kRowFill + (long long)planes * B - 1) / ((long long)planes * B);
    const long long most = fill > kRowBlocks ? fill : kRowBlocks;
    return runs < most ? runs : (int)most;
}

__global__ void paged_reset_status_kernel(WsHeader* hdr) {
    dependent_grid_sync();
    reset_status(hdr);
}

// ---- append -----------------------------------------------------------------------------------------------------

struct AppendArgs {
    const void *k_new, *v_new;
    void *k_pages, *v_pages;
    float *k_scales, *v_scales;
    const int32_t* reps;
    int32_t* seq_lens;
    const int32_t* new_lens;
    WsHeader* hdr;
    PagePool pool;
    FastDiv by_n;
    int H, k, N;
    int advance;
    bool wide;  // the dense arrays start on 32-byte boundaries
};

// Tokens of request b and whether they fit.  The lengths are read once a warp, or once a block where its threads meet at
// barriers later: what goes one way together follows from one reading, whatever another stream writes meanwhile.
__device__ __forceinline__ bool fits(const AppendArgs& a, int pos0, int n) { return pos0 >= 0 && (n == 0 || pos0 <= a.pool.capacity - n); }
__device__ __forceinline__ bool tokens_fit_warp(const AppendArgs& a, int b, int* pos0, int* n) {
    *pos0 = __shfl_sync(0xffffffffu, a.seq_lens[b], 0);
    *n = a.new_lens != nullptr ? __shfl_sync(0xffffffffu, min(max(a.new_lens[b], 0), a.N), 0) : a.N;
    return fits(a, *pos0, *n);
}
__device__ __forceinline__ bool tokens_fit_block(const AppendArgs& a, int b, int* pos0, int* n) {
    __shared__ int2 s;
    if (threadIdx.x == 0) s = make_int2(a.seq_lens[b], a.new_lens != nullptr ? min(max(a.new_lens[b], 0), a.N) : a.N);
    __syncthreads();
    *pos0 = s.x;
    *n = s.y;
    return fits(a, *pos0, *n);
}

// Stores the vector x of a row at `row` of plane `pl` (of the keys or the values) of a page; page -1: nothing.  The lanes
// of a row are neighbours in one warp and call this together.
template <typename TS, int D, bool FP8>
__device__ __forceinline__ void store_vector(const AppendArgs& a, bool key, int pl, int page, int row, int x, const Dense<FP8>& raw) {
    constexpr int EPV = Dense<FP8>::BYTES / (int)sizeof(TS);
    const size_t at = (size_t)page * (key ? a.pool.k_page_stride : a.pool.v_page_stride) +
                      ((size_t)pl * a.pool.page_size + row) * D + x * EPV;
    if constexpr (!FP8) {
        if (page >= 0) *reinterpret_cast<uint4*>(static_cast<TS*>(key ? a.k_pages : a.v_pages) + at) = raw.a;
    } else {
        float f[EPV];
        Vec16<TS>::unpack(raw.a, f);
        Vec16<TS>::unpack(raw.b, f + EPV / 2);
        const unsigned bits[8] = {raw.a.x, raw.a.y, raw.a.z, raw.a.w, raw.b.x, raw.b.y, raw.b.z, raw.b.w};
        const unsigned amax = row_max<TS, D * (int)sizeof(TS) / 32>(bits, f);
        const int e2 = amax == 0 ? 0 : scale_exponent(amax);
        unsigned w[EPV / 4];
        quantize<EPV>(f, pow2(-e2), w);
        if (page >= 0) {
            unsigned char* dst = static_cast<unsigned char*>(key ? a.k_pages : a.v_pages) + at;
            if constexpr (EPV == 16) *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
            else *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
            if (x == 0)
                (key ? a.k_scales : a.v_scales)[((size_t)page * (key ? a.k : a.H) + pl) * a.pool.page_size + row] = pow2(e2);
        }
    }
}

// A decode step's tokens: grid (1, B), one block moves all rows of a request and advances its length.
template <typename TS, int D, bool FP8>
__global__ void __launch_bounds__(kStepThreads) append_step_kernel(const AppendArgs a) {
    dependent_grid_sync();
    constexpr int LPR = D * (int)sizeof(TS) / Dense<FP8>::BYTES, EPV = Dense<FP8>::BYTES / (int)sizeof(TS);
    const int b = blockIdx.y, tid = threadIdx.x;
    int pos0, n;
    if (!tokens_fit_block(a, b, &pos0, &n)) {
        if (tid == 0) flag_status(a.hdr, CHAI_ERR_CACHE_FULL, b);
        return;
    }
    const int32_t* table = a.pool.block_table + (size_t)b * a.pool.max_pages;
    const int32_t* reps = a.reps + (size_t)b * a.k;
    const TS* k_new = static_cast<const TS*>(a.k_new) + (size_t)b * a.H * a.N * D;
    const TS* v_new = static_cast<const TS*>(a.v_new) + (size_t)b * a.H * a.N * D;
    const unsigned total = (unsigned)(a.k + a.H) * a.N * LPR;
    bool bad = false;
    for (unsigned base = 0; base < total; base += kStepThreads * kStepUnroll) {
        Dense<FP8> raw[kStepUnroll];
        int page[kStepUnroll], plane[kStepUnroll], row[kStepUnroll];  // page -1: nothing to store
#pragma unroll
        for (int u = 0; u < kStepUnroll; ++u) {
            const unsigned i = base + u * kStepThreads + tid, r = i / LPR;
            plane[u] = (int)a.by_n.div(r);
            const int t = (int)(r - (unsigned)plane[u] * (unsigned)a.N);
            raw[u].zero();
            page[u] = -1;
            row[u] = 0;
            if (i >= total || t >= n) continue;
            const unsigned pos = (unsigned)(pos0 + t), pi = a.pool.by_page.div(pos);
            row[u] = (int)(pos - pi * (unsigned)a.pool.page_size);
            const int pg = table[pi];
            const bool known = pg >= 0 && pg < a.pool.n_pages;
            bad |= !known;
            int head = plane[u] - a.k;
            if (plane[u] < a.k) {
                head = reps[plane[u]];
                if (head < 0 || head >= a.H) continue;  // unused cluster slot
            }
            raw[u].load((plane[u] < a.k ? k_new : v_new) + ((size_t)head * a.N + t) * D + (int)(i % LPR) * EPV, a.wide);
            page[u] = known ? pg : -1;
        }
#pragma unroll
        for (int u = 0; u < kStepUnroll; ++u) {
            const bool key = plane[u] < a.k;
            store_vector<TS, D, FP8>(a, key, key ? plane[u] : plane[u] - a.k, page[u], row[u], tid % LPR, raw[u]);
        }
    }
    if (bad) flag_status(a.hdr, CHAI_ERR_BAD_PAGE, b);
    bad = __syncthreads_or(bad);
    if (tid == 0 && a.advance && !bad) a.seq_lens[b] = pos0 + n;
}

// A prompt's tokens: grid (blocks, planes, B); a block takes a run of tokens, or (LOOP) every gridDim.x-th.
template <typename TS, int D, bool FP8, bool LOOP>
__global__ void __launch_bounds__(kRowThreads) append_rows_kernel(const AppendArgs a) {
    constexpr int LPR = D * (int)sizeof(TS) / Dense<FP8>::BYTES, EPV = Dense<FP8>::BYTES / (int)sizeof(TS), ROWS = kRowThreads / LPR;
    const int plane = blockIdx.y, b = blockIdx.z, x = threadIdx.x % LPR;
    int pos0, n;
    if (!tokens_fit_warp(a, b, &pos0, &n)) {
        if (threadIdx.x == 0 && blockIdx.x == 0 && plane == 0) flag_status(a.hdr, CHAI_ERR_CACHE_FULL, b);
        return;
    }
    if ((int)blockIdx.x * (ROWS * kRowUnroll) >= n) return;
    const bool key = plane < a.k;
    int head = plane - a.k;
    const int pl = key ? plane : head;
    if (key) {
        head = a.reps[(size_t)b * a.k + plane];
        if (head < 0 || head >= a.H) return;  // unused cluster slot
    }
    const int32_t* table = a.pool.block_table + (size_t)b * a.pool.max_pages;
    const TS* rows = static_cast<const TS*>(key ? a.k_new : a.v_new) + ((size_t)b * a.H + head) * a.N * D + x * EPV;
    bool bad = false;
#pragma unroll 1
    for (int run = (int)blockIdx.x * (ROWS * kRowUnroll); run < n; run = LOOP ? run + (int)gridDim.x * (ROWS * kRowUnroll) : n) {
        const int t0 = run + (int)threadIdx.x / LPR;
        const TS* src = rows + (size_t)t0 * D;
        Dense<FP8> raw[kRowUnroll];
        int page[kRowUnroll], row[kRowUnroll];  // page -1: nothing to store
#pragma unroll
        for (int u = 0; u < kRowUnroll; ++u) {
            const int t = t0 + u * ROWS;
            raw[u].zero();
            page[u] = -1;
            row[u] = 0;
            if (t < n) {
                raw[u].load(src + (size_t)u * ROWS * D, a.wide);
                const unsigned pos = (unsigned)(pos0 + t), pi = a.pool.by_page.div(pos);
                row[u] = (int)(pos - pi * (unsigned)a.pool.page_size);
                page[u] = table[pi];
            }
        }
#pragma unroll
        for (int u = 0; u < kRowUnroll; ++u) {
            if (page[u] < 0 || page[u] >= a.pool.n_pages) {
                bad |= t0 + u * ROWS < n;
                page[u] = -1;
            }
            store_vector<TS, D, FP8>(a, key, pl, page[u], row[u], x, raw[u]);
        }
    }
    if (bad) flag_status(a.hdr, CHAI_ERR_BAD_PAGE, b);
}

// Advances the lengths behind an append of many blocks: every request whose tokens fit and whose pages are all good.
__global__ void __launch_bounds__(128) advance_paged_kernel(const AppendArgs a) {
    dependent_grid_sync();
    const int b = blockIdx.x;
    int pos0, n;
    if (!tokens_fit_block(a, b, &pos0, &n) || n == 0) return;
    const int32_t* table = a.pool.block_table + (size_t)b * a.pool.max_pages;
    const unsigned last = a.pool.by_page.div((unsigned)(pos0 + n - 1));
    bool bad = false;
    for (unsigned p = a.pool.by_page.div((unsigned)pos0) + threadIdx.x; p <= last; p += blockDim.x)
        bad |= table[p] < 0 || table[p] >= a.pool.n_pages;
    bad = __syncthreads_or(bad);
    if (threadIdx.x == 0 && !bad) a.seq_lens[b] = pos0 + n;
}

template <typename TS, int D, bool FP8>
int launch_append(const AppendArgs& a, int B, cudaStream_t s) {
    constexpr int LPR = D * (int)sizeof(TS) / Dense<FP8>::BYTES, TOKENS = kRowThreads / LPR * kRowUnroll;
    // One block per request saves the launch that advances the lengths, as long as it has no more than two passes to make
    // (16 requests, 32 heads, one token: 2.6 us a call, 3.7 the other way; four tokens, three passes: 5.1 against 3.7).
    if ((size_t)(a.k + a.H) * a.N * LPR <= 2 * kStepThreads * kStepUnroll) {
        CHAI_LAUNCH_DEPENDENT("append_step_kernel launch", (append_step_kernel<TS, D, FP8>), dim3(1, B), dim3(kStepThreads), 0, s, a);
        return CHAI_OK;
    }
    const int runs = (a.N + TOKENS - 1) / TOKENS, blocks = row_blocks(runs, a.k + a.H, B);
    if (blocks == runs) append_rows_kernel<TS, D, FP8, false><<<dim3(blocks, a.k + a.H, B), kRowThreads, 0, s>>>(a);
    else append_rows_kernel<TS, D, FP8, true><<<dim3(blocks, a.k + a.H, B), kRowThreads, 0, s>>>(a);
    CHAI_LAUNCH_CHECK("append_rows_kernel launch");
    if (a.advance) CHAI_LAUNCH_DEPENDENT("advance_paged_kernel launch", advance_paged_kernel, dim3(B), dim3(128), 0, s, a);
    return CHAI_OK;
}

int append(const char* fn, bool fp8, AppendArgs a, int B, int n_pages, int page_size, int max_pages, int D,
           const int32_t* block_table, size_t k_page_stride, size_t v_page_stride, int dtype, cudaStream_t s) {
    CHAI_REQUIRE(a.k_new && a.v_new && a.k_pages && a.v_pages && a.reps && block_table && a.seq_lens, CHAI_ERR_INVALID_ARG,
                 "%s: null pointer", fn);
    CHAI_REQUIRE(!fp8 || (a.k_scales && a.v_scales), CHAI_ERR_INVALID_ARG, "%s: null pointer", fn);
    CHAI_REQUIRE(aligned16(a.k_new) && aligned16(a.v_new) && aligned16(a.k_pages) && aligned16(a.v_pages) &&
                     aligned16(a.k_scales) && aligned16(a.v_scales) && aligned16(a.hdr),
                 CHAI_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned", fn);
    CHAI_REQUIRE(dtype == CHAI_F32 || dtype == CHAI_BF16, CHAI_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, dtype);
    const int rc = make_pool(fn, block_table, B, a.H, a.k, n_pages, page_size, max_pages, D, k_page_stride, v_page_stride,
                             fp8 ? 1 : elem_size(dtype), &a.pool);
    if (rc != CHAI_OK) return rc;
    CHAI_REQUIRE(a.N > 0, CHAI_ERR_INVALID_ARG, "%s: need N > 0", fn);
    CHAI_REQUIRE((long long)a.H * a.N < (1ll << 30), CHAI_ERR_UNSUPPORTED, "%s: H*N must be below 2^30", fn);
    a.by_n = FastDiv((unsigned)a.N);
    a.wide = aligned32(a.k_new) && aligned32(a.v_new);
    CHAI_LOG_CALL("%s: B=%d H=%d k=%d N=%d D=%d dtype=%d page_size=%d", fn, B, a.H, a.k, a.N, D, dtype, page_size);
    if (a.hdr != nullptr)
        CHAI_LAUNCH_DEPENDENT("paged append: status reset", paged_reset_status_kernel, dim3(1), dim3(1), 0, s, a.hdr);
    using bf16 = __nv_bfloat16;
    if (dtype == CHAI_BF16) {
        if (D == 128) return fp8 ? launch_append<bf16, 128, true>(a, B, s) : launch_append<bf16, 128, false>(a, B, s);
        return fp8 ? launch_append<bf16, 64, true>(a, B, s) : launch_append<bf16, 64, false>(a, B, s);
    }
    if (D == 128) return fp8 ? launch_append<float, 128, true>(a, B, s) : launch_append<float, 128, false>(a, B, s);
    return fp8 ? launch_append<float, 64, true>(a, B, s) : launch_append<float, 64, false>(a, B, s);
}

// ---- read-back --------------------------------------------------------------------------------------------------

struct ReadArgs {
    const void *k_pages, *v_pages;
    const float *k_scales, *v_scales;
    const int32_t* seq_lens;
    void *k_out, *v_out;
    WsHeader* hdr;
    PagePool pool;
    int H, k, T_out;
    int nk, nv;  // planes that are wanted
    bool wide;   // the dense arrays start on 32-byte boundaries
};

template <typename TO>
__device__ __forceinline__ uint4 pack16(const float* f);
template <>
__device__ __forceinline__ uint4 pack16<float>(const float* f) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
template <>
__device__ __forceinline__ uint4 pack16<__nv_bfloat16>(const float* f) {
    uint4 r;
    unsigned* w = &r.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *reinterpret_cast<const unsigned*>(&p);
    }
    return r;
}

// x * scale for a type of fewer bits than fp32: rounded to odd (the last bit says that something was cut off), so that the
// rounding to that type is the only one.
__device__ __forceinline__ float product_to_odd(float x, float scale) {
    const float p = __fmul_rz(x, scale);
    return __uint_as_float(__float_as_uint(p) | (isfinite(p) && (double)p != (double)x * scale ? 1u : 0u));  // (28 bits: exact in fp64)
}

// grid (blocks, planes that are wanted, B); a block takes a run of tokens, or (LOOP) every gridDim.x-th.
template <typename TO, int D, bool FP8, bool LOOP>
__global__ void __launch_bounds__(kRowThreads) read_paged_kernel(const ReadArgs a) {
    constexpr int LPR = D * (int)sizeof(TO) / Dense<FP8>::BYTES, EPV = Dense<FP8>::BYTES / (int)sizeof(TO), ROWS = kRowThreads / LPR;
    const int plane = blockIdx.y, b = blockIdx.z, x = threadIdx.x % LPR;
    const int n = min(min(max(a.seq_lens[b], 0), a.pool.capacity), a.T_out);
    if ((int)blockIdx.x * (ROWS * kRowUnroll) >= n) return;
    const bool key = plane < a.nk;
    const int pl = key ? plane : plane - a.nk;
    const int32_t* table = a.pool.block_table + (size_t)b * a.pool.max_pages;
    using Raw = typename std::conditional<FP8, typename std::conditional<EPV == 16, uint4, uint2>::type, uint4>::type;
    const char* pages = static_cast<const char*>(key ? a.k_pages : a.v_pages);
    const size_t stride = key ? a.pool.k_page_stride : a.pool.v_page_stride;
    TO* rows = static_cast<TO*>(key ? a.k_out : a.v_out) + ((size_t)b * (key ? a.nk : a.nv) + pl) * a.T_out * D + x * EPV;
    bool bad = false;
#pragma unroll 1
    for (int run = (int)blockIdx.x * (ROWS * kRowUnroll); run < n; run = LOOP ? run + (int)gridDim.x * (ROWS * kRowUnroll) : n) {
        const int t0 = run + (int)threadIdx.x / LPR;
        Raw raw[kRowUnroll];
        [[maybe_unused]] float scale[kRowUnroll];
        int page[kRowUnroll], row[kRowUnroll];
#pragma unroll
        for (int u = 0; u < kRowUnroll; ++u) {
            const unsigned pos = (unsigned)min(t0 + u * ROWS, n - 1), pi = a.pool.by_page.div(pos);
            row[u] = (int)(pos - pi * (unsigned)a.pool.page_size);
            page[u] = table[pi];
        }
#pragma unroll
        for (int u = 0; u < kRowUnroll; ++u) {
            raw[u] = Raw{};
            scale[u] = 0.f;
            if (page[u] < 0 || page[u] >= a.pool.n_pages) {
                bad = true;  // the row is zero
            } else if (t0 + u * ROWS < n) {
                const size_t at = (size_t)page[u] * stride + ((size_t)pl * a.pool.page_size + row[u]) * D + x * EPV;
                raw[u] = __ldcs(reinterpret_cast<const Raw*>(pages + at * (FP8 ? 1 : sizeof(TO))));
                if constexpr (FP8)
                    scale[u] = __ldg((key ? a.k_scales : a.v_scales) + ((size_t)page[u] * (key ? a.k : a.H) + pl) * a.pool.page_size + row[u]);
            }
        }
        TO* dst = rows + (size_t)t0 * D;
#pragma unroll
        for (int u = 0; u < kRowUnroll; ++u) {
            if (t0 + u * ROWS >= n) break;
            Dense<FP8> v;
            if constexpr (FP8) {
                unsigned w[4] = {raw[u].x, raw[u].y, 0, 0};
                if constexpr (EPV == 16) w[2] = raw[u].z, w[3] = raw[u].w;
                float f[EPV];
#pragma unroll
                for (int e = 0; e < EPV / 2; ++e) {
                    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)((w[e / 2] >> (16 * (e & 1))) & 0xffffu), __NV_E4M3);
                    const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&h));
                    f[2 * e] = p.x;
                    f[2 * e + 1] = p.y;
                }
                // A power of two, as append writes it, multiplies without rounding.  Other scales do not: fp32, then bf16, would
                // round twice
                if (sizeof(TO) < 4 && (__float_as_uint(scale[u]) & 0x7fffffu) != 0) {
#pragma unroll
                    for (int e = 0; e < EPV; ++e) f[e] = product_to_odd(f[e], scale[u]);
                } else {
#pragma unroll
                    for (int e = 0; e < EPV; ++e) f[e] *= scale[u];
                }
                v.a = pack16<TO>(f);
                v.b = pack16<TO>(f + EPV / 2);
            } else {
                v.a = raw[u];
            }
            v.store(dst + (size_t)u * ROWS * D, a.wide);
        }
    }
    if (bad) flag_status(a.hdr, CHAI_ERR_BAD_PAGE, b);
}

template <typename TO, int D, bool FP8>
int launch_read(const ReadArgs& a, int B, cudaStream_t s) {
    constexpr int TOKENS = kRowThreads / (D * (int)sizeof(TO) / Dense<FP8>::BYTES) * kRowUnroll;
    const int runs = (a.T_out + TOKENS - 1) / TOKENS, blocks = row_blocks(runs, a.nk + a.nv, B);
    if (blocks == runs) read_paged_kernel<TO, D, FP8, false><<<dim3(blocks, a.nk + a.nv, B), kRowThreads, 0, s>>>(a);
    else read_paged_kernel<TO, D, FP8, true><<<dim3(blocks, a.nk + a.nv, B), kRowThreads, 0, s>>>(a);
    CHAI_LAUNCH_CHECK("read_paged_kernel launch");
    return CHAI_OK;
}

int read_back(const char* fn, bool fp8, ReadArgs a, int B, int n_pages, int page_size, int max_pages, int D,
              const int32_t* block_table, size_t k_page_stride, size_t v_page_stride, int dtype, cudaStream_t s) {
    CHAI_REQUIRE(block_table && a.seq_lens && (a.k_out || a.v_out), CHAI_ERR_INVALID_ARG, "%s: null pointer", fn);
    CHAI_REQUIRE((!a.k_out || (a.k_pages && (!fp8 || a.k_scales))) && (!a.v_out || (a.v_pages && (!fp8 || a.v_scales))),
                 CHAI_ERR_INVALID_ARG, "%s: null pointer to pages or scales of an output that is wanted", fn);
    CHAI_REQUIRE(aligned16(a.k_pages) && aligned16(a.v_pages) && aligned16(a.k_out) && aligned16(a.v_out) &&
                     aligned16(a.k_scales) && aligned16(a.v_scales) && aligned16(a.hdr),
                 CHAI_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned", fn);
    CHAI_REQUIRE(dtype == CHAI_F32 || dtype == CHAI_BF16, CHAI_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, dtype);
    const int rc = make_pool(fn, block_table, B, a.H, a.k, n_pages, page_size, max_pages, D, k_page_stride, v_page_stride,
                             fp8 ? 1 : elem_size(dtype), &a.pool);
    if (rc != CHAI_OK) return rc;
    CHAI_REQUIRE(a.T_out > 0, CHAI_ERR_INVALID_ARG, "%s: need T_out > 0", fn);
    CHAI_REQUIRE((long long)a.H * a.T_out < (1ll << 30), CHAI_ERR_UNSUPPORTED, "%s: H*T_out must be below 2^30", fn);
    a.wide = aligned32(a.k_out) && aligned32(a.v_out);
    a.nk = a.k_out != nullptr ? a.k : 0;
    a.nv = a.v_out != nullptr ? a.H : 0;
    CHAI_LOG_CALL("%s: B=%d H=%d k=%d T_out=%d D=%d dtype=%d page_size=%d", fn, B, a.H, a.k, a.T_out, D, dtype, page_size);
    if (a.hdr != nullptr)
        CHAI_LAUNCH_DEPENDENT("paged read: status reset", paged_reset_status_kernel, dim3(1), dim3(1), 0, s, a.hdr);
    using bf16 = __nv_bfloat16;
    if (dtype == CHAI_BF16) {
        if (D == 128) return fp8 ? launch_read<bf16, 128, true>(a, B, s) : launch_read<bf16, 128, false>(a, B, s);
        return fp8 ? launch_read<bf16, 64, true>(a, B, s) : launch_read<bf16, 64, false>(a, B, s);
    }
    if (D == 128) return fp8 ? launch_read<float, 128, true>(a, B, s) : launch_read<float, 128, false>(a, B, s);
    return fp8 ? launch_read<float, 64, true>(a, B, s) : launch_read<float, 64, false>(a, B, s);
}

AppendArgs append_args(const void* k_new, const void* v_new, void* k_pages, void* v_pages, float* k_scales,
                       float* v_scales, const int32_t* reps, int32_t* seq_lens, const int32_t* new_lens, int H, int k, int N,
                       int advance, void* workspace) {
    AppendArgs a = {};
    a.k_new = k_new;
    a.v_new = v_new;
    a.k_pages = k_pages;
    a.v_pages = v_pages;
    a.k_scales = k_scales;
    a.v_scales = v_scales;
    a.reps = reps;
    a.seq_lens = seq_lens;
    a.new_lens = new_lens;
    a.hdr = static_cast<WsHeader*>(workspace);
    a.H = H;
    a.k = k;
    a.N = N;
    a.advance = advance;
    return a;
}

ReadArgs read_args(const void* k_pages, const void* v_pages, const float* k_scales, const float* v_scales,
                   const int32_t* seq_lens, void* k_out, void* v_out, int H, int k, int T_out, void* workspace) {
    ReadArgs a = {};
    a.k_pages = k_pages;
    a.v_pages = v_pages;
    a.k_scales = k_scales;
    a.v_scales = v_scales;
    a.seq_lens = seq_lens;
    a.k_out = k_out;
    a.v_out = v_out;
    a.hdr = static_cast<WsHeader*>(workspace);
    a.H = H;
    a.k = k;
    a.T_out = T_out;
    return a;
}

}  // namespace
}  // namespace chai

extern "C" {

int chai_append_kv_paged(const void* k_new, const void* v_new, void* k_pages, void* v_pages, const int32_t* reps,
                         const int32_t* block_table, int32_t* seq_lens, const int32_t* new_lens, int B, int H, int k, int N,
                         int n_pages, int page_size, int max_pages, int D, size_t k_page_stride, size_t v_page_stride,
                         int dtype, int advance, void* workspace, void* stream) {
    return chai::append("chai_append_kv_paged", false,
                        chai::append_args(k_new, v_new, k_pages, v_pages, nullptr, nullptr, reps, seq_lens, new_lens, H, k,
                                          N, advance, workspace),
                        B, n_pages, page_size, max_pages, D, block_table, k_page_stride, v_page_stride, dtype,
                        static_cast<cudaStream_t>(stream));
}

int chai_append_kv_paged_fp8(const void* k_new, const void* v_new, void* k_pages, void* v_pages, float* k_scales,
                             float* v_scales, const int32_t* reps, const int32_t* block_table, int32_t* seq_lens,
                             const int32_t* new_lens, int B, int H, int k, int N, int n_pages, int page_size, int max_pages,
                             int D, size_t k_page_stride, size_t v_page_stride, int dtype, int advance, void* workspace,
                             void* stream) {
    return chai::append("chai_append_kv_paged_fp8", true,
                        chai::append_args(k_new, v_new, k_pages, v_pages, k_scales, v_scales, reps, seq_lens, new_lens, H,
                                          k, N, advance, workspace),
                        B, n_pages, page_size, max_pages, D, block_table, k_page_stride, v_page_stride, dtype,
                        static_cast<cudaStream_t>(stream));
}

int chai_read_kv_paged(const void* k_pages, const void* v_pages, const int32_t* block_table, const int32_t* seq_lens,
                       void* k_out, void* v_out, int B, int H, int k, int T_out, int n_pages, int page_size, int max_pages,
                       int D, size_t k_page_stride, size_t v_page_stride, int dtype, void* workspace, void* stream) {
    return chai::read_back("chai_read_kv_paged", false,
                           chai::read_args(k_pages, v_pages, nullptr, nullptr, seq_lens, k_out, v_out, H, k, T_out, workspace),
                           B, n_pages, page_size, max_pages, D, block_table, k_page_stride, v_page_stride, dtype,
                           static_cast<cudaStream_t>(stream));
}

int chai_read_kv_paged_fp8(const void* k_pages, const void* v_pages, const float* k_scales, const float* v_scales,
                           const int32_t* block_table, const int32_t* seq_lens, void* k_out, void* v_out, int B, int H,
                           int k, int T_out, int n_pages, int page_size, int max_pages, int D, size_t k_page_stride,
                           size_t v_page_stride, int dtype, void* workspace, void* stream) {
    return chai::read_back("chai_read_kv_paged_fp8", true,
                           chai::read_args(k_pages, v_pages, k_scales, v_scales, seq_lens, k_out, v_out, H, k, T_out, workspace),
                           B, n_pages, page_size, max_pages, D, block_table, k_page_stride, v_page_stride, dtype,
                           static_cast<cudaStream_t>(stream));
}

}  // extern "C"
