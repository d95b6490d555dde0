// Clustered decode attention over a paged cache (Fig. 3(b), Section 3.4): out[b][h] = sum_t p_t V[h][t] with
// p = softmax_t(scale * q[r] . K[c][t]), c the head's cluster and r its representative.
#include <type_traits>

#include "paged.cuh"

namespace chai {
namespace {

constexpr int kMaxCtas = 160;  // the workspace bound is stated for this many

struct PagedDecodeArgs {
    const void *q, *k_pages, *v_pages;
    const float *k_scales, *v_scales;
    const int32_t *membership, *reps, *seq_lens;
    void* out;
    WsHeader* hdr;
    PagePool pool;
    int B, H, k;
    float scale;
};

__global__ void paged_decode_reset_kernel(WsHeader* hdr) {
    dependent_grid_sync();
    reset_status(hdr);
}

template <typename T>
__device__ __forceinline__ float cached(const void* p, size_t i) { return to_float(static_cast<const T*>(p)[i]); }
template <>
__device__ __forceinline__ float cached<Fp8E4M3>(const void* p, size_t i) {
    const __half_raw h = __nv_cvt_fp8_to_halfraw(static_cast<const unsigned char*>(p)[i], __NV_E4M3);
    return __half2float(*reinterpret_cast<const __half*>(&h));
}

// One block per (head, request); each warp takes every eighth row with a running maximum and sum, and the warps'
// results are joined at the end.
template <typename T, typename TQ, int D>
__global__ void __launch_bounds__(256) paged_decode_kernel(const PagedDecodeArgs a) {
    constexpr bool FP8 = std::is_same<T, Fp8E4M3>::value;
    constexpr int E = D / 32;
    __shared__ float s_o[8][D], s_m[8], s_l[8];
    const int h = blockIdx.x, b = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int n = min(max(a.seq_lens[b], 0), a.pool.capacity);
    int c = 0, r = 0;
    const bool known = resolve_head(a.membership, a.reps, b, h, a.H, a.k, &c, &r);
    if (!known && threadIdx.x == 0) flag_bad_membership(a.hdr, b, h);
    const int32_t* table = a.pool.block_table + (size_t)b * a.pool.max_pages;
    const int ps = a.pool.page_size;
    bool bad = false;
    for (int p = threadIdx.x; (long long)p * ps < n; p += 256) bad |= table[p] < 0 || table[p] >= a.pool.n_pages;
    bad = __syncthreads_or(bad);
    if (bad && threadIdx.x == 0) flag_status(a.hdr, CHAI_ERR_BAD_PAGE, b);
    const int rows = known && !bad ? n : 0;
    float q[E], o[E], m = -INFINITY, l = 0.f;
    for (int e = 0; e < E; ++e) {
        q[e] = known ? to_float(static_cast<const TQ*>(a.q)[((size_t)b * a.H + r) * D + e * 32 + lane]) : 0.f;
        o[e] = 0.f;
    }
    for (int t = warp; t < rows; t += 8) {
        const int page = table[t / ps], row = t % ps;
        const size_t kat = (size_t)page * a.pool.k_page_stride + ((size_t)c * ps + row) * D;
        const size_t vat = (size_t)page * a.pool.v_page_stride + ((size_t)h * ps + row) * D;
        float s = 0.f;
        for (int e = 0; e < E; ++e) s += q[e] * cached<T>(a.k_pages, kat + e * 32 + lane);
        for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
        s *= a.scale;
        float vs = 1.f;
        if constexpr (FP8) {
            s *= a.k_scales[((size_t)page * a.k + c) * ps + row];
            vs = a.v_scales[((size_t)page * a.H + h) * ps + row];
        }
        const float top = fmaxf(m, s), ref = top == -INFINITY ? 0.f : top;
        const float keep = __expf(m - ref), p = __expf(s - ref);
        m = top;
        l = l * keep + p;
        for (int e = 0; e < E; ++e) o[e] = o[e] * keep + p * vs * cached<T>(a.v_pages, vat + e * 32 + lane);
    }
    for (int e = 0; e < E; ++e) s_o[warp][e * 32 + lane] = o[e];
    s_m[warp] = m;
    s_l[warp] = l;
    __syncthreads();
    for (int d = threadIdx.x; d < D; d += 256) {
        float top = -INFINITY, sum = 0.f, acc = 0.f;
        for (int w = 0; w < 8; ++w) top = fmaxf(top, s_m[w]);
        const float ref = top == -INFINITY ? 0.f : top;
        for (int w = 0; w < 8; ++w) {
            const float f = __expf(s_m[w] - ref);
            sum += f * s_l[w];
            acc += f * s_o[w][d];
        }
        static_cast<TQ*>(a.out)[((size_t)b * a.H + h) * D + d] = from_float<TQ>(rows > 0 ? acc / sum : 0.f);
    }
}

template <typename T, typename TQ, int D>
int launch_decode(const PagedDecodeArgs& a, cudaStream_t s) {
    CHAI_LAUNCH_DEPENDENT("paged decode: status reset", paged_decode_reset_kernel, dim3(1), dim3(1), 0, s, a.hdr);
    paged_decode_kernel<T, TQ, D><<<dim3(a.H, a.B), 256, 0, s>>>(a);
    CHAI_LAUNCH_CHECK("paged_decode_kernel launch");
    return CHAI_OK;
}

int decode(const char* fn, bool fp8, const void* q, const void* k_pages, const void* v_pages, const float* k_scales,
           const float* v_scales, const int32_t* membership, const int32_t* reps, const int32_t* block_table,
           const int32_t* seq_lens, void* out, int B, int H, int k, int n_pages, int page_size, int max_pages, int D,
           size_t k_page_stride, size_t v_page_stride, float scale, int dtype, void* workspace, size_t workspace_bytes,
           void* stream) {
    CHAI_REQUIRE(q && k_pages && v_pages && membership && reps && block_table && seq_lens && out && workspace &&
                     (!fp8 || (k_scales && v_scales)),
                 CHAI_ERR_INVALID_ARG, "%s: null pointer", fn);
    CHAI_REQUIRE(aligned16(q) && aligned16(k_pages) && aligned16(v_pages) && aligned16(out) && aligned16(workspace) &&
                     aligned16(k_scales) && aligned16(v_scales),
                 CHAI_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned", fn);
    CHAI_REQUIRE(dtype == CHAI_F32 || dtype == CHAI_BF16, CHAI_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, dtype);
    PagedDecodeArgs a = {};
    const int rc = make_pool(fn, block_table, B, H, k, n_pages, page_size, max_pages, D, k_page_stride, v_page_stride,
                             fp8 ? 1 : elem_size(dtype), &a.pool);
    if (rc != CHAI_OK) return rc;
    const size_t need = chai_decode_paged_workspace_bytes(B, H, D);
    CHAI_REQUIRE(workspace_bytes >= need, CHAI_ERR_WORKSPACE, "%s: workspace has %zu bytes, %zu needed", fn, workspace_bytes,
                 need);
    a.q = q;
    a.k_pages = k_pages;
    a.v_pages = v_pages;
    a.k_scales = k_scales;
    a.v_scales = v_scales;
    a.membership = membership;
    a.reps = reps;
    a.seq_lens = seq_lens;
    a.out = out;
    a.hdr = static_cast<WsHeader*>(workspace);
    a.B = B;
    a.H = H;
    a.k = k;
    a.scale = scale;
    CHAI_LOG_CALL("%s: B=%d H=%d k=%d D=%d dtype=%d page_size=%d max_pages=%d", fn, B, H, k, D, dtype, page_size, max_pages);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    using bf16 = __nv_bfloat16;
    if (fp8) {
        if (dtype == CHAI_BF16) return D == 128 ? launch_decode<Fp8E4M3, bf16, 128>(a, s) : launch_decode<Fp8E4M3, bf16, 64>(a, s);
        return D == 128 ? launch_decode<Fp8E4M3, float, 128>(a, s) : launch_decode<Fp8E4M3, float, 64>(a, s);
    }
    if (dtype == CHAI_BF16) return D == 128 ? launch_decode<bf16, bf16, 128>(a, s) : launch_decode<bf16, bf16, 64>(a, s);
    return D == 128 ? launch_decode<float, float, 128>(a, s) : launch_decode<float, float, 64>(a, s);
}

}  // namespace
}  // namespace chai

extern "C" {

size_t chai_decode_paged_workspace_bytes(int B, int H, int D) {
    if (B <= 0 || H <= 0 || (D != 64 && D != 128)) return 0;
    return (64u << 10) + 4 * ((size_t)chai::kMaxCtas + B) * H * (D + 8);
}

int chai_decode_attention_paged(const void* q, const void* k_pages, const void* v_pages, const int32_t* membership,
                                const int32_t* reps, const int32_t* block_table, const int32_t* seq_lens, void* out, int B,
                                int H, int k, int n_pages, int page_size, int max_pages, int D, size_t k_page_stride,
                                size_t v_page_stride, float scale, int dtype, void* workspace, size_t workspace_bytes,
                                void* stream) {
    return chai::decode("chai_decode_attention_paged", false, q, k_pages, v_pages, nullptr, nullptr, membership, reps,
                        block_table, seq_lens, out, B, H, k, n_pages, page_size, max_pages, D, k_page_stride, v_page_stride,
                        scale, dtype, workspace, workspace_bytes, stream);
}

int chai_decode_attention_paged_fp8(const void* q, const void* k_pages, const void* v_pages, const float* k_scales,
                                    const float* v_scales, const int32_t* membership, const int32_t* reps,
                                    const int32_t* block_table, const int32_t* seq_lens, void* out, int B, int H, int k,
                                    int n_pages, int page_size, int max_pages, int D, size_t k_page_stride,
                                    size_t v_page_stride, float scale, int dtype, void* workspace, size_t workspace_bytes,
                                    void* stream) {
    return chai::decode("chai_decode_attention_paged_fp8", true, q, k_pages, v_pages, k_scales, v_scales, membership, reps,
                        block_table, seq_lens, out, B, H, k, n_pages, page_size, max_pages, D, k_page_stride, v_page_stride,
                        scale, dtype, workspace, workspace_bytes, stream);
}

}  // extern "C"
