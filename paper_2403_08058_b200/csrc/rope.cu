// Rotary positions: queries and keys are rotated by their positions before their products are taken.
//
//   chai_rope                     q and k of whole prompts, any strides
//   chai_append_rope_paged, _fp8  a packed batch on its way into the pages: the representatives' q and k rotated, k and v
//                                 written to the tokens' slots (Section 3.5: only representatives' keys are cached, so only
//                                 they, and the queries that meet them, are read at all)
//   chai_rope_frequencies         the frequencies, on the host
//
// Pair i of a row, (x_i, x_{i + rot/2}) or (x_2i, x_2i+1), at position p turns by the angle a = 2 pi p f_i:
//   y1 = m (x1 cos a - x2 sin a),   y2 = m (x2 cos a + x1 sin a).
// f_i is held in turns a position and fp64, so that p f_i minus the nearest whole number is good to 2^-53 p f_i turns at any
// position; that remainder, rounded to fp32 (at most 2^-26 of a turn), goes to sincospi.  An angle in fp32 would be off by
// 0.008 at position 131072.
//
// Bound by HBM.  A block takes some tokens; their cosines and sines are worked out once, into shared memory; a thread owns one
// token and 16 (to e4m3: 32) bytes of its rows, keeps the factors of these in registers and goes from head to head, so that an
// angle costs nothing per head.  The other number of a pair comes from a neighbouring lane (half layout) or is the thread's
// own.  Few tokens are spread over more blocks by heads.
#include <math.h>

#include "paged.cuh"

namespace chai {
namespace {

constexpr int kThreads = 256, kUnroll = 4;
constexpr int kFill = 148 * 4;   // blocks that fill the GPU: four for each of its multiprocessors
constexpr int kEnterTokens = 4;  // of a block: few, so that most of a token's rows are in flight at once behind its angles (8: 3.2 -> 3.4 us for 16)
constexpr int kMaxPairs = 64;

struct Rotation {
    const double* turns;  // [rot / 2], device
    int rot;              // rotated elements of a row, a multiple of 16; 0: none
    int interleaved;
    double magnitude;
};

// cos and sin (times the magnitude) of a token's pair.
__device__ __forceinline__ float2 factors(const Rotation& r, int pos, int i) {
    const double t = __dmul_rn((double)pos, r.turns[i]);  // (rounded: the remainder is of this product)
    float s, c;
    sincospif(2.f * (float)(t - rint(t)), &s, &c);
    return make_float2(c * (float)r.magnitude, s * (float)r.magnitude);
}

// What a thread needs to rotate its vector of EPV elements: per element the factor of itself and of its partner.
template <int EPV>
struct Factors {
    float own[EPV], other[EPV];
};
// cs: the token's factors, [rot / 2].  x: the vector's index in the row.
template <int EPV>
__device__ __forceinline__ void gather(const Rotation& r, const float2* cs, int x, Factors<EPV>& f) {
    const int half = r.rot >> 1;
#pragma unroll
    for (int e = 0; e < EPV; ++e) {
        const int at = x * EPV + e;
        f.own[e] = 1.f;
        f.other[e] = 0.f;
        if (at < r.rot) {
            const bool second = r.interleaved ? (at & 1) : at >= half;
            const float2 v = cs[r.interleaved ? at >> 1 : second ? at - half : at];
            f.own[e] = v.x;
            f.other[e] = second ? v.y : -v.y;
        }
    }
}
// The lane that holds the partners of vector x (half layout); itself outside the rotated part.
template <int EPV>
__device__ __forceinline__ int partner_vector(const Rotation& r, int x) {
    if (r.interleaved || x * EPV >= r.rot) return x;
    const int half = r.rot / (2 * EPV);
    return x < half ? x + half : x - half;
}
// y = rotated x in fp32.  src_lane: the lane of the partner vector.  All lanes of the warp call this.
template <typename T, int EPV>
__device__ __forceinline__ void rotate(const uint4& raw, bool interleaved, bool rotated, int src_lane, const Factors<EPV>& f, float* y) {
    float a[EPV], b[EPV];
    Vec16<T>::unpack(raw, a);
    if (interleaved) {
#pragma unroll
        for (int e = 0; e < EPV; ++e) b[e] = a[e ^ 1];
    } else {
        uint4 o;
        o.x = __shfl_sync(0xffffffffu, raw.x, src_lane);
        o.y = __shfl_sync(0xffffffffu, raw.y, src_lane);
        o.z = __shfl_sync(0xffffffffu, raw.z, src_lane);
        o.w = __shfl_sync(0xffffffffu, raw.w, src_lane);
        Vec16<T>::unpack(o, b);
    }
#pragma unroll
    for (int e = 0; e < EPV; ++e) y[e] = rotated ? fmaf(a[e], f.own[e], b[e] * f.other[e]) : a[e];  // (outside the rotated part a bit copy)
}
template <typename T>
__device__ __forceinline__ uint4 pack(const float* f);
template <>
__device__ __forceinline__ uint4 pack<float>(const float* f) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
template <>
__device__ __forceinline__ uint4 pack<__nv_bfloat16>(const float* f) {
    uint4 r;
    unsigned* w = &r.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *reinterpret_cast<const unsigned*>(&p);
    }
    return r;
}

// ---- whole prompts ----------------------------------------------------------------------------------------------

struct Strided {
    const void* in;
    void* out;
    long long b, h, n, ob, oh, on;  // strides in elements, input and output
    int heads;
};
struct RopeArgs {
    Strided x[2];  // q, k
    const int32_t* positions;  // [B, N] or null: 0, 1, ...
    Rotation rot;
    int B, N, heads_per_block;
};

// grid (token groups, parts of the heads).  The rows of a pass are neighbouring tokens of one head: as much of an array that has
// tokens behind one another is read in one piece as the block is wide (with 8 tokens, two heads a pass, 8192 x 64 rows
// took 61 us, now 47: 268 MB at 5.7 TB/s).
template <typename T, int D>
struct RopeShape {
    static constexpr int EPV = 16 / (int)sizeof(T), LPR = D / EPV, TOKENS = kThreads / LPR;
};
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) rope_kernel(const __grid_constant__ RopeArgs a) {
    constexpr int EPV = RopeShape<T, D>::EPV, LPR = RopeShape<T, D>::LPR, TOKENS = RopeShape<T, D>::TOKENS;
    __shared__ float2 cs[TOKENS][D / 2 + 1];
    const int tid = threadIdx.x, x = tid % LPR, local = tid / LPR;
    const long long total = (long long)a.B * a.N, first = (long long)blockIdx.x * TOKENS;
    const int pairs = a.rot.rot >> 1;
    for (int i = tid; i < TOKENS * pairs; i += kThreads) {
        const int t = i / pairs, p = i - t * pairs;
        if (first + t >= total) break;
        const int pos = a.positions != nullptr ? a.positions[first + t] : (int)((first + t) % a.N);
        cs[t][p] = factors(a.rot, pos, p);
    }
    __syncthreads();
    const bool live = first + local < total;
    const long long token = live ? first + local : total - 1;
    const int b = (int)(token / a.N), n = (int)(token - (long long)b * a.N);
    Factors<EPV> f;
    gather<EPV>(a.rot, cs[live ? local : 0], x, f);
    const int lane = tid & 31, src_lane = lane - x + partner_vector<EPV>(a.rot, x);
    const bool rotated = x * EPV < a.rot.rot;
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {  // q, then k
        const Strided& s = a.x[which];
        const int from = which == 0 ? 0 : a.x[0].heads;
        const int h0 = max((int)blockIdx.y * a.heads_per_block - from, 0), h1 = min(((int)blockIdx.y + 1) * a.heads_per_block - from, s.heads);
        const T* in = static_cast<const T*>(s.in) + b * s.b + n * s.n + h0 * s.h + x * EPV;
        T* out = static_cast<T*>(s.out) + b * s.ob + n * s.on + h0 * s.oh + x * EPV;
#pragma unroll 1
        for (int h = h0; h < h1; h += kUnroll, in += kUnroll * s.h, out += kUnroll * s.oh) {
            uint4 raw[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                raw[u] = make_uint4(0, 0, 0, 0);
                if (h + u < h1 && live) raw[u] = __ldcs(reinterpret_cast<const uint4*>(in + u * s.h));  // (input and output may be one array)
            }
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                float y[EPV];
                rotate<T, EPV>(raw[u], a.rot.interleaved != 0, rotated, src_lane, f, y);
                if (h + u < h1 && live) __stcs(reinterpret_cast<uint4*>(out + u * s.oh), rotated ? pack<T>(y) : raw[u]);
            }
        }
    }
}

// Rows of an array: D elements each, `stride` elements apart along every index; a single index has no stride.
struct Rows {
    const char* base;
    long long stride[3], size[3];
};
Rows rows_of(const Strided& x, bool out, int B, int N) {
    Rows r = {static_cast<const char*>(out ? x.out : x.in), {out ? x.ob : x.b, out ? x.oh : x.h, out ? x.on : x.n}, {B, x.heads, N}};
    for (int i = 0; i < 3; ++i)
        if (r.size[i] == 1 || r.stride[i] == 0) r.size[i] = 1, r.stride[i] = 0;  // (one row for many is one row)
    return r;
}
// Whether strides in ascending order are each at least what the smaller ones span: then no two rows overlap.
bool nested(const Rows& r, int D) {
    __int128 span = D;
    bool done[3] = {};
    for (int n = 0; n < 3; ++n) {
        int at = -1;
        for (int i = 0; i < 3; ++i)
            if (!done[i] && (at < 0 || r.stride[i] < r.stride[at])) at = i;
        done[at] = true;
        if (r.size[at] == 1) continue;
        if (r.stride[at] < span) return false;
        span += (__int128)(r.size[at] - 1) * r.stride[at];
    }
    return true;
}
// Whether a row of x may overlap a row of y.  Exact where they have the same strides and are nested (parts of one array, say):
// a distance of two rows is e0 s0 + e1 s1 + e2 s2, and of the largest stride only the two multiples around what is
// to be bridged can do it.  Where strides differ, arrays are taken for the ranges that they span.
bool rows_meet(const Rows& x, const Rows& y, int D, int es) {
    __int128 x_span = D, y_span = D, to = ((__int128)(reinterpret_cast<intptr_t>(y.base)) - (__int128)(reinterpret_cast<intptr_t>(x.base))) / es;
    Rows both = x;
    bool same = true;
    for (int i = 0; i < 3; ++i) {
        x_span += (__int128)(x.size[i] - 1) * x.stride[i];
        y_span += (__int128)(y.size[i] - 1) * y.stride[i];
        if (x.size[i] > 1 && y.size[i] > 1 && x.stride[i] != y.stride[i]) same = false;
        both.stride[i] = x.size[i] > 1 ? x.stride[i] : y.stride[i];
        both.size[i] = x.size[i] > y.size[i] ? x.size[i] : y.size[i];
    }
    if (to >= x_span || -to >= y_span) return false;
    if (!same || !nested(both, D)) return true;
    int order[3] = {0, 1, 2};  // largest stride first
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2 - i; ++j)
            if (both.stride[order[j]] < both.stride[order[j + 1]]) {
                const int swap = order[j];
                order[j] = order[j + 1];
                order[j + 1] = swap;
            }
    for (int pick = 0; pick < 8; ++pick) {  // of the two multiples of every stride
        __int128 rest = to;
        bool there = true;
        for (int i = 0; i < 3 && there; ++i) {
            const int at = order[i];
            if (both.size[at] == 1) continue;
            const __int128 s = both.stride[at], below = -rest >= 0 ? -rest / s : -((rest + s - 1) / s), e = below + (pick >> i & 1);
            there = e >= -(__int128)(x.size[at] - 1) && e <= y.size[at] - 1;
            rest += e * s;
        }
        if (there && rest < D && -rest < D) return true;
    }
    return false;
}

template <typename T, int D>
int launch_rope(RopeArgs a, cudaStream_t s) {
    const int heads = a.x[0].heads + a.x[1].heads;
    const long long groups = ((long long)a.B * a.N + RopeShape<T, D>::TOKENS - 1) / RopeShape<T, D>::TOKENS;
    // Few tokens: the heads go to several blocks, so that there are four for every SM while each has a load for every slot
    const long long want = (kFill + groups - 1) / groups, most = (heads + kUnroll - 1) / kUnroll;
    const int parts = (int)(want < most ? want : most);
    a.heads_per_block = (heads + parts - 1) / parts;
    rope_kernel<T, D><<<dim3((unsigned)groups, (heads + a.heads_per_block - 1) / a.heads_per_block), kThreads, 0, s>>>(a);
    CHAI_LAUNCH_CHECK("rope_kernel launch");
    return CHAI_OK;
}

int check_rotation(const char* fn, const Rotation& r, int D) {
    CHAI_REQUIRE(r.rot >= 0 && r.rot <= D && r.rot % 16 == 0, CHAI_ERR_UNSUPPORTED,
                 "%s: rot %d (a multiple of 16 up to the head dimension supported)", fn, r.rot);
    CHAI_REQUIRE(r.rot == 0 || r.turns != nullptr, CHAI_ERR_INVALID_ARG, "%s: null pointer to the frequencies", fn);
    CHAI_REQUIRE((reinterpret_cast<uintptr_t>(r.turns) & 7u) == 0, CHAI_ERR_INVALID_ARG, "%s: frequencies must be 8-byte aligned", fn);
    CHAI_REQUIRE(isfinite(r.magnitude), CHAI_ERR_INVALID_ARG, "%s: magnitude must be finite", fn);
    return CHAI_OK;
}

// ---- into the pages ---------------------------------------------------------------------------------------------

struct EnterArgs {
    const void *q, *k, *v;
    void* q_out;
    void *k_pages, *v_pages;
    float *k_scales, *v_scales;
    const int32_t *reps, *token_request, *positions;
    const int64_t* slots;
    WsHeader* hdr;
    Rotation rot;
    long long q_stride, k_stride, v_stride;  // elements between tokens
    size_t k_page_stride, v_page_stride;
    FastDiv by_page;
    long long n_slots;
    int B, H, k_planes, n_tokens, page_size, rows_per_block;
    bool wide;  // q, k and v have tokens on 32-byte boundaries
};

// With R = hypot(x1, x2) m and u = 2^-24, a rotated number is off by at most 6 u R: the angle's remainder by 1.6 u, which turns the
// pair; the factors by 1.5 u and, with a magnitude, 1 u more; product and sum by 2 u.  The row's largest is at least R / sqrt 2,
// so the error is less than 9 u of it.  That decides two things where it should not: the scale, where the largest lies
// within 9 units of its mantissa of 1.75 * 2^i (once in 10^6 rows; it would be off by a factor of two), and the byte, where a
// number, 448 at most after scaling, lies within 9 u 448 of the middle between two e4m3 numbers (once in 10^4).  Such
// numbers are worked out in fp64, so that bytes and scales are those of the exact ones (5599 tokens of 52 heads: 58 us
// without, 68 with; with factors in fp64 for all, which would make this cheap: 76).  (Exact: of p f rounded to fp64, as the
// definition has it, about 2^-32 of a turn from the product at position 2^24, 2^-25 at 2^31.)
constexpr unsigned kBorder = 0x600000u, kNear = 16u;
constexpr float kMiddle = 9.f * 448.f / (1 << 24);
__device__ __forceinline__ bool near_border(unsigned amax_bits) { return (amax_bits & 0x7fffffu) - (kBorder - kNear) <= 2 * kNear; }
// How far a scaled number's magnitude is from the middle between the e4m3 numbers around it (below 2^-6 these are 2^-9 apart, as
// they are from there to 2^-5).
__device__ __forceinline__ float from_middle(float scaled) {
    float t = fabsf(scaled);
    t = t < 0.015625f ? t + 0.015625f : t;
    return fabsf(t - __uint_as_float((__float_as_uint(t) & 0xfff00000u) | 0x80000u));
}

// Element `at` of a row, rotated in fp64; rounded towards zero to fp32, with the last bit set where that is not the number:
// comparisons and a rounding to fewer bits go as the number's own would.  (Rare: the row is read once more.)
template <typename T>
__device__ __noinline__ float rotated_64(const Rotation& r, int pos, const T* row, int at) {
    const int half = r.rot >> 1;
    const bool second = r.interleaved ? (at & 1) : at >= half;
    const double t = __dmul_rn((double)pos, r.turns[r.interleaved ? at >> 1 : second ? at - half : at]);
    double s, c;
    sincospi(2.0 * (t - rint(t)), &s, &c);
    const double x = (float)row[at], other = (float)row[r.interleaved ? at ^ 1 : second ? at - half : at + half];
    const double z = (x * c + (second ? other : -other) * s) * r.magnitude;
    const float f = __double2float_rz(z);
    return (double)f == z ? f : __uint_as_float(__float_as_uint(f) | 1u);
}

// Stores what a thread has of a row (raw, or of a rotated one the numbers y) at `row` of plane `pl` of a page; store: whether at
// all.  The lanes of a row call this together.
template <typename T, int D>
__device__ __forceinline__ void put_row(const EnterArgs& a, bool key, int pl, unsigned page, int row, int x, bool store, const uint4& raw) {
    const size_t at = (size_t)page * (key ? a.k_page_stride : a.v_page_stride) + ((size_t)pl * a.page_size + row) * D + x * (16 / (int)sizeof(T));
    if (store) *reinterpret_cast<uint4*>(static_cast<T*>(key ? a.k_pages : a.v_pages) + at) = raw;
}
template <typename T, int D>
__device__ __forceinline__ void put_row_fp8(const EnterArgs& a, bool key, int pl, unsigned page, int row, int x, bool store, const float* y, int e2) {
    constexpr int EPL = 32 / (int)sizeof(T);
    unsigned w[EPL / 4];
    quantize<EPL>(y, pow2(-e2), w);
    if (!store) return;
    const size_t in_page = (size_t)pl * a.page_size + row;
    unsigned char* dst = static_cast<unsigned char*>(key ? a.k_pages : a.v_pages) + (size_t)page * (key ? a.k_page_stride : a.v_page_stride) + in_page * D + x * EPL;
    if constexpr (EPL == 16) *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
    else *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
    if (x == 0) (key ? a.k_scales : a.v_scales)[(size_t)page * (key ? a.k_planes : a.H) * a.page_size + in_page] = pow2(e2);
}

// grid (token groups, parts of the rows).  Rows of a token: k_planes keys, k_planes queries, then H values, which are not rotated and
// go through a loop of their own.  Blocks to an SM: what the registers of a rotated e4m3 row (its border check among them) allow is
// two; rows stored as they are gain from a third (bf16, 5599 tokens of 52 heads, 128 wide: 57 -> 50 us), and a fourth, 47 us there,
// spills what 568 tokens wait for (6.8 -> 7.6 us).
// To e4m3 the 5599 tokens take 68 us, 178 MB at 2.6 TB/s: bound by latency.  With 126 registers 16 warps stand on an SM, 21 % of what
// it holds; they issue in 42 % of the cycles, and of a warp's time between two instructions (8 cycles) 3 are waits for loads and 1.5
// for the result before.  The bf16 form, 50 us, is bound by the same at 24 warps: 7.8 of 13.9 cycles are waits for loads.
template <typename T, int D, bool FP8>
__global__ void __launch_bounds__(kThreads, FP8 ? 2 : 3) append_rope_kernel(const __grid_constant__ EnterArgs a) {
    constexpr int BYTES = Dense<FP8>::BYTES, VPL = BYTES / 16, EPV = 16 / (int)sizeof(T), EPL = EPV * VPL, LPR = D / EPL;
    constexpr int ROWS = kThreads / LPR, STEP = ROWS / kEnterTokens, UNROLL = kUnroll / VPL;
    static_assert(ROWS % kEnterTokens == 0, "a thread keeps its token");
    __shared__ float2 cs[kEnterTokens][kMaxPairs + 1];
    dependent_grid_sync();
    const int tid = threadIdx.x, x = tid % LPR, local = (tid / LPR) % kEnterTokens, r_off = tid / LPR / kEnterTokens;
    const int first = (int)blockIdx.x * kEnterTokens, token = first + local;
    const int turned = 2 * a.k_planes, r_begin = (int)blockIdx.y * a.rows_per_block;
    const int r_end = min(turned + a.H, r_begin + a.rows_per_block);
    const int pairs = a.rot.rot >> 1;
    // where the token goes
    long long slot = -1;
    int b = 0, pos = 0;
    bool bad = false;
    if (token < a.n_tokens) {
        slot = a.slots[token];
        b = a.token_request[token];
        pos = a.positions[token];
        if (slot >= 0 && (slot >= a.n_slots || b < 0 || b >= a.B)) bad = true, slot = -1;
    }
    const bool live = slot >= 0;
    const unsigned page = slot < 0x7fffffffll ? a.by_page.div((unsigned)max(slot, 0ll)) : (unsigned)(slot / a.page_size);
    const int row = live ? (int)(slot - (long long)page * a.page_size) : 0;
    if (r_begin < turned) {  // (block-uniform)
        const int32_t* reps = a.reps + (size_t)b * a.k_planes;
        const int t_end = min(r_end, turned);
        Dense<FP8> raw[UNROLL];
        int head[UNROLL];  // -1: nothing to do
        auto load = [&](int r0) {
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                const int r = r0 + u * STEP + r_off;
                head[u] = r < t_end && live ? reps[r < a.k_planes ? r : r - a.k_planes] : -1;
            }
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                const bool key = r0 + u * STEP + r_off < a.k_planes;
                raw[u].zero();
                if (head[u] < 0 || head[u] >= a.H) head[u] = -1;  // (-1: unused cluster slot)
                else raw[u].load(static_cast<const T*>(key ? a.k : a.q) + token * (key ? a.k_stride : a.q_stride) + (long long)head[u] * D + x * EPL, a.wide);
            }
        };
        load(r_begin);  // (on its way while the angles are worked out)
        for (int i = tid; i < kEnterTokens * pairs; i += kThreads) {
            const int t = i / pairs, p = i - t * pairs;
            if (first + t < a.n_tokens) cs[t][p] = factors(a.rot, a.positions[first + t], p);
        }
        __syncthreads();
        Factors<EPL> f;
        gather<EPL>(a.rot, cs[token < a.n_tokens ? local : 0], x, f);
        // (half layout) the lane that holds the partners of each of the thread's vectors, and which of that lane's they are
        const int lane = tid & 31, half_vectors = a.rot.rot / (2 * EPV), odd = VPL == 2 ? half_vectors & 1 : 0;
        int src_lane[VPL];
        bool in_rot[VPL];
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            src_lane[i] = lane - x + partner_vector<EPV>(a.rot, x * VPL + i) / VPL;
            in_rot[i] = (x * VPL + i) * EPV < a.rot.rot;
        }
#pragma unroll 1
        for (int r0 = r_begin; r0 < t_end; r0 += STEP * UNROLL) {
            if (r0 != r_begin) load(r0);
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                const int r = r0 + u * STEP + r_off;
                const bool key = r < a.k_planes, there = head[u] >= 0;
                float y[EPL];
                uint4 mine[VPL], other[VPL];
                mine[0] = raw[u].a;
                if constexpr (VPL == 2) mine[1] = raw[u].b;
#pragma unroll
                for (int i = 0; i < VPL; ++i) {
                    const uint4 give = VPL == 2 && odd != 0 ? mine[(i ^ 1) % VPL] : mine[i];
                    other[i] = give;
                    if (!a.rot.interleaved) {
                        other[i].x = __shfl_sync(0xffffffffu, give.x, src_lane[i]);
                        other[i].y = __shfl_sync(0xffffffffu, give.y, src_lane[i]);
                        other[i].z = __shfl_sync(0xffffffffu, give.z, src_lane[i]);
                        other[i].w = __shfl_sync(0xffffffffu, give.w, src_lane[i]);
                    }
                    float m[EPV], o[EPV];
                    Vec16<T>::unpack(mine[i], m);
                    Vec16<T>::unpack(other[i], o);
#pragma unroll
                    for (int e = 0; e < EPV; ++e) {
                        const float partner = a.rot.interleaved ? m[e ^ 1] : o[e];
                        y[i * EPV + e] = in_rot[i] ? fmaf(m[e], f.own[i * EPV + e], partner * f.other[i * EPV + e]) : m[e];
                    }
                }
                if (there && !key) {
                    uint4* to = reinterpret_cast<uint4*>(static_cast<T*>(a.q_out) + ((long long)token * a.H + head[u]) * D + x * EPL);
#pragma unroll
                    for (int i = 0; i < VPL; ++i) to[i] = in_rot[i] ? pack<T>(y + i * EPV) : mine[i];
                }
                if constexpr (!FP8) {
                    put_row<T, D>(a, true, r, page, row, x, there && key, in_rot[0] ? pack<T>(y) : mine[0]);
                } else {
                    if (!__any_sync(0xffffffffu, there && key)) continue;
                    auto largest = [&]() {
                        unsigned m = 0;
#pragma unroll
                        for (int e = 0; e < EPL; ++e) m = max(m, finite_magnitude(y[e]));
#pragma unroll
                        for (int o = LPR / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
                        return m;
                    };
                    unsigned m = largest();
                    int e2 = m == 0 ? 0 : scale_exponent(m);
                    float nearest = 1.f;
#pragma unroll
                    for (int e = 0; e < EPL; ++e)
                        if (in_rot[e / EPV]) nearest = fminf(nearest, from_middle(y[e] * pow2(-e2)));
                    const bool turns = key && there && a.rot.rot > 0, border = near_border(m);
                    if (__any_sync(0xffffffffu, turns && (border || nearest < kMiddle))) {
                        const T* from = static_cast<const T*>(a.k) + token * a.k_stride + (long long)head[u] * D;
                        bool again = true;  // twice at most: where the scale moves, the smallest numbers have other middles
#pragma unroll 1
                        for (int look = 0; look < 2 && again; ++look) {
                            unsigned which = 0;  // a bit an element
#pragma unroll
                            for (int e = 0; e < EPL; ++e) {
                                const unsigned size = finite_magnitude(y[e]);
                                const bool close = from_middle(y[e] * pow2(-e2)) < kMiddle || (border && near_border(size) && (size ^ m) >> 23 == 0);
                                if (turns && in_rot[e / EPV] && close) which |= 1u << e;
                            }
                            for (; which != 0; which &= which - 1) {
                                const int at = __ffs(which) - 1;
                                const float z = rotated_64<T>(a.rot, pos, from, x * EPL + at);
#pragma unroll
                                for (int e = 0; e < EPL; ++e)
                                    if (e == at) y[e] = z;
                            }
                            __syncwarp();
                            m = largest();
                            const int e_now = m == 0 ? 0 : scale_exponent(m);
                            again = __any_sync(0xffffffffu, e_now != e2);
                            e2 = e_now;
                        }
                    }
                    put_row_fp8<T, D>(a, true, r, page, row, x, there && key, y, e2);
                }
            }
        }
    }
    const T* v = static_cast<const T*>(a.v) + (live ? token * a.v_stride : 0) + x * EPL;
    const int h_end = r_end - turned;
#pragma unroll 1
    for (int h0 = max(r_begin - turned, 0); h0 < h_end; h0 += STEP * UNROLL) {
        Dense<FP8> raw[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int h = h0 + u * STEP + r_off;
            raw[u].zero();
            if (h < h_end && live) raw[u].load(v + (long long)h * D, a.wide);
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int h = h0 + u * STEP + r_off;
            const bool store = h < h_end && live;
            if constexpr (!FP8) {
                put_row<T, D>(a, false, h, page, row, x, store, raw[u].a);
            } else {
                float y[EPL];
                Vec16<T>::unpack(raw[u].a, y);
                Vec16<T>::unpack(raw[u].b, y + EPV);
                const unsigned bits[8] = {raw[u].a.x, raw[u].a.y, raw[u].a.z, raw[u].a.w, raw[u].b.x, raw[u].b.y, raw[u].b.z, raw[u].b.w};
                const unsigned m = row_max<T, LPR>(bits, y);
                put_row_fp8<T, D>(a, false, h, page, row, x, store, y, m == 0 ? 0 : scale_exponent(m));
            }
        }
    }
    if (bad) flag_status(a.hdr, CHAI_ERR_BAD_PAGE, b);
}

__global__ void enter_reset_status_kernel(WsHeader* hdr) {
    dependent_grid_sync();
    reset_status(hdr);
}

template <typename T, int D, bool FP8>
int launch_enter(EnterArgs a, cudaStream_t s) {
    constexpr int LPR = D * (int)sizeof(T) / Dense<FP8>::BYTES, STEP = kThreads / LPR / kEnterTokens, UNROLL = kUnroll * 16 / Dense<FP8>::BYTES;
    const int rows = 2 * a.k_planes + a.H;
    const long long groups = ((long long)a.n_tokens + kEnterTokens - 1) / kEnterTokens;
    const long long want = (kFill + groups - 1) / groups, most = (rows + STEP * UNROLL - 1) / (STEP * UNROLL);
    const int parts = (int)(want < most ? want : most);
    a.rows_per_block = ((rows + parts - 1) / parts + STEP - 1) / STEP * STEP;
    CHAI_LAUNCH_DEPENDENT("append_rope_kernel launch", (append_rope_kernel<T, D, FP8>),
                          dim3((unsigned)groups, (rows + a.rows_per_block - 1) / a.rows_per_block), dim3(kThreads), 0, s, a);
    return CHAI_OK;
}

int enter(const char* fn, bool fp8, EnterArgs a, int n_pages, int D, size_t k_page_stride, size_t v_page_stride, int dtype,
          cudaStream_t s) {
    CHAI_REQUIRE(a.q && a.k && a.v && a.q_out && a.k_pages && a.v_pages && a.reps && a.token_request && a.positions && a.slots,
                 CHAI_ERR_INVALID_ARG, "%s: null pointer", fn);
    CHAI_REQUIRE(!fp8 || (a.k_scales && a.v_scales), CHAI_ERR_INVALID_ARG, "%s: null pointer", fn);
    CHAI_REQUIRE(aligned16(a.q) && aligned16(a.k) && aligned16(a.v) && aligned16(a.q_out) && aligned16(a.k_pages) &&
                     aligned16(a.v_pages) && aligned16(a.hdr) && aligned16(a.k_scales) && aligned16(a.v_scales) &&
                     aligned16(a.reps) && aligned16(a.token_request) && aligned16(a.positions) && aligned16(a.slots),
                 CHAI_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned", fn);
    CHAI_REQUIRE(dtype == CHAI_F32 || dtype == CHAI_BF16, CHAI_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, dtype);
    CHAI_REQUIRE(a.n_tokens > 0, CHAI_ERR_INVALID_ARG, "%s: need n_tokens > 0", fn);
    CHAI_REQUIRE(a.n_tokens <= (1 << 30), CHAI_ERR_UNSUPPORTED, "%s: n_tokens must be <= 2^30", fn);
    PagePool pool = {};
    int rc = make_pool(fn, nullptr, a.B, a.H, a.k_planes, n_pages, a.page_size, 1, D, k_page_stride, v_page_stride,
                       fp8 ? 1 : elem_size(dtype), &pool);
    if (rc != CHAI_OK) return rc;
    rc = check_rotation(fn, a.rot, D);
    if (rc != CHAI_OK) return rc;
    const long long dense = (long long)a.H * D, es = (long long)elem_size(dtype);
    for (long long* st : {&a.q_stride, &a.k_stride, &a.v_stride}) {
        if (*st == 0) *st = dense;
        CHAI_REQUIRE(*st >= dense && *st <= (1ll << 56) / a.n_tokens && *st * es % 16 == 0, CHAI_ERR_INVALID_ARG,
                     "%s: token strides must be at least H*D=%lld elements, multiples of 16 bytes and below 2^56 / n_tokens", fn, dense);
    }
    const char* q_to = static_cast<const char*>(a.q_out);
    const long long apart[3] = {a.q_stride, a.k_stride, a.v_stride};
    const void* in[3] = {a.q, a.k, a.v};
    for (int i = 0; i < 3; ++i) {
        const char* from = static_cast<const char*>(in[i]);
        CHAI_REQUIRE(from + ((a.n_tokens - 1) * apart[i] + dense) * es <= q_to || q_to + a.n_tokens * dense * es <= from,
                     CHAI_ERR_INVALID_ARG, "%s: q_out must not overlap q, k or v", fn);
    }
    a.k_page_stride = pool.k_page_stride;
    a.v_page_stride = pool.v_page_stride;
    a.by_page = pool.by_page;
    a.n_slots = (long long)n_pages * a.page_size;
    a.wide = aligned32(a.q) && aligned32(a.k) && aligned32(a.v) && a.q_stride * es % 32 == 0 && a.k_stride * es % 32 == 0 && a.v_stride * es % 32 == 0;
    CHAI_LOG_CALL("%s: n_tokens=%d B=%d H=%d k=%d D=%d rot=%d dtype=%d page_size=%d", fn, a.n_tokens, a.B, a.H, a.k_planes, D,
                  a.rot.rot, dtype, a.page_size);
    if (a.hdr != nullptr)
        CHAI_LAUNCH_DEPENDENT("status reset", enter_reset_status_kernel, dim3(1), dim3(1), 0, s, a.hdr);
    using bf16 = __nv_bfloat16;
    if (dtype == CHAI_BF16) {
        if (D == 128) return fp8 ? launch_enter<bf16, 128, true>(a, s) : launch_enter<bf16, 128, false>(a, s);
        return fp8 ? launch_enter<bf16, 64, true>(a, s) : launch_enter<bf16, 64, false>(a, s);
    }
    if (D == 128) return fp8 ? launch_enter<float, 128, true>(a, s) : launch_enter<float, 128, false>(a, s);
    return fp8 ? launch_enter<float, 64, true>(a, s) : launch_enter<float, 64, false>(a, s);
}

EnterArgs enter_args(const void* q, const void* k, const void* v, void* q_out, void* k_pages, void* v_pages, float* k_scales,
                     float* v_scales, const int32_t* reps, const int32_t* token_request, const int32_t* positions,
                     const int64_t* slots, const double* turns, int rot, int interleaved, const double* magnitude_host, int B, int H,
                     int k_planes, int n_tokens, int page_size, size_t q_stride, size_t k_stride, size_t v_stride, void* workspace) {
    EnterArgs a = {};
    a.q = q;
    a.k = k;
    a.v = v;
    a.q_out = q_out;
    a.k_pages = k_pages;
    a.v_pages = v_pages;
    a.k_scales = k_scales;
    a.v_scales = v_scales;
    a.reps = reps;
    a.token_request = token_request;
    a.positions = positions;
    a.slots = slots;
    a.rot = {turns, rot, interleaved, magnitude_host != nullptr ? *magnitude_host : 1.0};
    a.B = B;
    a.H = H;
    a.k_planes = k_planes;
    a.n_tokens = n_tokens;
    a.page_size = page_size;
    a.q_stride = (long long)q_stride;
    a.k_stride = (long long)k_stride;
    a.v_stride = (long long)v_stride;
    a.hdr = static_cast<WsHeader*>(workspace);
    return a;
}

}  // namespace
}  // namespace chai

extern "C" {

int chai_rope(const void* q, const void* k, void* q_out, void* k_out, const int32_t* positions, const double* turns, int B,
              int Hq, int Hk, int N, int D, int rot, int interleaved, const double* magnitude_host, const int64_t* strides, int dtype,
              void* stream) {
    using namespace chai;
    const char* fn = "chai_rope";
    CHAI_REQUIRE(q && q_out && (Hk == 0 || (k && k_out)), CHAI_ERR_INVALID_ARG, "%s: null pointer", fn);
    CHAI_REQUIRE(aligned16(q) && aligned16(q_out) && aligned16(k) && aligned16(k_out) && (reinterpret_cast<uintptr_t>(positions) & 3u) == 0,
                 CHAI_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned", fn);
    CHAI_REQUIRE(B > 0 && Hq > 0 && Hk >= 0 && N > 0, CHAI_ERR_INVALID_ARG, "%s: need B, Hq, N > 0 and Hk >= 0", fn);
    CHAI_REQUIRE(dtype == CHAI_F32 || dtype == CHAI_BF16, CHAI_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, dtype);
    CHAI_REQUIRE(D == 64 || D == 128, CHAI_ERR_UNSUPPORTED, "%s: head_dim %d (64 or 128 supported)", fn, D);
    CHAI_REQUIRE(Hq <= 65535 && Hk <= 65535 && (long long)B * N < (1ll << 34), CHAI_ERR_UNSUPPORTED,
                 "%s: heads must be <= 65535 and B * N below 2^34", fn);
    RopeArgs a = {};
    a.positions = positions;
    a.rot = {turns, rot, interleaved, magnitude_host != nullptr ? *magnitude_host : 1.0};
    int rc = check_rotation(fn, a.rot, D);
    if (rc != CHAI_OK) return rc;
    a.B = B;
    a.N = N;
    const int heads[2] = {Hq, Hk};
    const void* in[2] = {q, k};
    void* out[2] = {q_out, k_out};
    const long long es = (long long)elem_size(dtype);
    for (int i = 0; i < 2; ++i) {
        Strided& x = a.x[i];
        x.in = in[i];
        x.out = out[i];
        x.heads = heads[i];
        long long* to[6] = {&x.b, &x.h, &x.n, &x.ob, &x.oh, &x.on};
        for (int j = 0; j < 6; ++j) {
            const long long dense[3] = {(long long)heads[i] * N * D, (long long)N * D, (long long)D};
            *to[j] = strides != nullptr ? strides[6 * i + j] : dense[j % 3];
            CHAI_REQUIRE(heads[i] == 0 || (*to[j] >= 0 && *to[j] * es % 16 == 0 && *to[j] <= (1ll << 40)), CHAI_ERR_INVALID_ARG,
                         "%s: strides must be multiples of 16 bytes, from 0 to 2^40 elements", fn);
            const long long sizes[3] = {B, heads[i], N};
            CHAI_REQUIRE(heads[i] == 0 || j < 3 || *to[j] > 0 || sizes[j % 3] <= 1, CHAI_ERR_INVALID_ARG, "%s: strides of an output must not be 0", fn);
        }
    }
    Rows from[2], to[2];
    const int arrays = Hk > 0 ? 2 : 1;
    for (int i = 0; i < arrays; ++i) {
        from[i] = rows_of(a.x[i], false, B, N);
        to[i] = rows_of(a.x[i], true, B, N);
        CHAI_REQUIRE(nested(to[i], D), CHAI_ERR_INVALID_ARG,
                     "%s: rows of an output must not overlap one another (strides, in ascending order, each at least what the smaller ones span)", fn);
    }
    for (int i = 0; i < arrays; ++i)
        for (int j = 0; j < arrays; ++j) {
            bool in_place = i == j && from[i].base == to[i].base;
            for (int d = 0; d < 3; ++d) in_place &= from[i].stride[d] == to[j].stride[d];
            CHAI_REQUIRE(in_place || !rows_meet(from[i], to[j], D, (int)es), CHAI_ERR_INVALID_ARG,
                         "%s: an output may be its own input, with the same strides, but not overlap an input otherwise", fn);
        }
    CHAI_REQUIRE(arrays < 2 || !rows_meet(to[0], to[1], D, (int)es), CHAI_ERR_INVALID_ARG, "%s: outputs must not overlap", fn);
    CHAI_LOG_CALL("%s: B=%d Hq=%d Hk=%d N=%d D=%d rot=%d interleaved=%d dtype=%d", fn, B, Hq, Hk, N, D, rot, interleaved, dtype);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (dtype == CHAI_BF16) return D == 128 ? launch_rope<__nv_bfloat16, 128>(a, s) : launch_rope<__nv_bfloat16, 64>(a, s);
    return D == 128 ? launch_rope<float, 128>(a, s) : launch_rope<float, 64>(a, s);
}

int chai_append_rope_paged(const void* q, const void* k, const void* v, void* q_out, void* k_pages, void* v_pages,
                           const int32_t* reps, const int32_t* token_request, const int32_t* positions, const int64_t* slots,
                           const double* turns, int rot, int interleaved, const double* magnitude_host, int B, int H, int k_planes,
                           int n_tokens, int n_pages, int page_size, int D, size_t q_token_stride, size_t k_token_stride,
                           size_t v_token_stride, size_t k_page_stride, size_t v_page_stride, int dtype, void* workspace,
                           void* stream) {
    return chai::enter("chai_append_rope_paged", false,
                       chai::enter_args(q, k, v, q_out, k_pages, v_pages, nullptr, nullptr, reps, token_request, positions, slots,
                                        turns, rot, interleaved, magnitude_host, B, H, k_planes, n_tokens, page_size, q_token_stride,
                                        k_token_stride, v_token_stride, workspace),
                       n_pages, D, k_page_stride, v_page_stride, dtype, static_cast<cudaStream_t>(stream));
}

int chai_append_rope_paged_fp8(const void* q, const void* k, const void* v, void* q_out, void* k_pages, void* v_pages,
                               float* k_scales, float* v_scales, const int32_t* reps, const int32_t* token_request,
                               const int32_t* positions, const int64_t* slots, const double* turns, int rot, int interleaved,
                               const double* magnitude_host, int B, int H, int k_planes, int n_tokens, int n_pages, int page_size, int D,
                               size_t q_token_stride, size_t k_token_stride, size_t v_token_stride, size_t k_page_stride,
                               size_t v_page_stride, int dtype, void* workspace, void* stream) {
    return chai::enter("chai_append_rope_paged_fp8", true,
                       chai::enter_args(q, k, v, q_out, k_pages, v_pages, k_scales, v_scales, reps, token_request, positions,
                                        slots, turns, rot, interleaved, magnitude_host, B, H, k_planes, n_tokens, page_size,
                                        q_token_stride, k_token_stride, v_token_stride, workspace),
                       n_pages, D, k_page_stride, v_page_stride, dtype, static_cast<cudaStream_t>(stream));
}

int chai_rope_frequencies(double* turns_host, double* magnitude_host, int rot, int scaling, const double* parameters_host) {
    using namespace chai;
    const char* fn = "chai_rope_frequencies";
    CHAI_REQUIRE(turns_host != nullptr && magnitude_host != nullptr && parameters_host != nullptr, CHAI_ERR_INVALID_ARG, "%s: null pointer", fn);
    const double base = parameters_host[0], factor = parameters_host[1], context = parameters_host[2], low = parameters_host[3], high = parameters_host[4];
    CHAI_REQUIRE(rot > 0 && rot % 2 == 0 && rot <= 1024, CHAI_ERR_INVALID_ARG, "%s: rot must be even, from 2 to 1024", fn);
    CHAI_REQUIRE(isfinite(base) && base > 1.0, CHAI_ERR_INVALID_ARG, "%s: base must be above 1", fn);
    CHAI_REQUIRE(scaling >= CHAI_ROPE_PLAIN && scaling <= CHAI_ROPE_BANDS, CHAI_ERR_UNSUPPORTED, "%s: unknown scaling %d", fn, scaling);
    CHAI_REQUIRE(scaling == CHAI_ROPE_PLAIN || (isfinite(factor) && factor >= 1.0), CHAI_ERR_INVALID_ARG, "%s: factor must be at least 1", fn);
    CHAI_REQUIRE(scaling != CHAI_ROPE_BASE || rot > 2, CHAI_ERR_INVALID_ARG, "%s: a scaled base needs rot > 2", fn);
    CHAI_REQUIRE(scaling < CHAI_ROPE_RAMP || (isfinite(context) && context > 0.0 && isfinite(low) && low > 0.0 && isfinite(high) && high > low),
                 CHAI_ERR_INVALID_ARG, "%s: need context > 0 and 0 < low < high", fn);
    const double pi = 3.14159265358979323846;
    const double used = scaling == CHAI_ROPE_BASE ? base * pow(factor, (double)rot / (rot - 2)) : base;
    *magnitude_host = 1.0;
    double first = 0, last = 0;
    if (scaling == CHAI_ROPE_RAMP) {
        // the pairs that turn `high` and `low` times over the context, as fractional indexes
        first = fmax(floor(rot * log(context / (high * 2 * pi)) / (2 * log(base))), 0.0);
        last = fmin(ceil(rot * log(context / (low * 2 * pi)) / (2 * log(base))), (double)(rot - 1));
        *magnitude_host = 0.1 * log(factor) + 1.0;
    }
    for (int i = 0; i < rot / 2; ++i) {
        const double f = pow(used, -2.0 * i / rot) / (2 * pi);
        double keep = 1.0;  // the share of the unscaled frequency
        if (scaling == CHAI_ROPE_LINEAR) keep = 0.0;
        if (scaling == CHAI_ROPE_RAMP) keep = 1.0 - fmin(fmax((i - first) / fmax(last - first, 0.001), 0.0), 1.0);
        if (scaling == CHAI_ROPE_BANDS) keep = fmin(fmax((context * f - low) / (high - low), 0.0), 1.0);
        turns_host[i] = f * keep + f / factor * (1.0 - keep);
        if (scaling == CHAI_ROPE_PLAIN || scaling == CHAI_ROPE_BASE) turns_host[i] = f;
    }
    return CHAI_OK;
}

}  // extern "C"
