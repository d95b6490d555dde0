// Clustered decode attention over a paged cache (Fig. 3(b), Section 3.4), bound by HBM:
//   out[b][h] = sum_t p_t V[h][t],  p = softmax_t(scale * q[r] . K[c][t]),  c the head's cluster, r its representative.
//
// The rows of all requests, in units of sixteen, are one line that is cut into equal pieces, one per CTA and one CTA per
// SM: ragged batches and a single long request are balanced alike, whatever the clusters' sizes, because a piece
// carries the key rows of all clusters and the value rows of all heads.  (Where pieces would be short or the layer has
// many planes, pieces are made longer, and the heads, ordered by cluster, are dealt to several CTAs instead.)  A CTA goes
// through its piece request by request in chunks that fit its score buffer:
//   K   its warps share the (cluster, tile) pairs of the chunk: scores into shared memory
//   S   per cluster: running maximum and sum, scores become probabilities
//   V   its warps share the (head, tile) pairs, in order of heads: sums of p_t V_t; a head that two warps share is
//       added up in warp order
// Every warp feeds itself: it owns two slots of shared memory, and as soon as it is done with a tile it starts the copies of
// the next one into the freed slot (bulk copies, a lane for each run of rows that are neighbours in memory; e4m3: 16 bytes
// a lane), values of the chunk and keys of the next one included, so that HBM is busy through the two barriers between
// the phases.
// A request that lies in one piece is written at once.  The others leave one partial result (maximum, sum, values) per
// piece, and a second kernel, launched as a programmatic dependent, joins them: all sums are taken in an order that
// follows from the lengths and memberships alone, and nothing in the workspace has to be cleared.  (Joining in this
// kernel, by the CTA of a request or the warp of a head that arrives last on a tagged word, was tried on an earlier form that
// took 11.3 us for one request of 256 tokens and 65 for the 7B shape below: 15.7 and 20, 76 and 79.  Few hands then do at
// the end what the second kernel spreads over the GPU.)
//
// Measured (GPU time a call, calls back to back, of the 6566 GB/s that a copy reaches): 7B shape (16 requests of 2048
// tokens, 32 heads, 8 clusters, bf16) 60.0 us = 85 %; one request of 131072 tokens 207 us = 99 %; the 7B shape in e4m3 with
// 32 clusters 54.5 us = 77 %.  Rows stream at the copy's rate or near it; what is left is constant, some 4 us from
// the start to the first tile's arrival (lengths, then tables and memberships, then rows: three round trips), 4 for the
// join, and the phases of the CTAs that two requests meet in.  e4m3 is also bound by the latencies of a warp's instructions
// (issue slots are half full, the tensor cores busy for a seventh of the time), which more warps hide: see Geom.
#include <type_traits>

#include "paged.cuh"

namespace chai {
namespace {

constexpr int kMaxCtas = 160;     // the workspace bound is stated for this many; a B200 has 148 SMs
constexpr int kQuantum = 8;       // rows; page sizes are multiples of it
constexpr int kJoinThreads = 128, kJoinBlocks = 37;  // blocks per head, at most
// Up to so many requests, their columns are dealt to D / 32 blocks a head: few requests have many pieces each and few blocks
// to join them.  One request of 2000 tokens 14.5 -> 12.6 us, of 20000 44.0 -> 41.4, of 131072 209.5 -> 206.8; two of 2048 19.1
// -> 17.4; four of 300 and less 11.6 -> 11.9, four of 2048 and less, e4m3, 28.8 -> 29.3.
constexpr int kJoinFew = 2;
constexpr int kUnit = 16;         // rows; the line of all rows is divided in units of so many
// Units that a request counts more than it has, in front: what a CTA loses where one request ends and the next begins, which
// a CTA without such a place makes up for.  In rows, 0 / 16 / 32 / 48 / 64 / 112: e4m3, 7B shape 58.4 / 56.7 / 56.9 / 55.9 /
// 54.5 / 54.8 us; 16 requests of 600 tokens 31.6 / 30.7 / 28.8 / 27.9 / 26.3 / 26.5; bf16, 7B shape 62.5 / 61.0 / 60.9 / 60.1 /
// 60.2 / 60.5.  Where all requests are short, CTAs meet several ends each, and more is lost to uneven pieces: 60 of up to 100
// tokens 32.5 / 30.7 / 27.1 / 27.0 / 28.2 / 30.3, 16 of up to 200 21.1 / 20.3 / 15.6 / 15.7 / 15.7 / 16.4.  So by the length, 32
// to 64.
__device__ __forceinline__ int overhead(int n) { return min(4, max(2, n >> 7)); }
__device__ __forceinline__ int units(int n) { return n > 0 ? (n + kUnit - 1) / kUnit + overhead(n) : 0; }
// e4m3: x as two fp16 numbers, h = fp16(x) and fp16(2^11 (x - h)).  2^11 keeps the second as large as the first: where both
// are normal numbers they hold x to 2^-22, and the error never exceeds 2^-36 (2^-25 if it were stored as it is).
constexpr float kLow = 2048.f;
constexpr float kProductFactor = 524288.f;  // brings products of 2^-12 ... 2^-4, as cached activations have, to 2^7 ... 2^15

template <typename T, typename TQ, int D>
struct Geom {
    static constexpr bool FP8 = std::is_same<T, Fp8E4M3>::value;
    // warps: e4m3, bound by the latency of a warp's instructions, as many as have registers enough (7B shape: 12 59.4 us,
    // 14 60.4, 16 54.5; 18 spill); the others as many as keep the copies going (bf16, 7B shape: 10 62.7 us, 12 60.0, 14 59.9, 16
    // 59.1, ragged 33B shape 60.3, 58.4, 58.3, 59.1; fp32, one request of 256 tokens 10.2, 10.1, 10.5, 10.7)
    static constexpr int W = FP8 ? 16 : 12, THREADS = W * 32;
    static constexpr int ROW = D * (int)sizeof(T);
    static constexpr int TR = FP8 ? 32 : 4096 / ROW;  // rows of a tile
    // Slots of a warp.  Two tiles of 4 KB in flight for each of 12 warps are 98 KB an SM, more than the rate takes; a third
    // only makes the queue longer, which every phase with few tiles a warp waits for (an earlier form, bf16: 131072 tokens 221
    // us with three, 211 with two; 7B shape 63.4 and 61.2).
    static constexpr int STAGES = 2;
    static constexpr int DATA = TR * ROW;
    static constexpr int QUERY = DATA + (FP8 ? TR * 4 : 0);  // e4m3: the rows' scales lie behind them ...
    static constexpr int QROW = D * (int)sizeof(TQ), SLOT = QUERY + QROW;  // ... and the query of a new cluster's keys
    static constexpr int HEADS = 112;    // heads a CTA handles at most
    static constexpr int SCORES = 8192;  // scores of a chunk: clusters * rows
    static constexpr int CHUNK_ROWS = 512;
    // types of 2 and 4 bytes: lanes a row, rows a warp-wide load, such loads a tile
    static constexpr int LPR = ROW / 16, RPW = 32 / LPR, IT = TR / RPW;
    // e4m3: the tensor cores take 16 rows a step; in phase V a quarter of the lanes reads four rows of them.  A row's
    // 16-byte pieces lie in its 128-byte line (two rows a line for D = 64) at a place that is the piece's number xor
    // 2 * (row / 4 % 4), for D = 128 also xor 4 * (row % 2): the lanes of a load then meet different banks
    static constexpr int STEPS = TR / 16;
    // how a lane holds a row of values: VPL neighbours from column col(lane) on, in the lanes that own(lane)
    static constexpr int VPL = FP8 ? D / 8 : 16 / (int)sizeof(T);
    __device__ static __forceinline__ bool own(int lane) { return FP8 ? (lane & 3) == 0 : lane < LPR; }
    __device__ static __forceinline__ int col(int lane) { return FP8 ? (lane >> 2) * VPL : (lane % LPR) * VPL; }
};

struct DecodeWs {
    int* err;      // [kMaxCtas] what each CTA met: a status, or CHAI_OK
    int* err_b;    // [kMaxCtas]
    int4* desc;    // [min(B, CTAs)] x: request (-1: nothing to join), y: first slot, z: slots
    int* slot_bad; // [kMaxCtas + B] a page of the slot's rows was bad
    float2* ml;    // [kMaxCtas + B][H] maximum (in powers of two) and sum; a sum of -1: no such head
    float* o;      // [kMaxCtas + B][H][D]
};
inline size_t decode_ws(char* base, int B, int H, int D, DecodeWs* w) {
    const size_t slots = (size_t)kMaxCtas + B;
    size_t off = sizeof(WsHeader);
    auto take = [&](size_t bytes) {
        char* p = base + off;
        off = round_up(off + bytes, 256);
        return p;
    };
    w->err = reinterpret_cast<int*>(take(4 * kMaxCtas));
    w->err_b = reinterpret_cast<int*>(take(4 * kMaxCtas));
    w->desc = reinterpret_cast<int4*>(take(16 * kMaxCtas));
    w->slot_bad = reinterpret_cast<int*>(take(4 * slots));
    w->ml = reinterpret_cast<float2*>(take(8 * slots * H));
    w->o = reinterpret_cast<float*>(take(4 * slots * H * D));
    return off;
}

struct DecodeArgs {
    const void *q, *k_pages, *v_pages;
    const float *k_scales, *v_scales;
    const int32_t *membership, *reps, *seq_lens;
    void* out;
    WsHeader* hdr;
    DecodeWs ws;
    PagePool pool;
    int B, H, k, n_desc;
    float scale_log2;
    long long wait_limit;
};

// ---- shared memory ----------------------------------------------------------------------------------------------

// n / d for 0 <= n < 2^20, 0 < d: (n + 1/2) / d is 1/(2 d) or more away from an integer, its rounding at most n / d * 2^-22.
__device__ __forceinline__ int small_div(int n, int d) { return (int)__fdividef((float)n + 0.5f, (float)d); }

template <int HEADS>
struct Segment {  // the rows of one request in this CTA's piece
    unsigned short head[HEADS];     // heads, ordered by cluster
    unsigned short cluster[HEADS];  // the head's cluster: its place among the clusters that have heads
    unsigned short id[HEADS];       // at place % HEADS: the cluster's own number ...
    unsigned short rep[HEADS];      // ... and representative
    int first, last;                      // places of this list's clusters (heads are many to a cluster: never more places than heads)
};
struct Chunk {
    int b, rows, stride;  // stride: floats between two clusters' scores
    int tiles, heads, clusters, run;
    int first, last, single, slot;  // first / last chunk of the segment; single: the segment is the whole request
    int seg;
};
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xffffffffu, x, 0); }  // the same in every lane, and known to be
struct Plan {  // how the line of all rows is divided; kept in shared memory, for registers are short
    int pieces, each, rest;  // a piece has each or each + 1 units
    int piece, group, groups;
    int q_hi;                // where this CTA's piece ends
    // place where piece i begins (i * total / pieces without 64-bit division; i and rest are at most kMaxCtas)
    __device__ __forceinline__ int start(int i) const { return i * each + small_div(i * rest, pieces); }
};
struct Division {  // how far the CTA has divided its piece
    int q_at, b;                    // place on the line, request
    int next_b, next_n, next_start; // the next request with rows (B: none), its length and place
    int t, end, rows;      // of the current segment: next row, last row, rows of a chunk
    int par, heads, clusters, slot, span_end;
    int single, first, opened_span;
};
template <int GROUPS>
struct Rows {  // where each eight rows of a chunk lie: byte offsets in plane 0 of the pages, page and row
    size_t k[GROUPS], v[GROUPS];
    int2 at[GROUPS];
};
template <typename G, int D>
struct Smem {
    alignas(128) unsigned char slot[G::W][G::STAGES][G::SLOT];
    alignas(16) float score[G::SCORES];
    union {
        alignas(16) float part[G::W][D];  // phase V: sums of a head's rows that another warp finishes
        struct {                          // while a segment is prepared, of every head:
            alignas(16) unsigned key[kPagedMaxHeads];  // cluster * 2048 + 2 * head, + 1 for a representative
            unsigned short mem[kPagedMaxHeads], rep[kPagedMaxHeads];
        } all;
    };
    float top[G::HEADS], sum[G::HEADS], keep[G::HEADS];  // per cluster: running maximum and sum, rescaling factor
    Segment<G::HEADS> seg[2];
    Chunk chunk[2];
    alignas(16) Rows<G::CHUNK_ROWS / kQuantum> rows[2];
    alignas(8) unsigned long long full[G::W][G::STAGES];
    int scan[G::W];
    Plan plan;
    Division division[2];
    int found_b, found_n, found_start;
    int err, err_b, any_bad;
};

// ---- small device helpers ---------------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.b32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
__device__ __forceinline__ bool bar_test(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.b32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
// A wait that does not succeed at once.  try_wait lets the hardware suspend the warp for a while, which a limit shorter
// than the default would not notice: such a limit polls instead.
__device__ __noinline__ bool bar_wait(uint32_t bar, uint32_t parity, long long limit) {
    const bool poll = limit < kDefaultWaitLimitCycles;
    const long long t0 = clock64();
    while (clock64() - t0 <= limit)
        if (poll ? bar_test(bar, parity) : bar_try(bar, parity)) return true;
    return false;
}
__device__ __forceinline__ void copy_rows(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
                 "r"(bytes), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// 16 bytes, of which `n` come from src and the others are zero
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, int n) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint4 lds16(const unsigned char* p) { return *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ uint2 lds8(const unsigned char* p) { return *reinterpret_cast<const uint2*>(p); }
__device__ __forceinline__ uint64_t pack2(float x, float y) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ float2 unpack2(uint64_t v) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
// four e4m3 numbers as two pairs of fp16 (exact): the low two bytes and the high two
__device__ __forceinline__ void e4m3_halves(uint32_t w, uint32_t* lo, uint32_t* hi) {
    asm("{\n\t.reg .b16 x, y;\n\tmov.b32 {x, y}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, x;\n\tcvt.rn.f16x2.e4m3x2 %1, y;\n\t}"
        : "=r"(*lo), "=r"(*hi)
        : "r"(w));
}
__device__ __forceinline__ uint32_t half_pair(float x, float y) {
    const __half2 h = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 half_floats(uint32_t h) { return __half22float2(*reinterpret_cast<const __half2*>(&h)); }
// c += a b with a 16 x 16 (row), b 16 x 8 (col), fp16, fp32 sums
__device__ __forceinline__ void mma16816(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The parts of two numbers times f, a power of two
__device__ __forceinline__ void two_halves(uint64_t x, float f, uint32_t* hi, uint32_t* lo) {
    const float2 y = unpack2(mul2(x, pack2(f, f)));
    *hi = half_pair(y.x, y.y);
    const float2 h = half_floats(*hi);
    const float2 rest = unpack2(fma2(pack2(h.x, h.y), pack2(-kLow, -kLow), mul2(pack2(y.x, y.y), pack2(kLow, kLow))));  // (exact)
    *lo = half_pair(rest.x, rest.y);
}
// A power of two f with |x| f in [1, 2) and its inverse; below 1 where x is subnormal or 0; 1 where x is infinite or NaN.
__device__ __forceinline__ void normaliser(float x, float* f, float* inv) {
    const unsigned e = max((__float_as_uint(x) >> 23) & 0xffu, 1u);
    *f = e == 254u ? __uint_as_float(1u << 22) : __uint_as_float((e == 255u ? 127u : 254u - e) << 23);  // (2^-127 is subnormal)
    *inv = __uint_as_float((e == 255u ? 127u : e) << 23);
}
// A power of two f with x f in [2^10, 2^11), for x of 2^-117 and more (below: f = 2^127); 1 where x is infinite.  1 / f is exact.
__device__ __forceinline__ float product_factor(float x) {
    const unsigned e = max((__float_as_uint(x) >> 23) & 0xffu, 10u);
    return __uint_as_float((e == 255u ? 127u : 264u - e) << 23);
}

// ---- the main kernel --------------------------------------------------------------------------------------------

// A warp's way through the tiles of a chunk: its share of the (cluster, tile) pairs, then of the (head, tile) pairs.
template <int W>
struct Walk {
    int phase, p, j, left;
    bool fresh;  // p has changed
    __device__ __forceinline__ void start(int ph, const Chunk& c, int warp) {
        const int tiles = uniform(c.tiles), n = uniform(ph == 0 ? c.clusters : c.heads) * tiles;
        const int lo = n * warp / W;
        phase = ph;
        left = n * (warp + 1) / W - lo;
        p = small_div(lo, tiles);
        j = lo - p * tiles;
        fresh = true;
    }
    __device__ __forceinline__ void step(int tiles) {
        --left;
        if (++j == tiles) {
            j = 0;
            ++p;
            fresh = true;
        }
    }
};

template <typename T, typename TQ, int D>
__global__ void __launch_bounds__(Geom<T, TQ, D>::THREADS, 1) paged_decode_kernel(const DecodeArgs a) {
    using G = Geom<T, TQ, D>;
    using S = Smem<G, D>;
    constexpr int W = G::W, THREADS = G::THREADS;
    extern __shared__ __align__(128) unsigned char smem_raw[];
    S& sm = *reinterpret_cast<S*>(smem_raw);
    const int tid = threadIdx.x, lane = tid & 31, warp = uniform(tid >> 5);
    const int ps = a.pool.page_size;
    if (lane == 0) {
        // types of 2 and 4 bytes: one arrival that announces the bytes of the bulk copies; e4m3: one a lane
        for (int s = 0; s < G::STAGES; ++s)
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(&sm.full[warp][s])), "r"(G::FP8 ? 32 : 1) : "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (tid == 0) sm.err = CHAI_OK, sm.err_b = -1;
    dependent_grid_sync();

    // -- the line of all rows, this CTA's piece [q_lo, q_hi) and the request it starts in
    auto length = [&](int b) { return min(max(a.seq_lens[b], 0), a.pool.capacity); };
    const bool few = a.B <= 32;  // every warp then looks at all requests by itself, a lane each: no barrier is needed
    const int per = few ? 1 : (a.B + THREADS - 1) / THREADS;
    const int b_lo = min((few ? lane : tid) * per, a.B), b_hi = min(b_lo + per, a.B);
    int mine = 0, n_last = 0;
#pragma unroll 1
    for (int b = b_lo; b < b_hi; ++b) mine += units(n_last = length(b));
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
    }
    int total = __shfl_sync(0xffffffffu, upto, 31);
    if (!few) {
        if (lane == 31) sm.scan[warp] = upto;
        __syncthreads();
        total = 0;
#pragma unroll 1
        for (int w = 0; w < W; ++w) {
            if (w < warp) upto += sm.scan[w];
            total += sm.scan[w];
        }
    }
    // Heads are dealt to several CTAs when a piece would be shorter than 32 rows, down to 4 heads a CTA: one request of 256
    // tokens takes 10.1 us a call instead of 11.4; of 512, 10.6 instead of 12.0.  With thresholds of 16 and 64 rows: one of 2000
    // 13.7 and 13.5 us, 13.0 with 32; four ragged to 500 12.8 and 12.0, 11.4; but e4m3, 66B shape, ragged to 400: 15.0 and 21.2,
    // 19.5.
    // To two CTAs, in layers of 40 planes and more, when that makes pieces longer at little cost: more even (in units), and
    // fewer partial results.  A cluster that both have a part of has its keys read twice, and a CTA meets twice the requests.
    // Worth it for few requests whatever the rows (32 heads, 8 clusters, e4m3: one of 16384 tokens 33.5 -> 28.5 us, five ragged
    // to 2000 21.4 -> 18.4, to 8000 37.9 -> 39.5); else where the planes' rows are 8 KB and more (bf16, 32 and 8: 8 requests 29.6
    // -> 28.7, 16 62.0 -> 60.8; 72 and 24, e4m3: 8 requests 42.9 -> 36.5) or more than 16 clusters shorten the chunks (32 and
    // 32, e4m3, D = 64: 16 requests 44.9 -> 42.2).  Not otherwise (32 and 8, e4m3: 8 requests ragged to 8000 54.2 -> 59.8, 16 of
    // 2048 41.3 -> 43.8), nor for many requests (64: 52.6 -> 60.5, bf16 76.7 -> 78.2).
    const int n_ctas = gridDim.x;
    const int base_groups = (a.H + G::HEADS - 1) / G::HEADS;
    int group_log = 0, most_pieces = base_groups == 1 ? n_ctas : small_div(n_ctas, base_groups);
    const bool two = a.H + a.k >= 40 && 4 * a.B <= n_ctas && (a.B < 8 || (a.H + a.k) * G::ROW >= 8192 || a.k > 16);
    while (((two && group_log == 0) || total < 2 * most_pieces) && (8 * base_groups << group_log) <= a.H && most_pieces > 1)
        ++group_log, most_pieces >>= 1;
    const int groups = base_groups << group_log;
    Plan plan;
    plan.pieces = max(1, min(most_pieces, total));
    plan.groups = groups;
    plan.piece = base_groups == 1 ? (int)blockIdx.x >> group_log : small_div(blockIdx.x, groups);
    plan.group = blockIdx.x - plan.piece * groups;
    plan.each = total / plan.pieces;
    plan.rest = total - plan.each * plan.pieces;
    const bool work = plan.piece < plan.pieces && total > 0;
    const int q_lo = work ? plan.start(plan.piece) : 0;
    plan.q_hi = work ? plan.start(plan.piece + 1) : 0;
    int found_b = 0, found_n = 0, found_start = 0;
    {
        const bool here = work && mine > 0 && q_lo >= upto - mine && q_lo < upto;
        if (few) {
            const unsigned who = __ballot_sync(0xffffffffu, here);
            found_b = who ? __ffs(who) - 1 : 0;
            found_n = __shfl_sync(0xffffffffu, n_last, found_b);
            found_start = __shfl_sync(0xffffffffu, upto - mine, found_b);
        } else {
            if (here) {
                int start = upto - mine, b = b_lo, n = length(b);
                while (b + 1 < b_hi && q_lo >= start + units(n)) start += units(n), n = length(++b);
                sm.found_b = b;
                sm.found_n = n;
                sm.found_start = start;
            }
            __syncthreads();
            if (work) found_b = sm.found_b, found_n = sm.found_n, found_start = sm.found_start;
        }
    }
    const bool by_request = a.n_desc == a.B;  // descriptions are kept per request, or (more requests than CTAs) per piece
    const bool some_empty = !few || __any_sync(0xffffffffu, lane < a.B && mine == 0);
    if (tid == 0) {
        sm.plan = plan;
        Division& d = sm.division[1];
        d.q_at = q_lo;
        d.next_b = found_b;
        d.next_n = found_n;
        d.next_start = found_start;
        d.t = d.end = 0;
        d.par = 1;
        d.opened_span = 0;
    }
    __syncthreads();

    // Prepares the next chunk into buffer `par`; false if the piece is done.  Called by all threads together, which
    // meet at a barrier afterwards.  Which way they take follows from the division in shared memory alone: one thread
    // reads a request's length, once (threads that read it for themselves would go apart, and read rows that nobody looked
    // up, if another stream wrote it meanwhile).
    auto prepare = [&](int par) -> bool {
        const Plan& plan = sm.plan;
        Division d = sm.division[par ^ 1];
        bool fresh = false, from_start = false;
        if (d.t >= d.end) {  // the next request that has rows here
            if (d.q_at >= plan.q_hi || d.next_b >= a.B) return false;
            const int n = d.next_n, stop = d.next_start + units(n), rows_at = d.next_start + overhead(n), q_end = min(plan.q_hi, stop);
            if (d.q_at >= stop || q_end <= rows_at) return false;  // (the piece ends before the request's first row)
            d.b = d.next_b;
            from_start = d.q_at <= rows_at;
            d.t = max(d.q_at - rows_at, 0) * kUnit;
            d.end = min(n, (q_end - rows_at) * kUnit);
            d.single = from_start && q_end == stop;
            d.span_end = from_start && !d.single ? stop : 0;
            d.slot = plan.piece + d.b;
            d.q_at = d.next_start = q_end;
            d.next_b = d.b + 1;
            fresh = true;
        }
        const int b = d.b, seg_t = d.t, seg_end = d.end, group = plan.group, groups = plan.groups;
        const bool look = tid == 0 && fresh && d.q_at < plan.q_hi && d.next_b < a.B;  // (its round trip passes beside those below)
        int next_n = look ? length(d.next_b) : 0;
        // pages of the rows that the chunk may have (how many it has follows from the number of clusters)
        const int32_t* table = a.pool.block_table + (size_t)b * a.pool.max_pages;
        const int reach = min(seg_end - seg_t, fresh ? G::CHUNK_ROWS : d.rows);
        int page = 0, row = 0;
        static_assert(G::CHUNK_ROWS / kQuantum <= THREADS, "one thread looks up eight rows");
        if (tid * kQuantum < reach) {
            const unsigned pos = (unsigned)(seg_t + tid * kQuantum), pi = a.pool.by_page.div(pos);
            page = table[pi];
            row = (int)(pos - pi * (unsigned)ps);
        }
        if (fresh) {
            d.par ^= 1;
            d.first = 1;
            auto& sg = sm.seg[d.par];
            const bool opens = from_start && group == 0;  // this CTA answers for the request's unknown heads
            if (d.span_end > 0) d.opened_span = 1;
            if (tid == THREADS - 1 && opens && (by_request || !d.single)) {
                int end = plan.piece;  // the piece that the request ends in
                if (!d.single) {
                    end = max(end, min((d.span_end - 1) / (plan.each + 1), plan.pieces - 1));
                    while (end + 1 < plan.pieces && plan.start(end + 1) < d.span_end) ++end;
                }
                a.ws.desc[by_request ? b : plan.piece] = make_int4(d.single ? -1 : b, d.slot, end - plan.piece + 1, 0);
            }
            // heads ordered by cluster; unknown ones get zeros and are left out
            const int32_t* mem = a.membership + (size_t)b * a.H;
            const int32_t* reps = a.reps + (size_t)b * a.k;
            const int padded = (a.H + 7) & ~7;
            for (int h = tid; h < a.H; h += THREADS) {
                const unsigned c = (unsigned)mem[h], r = h < a.k ? (unsigned)reps[h] : 0u;
                sm.all.mem[h] = c < (unsigned)a.k ? (unsigned short)c : 0xffff;
                sm.all.rep[h] = r < (unsigned)a.H ? (unsigned short)r : 0xffff;
            }
            if (tid == 0) sm.any_bad = 0, sg.last = -1;
            __syncthreads();
            int known = 0;
            for (int h0 = 0; h0 < padded; h0 += THREADS) {
                const int h = h0 + tid;
                bool ok = false;
                unsigned c = 0xffff, r = 0xffff;
                if (h < a.H) {
                    c = sm.all.mem[h];
                    if (c != 0xffff) r = sm.all.rep[c];
                    ok = r != 0xffff && sm.all.mem[r] == c;
                }
                if (h < padded) sm.all.key[h] = ok ? c * 2048 + 2 * h + (r == (unsigned)h) : 0xfffffffeu;
                known += __syncthreads_count(ok);
                if (h < a.H && !ok && opens) {
                    atomicCAS(&sm.err, CHAI_OK, CHAI_ERR_BAD_MEMBERSHIP);
                    sm.err_b = b;
                    if (!d.single) a.ws.ml[(size_t)d.slot * a.H + h] = make_float2(0.f, -1.f);
                    TQ* o = static_cast<TQ*>(a.out) + ((size_t)b * a.H + h) * D;
                    for (int d = 0; d < D; ++d) o[d] = from_float<TQ>(0.f);
                }
            }
            // the group's heads: of two groups half the planes (keys of the clusters and values, in order), else as many heads
            // as any (half the heads instead of half the planes: 7B shape 61.6 us, 60.0 this way, 66B shape in e4m3 30.4 and 29.2;
            // many groups have short pieces, where the barrier that this takes costs more than it gains, 0.3 us)
            const bool by_planes = groups == 2 && a.H <= G::HEADS;
            int lo = groups == 1 ? 0 : small_div(known * group, groups), n_heads = groups == 1 ? known : small_div(known * (group + 1), groups) - lo;
            int mine = -1;
            for (int h0 = 0; h0 < a.H; h0 += THREADS) {
                const int h = h0 + tid;
                const unsigned own = h < a.H ? sm.all.key[h] : 0xfffffffeu, c = own / 2048;
                const bool ok = own != 0xfffffffeu;
                int rank = 0, place = 0, places = 0;  // heads before this one, clusters (their representatives) before its own, clusters
                if (ok) {
#pragma unroll 2
                    for (int x = 0; x < padded; x += 4) {
                        const uint4 u = *reinterpret_cast<const uint4*>(&sm.all.key[x]);
                        rank += (u.x < own) + (u.y < own) + (u.z < own) + (u.w < own);
                        place += (u.x & (u.x < c * 2048)) + (u.y & (u.y < c * 2048)) + (u.z & (u.z < c * 2048)) + (u.w & (u.w < c * 2048));
                        places += (u.x & 1) + (u.y & 1) + (u.z & 1) + (u.w & 1);
                    }
                }
                bool in = ok && rank >= lo && rank < lo + n_heads;
                if (by_planes) {  // (one turn of the loop)
                    mine = ok ? small_div((rank + place + 1) * groups, known + places) : -1;
                    lo = __syncthreads_count(ok && mine < group);
                    in = mine == group;
                }
                if (in) {
                    sg.head[rank - lo] = (unsigned short)h;
                    sg.cluster[rank - lo] = (unsigned short)place;
                    sg.id[place % G::HEADS] = (unsigned short)c;
                    sg.rep[place % G::HEADS] = sm.all.rep[c];
                    if (rank == lo) sg.first = place;
                    atomicMax(&sg.last, place);
                }
            }
            if (by_planes) n_heads = __syncthreads_count(mine == group);
            else __syncthreads();
            d.heads = n_heads;
            d.clusters = d.heads > 0 ? sg.last - sg.first + 1 : 0;
            d.rows = min(G::CHUNK_ROWS, small_div(G::SCORES, max(d.clusters, 1)) / G::TR * G::TR);
        }
        const int rows = min(d.rows, seg_end - seg_t);
        if (tid * kQuantum < ((reach + 31) & ~31)) {  // (behind the rows: page 0, an address that is never read)
            if (page < 0 || page >= a.pool.n_pages) {
                sm.any_bad = 1;  // of the segment so far
                page = 0;
            }
            sm.rows[par].k[tid] = ((size_t)page * a.pool.k_page_stride + (size_t)row * D) * sizeof(T);
            sm.rows[par].v[tid] = ((size_t)page * a.pool.v_page_stride + (size_t)row * D) * sizeof(T);
            sm.rows[par].at[tid] = make_int2(page, row);
        }
        if (tid == 0) {
            Chunk& c = sm.chunk[par];
            c.b = b;
            c.rows = rows;
            c.stride = (rows + G::TR - 1) / G::TR * G::TR;
            c.tiles = (rows + G::TR - 1) / G::TR;
            c.heads = d.heads;
            c.clusters = d.clusters;
            const int align = ps | seg_t;
            c.run = min(align & -align, G::TR);
            c.first = d.first;
            c.last = seg_t + rows >= seg_end;
            c.single = d.single;
            c.slot = d.slot;
            c.seg = d.par;
            d.first = 0;
            d.t += rows;
            if (look) {
                while (next_n == 0 && ++d.next_b < a.B) next_n = length(d.next_b);
                d.next_n = next_n;
            }
            sm.division[par] = d;
        }
        return true;
    };

    // -- the warp's own slots
    int issued = 0, used = 0;                                            // tiles started / finished: the next slots follow from them
    static_assert(G::STAGES == 2, "slots and phases are bits of the counts");
    bool dead = false;                                                   // a wait ran out: no more copies, no more waits
    Walk<W> ahead;                                                       // the next tile to start, of chunk number ahead_no
    int ahead_no = 0, ahead_par = 1, ready_no = 0;                       // chunks up to ready_no are prepared
    const char* ahead_plane = nullptr;                                   // the plane of the next tile, in page 0 ...
    [[maybe_unused]] const float* ahead_scales = nullptr;                // ... and its rows' scales
    ahead.left = 0;
    ahead.phase = 1;
    const size_t plane_bytes = (size_t)ps * D * sizeof(T);
    const uint32_t slots = smem_addr(sm.slot[warp][0]), bars = smem_addr(&sm.full[warp][0]);
    // e4m3: a lane's place in a warp-wide copy of 512 bytes (see Geom) whose first row is one of the first four of sixteen:
    // four rows a copy for D = 128; eight for D = 64, where the lane's own row matters too
    [[maybe_unused]] const uint32_t copy_at = (lane >> 3) * 128 + 16 * ((lane & 7) ^ (D == 128 ? 4 * ((lane >> 3) & 1) : 2 * (lane >> 4)));

    // Starts copies until the warp's slots are in flight or nothing is known to copy.  (Addresses are worked out when a slot
    // is free.  Held ready from a tile earlier they cost registers, which are worth more as warps: in an earlier form
    // e4m3 with 16 warps, 7B shape, 61.9 us that way and 56.5 this way, bf16 61.3 and 60.6.)
    auto fill = [&]() __attribute__((always_inline)) {
#pragma unroll 1
        while (!dead && issued - used < G::STAGES) {
            while (ahead.left == 0) {
                if (ahead.phase == 0) {
                    ahead.start(1, sm.chunk[ahead_par], warp);
                } else {
                    if (ahead_no >= ready_no) return;
                    ++ahead_no;
                    ahead_par ^= 1;
                    ahead.start(0, sm.chunk[ahead_par], warp);
                }
            }
            const Chunk& in = sm.chunk[ahead_par];
            const bool key = ahead.phase == 0, query = key && ahead.fresh;
            int query_row = 0;
            if (ahead.fresh) {
                ahead.fresh = false;
                const auto& sg = sm.seg[in.seg];
                const int plane = key ? sg.id[(sg.first + ahead.p) % G::HEADS] : sg.head[ahead.p];
                ahead_plane = static_cast<const char*>(key ? a.k_pages : a.v_pages) + plane * plane_bytes;
                if constexpr (G::FP8) ahead_scales = (key ? a.k_scales : a.v_scales) + plane * (size_t)ps;
                if (key) query_row = in.b * a.H + sg.rep[(sg.first + ahead.p) % G::HEADS];
            }
            const uint32_t slot = slots + (issued & 1) * G::SLOT, bar = bars + (issued & 1) * 8;
            const int row0 = ahead.j * G::TR, n = min(G::TR, in.rows - row0);
            const auto& rows = sm.rows[ahead_par];
            const size_t* off = (key ? rows.k : rows.v) + row0 / kQuantum;
            const char* q = static_cast<const char*>(a.q) + (size_t)(unsigned)query_row * G::QROW;
            ahead.step(in.tiles);
            if constexpr (!G::FP8) {
                const int run = in.run, r0 = lane * run;
                if (lane == 0)
                    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(n * G::ROW + (query ? G::QROW : 0))
                                 : "memory");
                __syncwarp();
                if (r0 < n) copy_rows(slot + r0 * G::ROW, ahead_plane + off[r0 / kQuantum], min(run, n - r0) * G::ROW, bar);
                if (query && lane == 31) copy_rows(slot + G::QUERY, q, G::QROW, bar);
            } else {
                // 16 bytes a lane, and as many of the scales.  Behind the last row the tile is filled with zeros, up to the
                // end of a step
                constexpr int UNITS = kQuantum * G::ROW / 512, EACH = 512 / G::ROW;  // warp-wide copies of eight rows, rows of one
                constexpr int GROUPS = G::TR / kQuantum;
                static_assert(GROUPS == 4 && G::SLOT % 128 == 0, "two loads of offsets; places within a line are found by xor");
                auto place = [&](int g, int u) { return ((slot + copy_at) ^ (32 * ((2 * g + u) & (D == 128 ? 3 : 2)))) + (g * kQuantum + u * EACH) * G::ROW; };
                const ulonglong2 x = reinterpret_cast<const ulonglong2*>(off)[0], y = reinterpret_cast<const ulonglong2*>(off)[1];
                const char* mine = ahead_plane + lane * 16;
                const char* src[GROUPS] = {mine + x.x, mine + x.y, mine + y.x, mine + y.y};
                const int2 at = rows.at[row0 / kQuantum + (lane & 7) / 2];
                const float* scales = ahead_scales + (size_t)(unsigned)at.x * (unsigned)((key ? a.k : a.H) * ps) + (at.y + (lane & 1) * 4);
                if (n == G::TR) {
#pragma unroll
                    for (int g = 0; g < GROUPS; ++g)
#pragma unroll
                        for (int u = 0; u < UNITS; ++u) copy16(place(g, u), src[g] + u * 512);
                    if (lane < 8) copy16(slot + G::DATA + lane * 16, scales);
                } else {
                    const int left = n - lane / (G::ROW / 16);
#pragma unroll 1
                    for (int s = 0; s * 16 < n; ++s)
#pragma unroll
                        for (int g = 0; g < 2; ++g)
#pragma unroll
                            for (int u = 0; u < UNITS; ++u)
                                copy16(place(g, u) + s * 16 * G::ROW, (s == 0 ? src[g] : src[g + 2]) + u * 512, left > s * 16 + g * kQuantum + u * EACH ? 16 : 0);
                    if (lane < 8) copy16(slot + G::DATA + lane * 16, scales, min(max(n - lane * 4, 0), 4) * 4);
                }
                if (query && lane * 16 < G::QROW) copy16(slot + G::QUERY + lane * 16, q + lane * 16);
                asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
            }
            ++issued;
        }
    };
    // Waits for the warp's next tile; nothing if the wait ran out, now or earlier.
    auto take = [&]() -> const unsigned char* {
        if (dead) return nullptr;
        const uint32_t bar = bars + (used & 1) * 8, phase = (used >> 1) & 1;
        if (!__all_sync(0xffffffffu, bar_test(bar, phase))) {
            dead = __any_sync(0xffffffffu, !bar_wait(bar, phase, a.wait_limit));
            if (dead) {
                if (lane == 0) sm.err = CHAI_ERR_TIMEOUT;
                return nullptr;
            }
        }
        return sm.slot[warp][used & 1];
    };
    auto release = [&]() {
        ++used;
        __syncwarp();  // every lane has read the tile before a copy overwrites it
    };

    // -- chunk by chunk
    int no = 0, par = 1;
    bool more = prepare(0);
    __syncthreads();
    if (more) ready_no = 1;

    // -- requests without rows get zeros
    if (some_empty) {
#pragma unroll 1
        for (int z = blockIdx.x; z < a.B; z += n_ctas) {
            if (length(z) > 0) continue;
            if (by_request && tid == 0) a.ws.desc[z] = make_int4(-1, 0, 0, 0);
            uint4* o = reinterpret_cast<uint4*>(static_cast<TQ*>(a.out) + (size_t)z * a.H * D);
#pragma unroll 1
            for (int i = tid; i < a.H * D * (int)sizeof(TQ) / 16; i += THREADS) o[i] = make_uint4(0, 0, 0, 0);
        }
    }
#pragma unroll 1
    while (more) {
        ++no;
        par ^= 1;
        const Chunk& c = sm.chunk[par];
        const auto& sg = sm.seg[c.seg];
        const int first_place = uniform(sg.first), chunk_rows = uniform(c.rows), chunk_tiles = uniform(c.tiles), stride = uniform(c.stride);

        // K: scores of the warp's tiles, in powers of two
        {
            Walk<W> w;
            w.start(0, c, warp);
            int have = -1;
            float factor = 1.f;
            constexpr int QN = G::FP8 ? 1 : 16 / (int)sizeof(T);
            [[maybe_unused]] uint64_t qf[QN / 2 + 1];
            [[maybe_unused]] uint32_t qb[G::FP8 ? D / 8 : 1];  // e4m3: fp16 fragments, column 0 the leading and column 1 the trailing part
#pragma unroll 1
            for (;; w.step(chunk_tiles)) {
                fill();
                if (w.left == 0) break;
                const int row0 = w.j * G::TR;
                const unsigned char* tile = take();
                if (tile == nullptr) break;
                if (w.p != have) {
                    have = w.p;
                    const TQ* q = reinterpret_cast<const TQ*>(tile + G::QUERY);
                    if constexpr (!G::FP8) {
                        float x[QN];
                        Vec16<T>::unpack(*reinterpret_cast<const uint4*>(q + (lane % G::LPR) * QN), x);
#pragma unroll
                        for (int e = 0; e < QN / 2; ++e) qf[e] = pack2(x[2 * e] * a.scale_log2, x[2 * e + 1] * a.scale_log2);
                    } else {
                        // lane (g, t) holds the columns 16 (t + 4 j) ... + 15 of its keys
                        constexpr int J = D / 64, QV = 16 / (int)sizeof(TQ);
                        float x[16 * J], top = 0.f, inv;
#pragma unroll
                        for (int j = 0; j < J; ++j)
#pragma unroll
                            for (int v = 0; v < 16 / QV; ++v)
                                Vec16<TQ>::unpack(reinterpret_cast<const uint4*>(q + ((lane & 3) + 4 * j) * 16)[v], x + 16 * j + v * QV);
#pragma unroll
                        for (int e = 0; e < 16 * J; ++e) top = fmaxf(top, fabsf(x[e]));
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                        float f;
                        normaliser(top, &f, &inv);
                        factor = a.scale_log2 * inv;
#pragma unroll
                        for (int i = 0; i < 8 * J; ++i) {
                            uint32_t hi, lo;
                            two_halves(pack2(x[2 * i], x[2 * i + 1]), f, &hi, &lo);
                            qb[i] = lane < 4 ? hi : (lane < 8 ? lo : 0u);
                        }
                    }
                }
                float* score = sm.score + w.p * stride + row0;
                if constexpr (!G::FP8) {
                    // lanes of a group hold 16 bytes each of rows group * IT + i; a butterfly turns 16 partial sums a
                    // lane into whole sums, halving the rows a lane answers for at every step
                    const unsigned char* base = tile + (lane / G::LPR) * G::IT * G::ROW + (lane % G::LPR) * 16;
                    uint4 raw[G::IT];
                    float s[G::IT];
#pragma unroll
                    for (int i = 0; i < G::IT; ++i) raw[i] = lds16(base + i * G::ROW);
#pragma unroll
                    for (int i = 0; i < G::IT; ++i) {
                        float kf[QN];
                        Vec16<T>::unpack(raw[i], kf);
                        uint64_t sum = 0;
#pragma unroll
                        for (int e = 0; e < QN / 2; ++e) sum = fma2(qf[e], pack2(kf[2 * e], kf[2 * e + 1]), sum);
                        const float2 x = unpack2(sum);
                        s[i] = x.x + x.y;
                    }
                    int row = (lane / G::LPR) * G::IT;
#pragma unroll
                    for (int lv = 1; (1 << lv) <= G::LPR; ++lv) {
                        const int o = G::LPR >> lv, n = G::IT >> lv;
                        if (n >= 1) {
                            const bool up = lane & o;
#pragma unroll
                            for (int i = 0; i < G::IT / 2; ++i) {
                                if (i < n) {
                                    const float send = up ? s[i] : s[i + n], keep = up ? s[i + n] : s[i];
                                    s[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
                                }
                            }
                            row += up ? n : 0;
                        } else {
                            s[0] += __shfl_xor_sync(0xffffffffu, s[0], o);
                        }
                    }
                    constexpr int LEFT = G::IT > G::LPR ? G::IT / G::LPR : 1;  // rows a lane ends with
                    constexpr int SAME = G::LPR > G::IT ? G::LPR / G::IT : 1;  // lanes that end with the same row
#pragma unroll
                    for (int i = 0; i < LEFT; ++i)
                        if (lane % SAME == 0) score[row + i] = s[i];  // (rows behind the last get scores that nothing reads)
                } else {
                    // 16 keys are the rows of A, 16 columns of them a step; B holds the query (leading and trailing part)
                    const int g = lane >> 2, t = lane & 3;
                    const float* scales = reinterpret_cast<const float*>(tile + G::DATA) + g;
                    // rows 16 m + g and 16 m + g + 8, pieces t + 4 j (see Geom; the lane's share taken out)
                    const int lane_at = (D == 128 ? g * 128 + 16 * (t + 4 * (g & 1)) : (g >> 1) * 128 + 16 * ((g & 1) * 4 + t)) ^ (32 * (g >> 2));
#pragma unroll
                    for (int m = 0; m < G::STEPS; ++m) {
                        if (16 * m >= chunk_rows - row0) break;
                        float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int j = 0; j < D / 64; ++j) {
                            const uint4 x = lds16(tile + 16 * m * G::ROW + (lane_at ^ (64 * j)));
                            const uint4 y = lds16(tile + (16 * m + 8) * G::ROW + (lane_at ^ (64 * j) ^ 64));
                            const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                uint32_t a0, a1, a2, a3;
                                e4m3_halves(xs[i], &a0, &a2);
                                e4m3_halves(ys[i], &a1, &a3);
                                mma16816(acc, a0, a1, a2, a3, qb[8 * j + 2 * i], qb[8 * j + 2 * i + 1]);
                            }
                        }
                        // (rows behind the last get scores that nothing reads)
                        const float ks = scales[16 * m], ks8 = scales[16 * m + 8];
                        if (t == 0) {
                            score[16 * m + g] = fmaf(acc[1], 1.f / kLow, acc[0]) * (ks * factor);
                            score[16 * m + g + 8] = fmaf(acc[3], 1.f / kLow, acc[2]) * (ks8 * factor);
                        }
                    }
                }
                release();
            }
        }
        __syncthreads();

        // S: running maximum and sum of every cluster, probabilities relative to the new maximum
#pragma unroll 1
        for (int cl = warp; cl < c.clusters; cl += W) {
            float* score = sm.score + cl * stride;
            float top = -INFINITY, old = c.first ? -INFINITY : sm.top[cl], sum = 0.f;
#pragma unroll 4
            for (int r = lane; r < chunk_rows; r += 32) top = fmaxf(top, score[r]);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            top = fmaxf(top, old);
            const float ref = top == -INFINITY ? 0.f : top;  // scores of -inf leave their rows out
#pragma unroll 4
            for (int r = lane; r < chunk_rows; r += 32) {
                const float p = exp2_approx(score[r] - ref);
                score[r] = p;
                sum += p;
            }
            const int r0 = chunk_rows + lane;
            if (r0 < stride) score[r0] = 0.f;  // (a tile has 32 rows at most)
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (lane == 0) {
                const float keep = exp2_approx(old - ref);
                sm.top[cl] = top;
                sm.keep[cl] = keep;
                sm.sum[cl] = (c.first ? 0.f : sm.sum[cl] * keep) + sum;
            }
        }
        const int bad_so_far = sm.any_bad;
        __syncthreads();  // (the next chunk may be of another request, whose pages count anew)
        more = prepare(par ^ 1);
        if (more) {
            __syncthreads();
            ready_no = no + 1;
        }

        // V: sums of the warp's share
        float acc[G::VPL];
#pragma unroll
        for (int e = 0; e < G::VPL; ++e) acc[e] = 0.f;
        // e4m3: sums on the tensor cores, of products that are `factor` too large
        constexpr int PARTS = G::FP8 ? D / 16 : 1;
        [[maybe_unused]] float part[PARTS][4];
        [[maybe_unused]] float factor = 1.f;
        // Writes the finished sums of a head.
        auto emit = [&](int p) __attribute__((always_inline)) {
            const int h = sg.head[p], cl = sg.cluster[p] - first_place;
            float* o = a.ws.o + ((size_t)c.slot * a.H + h) * D + G::col(lane);
            if (G::own(lane)) {
                if (!c.first) {
                    const float keep = sm.keep[cl];
#pragma unroll
                    for (int e = 0; e < G::VPL; e += 4) {
                        const float4 x = *reinterpret_cast<const float4*>(o + e);
                        acc[e] = fmaf(x.x, keep, acc[e]);
                        acc[e + 1] = fmaf(x.y, keep, acc[e + 1]);
                        acc[e + 2] = fmaf(x.z, keep, acc[e + 2]);
                        acc[e + 3] = fmaf(x.w, keep, acc[e + 3]);
                    }
                }
                if (c.last && c.single) {
                    const float sum = sm.sum[cl];
                    const bool zero = bad_so_far || sum == 0.f;  // (no score above -inf: nothing is left of the row)
                    TQ* dst = static_cast<TQ*>(a.out) + ((size_t)c.b * a.H + h) * D + G::col(lane);
#pragma unroll
                    for (int e = 0; e < G::VPL; ++e) dst[e] = from_float<TQ>(zero ? 0.f : acc[e] / sum);
                } else {
#pragma unroll
                    for (int e = 0; e < G::VPL; e += 4)
                        *reinterpret_cast<float4*>(o + e) = make_float4(acc[e], acc[e + 1], acc[e + 2], acc[e + 3]);
                }
            }
            if (c.last && !c.single && lane == 0) a.ws.ml[(size_t)c.slot * a.H + h] = make_float2(sm.top[cl], sm.sum[cl]);
        };
        int open = -1;  // a head whose first rows are in acc and whose last rows another warp has
        {
            Walk<W> w;
            w.start(1, c, warp);
            bool from_start = w.j == 0, begins = true;  // begins: the sums of a head start with this tile
#pragma unroll 1
            for (;;) {
                fill();
                if (w.left == 0) break;
                const int row0 = w.j * G::TR;
                const float* prob = sm.score + (sg.cluster[w.p] - first_place) * stride + row0;
                const unsigned char* tile = take();
                if (tile == nullptr) break;
                if constexpr (!G::FP8) {
                    const int first = (lane / G::LPR) * G::IT, rows = chunk_rows - row0;
                    if (rows < G::TR) {  // rows behind the last hold anything: zeros instead
#pragma unroll 1
                        for (int i = rows * G::LPR + lane; i < G::TR * G::LPR; i += 32)
                            *reinterpret_cast<uint4*>(sm.slot[warp][used & 1] + i * 16) = make_uint4(0, 0, 0, 0);
                        __syncwarp();
                    }
                    const unsigned char* base = tile + first * G::ROW + (lane % G::LPR) * 16;
                    uint64_t sum[G::VPL / 2];
#pragma unroll
                    for (int e = 0; e < G::VPL / 2; ++e) sum[e] = pack2(acc[2 * e], acc[2 * e + 1]);
                    uint4 raw[G::IT];
                    float pr[G::IT];
#pragma unroll
                    for (int i = 0; i < G::IT; ++i) raw[i] = lds16(base + i * G::ROW);
#pragma unroll
                    for (int i = 0; i < G::IT; i += 4) *reinterpret_cast<float4*>(pr + i) = *reinterpret_cast<const float4*>(prob + first + i);
#pragma unroll
                    for (int i = 0; i < G::IT; ++i) {
                        float vf[G::VPL];
                        Vec16<T>::unpack(raw[i], vf);
                        const uint64_t pp = pack2(pr[i], pr[i]);
#pragma unroll
                        for (int e = 0; e < G::VPL / 2; ++e) sum[e] = fma2(pp, pack2(vf[2 * e], vf[2 * e + 1]), sum[e]);
                    }
                    if (rows < G::TR) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // (the slot's next rows come by bulk copies)
#pragma unroll
                    for (int e = 0; e < G::VPL / 2; ++e) {
                        const float2 x = unpack2(sum[e]);
                        acc[2 * e] = x.x;
                        acc[2 * e + 1] = x.y;
                    }
                } else {
                    // 16 columns are the rows of A, 16 cache rows a step; B holds the probabilities times the rows' scales, as
                    // two fp16 numbers each, times a power of two that brings the largest product of a head's first tile to
                    // 2^7 ... 2^15.  Where a later one passes 2^15 the sums so far are brought to a new one.  So every
                    // product is held to 2^-22 of itself or 2^-43 of the head's largest, whichever is more.  (By the largest
                    // scale instead of the largest product, and with the second number stored as it is, rows whose scale is
                    // large and whose probability is not took the others' bits.  This way costs 0.3 to 0.6 %: 7B shape 54.1
                    // -> 54.3 us, 66B shape 28.8 -> 29.0; with a power found anew for every head, 54.4 and 29.5.)
                    const int g = lane >> 2, t = lane & 3;
                    const float4* scales = reinterpret_cast<const float4*>(tile + G::DATA + 16 * t);
                    const bool both = chunk_rows - row0 > 16;  // the tile has rows for both steps
                    uint64_t x[G::STEPS][2];
                    float top = 0.f;
#pragma unroll
                    for (int s = 0; s < G::STEPS; ++s) {
                        const float4 vs = s == 0 || both ? scales[4 * s] : make_float4(0.f, 0.f, 0.f, 0.f);
                        const float4 pr = *reinterpret_cast<const float4*>(prob + 16 * s + 4 * t);  // (zeros behind the last row)
                        x[s][0] = mul2(pack2(pr.x, pr.y), pack2(vs.x, vs.y));
                        x[s][1] = mul2(pack2(pr.z, pr.w), pack2(vs.z, vs.w));
                        const float2 u = unpack2(x[s][0]), v = unpack2(x[s][1]);
                        top = fmaxf(top, fmaxf(fmaxf(fabsf(u.x), fabsf(u.y)), fmaxf(fabsf(v.x), fabsf(v.y))));
                    }
                    if (begins) {
                        factor = kProductFactor;
#pragma unroll
                        for (int i = 0; i < PARTS; ++i) part[i][0] = part[i][1] = part[i][2] = part[i][3] = 0.f;
                    }
                    const unsigned high = __ballot_sync(0xffffffffu, top * factor > 32768.f);
                    const unsigned low = __ballot_sync(0xffffffffu, begins && top * factor < 128.f);
                    if (high != 0 || low == 0xffffffffu) {
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                        const float old = factor;
                        factor = product_factor(top);
                        const float change = factor / old;
#pragma unroll
                        for (int i = 0; i < PARTS; ++i)
#pragma unroll
                            for (int e = 0; e < 4; ++e) part[i][e] *= change;
                    }
                    constexpr int WORDS = D / 32;  // 32-bit words a lane holds of a row
                    const int lane_at = 4 * t * G::ROW + (D == 128 ? 16 * (g ^ (2 * t)) : (16 * ((g >> 1) ^ (2 * t)) + 8 * (g & 1)));
#pragma unroll
                    for (int s = 0; s < G::STEPS; ++s) {
                        if (s == 1 && !both) break;
                        uint32_t h0, h1, l0, l1;
                        two_halves(x[s][0], factor, &h0, &l0);
                        two_halves(x[s][1], factor, &h1, &l1);
                        const uint32_t b0 = g == 0 ? h0 : (g == 1 ? l0 : 0u), b1 = g == 0 ? h1 : (g == 1 ? l1 : 0u);
                        uint32_t v[4][WORDS];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            // row 16 s + 4 t + i (see Geom; the lane's share taken out)
                            const unsigned char* at = tile + 16 * s * G::ROW + i / (D == 128 ? 1 : 2) * 128 + (lane_at ^ (64 * (i & 1)));
                            if constexpr (WORDS == 4) {
                                const uint4 x = lds16(at);
                                v[i][0] = x.x; v[i][1] = x.y; v[i][2] = x.z; v[i][3] = x.w;
                            } else {
                                const uint2 x = lds8(at);
                                v[i][0] = x.x; v[i][1] = x.y;
                            }
                        }
#pragma unroll
                        for (int wd = 0; wd < WORDS; ++wd) {
                            // columns 4 wd .. + 3 of two rows each, side by side
#pragma unroll
                            for (int x = 0; x < 2; ++x) {
                                const unsigned sel = x == 0 ? 0x5140 : 0x7362;
                                uint32_t a0, a1, a2, a3;
                                e4m3_halves(__byte_perm(v[0][wd], v[1][wd], sel), &a0, &a1);
                                e4m3_halves(__byte_perm(v[2][wd], v[3][wd], sel), &a2, &a3);
                                mma16816(part[2 * wd + x], a0, a1, a2, a3, b0, b1);
                            }
                        }
                    }
                }
                release();
                const int p = w.p;
                const bool ends = w.j + 1 == chunk_tiles;
                w.step(chunk_tiles);
                begins = ends;
                if (!ends && w.left > 0) continue;
                if constexpr (G::FP8) {
                    const float f = 1.f / factor;
#pragma unroll
                    for (int i = 0; i < PARTS; ++i) {
                        acc[2 * i] = fmaf(part[i][1], 1.f / kLow, part[i][0]) * f;
                        acc[2 * i + 1] = fmaf(part[i][3], 1.f / kLow, part[i][2]) * f;
                    }
                } else {
#pragma unroll
                    for (int o = G::LPR; o < 32; o <<= 1)
#pragma unroll
                        for (int e = 0; e < G::VPL; ++e) acc[e] += __shfl_xor_sync(0xffffffffu, acc[e], o);
                }
                if (!from_start) {  // the head began in an earlier warp
                    if (G::own(lane))
#pragma unroll
                        for (int e = 0; e < G::VPL; ++e) sm.part[warp][G::col(lane) + e] = acc[e];
                } else if (ends) {
                    emit(p);
                } else {
                    open = p;
                    fill();
                    break;
                }
#pragma unroll
                for (int e = 0; e < G::VPL; ++e) acc[e] = 0.f;
                from_start = true;
            }
        }
        __syncthreads();
        if (open >= 0) {
            const int n = c.heads * chunk_tiles, stop = (open + 1) * chunk_tiles;
#pragma unroll 1
            for (int w = warp + 1; w < W; ++w) {
                const int lo = n * w / W;
                if (lo >= stop) break;
                if (lo == n * (w + 1) / W) continue;  // a warp without tiles
                if (G::own(lane))
#pragma unroll
                    for (int e = 0; e < G::VPL; ++e) acc[e] += sm.part[w][G::col(lane) + e];
            }
            emit(open);
        }
        if (c.last && tid == 0) {
            if (!c.single && sm.plan.group == 0) a.ws.slot_bad[c.slot] = bad_so_far;
            if (bad_so_far && atomicCAS(&sm.err, CHAI_OK, CHAI_ERR_BAD_PAGE) == CHAI_OK) sm.err_b = c.b;
        }
    }
    if (dead)  // copies in flight end before the shared memory goes
        for (int i = used; i < issued; ++i) bar_wait(bars + (i & 1) * 8, (i >> 1) & 1, kDefaultWaitLimitCycles);

    if (!by_request && tid == 0) {  // pieces that open no request that goes on say so
        const Plan& plan = sm.plan;
        if ((int)blockIdx.x >= plan.pieces && (int)blockIdx.x < a.n_desc) a.ws.desc[blockIdx.x] = make_int4(-1, 0, 0, 0);
        if (plan.piece < plan.pieces && plan.group == 0 && !sm.division[par].opened_span) a.ws.desc[plan.piece] = make_int4(-1, 0, 0, 0);
    }
    __syncthreads();
    if (tid == 0) {
        a.ws.err[blockIdx.x] = sm.err;
        a.ws.err_b[blockIdx.x] = sm.err_b;
    }
}

// ---- joining the pieces of a request ----------------------------------------------------------------------------

// grid (H, blocks, SPLIT): out[b][h] from the partial results of consecutive pieces, a SPLIT-th of its columns.  Bound by the
// round trips to L2, one for the description and one for everything else: the first rows are on their way before the
// weights are known.  The order of the sums is the same for every SPLIT, and does not depend on the width of the tables.
template <typename TQ, int D, int SPLIT>
__global__ void __launch_bounds__(kJoinThreads) paged_join_kernel(const DecodeArgs a, int n_ctas) {
    constexpr int THREADS = kJoinThreads, WARPS = THREADS / 32, COLS = D / SPLIT, E = COLS / 32;
    constexpr int AHEAD = SPLIT == 1 ? 4 : 16, THEN = SPLIT == 1 ? 8 : 24;  // rows a warp has on their way, at first and later
    __shared__ float s_w[kMaxCtas], s_top[WARPS], s_sum[WARPS], s_o[WARPS][COLS];
    dependent_grid_sync();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, h = blockIdx.x, col = blockIdx.z * COLS;
    if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0 && warp == 0) {  // the call's status
        int code = CHAI_OK, at = -1;
        for (int i = lane; i < n_ctas; i += 32) {
            const int e = a.ws.err[i];
            if (e != CHAI_OK && (code == CHAI_OK || e == CHAI_ERR_TIMEOUT)) {
                code = e;
                at = a.ws.err_b[i];
            }
        }
        const unsigned late = __ballot_sync(0xffffffffu, code == CHAI_ERR_TIMEOUT), any = __ballot_sync(0xffffffffu, code != CHAI_OK);
        const int from = late ? __ffs(late) - 1 : (any ? __ffs(any) - 1 : 0);
        code = __shfl_sync(0xffffffffu, code, from);
        at = __shfl_sync(0xffffffffu, at, from);
        if (lane == 0) {
            reset_status(a.hdr);
            a.hdr->status = code;
            a.hdr->bad_b = at;
        }
    }
    struct alignas(4 * E) Row {
        float x[E];
    };
    auto add = [&](float* o, float w, const Row& r) {
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = fmaf(w, r.x[e], o[e]);
    };
#pragma unroll 1
    for (int di = blockIdx.y; di < a.n_desc; di += gridDim.y) {
        const int4 d = a.ws.desc[di];
        const int b = d.x, first = d.y, n = d.z;
        // -1: nothing to join.  (The other bounds hold unless another stream changes lengths under the call, which leaves
        // descriptions unwritten; results are anyone's guess then, addresses are not.)
        if (b < 0 || b >= a.B || n < 1 || n > n_ctas || first < 0 || first > kMaxCtas + a.B - n) continue;
        const float* src = a.ws.o + ((size_t)first * a.H + h) * D + col + lane * E;
        const size_t apart = (size_t)a.H * D;
        Row ahead[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (warp + u * WARPS < n) ahead[u] = *reinterpret_cast<const Row*>(src + (warp + u * WARPS) * apart);
        float2 ml[2];
        bool bad = false, unknown = false;
        float top = -INFINITY;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int i = tid + u * THREADS;
            ml[u] = make_float2(-INFINITY, 0.f);
            if (i < n) {
                ml[u] = a.ws.ml[(size_t)(first + i) * a.H + h];
                bad |= a.ws.slot_bad[first + i] != 0;
                unknown |= i == 0 && ml[u].y == -1.f;
            }
            top = fmaxf(top, ml[u].x);
        }
        static_assert(2 * THREADS >= kMaxCtas, "two slots a thread");
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        if (lane == 0) s_top[warp] = top;
        if (__syncthreads_or(unknown)) continue;  // an unknown head: zeros are written already
        const bool zero = __syncthreads_or(bad);
#pragma unroll
        for (int w = 0; w < WARPS; ++w) top = fmaxf(top, s_top[w]);
        const float ref = top == -INFINITY ? 0.f : top;
        float sum = 0.f;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int i = tid + u * THREADS;
            if (i < n) {
                const float weight = exp2_approx(ml[u].x - ref);
                s_w[i] = weight;
                sum += weight * ml[u].y;
            }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) s_sum[warp] = sum;
        __syncthreads();
        float o[E];
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = 0.f;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (warp + u * WARPS < n) add(o, s_w[warp + u * WARPS], ahead[u]);
#pragma unroll THEN
        for (int i = warp + AHEAD * WARPS; i < n; i += WARPS) add(o, s_w[i], *reinterpret_cast<const Row*>(src + i * apart));
#pragma unroll
        for (int e = 0; e < E; ++e) s_o[warp][lane * E + e] = o[e];
        __syncthreads();
        if (tid < COLS) {
            float l = 0.f, x = 0.f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                l += s_sum[w];
                x += s_o[w][tid];
            }
            static_cast<TQ*>(a.out)[((size_t)b * a.H + h) * D + col + tid] = from_float<TQ>(zero || l == 0.f ? 0.f : x / l);
        }
        __syncthreads();  // s_* are free for the next description
    }
}

// ---- host -------------------------------------------------------------------------------------------------------

template <typename T, typename TQ, int D>
int launch_decode(const DecodeArgs& args, cudaStream_t s) {
    using G = Geom<T, TQ, D>;
    constexpr size_t smem = sizeof(Smem<G, D>);
    static_assert(smem <= 227 * 1024, "one CTA's shared memory");
    static_assert(G::SLOT % 16 == 0 && (G::FP8 || G::IT == 8) && G::TR % 8 == 0 && G::TR <= 32, "tile geometry");
    static PerDeviceOnce once;  // (one per instantiation)
    static int sm_count[kMaxDevices];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return cuda_fail(e, "paged decode: current device");
    const int rc = once.run(dev, [&]() -> int {
        cudaError_t err = cudaDeviceGetAttribute(&sm_count[dev & (kMaxDevices - 1)], cudaDevAttrMultiProcessorCount, dev);
        if (err == cudaSuccess)
            err = cudaFuncSetAttribute(paged_decode_kernel<T, TQ, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        return err == cudaSuccess ? CHAI_OK : cuda_fail(err, "paged_decode_kernel set-up");
    });
    if (rc != CHAI_OK) return rc;
    const int n_ctas = sm_count[dev & (kMaxDevices - 1)] < kMaxCtas ? sm_count[dev & (kMaxDevices - 1)] : kMaxCtas;
    DecodeArgs a = args;
    a.n_desc = a.B < n_ctas ? a.B : n_ctas;
    CHAI_LAUNCH_DEPENDENT("paged_decode_kernel launch", (paged_decode_kernel<T, TQ, D>), dim3(n_ctas), dim3(G::THREADS), smem, s, a);
    const int blocks = a.n_desc < kJoinBlocks ? a.n_desc : kJoinBlocks;
    if (a.n_desc <= kJoinFew)
        CHAI_LAUNCH_DEPENDENT("paged_join_kernel launch", (paged_join_kernel<TQ, D, D / 32>), dim3(a.H, blocks, D / 32),
                              dim3(kJoinThreads), 0, s, a, n_ctas);
    else
        CHAI_LAUNCH_DEPENDENT("paged_join_kernel launch", (paged_join_kernel<TQ, D, 1>), dim3(a.H, blocks), dim3(kJoinThreads), 0,
                              s, a, n_ctas);
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
    DecodeArgs a = {};
    const int rc = make_pool(fn, block_table, B, H, k, n_pages, page_size, max_pages, D, k_page_stride, v_page_stride,
                             fp8 ? 1 : elem_size(dtype), &a.pool);
    if (rc != CHAI_OK) return rc;
    CHAI_REQUIRE((long long)B * a.pool.capacity < (1ll << 33), CHAI_ERR_UNSUPPORTED,
                 "%s: B * max_pages * page_size must be below 2^33", fn);
    const size_t need = chai_decode_paged_workspace_bytes(B, H, D);
    CHAI_REQUIRE(workspace_bytes >= need, CHAI_ERR_WORKSPACE, "%s: workspace has %zu bytes, %zu needed", fn, workspace_bytes,
                 need);
    CHAI_REQUIRE(decode_ws(static_cast<char*>(workspace), B, H, D, &a.ws) <= need, CHAI_ERR_WORKSPACE, "%s: workspace layout", fn);
    const size_t rows = (size_t)B * H * D * elem_size(dtype);
    CHAI_REQUIRE(static_cast<const char*>(q) + rows <= out || static_cast<const char*>(out) + rows <= q, CHAI_ERR_INVALID_ARG,
                 "%s: q and out overlap (a head's query is read until the call ends)", fn);
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
    a.scale_log2 = scale * 1.44269504088896340736f;
    a.wait_limit = decode_wait_limit_cycles();
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
    // a plain bound of what decode_ws lays out: 64 KiB for the words per CTA and the rounding, and per slot and head D
    // sums, a maximum and a sum, with room for the slot's own word
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
