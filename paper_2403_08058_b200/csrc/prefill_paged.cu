// Clustered attention of packed tokens over a paged cache: a prompt's chunk behind what is cached of it, guessed tokens that are
// verified at once, a batch that mixes chunks and single tokens, or queries over states of another length without a mask.
// The entry points, and the kernel on the 5th-generation tensor cores (tcgen05 + TMEM + TMA) for bf16; 32-bit queries run on
// the CUDA cores (prefill_paged_simt.cu).
//
// The arithmetic is prefill_tc.cu's: S = Q K^T of a tile of 128 query rows and 128 keys into tensor memory, the softmax against
// a reference that moves only when a row's maximum leaves a window of 2^32 around it, P as bf16 in tensor memory, O_g += P V_g
// for the members of a cluster, two at a time (head_dim 64: four).  P is rounded to bf16, at most 2^-8 of each
// probability, because that is the tensor core's type beside bf16 values; row sums are of the rounded ones, in fp32, so that a
// row which sees one position, or nearly one, gets its values (sums of the unrounded ones, two additions an instruction, left such
// a row 0.0016 off; they are 2 % faster for 2048 tokens behind 30720).
// What differs:
//   - keys and values come from pages, in boxes of as many rows as divide both the page size and 128, whole rows each: a box
//     costs about 90 cycles of the copy engine whatever it holds.  A box lands as one piece of shared memory, so tiles are
//     laid out by boxes: keys as 8-row groups of both column halves (one distance between groups), values as boxes of
//     all members side by side (one distance between 64-column blocks).  The lanes of the loading warp look up and issue
//     one box each, tables a tile ahead.
//   - rows behind a request's length are never used, whatever they hold: their scores are masked, and their values, which
//     would meet probabilities of zero, are zeroed in shared memory before the last tile is multiplied.
//   - a request may have few tokens: rows that it does not have cost tensor work but no softmax, and all tiles are one line that
//     is cut into equal shares (prefill_paged.cuh); a query tile on both sides of a cut leaves unnormalised accumulators, joined
//     in order of the pieces by the CTA that finishes its last piece, at the end of that CTA's work: its softmax warps have
//     nothing else to do then and registers for the loads (by the warp that writes accumulators out, in between, 64 tokens
//     over 8192 in e4m3 took 243 us, not 205).
// Bound by the cache's bytes for few tokens a request, by the softmax chain of a tile (as in prefill_tc.cu) for many; with e4m3
// pages by their conversion to bf16, which stands in the chain between a tile's products and the next one's (instructions issue in
// 45 % of the cycles, the tensor pipe is busy in 22 %).
// Measured (of 6567 GB/s, or of 1638 TFLOP/s), in bursts of some ten ms at 1965 MHz: 16 requests of 4 tokens over up to 2048, 32 heads,
// 8 clusters: 54 us, 54 %; 2048 tokens behind 30720: 760 - 800 us, 51 - 53 %; 24 mixed requests over up to 4096, 52 heads: 305 us, 42 %
// (the chunks' query tiles read their rows again, after they have left L2: 1.7 GB at 5.7 TB/s, where 0.80 would do); e4m3, 4 x 64 tokens
// over up to 8192, 72 heads, 24 clusters: 199 us, 21 %.  Without a pause the chunk and the mixed batch draw 1000 W, the clock falls
// to 1570 and 1450 MHz, and they take 840 - 890 and 340 - 360 us.  Before the first tile stand some 10 us: the planner 3.5, the
// launch 1.7, finding the share 1.5, its first rows 3.
#include <cuda.h>
#include <math.h>

#include "prefill_paged.cuh"
#include "tc_ptx.cuh"

namespace chai {

void prefill_paged_simt_tile(int B, int n_tokens, int D, int* rows, int* keys);
int prefill_paged_simt(const PagedCall& a, int D, bool fp8, cudaStream_t s);

namespace pp {

using namespace tcx;

constexpr int BM = 128, BN = 128;
constexpr int GMAX = 4;
constexpr int KST = 2;                       // key tile stages: tile kt uses stage kt & 1
constexpr int TILE_BYTES = BN * 128 * 2;     // a tile slot (head_dim 64: two members' value tiles share one)
constexpr int HALF_BYTES = TILE_BYTES / 2;   // 128 rows x 64 columns, 128-byte swizzled rows
constexpr int SOFTMAX_WARPS = 8, EPILOGUE_WARPS = 4;
// Warps of the roles.  With e4m3 pages eight warps convert, four of which are the epilogue's too, one brings row scales, and roles are
// whole warpgroups, which trade registers.  (Spills cost more than they look: beside this much shared memory there is hardly any L1.)
template <bool FP8>
struct Roles {
    static constexpr int QK = 1, SCALES = FP8 ? 3 : -1, SOFTMAX = FP8 ? 4 : 2, EPILOGUE = SOFTMAX + SOFTMAX_WARPS, CONVERT_WARPS = FP8 ? 8 : 0;
    static constexpr int PV = FP8 ? 2 : EPILOGUE + EPILOGUE_WARPS;
    static constexpr int THREADS = FP8 ? 640 : 480;
};
constexpr int LAUNCH_REGS = 96, WORKER_REGS = 80, CONVERT_REGS = 72, SOFTMAX_REGS = 128;  // e4m3, a thread
static_assert(128 * WORKER_REGS + 256 * CONVERT_REGS + 256 * SOFTMAX_REGS <= 640 * LAUNCH_REGS, "registers are only moved");
template <int N>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
constexpr int JOIN_BARRIER = 5;  // (1 - 4: the quadrants' pairs of softmax warps)
constexpr float REF_WINDOW = 32.f, EXACT_FROM = 2048.f;  // log2
constexpr uint32_t TMEM_COLS = 512;
constexpr uint32_t S_COL0 = 0, P_COL0 = 128, O_COL0 = 256;

// shared memory map (offsets from a 1024-byte aligned base)
constexpr int OFF_Q = 0;
constexpr int OFF_K = OFF_Q + TILE_BYTES;
constexpr int OFF_V = OFF_K + KST * TILE_BYTES;
constexpr int OFF_BAR = OFF_V + 4 * TILE_BYTES;
constexpr int NUM_BARS = 35;
// e4m3: keys and values have one stage each; in the others' places lie units (128 rows of one plane) as they come from the
// pages, and their scales.
template <int HD>
struct Units {
    static constexpr int SLOTS = HD == 128 ? 4 : 6;
};
constexpr int RAW_SLOTS = 6, OFF_RAW = OFF_V + 2 * TILE_BYTES, OFF_SCALES = OFF_K + TILE_BYTES;
static_assert(OFF_RAW + Units<128>::SLOTS * BN * 128 <= OFF_BAR && OFF_RAW + Units<64>::SLOTS * BN * 64 <= OFF_BAR && OFF_SCALES + RAW_SLOTS * BN * 4 <= OFF_V,
              "units and scales fit");
constexpr int OFF_XCH = OFF_BAR + 8 * NUM_BARS + 24;  // (the barriers, the tensor-memory address, the abort flag)
constexpr int OFF_LSUM = OFF_XCH + 2 * BM * 4;       // [half][row] sums
constexpr int OFF_REF = OFF_LSUM + 2 * BM * 4;       // [row] reference of the exponentials
constexpr int OFF_ITEM = OFF_REF + BM * 4;
constexpr int ITEM_BYTES = 64;
constexpr int OFF_JOINS = OFF_ITEM + 3 * ITEM_BYTES;  // bits: which query tiles' (begun before the share, in it) quadrants to join
constexpr int SMEM_BYTES = OFF_JOINS + 16;
static_assert(ITEM_BYTES == kPagedJoinBytes && OFF_ITEM % 16 == 0 && SMEM_BYTES <= 232448, "shared memory budget");

struct Bars {
    uint32_t base;
    __device__ __forceinline__ uint32_t q_full() const { return base; }
    __device__ __forceinline__ uint32_t q_empty() const { return base + 8; }
    __device__ __forceinline__ uint32_t o_free(int g) const { return g == 0 ? base + 16 : base + 8 * (18 + g); }
    __device__ __forceinline__ uint32_t p_full(int i) const { return i == 0 ? base + 24 : base + 8 * 22; }
    __device__ __forceinline__ uint32_t item_full(int i) const { return base + 8 * (4 + i); }
    __device__ __forceinline__ uint32_t item_empty(int i) const { return base + 8 * (6 + i); }
    __device__ __forceinline__ uint32_t k_full(int i) const { return base + 8 * (8 + i); }
    __device__ __forceinline__ uint32_t v_full(int i) const { return base + 8 * (10 + i); }
    __device__ __forceinline__ uint32_t qk_done(int i) const { return base + 8 * (12 + i); }
    __device__ __forceinline__ uint32_t pv_done(int i) const { return base + 8 * (14 + i); }
    __device__ __forceinline__ uint32_t epi_full() const { return base + 8 * 16; }
    __device__ __forceinline__ uint32_t epi_empty() const { return base + 8 * 17; }
    __device__ __forceinline__ uint32_t s_free() const { return base + 8 * 18; }
    __device__ __forceinline__ uint32_t raw_full(int i) const { return base + 8 * (23 + i); }
    __device__ __forceinline__ uint32_t raw_free(int i) const { return base + 8 * (29 + i); }
};
static_assert(NUM_BARS == 29 + RAW_SLOTS, "barrier count");

// One unit of work, published by the loading warp to the other roles through shared memory.
struct Item {
    int n_kv;         // key tiles to walk; 0: zero rows (no keys, unresolved heads); -1: no more work
    int n_members;
    int row0;         // first row of the packed arrays
    int rows;         // rows of the tile that exist
    int first, tiles; // the walk begins at key tile `first` and wraps around at `tiles`
    int sees;         // positions that row 0 sees; row r: r more, at most kv (unmasked: kv)
    int kv;
    int pieces, owner;
    short piece, cluster;
    int heads[GMAX];
    int b;
};
static_assert(sizeof(Item) == ITEM_BYTES, "item descriptor");

// First position of the j-th tile of a walk.
__device__ __forceinline__ int tile_col(int first, int tiles, int j) { return (first + j < tiles ? first + j : first + j - tiles) * BN; }

struct Tma {
    CUtensorMap q, k, v;
};

// e4m3: the slot of the next unit, and the parity of its filling.
template <int HD>
struct Unit {
    int slot = 0, phase = 0;
    __device__ __forceinline__ void next() {
        if (++slot == Units<HD>::SLOTS) slot = 0, phase ^= 1;
    }
};

// Four e4m3 numbers times a scale, as bf16 (rounded once where the scale is a power of two, twice otherwise).
__device__ __forceinline__ void e4m3x4_to_bf16(uint32_t w, float scale, uint32_t* o) {
    const __half2_raw lo = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w & 0xffffu), __NV_E4M3);
    const __half2_raw hi = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w >> 16), __NV_E4M3);
    const float2 u = __half22float2(*reinterpret_cast<const __half2*>(&lo)), v = __half22float2(*reinterpret_cast<const __half2*>(&hi));
    const __nv_bfloat162 p = __floats2bfloat162_rn(u.x * scale, u.y * scale), q = __floats2bfloat162_rn(v.x * scale, v.y * scale);
    o[0] = *reinterpret_cast<const uint32_t*>(&p);
    o[1] = *reinterpret_cast<const uint32_t*>(&q);
}
// The same by moving bits, for a scale 2^e with -126 <= e <= 7: the byte s eeee mmm is, as the bf16 number s 0000eeee mmm0000, its
// value times 2^-120 (the exponents' biases are 7 and 127; e4m3's subnormal numbers become bf16's), and the product with 2^(120 + e)
// is exact.  The result has the highest bit of a byte set where that number is a NaN, which this does not know: 1111 111 would
// be 480.  (The conversion instructions run on a pipe that takes them some thirty cycles a warp.)
__device__ __forceinline__ uint32_t e4m3_factor(float scale) {  // (two bf16 numbers: the upper halves of fp32's)
    const uint32_t f = __float_as_uint(scale * 0x1p120f);
    return __byte_perm(f, f, 0x3232);
}
__device__ __forceinline__ uint32_t e4m3x4_to_bf16_bits(uint32_t w, uint32_t factor, uint32_t* o) {
    const uint32_t high = (w & 0x80808080u) | ((w >> 4) & 0x07070707u), low = (w << 4) & 0xf0f0f0f0u;
    uint32_t p[2] = {__byte_perm(low, high, 0x5140), __byte_perm(low, high, 0x7362)};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const __nv_bfloat162 v = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&p[i]), *reinterpret_cast<const __nv_bfloat162*>(&factor));
        o[i] = *reinterpret_cast<const uint32_t*>(&v);
    }
    return (w & 0x7f7f7f7fu) + 0x01010101u;
}

// Writes out the ei-th finished item, by the four epilogue warps, one thread per query row; false: there is none any more, or a wait ran
// out.
template <int HD>
__device__ __forceinline__ bool finish_item(const PagedCall& a, uint8_t* smem, uint32_t tmem_base, volatile int* abort_flag, int ei) {
    constexpr int GM = HD == 128 ? 2 : 4;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Item* items = reinterpret_cast<const Item*>(smem + OFF_ITEM);
    const Bars bar{smem_u32(smem) + OFF_BAR};
    const int quad = warp & 3, row = quad * 32 + lane;
    const uint32_t lane_addr = tmem_base + ((uint32_t)(quad * 32) << 16);
    const float* lsum = reinterpret_cast<const float*>(smem + OFF_LSUM);
    const float* refs = reinterpret_cast<const float*>(smem + OFF_REF);
    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out);
    const bool wide = (reinterpret_cast<uintptr_t>(out) & 31u) == 0;
    const size_t slot_bytes = (size_t)a.slot_rows * kSlotRowBytes, stats = (size_t)a.slot_rows * 1024;
    bool ok = __all_sync(0xffffffffu, mbar_wait(bar.epi_full(), ei & 1, abort_flag));
    if (!ok) return false;
    const Item ep = items[2];
    const float l = lsum[row] + lsum[BM + row], ref = refs[row];
    if (ep.n_members < 0) return false;
    const int last = ep.n_kv;
    ok = __all_sync(0xffffffffu, mbar_wait(bar.pv_done(last & 1), (last >> 1) & 1, abort_flag));
    if (!ok) return false;
    tc_fence_after();
    __syncwarp();
    if (lane == 0) mbar_arrive(bar.epi_empty());
    const bool live = row < ep.rows, split = ep.pieces > 1;
    const float inv = split ? 1.f : l == 0.f ? 0.f : 1.f / l;  // (a NaN stays one)
    const uint64_t inv2 = pack2(inv, inv);
    auto slot = [&](int piece) { return a.slots + (size_t)piece_slot(ep.owner, piece) * slot_bytes; };
    float* part = reinterpret_cast<float*>(slot(ep.piece));
    constexpr int NSUB = HD / 32;
    const int n_sub = ep.n_members * NSUB;
    uint32_t cur[32];
#pragma unroll
    for (int c = 0; c < GM * NSUB; ++c) {
        if (c >= n_sub) break;
        __syncwarp();  // (the stores below are for some lanes only, the load is for the warp as a whole)
        tc_ld32_wait(lane_addr + O_COL0 + c * 32, cur);  // (members' accumulators are contiguous)
        const int g = c / NSUB, sc = c % NSUB;
        if (sc == NSUB - 1) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(bar.o_free(g));
                if (g == ep.n_members - 1)
                    for (int x = ep.n_members; x < GM; ++x) mbar_arrive(bar.o_free(x));
            }
        }
        if (live && !split) {
            int h = ep.heads[0];
#pragma unroll
            for (int x = 1; x < GM; ++x)
                if (g == x) h = ep.heads[x];
            __nv_bfloat16* orow = out + ((size_t)(ep.row0 + row) * a.H + h) * HD + sc * 32;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                uint32_t w[8];
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    float y0, y1;
                    unpack2(mul2(pack2(__uint_as_float(cur[16 * u + 2 * x]), __uint_as_float(cur[16 * u + 2 * x + 1])), inv2), y0, y1);
                    if (inv == 0.f) y0 = y1 = 0.f;
                    __nv_bfloat162 pk = __floats2bfloat162_rn(y0, y1);
                    w[x] = *reinterpret_cast<uint32_t*>(&pk);
                }
                st_global_row32(orow + u * 16, w, wide);
            }
        } else if (live) {
            float* prow = part + ((size_t)g * a.slot_rows + row) * HD + sc * 32;
#pragma unroll
            for (int u = 0; u < 8; ++u)
                reinterpret_cast<uint4*>(prow)[u] = make_uint4(cur[4 * u], cur[4 * u + 1], cur[4 * u + 2], cur[4 * u + 3]);
        }
    }
    if (!split || quad * 32 >= ep.rows) return true;
    // A piece: its rows' references and sums; the CTA whose warp finishes its rows' last piece joins them, in order of the
    // pieces.  (A byte of the counter per warp.)
    if (live) reinterpret_cast<float2*>(reinterpret_cast<char*>(part) + stats)[row] = make_float2(ref, l);
    __threadfence();
    __syncwarp();
    unsigned before = 0;
    if (lane == 0) {
        before = (unsigned)atomicAdd(&a.done[ep.owner], 1 << (8 * quad)) >> (8 * quad) & 255u;
        __threadfence();
    }
    before = __shfl_sync(0xffffffffu, before, 0);
    if ((int)before != ep.pieces - 1) return true;
    if (lane == 0) {  // (at the end of the CTA's work, by warps that have nothing else to do then)
        const int which = ep.piece > 0 ? 0 : 1;
        reinterpret_cast<Item*>(a.joins)[blockIdx.x * 2 + which] = ep;
        atomicOr(reinterpret_cast<unsigned*>(smem + OFF_JOINS), 1u << (which * 4 + quad));
        __threadfence_block();
    }
    return true;
}

// Joins the pieces that the CTA finished last, by the softmax warps: a warp takes ROWS rows of a quadrant at a time, a lane 8 columns
// of one member (a row of both or all members is 1 KB), whose loads of the next piece are under way meanwhile.
template <int HD>
__device__ __forceinline__ void join_pieces(const PagedCall& a, const uint8_t* smem, int warp) {
    constexpr int ROWS = 4;
    const int lane = threadIdx.x & 31;
    const unsigned todo = *reinterpret_cast<const volatile unsigned*>(smem + OFF_JOINS);
    const size_t slot_bytes = (size_t)a.slot_rows * kSlotRowBytes, stats = (size_t)a.slot_rows * 1024;
    const int g = lane / (HD / 8), x = lane % (HD / 8);
#pragma unroll 1
    for (int i = warp; i < 8 * (32 / ROWS); i += SOFTMAX_WARPS) {
        const int bit = i / (32 / ROWS), row0 = (bit & 3) * 32 + i % (32 / ROWS) * ROWS;
        if (!(todo >> bit & 1u)) continue;
        const Item* ep = reinterpret_cast<const Item*>(a.joins) + blockIdx.x * 2 + (bit >> 2);
        const int rows = ep->rows, pieces = ep->pieces, owner = ep->owner;
        if (row0 >= rows) continue;
        auto slot = [&](int piece) { return a.slots + (size_t)piece_slot(owner, piece) * slot_bytes; };
        const bool mine = g < ep->n_members;
        const size_t offset = (((size_t)(mine ? g : 0) * a.slot_rows + row0) * HD + x * 8) * 4;
        float4 v[ROWS][2];
        auto load = [&](int p) {
            const float* src = reinterpret_cast<const float*>(slot(p) + offset);
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const int at = row0 + r < rows ? r : 0;
                v[r][0] = __ldcg(reinterpret_cast<const float4*>(src + at * HD));
                v[r][1] = __ldcg(reinterpret_cast<const float4*>(src + at * HD) + 1);
            }
        };
        // A lane a piece: its share of every row, relative to the reference of all.
        float share[ROWS];
        float2 st[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            st[r] = make_float2(0.f, 0.f);
            if (lane < pieces && row0 + r < rows) st[r] = __ldcg(reinterpret_cast<const float2*>(slot(lane) + stats) + row0 + r);
        }
        load(0);  // (on its way meanwhile)
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const bool sees = st[r].y != 0.f;  // (a piece that the row sees nothing of)
            float m = sees ? st[r].x : -INFINITY;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            const float w = sees ? fast_exp2(st[r].x - m) : 0.f;
            float sum = w * st[r].y;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            share[r] = sees ? w / sum : 0.f;
        }
        float o8[ROWS][8];
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
#pragma unroll
            for (int y = 0; y < 8; ++y) o8[r][y] = 0.f;
#pragma unroll 1
        for (int p = 0; p < pieces; ++p) {
            float4 u[ROWS][2];
#pragma unroll
            for (int r = 0; r < ROWS; ++r) u[r][0] = v[r][0], u[r][1] = v[r][1];
            if (p + 1 < pieces) load(p + 1);
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const float w = __shfl_sync(0xffffffffu, share[r], p);
                if (w == 0.f) continue;  // (what such a piece holds is not a number it may be)
                o8[r][0] += w * u[r][0].x, o8[r][1] += w * u[r][0].y, o8[r][2] += w * u[r][0].z, o8[r][3] += w * u[r][0].w;
                o8[r][4] += w * u[r][1].x, o8[r][5] += w * u[r][1].y, o8[r][6] += w * u[r][1].z, o8[r][7] += w * u[r][1].w;
            }
        }
        if (!mine) continue;
        __nv_bfloat16* to = static_cast<__nv_bfloat16*>(a.out) + ((size_t)(ep->row0 + row0) * a.H + ep->heads[g]) * HD + x * 8;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            uint4 w;
            uint32_t* words = &w.x;
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const __nv_bfloat162 pk = __floats2bfloat162_rn(o8[r][2 * y], o8[r][2 * y + 1]);
                words[y] = *reinterpret_cast<const uint32_t*>(&pk);
            }
            if (row0 + r < rows) *reinterpret_cast<uint4*>(to + (size_t)r * a.H * HD) = w;
        }
    }
}

template <int HD, bool FP8>
__global__ void __launch_bounds__(Roles<FP8>::THREADS, 1)
prefill_paged_kernel(const __grid_constant__ Tma maps, const __grid_constant__ PagedCall a, const int box_rows, const float scale_log2) {
    using R = Roles<FP8>;
    constexpr int GM = HD == 128 ? 2 : 4, HALVES = HD / 64, ROW_BYTES = HD * 2;
    // Bytes between two 64-column blocks of a value box, and between two boxes of a value tile (those of all members).  (e4m3: the
    // converting warps write a tile as one box.)
    const int tile_rows = FP8 ? BN : box_rows, v_block = tile_rows * 128, v_box = GM * HALVES * v_block;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    extern __shared__ uint8_t smem[];
    const uint32_t sbase = smem_u32(smem);
    if ((sbase & 1023u) != 0) {  // swizzled tiles need it; a kernel without static shared memory has it
        asm volatile("griddepcontrol.wait;" ::: "memory");
        if (tid == 0) atomicExch(&a.hdr->status, CHAI_ERR_TIMEOUT);
        return;
    }
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + OFF_BAR + 8 * NUM_BARS);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    Item* items = reinterpret_cast<Item*>(smem + OFF_ITEM);  // [2] to the issuers and softmax warps, [2] = to the epilogue
    const Bars bar{sbase + OFF_BAR};

    if (tid == 0) {
        mbar_init(bar.q_full(), 1);
        mbar_init(bar.q_empty(), 1);
        for (int g = 0; g < GMAX; ++g) mbar_init(bar.o_free(g), EPILOGUE_WARPS);
        mbar_init(bar.epi_full(), SOFTMAX_WARPS);
        mbar_init(bar.epi_empty(), EPILOGUE_WARPS);
        mbar_init(bar.s_free(), SOFTMAX_WARPS);
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar.p_full(i), SOFTMAX_WARPS);
            mbar_init(bar.item_full(i), 1);
            mbar_init(bar.item_empty(i), 2 + SOFTMAX_WARPS + R::CONVERT_WARPS + (FP8 ? 1 : 0));
            mbar_init(bar.k_full(i), FP8 ? R::CONVERT_WARPS : 1);
            mbar_init(bar.v_full(i), FP8 ? R::CONVERT_WARPS : 1);
            mbar_init(bar.qk_done(i), 1);
            mbar_init(bar.pv_done(i), 1);
        }
        for (int i = 0; i < RAW_SLOTS; ++i) {
            mbar_init(bar.raw_full(i), 2);  // the copies, and the scales
            mbar_init(bar.raw_free(i), 8);  // (e4m3: R::CONVERT_WARPS)
        }
        *abort_flag = 0;
        *reinterpret_cast<unsigned*>(smem + OFF_JOINS) = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_proxy();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;

    if (warp == 0) {
        // ---------------- work distribution and loads, by all lanes ----------------
        if constexpr (FP8) fewer_registers<WORKER_REGS>();
        auto wait_all = [&](uint32_t b, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(b, parity, abort_flag)); };
        const int blocks = BN / box_rows;                    // boxes of a tile
        bool ok = true;
        int it = 0, qi = 0, kt = 0;                          // items published, items with loads, key tiles issued
        PagedGroup e, e_next;
        PagedItem cur = {}, nxt = {};
        [[maybe_unused]] Unit<HD> unit;
        PagedWalk walk;
        walk.begin(a, lane);
        bool more = walk.next(a, cur, e);
        while (ok) {
            const int is = it & 1;
            ok = wait_all(bar.item_empty(is), ((it >> 1) & 1) ^ 1);
            if (!ok) break;
            if (!more) {
                if (lane == 0) {
                    items[is].n_kv = -1;
                    mbar_arrive(bar.item_full(is));
                }
                break;
            }
            const int n_kv = cur.count, n_members = min(e.n, GM), kv = cur.kv;
            if (lane == 0) {
                Item& item = items[is];
                item.n_kv = n_kv;
                item.n_members = n_members;
                item.row0 = cur.q0;
                item.rows = cur.rows;
                item.first = cur.first;
                item.tiles = cur.tiles;
                item.kv = kv;
                item.sees = a.causal ? kv - cur.n + cur.t0 + 1 : kv;
                item.pieces = cur.pieces;
                item.piece = (short)cur.piece;
                item.cluster = (short)e.cluster;
                item.b = cur.b;
                item.owner = cur.owner;
#pragma unroll
                for (int g = 0; g < GMAX; ++g) item.heads[g] = g < n_members ? e.heads[g] : e.heads[0];
                mbar_arrive(bar.item_full(is));
            }
            __syncwarp();
            ++it;
            if (n_kv == 0) {
                more = walk.next(a, cur, e);
                continue;
            }
            // Lane l knows the place of box l of a tile: page and first row in it.
            const int32_t* table = a.pool.block_table + (size_t)cur.b * a.pool.max_pages;
            auto col = [&](int j) { return tile_col(cur.first, cur.tiles, j); };
            auto boxes = [&](int j) { return (min(BN, kv - col(j)) + box_rows - 1) / box_rows; };  // that hold rows
            auto look_up = [&](int j, int& page, int& row) {
                page = -1;
                row = 0;
                if (j >= n_kv || lane >= blocks) return;
                const int pos = col(j) + lane * box_rows;
                if (pos >= kv) return;
                const int pi = (int)a.pool.by_page.div((unsigned)pos);
                row = pos - pi * a.pool.page_size;
                page = table[pi];  // (an entry that is no page: outside the map, zeros arrive)
            };
            int page_v, row_v, page_k, row_k, page_n, row_n;
            look_up(0, page_v, row_v);
            look_up(1, page_k, row_k);
            // queries: wait until the previous item's last S = Q K^T has been computed
            ok = wait_all(bar.q_empty(), (qi & 1) ^ 1);
            if (!ok) break;
            if (lane == 0) {
                mbar_expect_tx(bar.q_full(), BM * ROW_BYTES);
#pragma unroll
                for (int h = 0; h < HALVES; ++h)
                    tma_load_3d(sbase + OFF_Q + h * HALF_BYTES, &maps.q, h * 64, e.rep, cur.q0, bar.q_full());
            }
            __syncwarp();
            if constexpr (FP8) {  // units in order: K(0), K(1), V(0) of every member, K(2), V(1), ...
                auto load_unit = [&](bool key, int plane, int j, int page, int row) -> bool {
                    const int count = boxes(j);
                    if (!wait_all(bar.raw_free(unit.slot), unit.phase ^ 1)) return false;
                    if (lane == 0) mbar_expect_tx(bar.raw_full(unit.slot), count * box_rows * HD);
                    __syncwarp();
                    if (lane < count)
                        tma_load_3d(sbase + OFF_RAW + (unit.slot * BN + lane * box_rows) * HD, key ? &maps.k : &maps.v, 0, plane * a.pool.page_size + row, page, bar.raw_full(unit.slot));
                    unit.next();
                    return true;
                };
                ok = load_unit(true, e.cluster, 0, page_v, row_v);
                for (int j = 0; j < n_kv && ok; ++j) {
                    look_up(j + 2, page_n, row_n);
                    if (j + 1 < n_kv) ok = load_unit(true, e.cluster, j + 1, page_k, row_k);
#pragma unroll
                    for (int g = 0; g < GM; ++g)
                        if (g < n_members && ok) ok = load_unit(false, e.heads[g], j, page_v, row_v);
                    if (j == 0) more = walk.next(a, nxt, e_next);
                    page_v = page_k, row_v = row_k;
                    page_k = page_n, row_k = row_n;
                }
                kt += n_kv;
                ++qi;
                cur = nxt;
                e = e_next;
                continue;
            }
            auto load_k = [&](int j, int page, int row) -> bool {
                const int n = kt + j, ts = n & 1, count = boxes(j);
                if (!wait_all(bar.qk_done(ts), ((n >> 1) & 1) ^ 1)) return false;  // stage free
                if (lane == 0) mbar_expect_tx(bar.k_full(ts), count * box_rows * ROW_BYTES);
                __syncwarp();
                if (lane < count) {
                    const uint32_t dst = sbase + OFF_K + ts * TILE_BYTES + lane * box_rows * ROW_BYTES;
                    const int at = e.cluster * a.pool.page_size + row;
                    if constexpr (HD == 128) tma_load_5d(dst, &maps.k, 0, 0, 0, at >> 3, page, bar.k_full(ts));
                    else tma_load_3d(dst, &maps.k, 0, at, page, bar.k_full(ts));
                }
                return true;
            };
            // order of need: K(0), K(1), V(0), K(2), V(1), ...
            ok = load_k(0, page_v, row_v);
            for (int j = 0; j < n_kv && ok; ++j) {
                look_up(j + 2, page_n, row_n);
                if (j + 1 < n_kv) ok = load_k(j + 1, page_k, row_k);
                if (!ok) break;
                const int n = kt + j, ts = n & 1, count = boxes(j);
                ok = wait_all(bar.pv_done(ts), ((n >> 1) & 1) ^ 1);  // the tile's value slots are free
                if (!ok) break;
                if (lane == 0) mbar_expect_tx(bar.v_full(ts), n_members * count * box_rows * ROW_BYTES);
                __syncwarp();
                if (lane < count) {
                    const uint32_t dst = sbase + OFF_V + ts * 2 * TILE_BYTES + lane * v_box;
#pragma unroll
                    for (int g = 0; g < GM; ++g) {
                        if (g >= n_members) break;
                        const int at = e.heads[g] * a.pool.page_size + row_v;
                        if constexpr (HD == 128) tma_load_page(dst + g * HALVES * v_block, &maps.v, 0, at, 0, page_v, bar.v_full(ts));
                        else tma_load_3d(dst + g * v_block, &maps.v, 0, at, page_v, bar.v_full(ts));
                    }
                }
                if (j == 0) more = walk.next(a, nxt, e_next);
                page_v = page_k, row_v = row_k;
                page_k = page_n, row_k = row_n;
            }
            kt += n_kv;
            ++qi;
            cur = nxt;
            e = e_next;
        }
    } else if (warp == R::QK || warp == R::PV) {
        // ---------------- MMA issuers ----------------
        if constexpr (FP8) fewer_registers<WORKER_REGS>();
        constexpr uint32_t IDESC_QK = make_idesc(false);
        auto desc = [](uint32_t hi, uint32_t lo) { return ((uint64_t)hi << 32) | lo; };
        // (e4m3: polling takes issue slots from the converting warps, 2 % of the kernel's time)
        auto wait_all = [&](uint32_t b, uint32_t parity) { return __all_sync(0xffffffffu, (FP8 ? mbar_wait(b, parity, abort_flag) : mbar_wait_polling(b, parity, abort_flag))); };
        const bool qk_role = warp == R::QK;
        const uint64_t dq = make_desc(sbase + OFF_Q, 16, 1024);
        // keys: 8-row groups of HALVES blocks of 1 KB; values: 8-row groups of a block 1 KB apart, or (boxes of 8 rows) a box apart
        const uint64_t dk = make_desc(sbase + OFF_K, 16, HALVES * 1024);
        const uint64_t dv = make_desc(sbase + OFF_V, v_block, tile_rows == 8 ? v_box : 1024);
        const uint32_t hi_q = (uint32_t)(dq >> 32), hi_k = (uint32_t)(dk >> 32), hi_v = (uint32_t)(dv >> 32);
        const uint32_t q_lo = (uint32_t)dq, k_lo = (uint32_t)dk, v_lo = (uint32_t)dv;
        // 16 keys further in a value tile: within a box of 128 rows or less, or in another box
        const int box_shift = __ffs(tile_rows) - 1;
        const int steps_of_box = tile_rows >= 16 ? tile_rows / 16 : 1, box_step = tile_rows >= 16 ? v_box : 2 * v_box, step_shift = __ffs(steps_of_box) - 1;
        bool ok = true;
        int it = 0, qi = 0, kt = 0;
        while (ok) {
            const int is = it & 1;
            ok = wait_all(bar.item_full(is), (it >> 1) & 1);
            if (!ok) break;
            const int n_kv = items[is].n_kv, n_members = items[is].n_members, first = items[is].first, tiles = items[is].tiles, kv = items[is].kv;
            __syncwarp();
            if (lane == 0) mbar_arrive(bar.item_empty(is));
            if (n_kv < 0) break;
            ++it;
            if (n_kv == 0) continue;
            if (qk_role) {
                ok = wait_all(bar.q_full(), qi & 1);
                for (int j = 0; j < n_kv && ok; ++j, ++kt) {
                    const int ts = kt & 1;
                    ok = wait_all(bar.k_full(ts), (kt >> 1) & 1) && (kt == 0 || wait_all(bar.s_free(), (kt - 1) & 1));
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t d = tmem_base + S_COL0;
                    const uint32_t kb = k_lo + (FP8 ? 0 : ts) * (TILE_BYTES >> 4);
                    if (elect_one()) {
#pragma unroll
                        for (int s = 0; s < HD / 16; ++s) {
                            const uint32_t q_off = ((s >> 2) * HALF_BYTES + (s & 3) * 32) >> 4, k_off = ((s >> 2) * 1024 + (s & 3) * 32) >> 4;
                            tc_mma(d, desc(hi_q, q_lo + q_off), desc(hi_k, kb + k_off), IDESC_QK, s > 0);
                        }
                        tc_commit(bar.qk_done(ts));
                        if (j + 1 == n_kv) tc_commit(bar.q_empty());
                    }
                    __syncwarp();
                }
            } else {
                for (int j = 0; j < n_kv && ok; ++j, ++kt) {
                    const int ts = kt & 1;
                    ok = wait_all(bar.v_full(ts), (kt >> 1) & 1);
                    if (!ok) break;
                    const int valid = kv - tile_col(first, tiles, j);
                    if (!FP8 && valid < BN) {  // rows behind the request's length: zeros, whatever is there
                        const int strip = lane >> 3;  // a 64-column block of a member: 4 in all
                        if (strip < n_members * HALVES)
                            for (int r = valid; r < BN; ++r) {
                                const uint32_t at = sbase + OFF_V + ts * 2 * TILE_BYTES + (r >> box_shift) * v_box + strip * v_block + (r & (box_rows - 1)) * 128 + (lane & 7) * 16;
                                asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at), "r"(0) : "memory");
                            }
                        fence_async_proxy();
                        __syncwarp();
                    }
                    ok = wait_all(bar.p_full(ts), (kt >> 1) & 1);
                    if (!ok) break;
                    const uint32_t p_addr = tmem_base + P_COL0 + ts * 64;
                    if (j == 0 && qi > 0)  // the accumulators still hold the previous item's output
                        for (int g = 0; g < n_members && ok; ++g) ok = wait_all(bar.o_free(g), (qi - 1) & 1);
                    if (!ok) break;
                    tc_fence_after();
                    if (elect_one()) {
                        const uint32_t d = tmem_base + O_COL0;
                        const uint32_t vb = v_lo + (FP8 ? 0 : ts * 2) * (TILE_BYTES >> 4);
                        const uint32_t idesc_all = make_idesc_n(true, (unsigned)(HD * n_members));
#pragma unroll
                        for (int s = 0; s < BN / 16; ++s)
                            tc_mma_ts(d, p_addr + s * 8, desc(hi_v, vb + (uint32_t)(((s >> step_shift) * box_step + (s & (steps_of_box - 1)) * 2048) >> 4)), idesc_all, (j > 0 || s > 0) ? 1u : 0u);
                        tc_commit(bar.pv_done(ts));
                    }
                    __syncwarp();
                }
            }
            ++qi;
        }
    } else if (warp >= R::SOFTMAX && warp < R::EPILOGUE) {
        // ---------------- softmax / correction: two threads per query row ----------------
        if constexpr (FP8) more_registers<SOFTMAX_REGS>();
        const int quad = warp & 3, half = (warp - R::SOFTMAX) >> 2;
        const int row = quad * 32 + lane, cbase = half * 64;
        const uint32_t lane_addr = tmem_base + ((uint32_t)(quad * 32) << 16);
        // row maxima: bf16 [half][row][tile parity], or fp32 [half][row]
        uint8_t* const xch = smem + OFF_XCH + (half * BM + row) * 4;
        const uint8_t* const xch_other = smem + OFF_XCH + ((half ^ 1) * BM + row) * 4;
        float* lsum = reinterpret_cast<float*>(smem + OFF_LSUM);
        float* refs = reinterpret_cast<float*>(smem + OFF_REF);
        bool ok = true;
        int it = 0, ei = 0, kt = 0;
        uint32_t r[64];
        while (true) {
            const int is = it & 1;
            ok = ok && mbar_wait(bar.item_full(is), (it >> 1) & 1, abort_flag);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            const int n_kv = items[is].n_kv, n_members = items[is].n_members, rows = items[is].rows;
            const int first = items[is].first, tiles = items[is].tiles, kv = items[is].kv, sees0 = items[is].sees;
            // (the warp that hands the item on to the epilogue keeps it until then)
            const bool keeps = warp == R::SOFTMAX && n_kv > 0;
            if (n_kv == 0 && row < rows)
#pragma unroll
                for (int g = 0; g < GM; ++g) {
                    if (g >= n_members) break;
                    uint4* o = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.out) + ((size_t)(items[is].row0 + row) * a.H + items[is].heads[g]) * HD + half * (HD / 2));
#pragma unroll
                    for (int u = 0; u < HD / 16; ++u) o[u] = make_uint4(0, 0, 0, 0);
                }
            __syncwarp();
            if (lane == 0 && !keeps) mbar_arrive(bar.item_empty(is));
            if (n_kv < 0) break;
            ++it;
            if (n_kv == 0) continue;
            const bool idle = quad * 32 >= rows;  // none of the warp's rows exists: it only keeps step
            // positions that the row sees (a row that does not exist: none, so that it cannot move a reference)
            const int sees = row < rows ? min(kv, a.causal ? sees0 + row : kv) : 0;
            // The reference starts at 0, may be lowered by the first tile that the row sees something of, and grows when a
            // tile's maximum leaves the window around it.
            float m_used = 0.f, l_run = 0.f;
            bool fresh = true;  // the row has seen nothing so far
            for (int j = 0; j < n_kv && ok; ++j, ++kt) {
                const int sb = kt & 1;
                ok = __all_sync(0xffffffffu, mbar_wait(bar.qk_done(sb), (kt >> 1) & 1, abort_flag));
                if (!ok) break;
                if (idle) {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar.s_free());
                    if (kt >= 2) ok = __all_sync(0xffffffffu, mbar_wait(bar.pv_done(sb), ((kt >> 1) & 1) ^ 1, abort_flag));
                    if (!ok) break;
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar.p_full(sb));
                    continue;
                }
                tc_fence_after();
                const uint32_t s_addr = lane_addr + S_COL0;
                const uint32_t p_st = lane_addr + P_COL0 + sb * 64 + half * 32;
                const int col0 = tile_col(first, tiles, j);
                const int vis = max(0, min(sees - col0 - cbase, 64));
                const bool full_tile = col0 + BN <= min(kv, sees0) && quad * 32 + 32 <= rows;
                tc_ld64_wait(s_addr + cbase, r);
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar.s_free());
                if (!full_tile) {
#pragma unroll
                    for (int i = 0; i < 64; ++i)
                        if (i >= vis) r[i] = 0xff800000u;
                }
                float mxa[8];
#pragma unroll
                for (int c = 0; c < 8; ++c) mxa[c] = -INFINITY;
                auto publish = [&]() {
                    *reinterpret_cast<__nv_bfloat16*>(xch + (kt & 1) * 2) = __float2bfloat16_ru(max3(max3(mxa[0], mxa[1], mxa[2]), max3(mxa[3], mxa[4], mxa[5]), fmaxf(mxa[6], mxa[7])));
                };
                auto together = [&]() -> bool {
                    // (the two warps of a quadrant; whoever gives up arrives once on its way out)
                    asm volatile("bar.sync %0, 64;" ::"r"(quad + 1) : "memory");
                    return !*abort_flag;
                };
                auto leaves = [&](float m) { return m > m_used + REF_WINDOW || (fresh && m > -INFINITY && m < m_used - REF_WINDOW); };
                auto emit = [&](float m, auto with_max) -> float {
                    const uint64_t sc2 = pack2(scale_log2, scale_log2), nm2 = pack2(-m, -m);
                    float l0 = 0.f, l1 = 0.f, l2 = 0.f, l3 = 0.f;  // of the rounded probabilities
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t packed[8];
#pragma unroll
                        for (int u = 0; u < 16; u += 4) {
                            const int i = c * 16 + u;
                            float x0, x1, x2, x3;
                            unpack2(fma2(pack2(__uint_as_float(r[i]), __uint_as_float(r[i + 1])), sc2, nm2), x0, x1);
                            unpack2(fma2(pack2(__uint_as_float(r[i + 2]), __uint_as_float(r[i + 3])), sc2, nm2), x2, x3);
                            const float p0 = fast_exp2(x0), p1 = fast_exp2(x1), p2 = fast_exp2(x2), p3 = fast_exp2(x3);
                            if constexpr (decltype(with_max)::value) {
                                mxa[(i >> 1) & 7] = max3(mxa[(i >> 1) & 7], __uint_as_float(r[i]), __uint_as_float(r[i + 1]));
                                mxa[((i >> 1) + 1) & 7] = max3(mxa[((i >> 1) + 1) & 7], __uint_as_float(r[i + 2]), __uint_as_float(r[i + 3]));
                            }
                            __nv_bfloat162 pa = __floats2bfloat162_rn(p0, p1), pb = __floats2bfloat162_rn(p2, p3);
                            packed[u >> 1] = *reinterpret_cast<uint32_t*>(&pa);
                            packed[(u >> 1) + 1] = *reinterpret_cast<uint32_t*>(&pb);
                            add_bf16x2(l0, l1, packed[u >> 1]);
                            add_bf16x2(l2, l3, packed[(u >> 1) + 1]);
                        }
                        tc_st8(p_st + c * 8, packed);
                    }
                    return (l0 + l1) + (l2 + l3);
                };
                if (kt >= 2) {  // P buffer kt & 1 was last read by the P V of tile kt - 2
                    ok = __all_sync(0xffffffffu, mbar_wait(bar.pv_done(sb), ((kt >> 1) & 1) ^ 1, abort_flag));
                    if (!ok) break;
                    tc_fence_after();
                }
                float ls = emit(m_used, std::true_type{});
                publish();
                ok = together();
                if (!ok) break;
                // The maximum rounded up to bf16 says whether a reference may move.  It is less than 2^-7 of itself too large: up
                // to EXACT_FROM that is less than 16 binary orders, and as good a reference; beyond, rows would lie further below
                // it than exponentials reach, and the two warps exchange the maximum in fp32.  (They see the same numbers and
                // decide alike.  The fp32 maximum is taken again, for nothing is free to hold it.)
                float m_tile = fmaxf(__bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(xch + (kt & 1) * 2)), __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(xch_other + (kt & 1) * 2))) * scale_log2;
                float corr = 1.f;
                bool moved = __any_sync(0xffffffffu, leaves(m_tile));
                if (moved) {
                    if (__any_sync(0xffffffffu, fabsf(m_tile) > EXACT_FROM)) {
                        ok = together();  // (both have read)
                        if (!ok) break;
                        float mx = -INFINITY;
#pragma unroll
                        for (int i = 0; i < 64; ++i) mx = fmaxf(mx, __uint_as_float(r[i]));
                        *reinterpret_cast<float*>(xch) = mx;
                        ok = together();
                        if (!ok) break;
                        if (fabsf(m_tile) > EXACT_FROM) m_tile = fmaxf(mx, *reinterpret_cast<const float*>(xch_other)) * scale_log2;  // (a row's reference follows from its own scores)
                        ok = together();  // (the next tile writes there)
                        if (!ok) break;
                    }
                    const float m_old = m_used;
                    if (leaves(m_tile)) {
                        corr = fresh ? 1.f : fast_exp2(m_used - m_tile);  // (nothing has been accumulated yet)
                        m_used = m_tile;
                    }
                    moved = __any_sync(0xffffffffu, m_used != m_old);
                    if (moved) ls = emit(m_used, std::false_type{});
                }
                if (m_tile > -INFINITY) fresh = false;
                l_run = l_run * corr + ls;
                if (j > 0 && moved) {
                    ok = __all_sync(0xffffffffu, mbar_wait(bar.pv_done((kt - 1) & 1), ((kt - 1) >> 1) & 1, abort_flag));
                    if (!ok) break;
                    tc_fence_after();
                    for (int g = 0; g < n_members; ++g) {
                        const uint32_t o_addr = lane_addr + O_COL0 + g * HD + half * (HD / 2);
                        if constexpr (HD == 128) tc_ld64_wait(o_addr, r);
                        else tc_ld32_wait(o_addr, r);
#pragma unroll
                        for (int i = 0; i < HD / 2; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * corr);
                        tc_st32(o_addr, r);
                        if constexpr (HD == 128) tc_st32(o_addr + 32, r + 32);
                    }
                }
                tc_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar.p_full(sb));
            }
            ok = __all_sync(0xffffffffu, ok && mbar_wait(bar.epi_empty(), (ei & 1) ^ 1, abort_flag));
            if (!ok) break;
            lsum[half * BM + row] = l_run;
            if (half == 0) refs[row] = m_used;
            if (tid == 32 * R::SOFTMAX) {
                items[2] = items[is];
                items[2].n_kv = kt - 1;  // number of the item's last key tile (its P V is awaited)
                mbar_arrive(bar.item_empty(is));
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar.epi_full());
            ++ei;
        }
        if (__all_sync(0xffffffffu, mbar_wait(bar.epi_empty(), (ei & 1) ^ 1, abort_flag))) {
            if (tid == 32 * R::SOFTMAX) items[2].n_members = -1;
            __syncwarp();
            if (lane == 0) mbar_arrive(bar.epi_full());
        }
        if (!ok) asm volatile("bar.arrive %0, 64;" ::"r"(quad + 1) : "memory");
        asm volatile("bar.sync %0, %1;" ::"n"(JOIN_BARRIER), "n"(32 * (SOFTMAX_WARPS + EPILOGUE_WARPS)) : "memory");
        if (!*abort_flag) join_pieces<HD>(a, smem, warp - R::SOFTMAX);
    } else if (warp >= R::EPILOGUE) {
        // ---------------- epilogue: one thread per query row ----------------
        if constexpr (!FP8) {
            for (int ei = 0; finish_item<HD>(a, smem, tmem_base, abort_flag, ei); ++ei) {}
            asm volatile("bar.arrive %0, %1;" ::"n"(JOIN_BARRIER), "n"(32 * (SOFTMAX_WARPS + EPILOGUE_WARPS)) : "memory");
        } else {
            // e4m3: units become bf16 tiles, by eight warps; a thread takes 16 numbers of NV rows, a row at a time: there are no
            // registers for more, and what is spilled comes back from L2.  The first four warps write the item before
            // out ahead of V(0), whose product waits for its accumulators.  (Two teams that take turns would hide more of the
            // waits, but a team that does not wait for every tile's products in order can mistake a barrier's phase for another.)
            fewer_registers<CONVERT_REGS>();
            constexpr int CHUNKS = HD / 16, STEP = 32 * R::CONVERT_WARPS / CHUNKS, NV = BN / STEP;
            const int ct = tid - 32 * R::EPILOGUE, x = ct % CHUNKS, row = ct / CHUNKS;  // row + i * STEP
            const bool writes_out = warp < R::EPILOGUE + EPILOGUE_WARPS;
            // 16 numbers are two 16-byte vectors of the bf16 row, in its 64-column block x / 4; vectors are swizzled within 128 bytes
            const uint32_t swizzled = (((x & 3) * 2) ^ (row & 7)) << 4;  // (STEP is a multiple of 8; the other vector: ^ 16)
            const uint32_t k_row = sbase + OFF_K + (row >> 3) * (HALVES * 1024) + (row & 7) * 128 + (x >> 2) * 1024 + swizzled;
            const uint32_t v_row = sbase + OFF_V + row * 128 + (x >> 2) * HALF_BYTES + swizzled;
            auto wait_all = [&](uint32_t b, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(b, parity, abort_flag)); };
            Unit<HD> unit;
            bool ok = true, pending = false;
            int it = 0, kt = 0, ei = 0;  // items seen, key tiles, items written out
            // The next unit to dst, rows STEP apart `apart` bytes; rows from `valid` on become zeros.
            auto convert = [&](uint32_t dst, uint32_t apart, int valid) -> bool {
                if (!wait_all(bar.raw_full(unit.slot), unit.phase)) return false;
                valid -= row;
                const uint8_t* raw = smem + OFF_RAW + (unit.slot * BN + row) * HD + x * 16;
                const float* scales = reinterpret_cast<const float*>(smem + OFF_SCALES) + unit.slot * BN + row;
                // Two rows at a time, for one chain of dependent instructions leaves most of the issue slots empty; not unrolled, for
                // what does not fit the instruction caches beside the other roles' loops waits for them.
#pragma unroll 1
                for (int i0 = 0; i0 < NV; i0 += 2) {
                    uint4 v[2];
                    float scale[2];
                    uint32_t o[2][8];
                    bool other = false;  // a NaN, or a scale that is no power of two or above 2^7
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        v[i] = *reinterpret_cast<const uint4*>(raw + i * STEP * HD);
                        scale[i] = scales[i * STEP];
                        if (i * STEP >= valid) v[i] = make_uint4(0, 0, 0, 0), scale[i] = 1.f;
                    }
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint32_t words[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
                        const uint32_t f = e4m3_factor(scale[i]);
                        uint32_t nan = 0;
#pragma unroll
                        for (int w = 0; w < 4; ++w) nan |= e4m3x4_to_bf16_bits(words[w], f, o[i] + 2 * w);
                        other |= (nan & 0x80808080u) != 0 || (__float_as_uint(scale[i]) & 0x007fffffu) != 0 || __float_as_uint(scale[i]) - 0x00800000u > 0x42800000u;
                    }
                    if (__any_sync(0xffffffffu, other))
#pragma unroll
                        for (int w = 0; w < 8; ++w)
                            e4m3x4_to_bf16(w % 4 == 0 ? v[w / 4].x : w % 4 == 1 ? v[w / 4].y : w % 4 == 2 ? v[w / 4].z : v[w / 4].w, scale[w / 4], o[w / 4] + 2 * (w % 4));
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        st_shared16(dst + i * apart, o[i]);
                        st_shared16((dst + i * apart) ^ 16, o[i] + 4);
                    }
                    raw += 2 * STEP * HD;
                    scales += 2 * STEP;
                    dst += 2 * apart;
                    valid -= 2 * STEP;
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(bar.raw_free(unit.slot));
                unit.next();
                return true;
            };
            while (ok) {
                const int is = it & 1;
                ok = wait_all(bar.item_full(is), (it >> 1) & 1);
                if (!ok) break;
                const int n_kv = items[is].n_kv, n_members = items[is].n_members, first = items[is].first, tiles = items[is].tiles, kv = items[is].kv;
                if (n_kv < 0) break;
                ++it;
                __syncwarp();
                if (lane == 0) mbar_arrive(bar.item_empty(is));
                if (n_kv == 0) continue;
                auto done = [&](uint32_t b0, uint32_t b1, int n) { return n < 0 || wait_all((n & 1) ? b1 : b0, (n >> 1) & 1); };
                auto put_k = [&](int j) -> bool {  // once the products of the tile before have read theirs
                    const int n = kt + j;
                    if (!done(bar.qk_done(0), bar.qk_done(1), n - 1) || !convert(k_row, STEP / 8 * (HALVES * 1024), kv - tile_col(first, tiles, j))) return false;
                    fence_async_proxy();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar.k_full(n & 1));
                    return true;
                };
                ok = put_k(0);
                for (int j = 0; j < n_kv && ok; ++j) {
                    if (j + 1 < n_kv) ok = put_k(j + 1);
                    if (!ok) break;
                    if (j == 0 && pending && writes_out) {
                        ok = finish_item<HD>(a, smem, tmem_base, abort_flag, ei++);
                        if (!ok) break;
                    }
                    const int n = kt + j;
                    ok = done(bar.pv_done(0), bar.pv_done(1), n - 1);
                    for (int g = 0; g < n_members && ok; ++g) ok = convert(v_row + g * HALVES * HALF_BYTES, STEP * 128, kv - tile_col(first, tiles, j));
                    if (!ok) break;
                    fence_async_proxy();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar.v_full(n & 1));
                }
                kt += n_kv;
                pending = true;
            }
            if (ok && pending && writes_out) finish_item<HD>(a, smem, tmem_base, abort_flag, ei);
            if (writes_out) asm volatile("bar.arrive %0, %1;" ::"n"(JOIN_BARRIER), "n"(32 * (SOFTMAX_WARPS + EPILOGUE_WARPS)) : "memory");
        }
    } else if constexpr (FP8) {
        // ---------------- row scales of the units, four rows a lane (of one page: page sizes are multiples of 8) ----------------
        fewer_registers<WORKER_REGS>();
        auto wait_all = [&](uint32_t b, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(b, parity, abort_flag)); };
        Unit<HD> unit;
        bool ok = true;
        for (int it = 0; ok; ++it) {
            const int is = it & 1;
            ok = wait_all(bar.item_full(is), (it >> 1) & 1);
            if (!ok) break;
            const int n_kv = items[is].n_kv, n_members = items[is].n_members, first = items[is].first, tiles = items[is].tiles, kv = items[is].kv;
            const int b = items[is].b, cluster = items[is].cluster;
            int heads[GM];
#pragma unroll
            for (int g = 0; g < GM; ++g) heads[g] = items[is].heads[g];
            __syncwarp();
            if (lane == 0) mbar_arrive(bar.item_empty(is));
            if (n_kv < 0) break;
            if (n_kv == 0) continue;
            const int32_t* table = a.pool.block_table + (size_t)b * a.pool.max_pages;
            auto look_up = [&](int j, int& page, int& row) {
                page = -1;
                row = 0;
                if (j >= n_kv) return;
                const int pos = tile_col(first, tiles, j) + lane * 4;
                if (pos >= kv) return;
                const int pi = (int)a.pool.by_page.div((unsigned)pos);
                row = pos - pi * a.pool.page_size;
                page = table[pi];
            };
            auto load = [&](bool key, int plane, int page, int row) {
                if ((unsigned)page >= (unsigned)a.pool.n_pages) return make_float4(0.f, 0.f, 0.f, 0.f);
                return __ldg(reinterpret_cast<const float4*>((key ? a.k_scales : a.v_scales) + ((size_t)page * (key ? a.k : a.H) + plane) * a.pool.page_size + row));
            };
            auto put = [&](const float4& v) -> bool {
                if (!wait_all(bar.raw_free(unit.slot), unit.phase ^ 1)) return false;
                *reinterpret_cast<float4*>(smem + OFF_SCALES + (unit.slot * BN + lane * 4) * 4) = v;
                __syncwarp();
                if (lane == 0) mbar_arrive(bar.raw_full(unit.slot));
                unit.next();
                return true;
            };
            // the scales of tile j's values and of key tile j + 1 are loaded while the ones before wait for their slots
            int page_v, row_v, page_k, row_k, page_n, row_n;
            look_up(0, page_v, row_v);
            look_up(1, page_k, row_k);
            look_up(2, page_n, row_n);
            ok = put(load(true, cluster, page_v, row_v));
            float4 k_next = load(true, cluster, page_k, row_k), v_now[GM];
#pragma unroll
            for (int g = 0; g < GM; ++g) v_now[g] = load(false, heads[g], g < n_members ? page_v : -1, row_v);
            for (int j = 0; j < n_kv && ok; ++j) {
                page_v = page_k, row_v = row_k;
                page_k = page_n, row_k = row_n;
                look_up(j + 3, page_n, row_n);
                if (j + 1 < n_kv) ok = put(k_next);
                k_next = load(true, cluster, page_k, row_k);
#pragma unroll
                for (int g = 0; g < GM; ++g)
                    if (g < n_members && ok) {
                        ok = put(v_now[g]);
                        v_now[g] = load(false, heads[g], page_v, row_v);
                    }
            }
        }
    }

    // teardown: every tcgen05 operation of this CTA has completed or been abandoned after a timeout
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM_COLS) : "memory");
    }
    if (tid == 0 && *abort_flag) atomicExch(&a.hdr->status, CHAI_ERR_TIMEOUT);
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static EncodeTiledFn encode_tiled_fn() {
    static const EncodeTiledFn fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        const bool ok = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess &&
                        q == cudaDriverEntryPointSuccess;
        return ok ? reinterpret_cast<EncodeTiledFn>(p) : nullptr;
    }();
    return fn;
}

static bool make_map(CUtensorMap* map, const void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box, bool bytes = false) {
    const EncodeTiledFn fn = encode_tiled_fn();
    if (fn == nullptr) return false;
    const cuuint32_t estr[5] = {1, 1, 1, 1, 1};
    return fn(map, bytes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              bytes ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// Keys, D = 128: (64 columns, 8 rows, 2 column halves, row groups of all planes, pages); a box of box_rows whole rows lands as
// 8-row groups of both halves.  Values: (64 columns, rows of all planes, 2 halves, pages); a box lands as one half behind the
// other.  D = 64 needs no halves: (64 columns, rows of all planes, pages).  e4m3: (D bytes, rows of all planes, pages), not swizzled.
static bool make_page_map(CUtensorMap* map, const void* base, int D, const PagePool& p, int planes, size_t page_stride, int box_rows, bool keys, bool fp8) {
    const cuuint64_t rows = (cuuint64_t)planes * p.page_size, pages = (cuuint64_t)p.n_pages, apart = (cuuint64_t)page_stride * (fp8 ? 1 : 2);
    const cuuint32_t box = (cuuint32_t)box_rows;
    if (fp8) {
        const cuuint64_t dims[3] = {(cuuint64_t)D, rows, pages}, strides[2] = {(cuuint64_t)D, apart};
        const cuuint32_t b[3] = {(cuuint32_t)D, box, 1};
        return make_map(map, base, 3, dims, strides, b, true);
    }
    if (D == 64) {
        const cuuint64_t dims[3] = {64, rows, pages}, strides[2] = {128, apart};
        const cuuint32_t b[3] = {64, box, 1};
        return make_map(map, base, 3, dims, strides, b);
    }
    if (keys) {
        const cuuint64_t dims[5] = {64, 8, 2, rows / 8, pages}, strides[4] = {256, 128, 2048, apart};
        const cuuint32_t b[5] = {64, 8, 2, box / 8, 1};
        return make_map(map, base, 5, dims, strides, b);
    }
    const cuuint64_t dims[4] = {64, rows, 2, pages}, strides[3] = {256, 128, apart};
    const cuuint32_t b[4] = {64, box, 2, 1};
    return make_map(map, base, 4, dims, strides, b);
}

}  // namespace pp

static int prefill_paged(const char* fn, bool fp8, PagedCall a, int n_pages, int page_size, int max_pages, int D,
                         const int32_t* block_table, size_t k_page_stride, size_t v_page_stride, int dtype, void* workspace,
                         size_t workspace_bytes, cudaStream_t s) {
    CHAI_REQUIRE(a.q && a.k_pages && a.v_pages && a.membership && a.reps && block_table && a.kv_lens && a.token_start && a.out && workspace,
                 CHAI_ERR_INVALID_ARG, "%s: null pointer", fn);
    CHAI_REQUIRE(!fp8 || (a.k_scales && a.v_scales), CHAI_ERR_INVALID_ARG, "%s: null pointer", fn);
    const void* all[] = {a.q, a.k_pages, a.v_pages, a.membership, a.reps, block_table, a.kv_lens, a.token_start, a.out, workspace, a.k_scales, a.v_scales};
    for (const void* p : all) CHAI_REQUIRE(aligned16(p), CHAI_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned", fn);
    CHAI_REQUIRE(dtype == CHAI_F32 || dtype == CHAI_BF16, CHAI_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, dtype);
    const int rc = make_pool(fn, block_table, a.B, a.H, a.k, n_pages, page_size, max_pages, D, k_page_stride, v_page_stride,
                             fp8 ? 1 : elem_size(dtype), &a.pool);
    if (rc != CHAI_OK) return rc;
    CHAI_REQUIRE(a.n_tokens > 0, CHAI_ERR_INVALID_ARG, "%s: need n_tokens > 0", fn);
    CHAI_REQUIRE(isfinite(a.scale) && a.scale > 0.f, CHAI_ERR_INVALID_ARG, "%s: scale must be positive and finite", fn);
    CHAI_REQUIRE(a.n_tokens <= (1 << 26), CHAI_ERR_UNSUPPORTED, "%s: n_tokens must be <= 2^26", fn);
    constexpr size_t plan_limit = 48 * 1024 - 256;  // (beside what the planner has anyway)
    CHAI_REQUIRE(prefill_paged_plan_smem(a.H, a.k) <= plan_limit, CHAI_ERR_UNSUPPORTED,
                 "%s: too many heads and clusters for the planner (H=%d, k=%d need %zu bytes of shared memory, limit %zu)", fn, a.H,
                 a.k, prefill_paged_plan_smem(a.H, a.k), plan_limit);
    const long long dense = (long long)a.H * D, es = (long long)elem_size(dtype);
    if (a.q_stride == 0) a.q_stride = dense;
    CHAI_REQUIRE(a.q_stride >= dense && a.q_stride < (1ll << 40) / es && a.q_stride <= (1ll << 56) / a.n_tokens && a.q_stride * es % 16 == 0,
                 CHAI_ERR_INVALID_ARG,
                 "%s: the token stride of q must be at least H*D=%lld elements, a multiple of 16 bytes and below 2^40 bytes", fn, dense);
    CHAI_REQUIRE(a.pool.k_page_stride * 2 < (1ull << 40) && a.pool.v_page_stride * 2 < (1ull << 40), CHAI_ERR_UNSUPPORTED,
                 "%s: page strides must be below 2^39 elements", fn);
    const char *q_at = static_cast<const char*>(a.q), *o_at = static_cast<const char*>(a.out);
    CHAI_REQUIRE(q_at + ((a.n_tokens - 1) * a.q_stride + dense) * es <= o_at || o_at + a.n_tokens * dense * es <= q_at,
                 CHAI_ERR_INVALID_ARG, "%s: q and out must not overlap", fn);
    const bool tensor = dtype == CHAI_BF16;
    a.bq = pp::BM;
    a.bk = pp::BN;
    if (!tensor) prefill_paged_simt_tile(a.B, a.n_tokens, D, &a.bq, &a.bk);
    // (the work's line is counted in 32 bits for a group, and shares of all of it are)
    const long long row_tiles = (long long)a.n_tokens / a.bq + 1, keys = a.pool.capacity / a.bk + 2;
    CHAI_REQUIRE(row_tiles * keys < (1ll << 27) && (row_tiles + a.B) * keys * a.H < (1ll << 32), CHAI_ERR_UNSUPPORTED,
                 "%s: tokens x table too large: with query tiles of %d rows and key tiles of %d, (tiles + B) * key tiles * H must be below "
                 "2^32, and tiles * key tiles below 2^27", fn, a.bq, a.bk);
    const size_t need = chai_prefill_paged_workspace_bytes(a.B, a.H, a.n_tokens);
    CHAI_REQUIRE(workspace_bytes >= need, CHAI_ERR_WORKSPACE, "%s: workspace has %zu bytes, %zu needed", fn, workspace_bytes, need);

    static PerDeviceOnce once;
    static int sms_of_device[kMaxDevices] = {};
    int dev = 0;
    cudaError_t de = cudaGetDevice(&dev);
    if (de != cudaSuccess) return cuda_fail(de, "prefill_paged_kernel set-up");
    CHAI_REQUIRE(dev >= 0 && dev < kMaxDevices, CHAI_ERR_UNSUPPORTED, "%s: device index %d out of range", fn, dev);
    const int set_up = once.run(dev, [&]() -> int {
        int count = 0;
        cudaError_t e = cudaDeviceGetAttribute(&count, cudaDevAttrMultiProcessorCount, dev);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(pp::prefill_paged_kernel<128, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, pp::SMEM_BYTES);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(pp::prefill_paged_kernel<64, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, pp::SMEM_BYTES);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(pp::prefill_paged_kernel<128, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, pp::SMEM_BYTES);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(pp::prefill_paged_kernel<64, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, pp::SMEM_BYTES);
        // the e4m3 kernels move registers between their warpgroups: no more than they were launched with
        for (const void* f : {(const void*)pp::prefill_paged_kernel<128, true>, (const void*)pp::prefill_paged_kernel<64, true>}) {
            cudaFuncAttributes attr = {};
            if (e == cudaSuccess) e = cudaFuncGetAttributes(&attr, f);
            CHAI_REQUIRE(e != cudaSuccess || attr.numRegs == pp::LAUNCH_REGS, CHAI_ERR_CUDA,
                         "prefill_paged_kernel was compiled for %d registers a thread, %d expected", attr.numRegs, pp::LAUNCH_REGS);
        }
        if (e != cudaSuccess) return cuda_fail(e, "prefill_paged_kernel set-up");
        sms_of_device[dev] = count;
        return CHAI_OK;
    });
    if (set_up != CHAI_OK) return set_up;

    const PagedLayout L = paged_layout(a.B, a.H, a.n_tokens);
    char* ws = static_cast<char*>(workspace);
    a.hdr = reinterpret_cast<WsHeader*>(ws);
    a.done = reinterpret_cast<int*>(ws + L.off_done);
    a.joins = ws + L.off_joins;
    a.req = reinterpret_cast<PagedRequest*>(ws + L.off_req);
    a.groups = reinterpret_cast<PagedGroup*>(ws + L.off_groups);
    a.slots = ws + L.off_slots;
    a.gmax = 256 / D;
    const int ctas = sms_of_device[dev] * (tensor ? 1 : 2);
    a.ctas = ctas < kPagedMaxCtas ? ctas : kPagedMaxCtas;
    a.slot_rows = ((a.bq < a.n_tokens ? a.bq : a.n_tokens) + 1) & ~1;  // (even: slots are multiples of 16 bytes)
    CHAI_LOG_CALL("%s: B=%d H=%d k=%d n_tokens=%d D=%d dtype=%d page_size=%d causal=%d, query tiles of %d rows", fn, a.B, a.H, a.k,
                  a.n_tokens, D, dtype, page_size, a.causal, a.bq);
    CHAI_LAUNCH_DEPENDENT("prefill_paged_plan_kernel launch", prefill_paged_plan_kernel, dim3(a.B), dim3(kPagedPlanThreads), prefill_paged_plan_smem(a.H, a.k), s, a);
    if (!tensor) return prefill_paged_simt(a, D, fp8, s);
    pp::Tma maps;
    int box_rows = 128;
    while (page_size % box_rows != 0) box_rows >>= 1;
    const cuuint64_t q_dims[3] = {(cuuint64_t)D, (cuuint64_t)a.H, (cuuint64_t)a.n_tokens};
    const cuuint64_t q_strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)a.q_stride * 2};
    const cuuint32_t q_box[3] = {64, 1, pp::BM};
    CHAI_REQUIRE(pp::make_map(&maps.q, a.q, 3, q_dims, q_strides, q_box) &&
                     pp::make_page_map(&maps.k, a.k_pages, D, a.pool, a.k, a.pool.k_page_stride, box_rows, true, fp8) &&
                     pp::make_page_map(&maps.v, a.v_pages, D, a.pool, a.H, a.pool.v_page_stride, box_rows, false, fp8),
                 CHAI_ERR_CUDA, "%s: cuTensorMapEncodeTiled failed", fn);
    const float scale_log2 = a.scale * 1.4426950408889634f;
    auto kernel = D == 128 ? (fp8 ? pp::prefill_paged_kernel<128, true> : pp::prefill_paged_kernel<128, false>)
                           : (fp8 ? pp::prefill_paged_kernel<64, true> : pp::prefill_paged_kernel<64, false>);
    CHAI_LAUNCH_DEPENDENT("prefill_paged_kernel launch", kernel, dim3(a.ctas), dim3(fp8 ? pp::Roles<true>::THREADS : pp::Roles<false>::THREADS), pp::SMEM_BYTES, s, maps, a, box_rows, scale_log2);
    return CHAI_OK;
}

static PagedCall paged_call(const void* q, const void* k_pages, const void* v_pages, const float* k_scales, const float* v_scales,
                            const int32_t* membership, const int32_t* reps, const int32_t* kv_lens, const int32_t* token_start,
                            void* out, int B, int H, int k, int n_tokens, size_t q_token_stride, float scale, int causal) {
    PagedCall a = {};
    a.q = q;
    a.k_pages = k_pages;
    a.v_pages = v_pages;
    a.k_scales = k_scales;
    a.v_scales = v_scales;
    a.membership = membership;
    a.reps = reps;
    a.kv_lens = kv_lens;
    a.token_start = token_start;
    a.out = out;
    a.B = B;
    a.H = H;
    a.k = k;
    a.n_tokens = n_tokens;
    a.q_stride = (long long)q_token_stride;
    a.scale = scale;
    a.causal = causal != 0;
    return a;
}

}  // namespace chai

extern "C" {

size_t chai_prefill_paged_workspace_bytes(int B, int H, int n_tokens) {
    if (B <= 0 || H <= 0 || n_tokens <= 0) return 0;
    return ((size_t)1 << 20) + 64 * (size_t)B + 36 * (size_t)H * ((size_t)B + n_tokens / 128 + 1) +
           chai::kSlotBytesPerToken * (size_t)(n_tokens < 128 ? n_tokens : 128);
}

int chai_prefill_attention_paged(const void* q, const void* k_pages, const void* v_pages, const int32_t* membership,
                                 const int32_t* reps, const int32_t* block_table, const int32_t* kv_lens, const int32_t* token_start,
                                 void* out, int B, int H, int k, int n_tokens, int n_pages, int page_size, int max_pages, int D,
                                 size_t q_token_stride, size_t k_page_stride, size_t v_page_stride, float scale, int causal,
                                 int dtype, void* workspace, size_t workspace_bytes, void* stream) {
    return chai::prefill_paged("chai_prefill_attention_paged", false,
                               chai::paged_call(q, k_pages, v_pages, nullptr, nullptr, membership, reps, kv_lens, token_start, out, B,
                                                H, k, n_tokens, q_token_stride, scale, causal),
                               n_pages, page_size, max_pages, D, block_table, k_page_stride, v_page_stride, dtype, workspace,
                               workspace_bytes, static_cast<cudaStream_t>(stream));
}

int chai_prefill_attention_paged_fp8(const void* q, const void* k_pages, const void* v_pages, const float* k_scales,
                                     const float* v_scales, const int32_t* membership, const int32_t* reps,
                                     const int32_t* block_table, const int32_t* kv_lens, const int32_t* token_start, void* out, int B,
                                     int H, int k, int n_tokens, int n_pages, int page_size, int max_pages, int D,
                                     size_t q_token_stride, size_t k_page_stride, size_t v_page_stride, float scale, int causal,
                                     int dtype, void* workspace, size_t workspace_bytes, void* stream) {
    return chai::prefill_paged("chai_prefill_attention_paged_fp8", true,
                               chai::paged_call(q, k_pages, v_pages, k_scales, v_scales, membership, reps, kv_lens, token_start, out,
                                                B, H, k, n_tokens, q_token_stride, scale, causal),
                               n_pages, page_size, max_pages, D, block_table, k_page_stride, v_page_stride, dtype, workspace,
                               workspace_bytes, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
