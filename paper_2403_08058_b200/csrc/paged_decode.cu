// Clustered decode attention over a paged cache (Fig. 3(b), Section 3.4), bound by HBM:
//   out[b][h] = sum_t p_t V[h][t],  p = softmax_t(scale * q[r] . K[c][t]),  c the head's cluster, r its representative.
//
// The rows of all requests, in units of eight, are one line that is cut into equal pieces, one per CTA and one CTA per
// SM: ragged batches and a single long request are balanced alike, whatever the clusters' sizes, because a piece
// carries the key rows of all clusters and the value rows of all heads.  (Pieces too short to be worth a CTA are made
// longer, and the heads, ordered by cluster, are dealt to several CTAs instead.)  A CTA goes through its piece request
// by request in chunks that fit its score buffer:
//   K   its warps share the (cluster, tile) pairs of the chunk: scores into shared memory
//   S   per cluster: running maximum and sum, scores become probabilities
//   V   its warps share the (head, tile) pairs, in order of heads: sums of p_t V_t; a head that two warps share is
//       added up in warp order
// Every warp feeds itself: it owns a few slots of shared memory, and as soon as it is done with a tile one of its lanes
// per page starts the bulk copies of the next tile into the freed slot, values of the chunk (and keys of the next one)
// included, so that HBM is busy through the two barriers between the phases.  A tile's rows may come from several
// pages; a copy is a run of rows that are neighbours in memory.
// A request that lies in one piece is written at once.  The others leave one partial result (maximum, sum, values) per
// piece, and a second kernel, launched as a programmatic dependent, joins them: all sums are taken in an order that
// follows from the lengths alone, and nothing in the workspace has to be cleared.
#include <type_traits>

#include "paged.cuh"

namespace chai {
namespace {

constexpr int kWarps = 8, kThreads = kWarps * 32;
constexpr int kMaxCtas = 160;       // the workspace bound is stated for this many; a B200 has 148 SMs
constexpr int kQuantum = 8;         // rows; page sizes are multiples of it
constexpr int kMaxChunkRows = 512;
constexpr int kScoreFloats = 4096;  // scores of a chunk: clusters * rows
constexpr int kGroupHeads = 128;    // heads a CTA handles at most
constexpr int kJoinThreads = 256;

template <typename T, int D>
struct Geom {
    static constexpr bool FP8 = std::is_same<T, Fp8E4M3>::value;
    static constexpr int ROW = D * (int)sizeof(T);
    static constexpr int TR = FP8 ? 64 : 8192 / ROW;       // rows of a tile
    static constexpr int STAGES = FP8 && D == 64 ? 5 : 3;  // slots of a warp (about 24 KB)
    static constexpr int LPR = ROW / 16, RPW = 32 / LPR;   // lanes a row, rows a warp-wide load (types of 2 and 4 bytes)
    static constexpr int IT = TR / RPW;                    // ... and such loads a tile
    // e4m3: a tile is four runs of 16 rows, each 32 bytes further than dense, so that the four lanes which read rows of
    // the four runs at once meet different banks
    static constexpr int RUN = FP8 ? TR / 4 : TR;
    static constexpr int RUN_STRIDE = RUN * ROW + (FP8 ? 32 : 0);
    static constexpr int DATA = FP8 ? 4 * RUN_STRIDE : TR * ROW;
    static constexpr int SLOT = DATA + (FP8 ? TR * 4 : 0);  // e4m3: the rows' scales lie behind them
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

struct Segment {  // the rows of one request in this CTA's piece
    unsigned short head[kGroupHeads];     // heads, ordered by cluster
    unsigned short cluster[kGroupHeads];  // the head's cluster, counted within this list
    unsigned short id[kGroupHeads];       // a counted cluster's own number ...
    unsigned short rep[kGroupHeads];      // ... and representative
};
struct Chunk {
    int b, t0, rows, stride;  // stride: floats between two clusters' scores
    int tiles, heads, clusters, run;
    int first, last, single, slot;  // first / last chunk of the segment; single: the segment is the whole request
    int seg, bad;
};
template <int SLOT, int STAGES, int D>
struct Smem {
    alignas(128) unsigned char slot[kWarps][STAGES][SLOT];
    alignas(16) float score[kScoreFloats];
    union {
        alignas(16) float part[kWarps][D];   // phase V: sums of a head's rows that another warp finishes
        unsigned short cl[kPagedMaxHeads];   // while a segment is prepared: every head's cluster (0xffff: unknown)
    };
    float top[kGroupHeads], sum[kGroupHeads], keep[kGroupHeads];  // per cluster: running maximum and sum, rescaling factor
    Segment seg[2];
    Chunk chunk[2];
    int2 at[2][kMaxChunkRows / kQuantum];  // page and row of every eighth row of the chunk
    alignas(8) unsigned long long full[kWarps][STAGES];
    int scan[kWarps];
    int found_b, found_start;
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
// try_wait lets the hardware suspend the warp for a while, which a limit shorter than the default would not notice:
// such a limit polls instead.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, long long limit) {
    const bool poll = limit < kDefaultWaitLimitCycles;
    if (poll ? bar_test(bar, parity) : bar_try(bar, parity)) return true;
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
__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint4 lds16(uint32_t a) {
    uint4 r;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(a));
    return r;
}
__device__ __forceinline__ uint2 lds8(uint32_t a) {
    uint2 r;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(r.x), "=r"(r.y) : "r"(a));
    return r;
}
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
__device__ __forceinline__ uint32_t e4m3_pair(uint32_t two_bytes) {  // two numbers as two fp16 (exact)
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two_bytes, __NV_E4M3);
    return (uint32_t)h.x | ((uint32_t)h.y << 16);
}
__device__ __forceinline__ uint32_t half_pair(float x, float y) {
    const __half2 h = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 half_floats(uint32_t h) { return __half22float2(*reinterpret_cast<const __half2*>(&h)); }
// c += a b with a 16 x 16 (row), b 16 x 8 (col), fp16, fp32 sums
__device__ __forceinline__ void mma16816(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// A power of two f with |x| f in [1, 2) and its inverse; 1 where x is 0, tiny, infinite or NaN.
__device__ __forceinline__ void normaliser(float x, float* f, float* inv) {
    const unsigned e = (__float_as_uint(x) >> 23) & 0xffu;
    const bool plain = e >= 1 && e <= 253;
    *f = plain ? __uint_as_float((254u - e) << 23) : 1.f;
    *inv = plain ? __uint_as_float(e << 23) : 1.f;
}

// ---- the main kernel --------------------------------------------------------------------------------------------

// A warp's way through the tiles of a chunk: its share of the (cluster, tile) pairs, then of the (head, tile) pairs.
struct Walk {
    int phase, p, j, left;
    __device__ __forceinline__ void start(int ph, const Chunk& c, int warp) {
        const int n = (ph == 0 ? c.clusters : c.heads) * c.tiles;
        const int lo = n * warp / kWarps;
        phase = ph;
        left = n * (warp + 1) / kWarps - lo;
        p = lo / c.tiles;
        j = lo - p * c.tiles;
    }
    __device__ __forceinline__ void step(int tiles) {
        --left;
        if (++j == tiles) {
            j = 0;
            ++p;
        }
    }
};

template <typename T, typename TQ, int D>
__global__ void __launch_bounds__(kThreads, 1) paged_decode_kernel(const DecodeArgs a) {
    using G = Geom<T, D>;
    using S = Smem<G::SLOT, G::STAGES, D>;
    extern __shared__ __align__(128) unsigned char smem_raw[];
    S& sm = *reinterpret_cast<S*>(smem_raw);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int ps = a.pool.page_size;
    dependent_grid_sync();

    if (lane == 0) {
        for (int s = 0; s < G::STAGES; ++s)
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_addr(&sm.full[warp][s])) : "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (tid == 0) sm.err = CHAI_OK, sm.err_b = -1;

    // -- the line of all rows, this CTA's piece [q_lo, q_hi) and the request it starts in
    auto length = [&](int b) { return min(max(a.seq_lens[b], 0), a.pool.capacity); };
    auto quanta = [](int n) { return (n + kQuantum - 1) / kQuantum; };
    const int per = (a.B + kThreads - 1) / kThreads;
    const int b_lo = min(tid * per, a.B), b_hi = min(b_lo + per, a.B);
    int mine = 0;
    for (int b = b_lo; b < b_hi; ++b) mine += quanta(length(b));
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
    }
    if (lane == 31) sm.scan[warp] = upto;
    __syncthreads();
    int total = 0;
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) upto += sm.scan[w];
        total += sm.scan[w];
    }
    // Heads are dealt to several CTAs when a piece would be shorter than 32 rows, down to 4 heads a CTA.
    int groups = (a.H + kGroupHeads - 1) / kGroupHeads;
    while ((long long)total * groups < 4ll * gridDim.x && 8 * groups <= a.H && 2 * groups <= (int)gridDim.x) groups *= 2;
    const int pieces = max(1, min((int)gridDim.x / groups, total));
    const int piece = blockIdx.x / groups, group = blockIdx.x - piece * groups;
    const bool by_request = a.n_desc == a.B;  // descriptions are kept per request, or (more requests than CTAs) per piece
    if (!by_request && (int)blockIdx.x >= pieces && (int)blockIdx.x < a.n_desc && tid == 0) a.ws.desc[blockIdx.x] = make_int4(-1, 0, 0, 0);
    for (int b = blockIdx.x; b < a.B; b += gridDim.x) {  // requests without rows: zeros
        if (length(b) > 0) continue;
        if (by_request && tid == 0) a.ws.desc[b] = make_int4(-1, 0, 0, 0);
        uint4* o = reinterpret_cast<uint4*>(static_cast<TQ*>(a.out) + (size_t)b * a.H * D);
        for (int i = tid; i < a.H * D * (int)sizeof(TQ) / 16; i += kThreads) o[i] = make_uint4(0, 0, 0, 0);
    }
    auto piece_start = [&](int i) { return (int)((long long)i * total / pieces); };
    const bool work = piece < pieces && total > 0;
    const int q_lo = work ? piece_start(piece) : 0, q_hi = work ? piece_start(piece + 1) : 0;
    if (work && mine > 0 && q_lo >= upto - mine && q_lo < upto) {
        int start = upto - mine, b = b_lo;
        while (q_lo >= start + quanta(length(b))) start += quanta(length(b++));
        sm.found_b = b;
        sm.found_start = start;
    }
    __syncthreads();

    // -- state of the division into segments and chunks, the same in every thread
    int q_at = q_lo, b = work ? sm.found_b : 0, b_start = work ? sm.found_start : 0;
    int seg_t = 0, seg_end = 0, seg_par = 1, seg_rows = 0, seg_heads = 0, seg_clusters = 0, seg_slot = 0;
    bool seg_single = false, seg_first = false;
    bool opened_span = false;

    // Prepares the next chunk into buffer `par`; false if the piece is done.  Called by all threads together.
    auto prepare = [&](int par) -> bool {
        if (seg_t >= seg_end) {
            if (q_at >= q_hi) return false;
            int n = length(b);
            while (q_at >= b_start + quanta(n)) {
                b_start += quanta(n);
                n = length(++b);
            }
            const int nq = quanta(n), q_end = min(q_hi, b_start + nq);
            seg_t = (q_at - b_start) * kQuantum;
            seg_end = min(n, (q_end - b_start) * kQuantum);
            seg_single = q_at == b_start && q_end == b_start + nq;
            seg_first = true;
            seg_slot = piece + b;
            seg_par ^= 1;
            Segment& sg = sm.seg[seg_par];
            const bool opens = q_at == b_start && group == 0;  // this CTA answers for the request's unknown heads
            if (q_at == b_start && !seg_single) opened_span = true;
            if (tid == 0 && opens && (by_request || !seg_single)) {
                const long long last = b_start + nq - 1;
                const int end = (int)(((last + 1) * pieces - 1) / total);
                a.ws.desc[by_request ? b : piece] = make_int4(seg_single ? -1 : b, seg_slot, end - piece + 1, 0);
            }
            q_at = q_end;
            // heads ordered by cluster; unknown ones get zeros and are left out
            const int32_t* reps = a.reps + (size_t)b * a.k;
            int known = 0;
            for (int h0 = 0; h0 < a.H; h0 += kThreads) {
                const int h = h0 + tid;
                int c = 0xffff, r;
                bool ok = false;
                if (h < a.H) {
                    ok = resolve_head(a.membership, a.reps, b, h, a.H, a.k, &c, &r);
                    sm.cl[h] = ok ? (unsigned short)c : 0xffff;
                    if (!ok && opens) {
                        atomicCAS(&sm.err, CHAI_OK, CHAI_ERR_BAD_MEMBERSHIP);
                        sm.err_b = b;
                        if (!seg_single) a.ws.ml[(size_t)seg_slot * a.H + h] = make_float2(0.f, -1.f);
                        TQ* o = static_cast<TQ*>(a.out) + ((size_t)b * a.H + h) * D;
                        for (int d = 0; d < D; ++d) o[d] = from_float<TQ>(0.f);
                    }
                }
                known += __syncthreads_count(ok);
            }
            const int lo = (int)((long long)known * group / groups), hi = (int)((long long)known * (group + 1) / groups);
            for (int h = tid; h < a.H; h += kThreads) {
                const unsigned c = sm.cl[h];
                if (c == 0xffff) continue;
                int rank = 0;
                for (int x = 0; x < a.H; ++x) rank += sm.cl[x] < c || (sm.cl[x] == c && x < h);
                if (rank >= lo && rank < hi) {
                    sg.head[rank - lo] = (unsigned short)h;
                    sg.cluster[rank - lo] = (unsigned short)c;
                }
            }
            __syncthreads();
            seg_heads = hi - lo;
            // number the clusters that occur: one warp, 32 heads at a time
            if (warp == 0) {
                int before = 0;
                for (int i0 = 0; i0 < seg_heads; i0 += 32) {
                    const int i = i0 + lane;
                    const int c = i < seg_heads ? sg.cluster[i] : -1;
                    const bool opens_cluster = i < seg_heads && (i == 0 || sm.cl[sg.head[i - 1]] != c);
                    const unsigned bits = __ballot_sync(0xffffffffu, opens_cluster);
                    const int idx = before + __popc(bits & (0xffffffffu >> (31 - lane))) - 1;
                    if (opens_cluster) {
                        sg.id[idx] = (unsigned short)c;
                        sg.rep[idx] = (unsigned short)reps[c];
                    }
                    __syncwarp();
                    if (i < seg_heads) sg.cluster[i] = (unsigned short)idx;
                    before += __popc(bits);
                }
                if (lane == 0) sm.scan[0] = before;
            }
            if (tid == 0) sm.any_bad = 0;
            __syncthreads();
            seg_clusters = sm.scan[0];
            const int most = min(kMaxChunkRows, kScoreFloats / max(seg_clusters, 1) / kQuantum * kQuantum);
            const int rows = seg_end - seg_t, chunks = (rows + most - 1) / most;
            seg_rows = ((rows + chunks - 1) / chunks + kQuantum - 1) / kQuantum * kQuantum;
        }
        const int rows = min(seg_rows, seg_end - seg_t);
        const int32_t* table = a.pool.block_table + (size_t)b * a.pool.max_pages;
        bool bad = false;
        for (int i = tid; i * kQuantum < rows; i += kThreads) {
            const unsigned pos = (unsigned)(seg_t + i * kQuantum), pi = a.pool.by_page.div(pos);
            int page = table[pi];
            if (page < 0 || page >= a.pool.n_pages) {
                bad = true;
                page = 0;
            }
            sm.at[par][i] = make_int2(page, (int)(pos - pi * (unsigned)ps));
        }
        if (bad) sm.any_bad = 1;  // of the segment so far
        if (tid == 0) {
            Chunk& c = sm.chunk[par];
            c.b = b;
            c.t0 = seg_t;
            c.rows = rows;
            c.stride = (rows + 7) & ~7;
            c.tiles = (rows + G::TR - 1) / G::TR;
            c.heads = seg_heads;
            c.clusters = seg_clusters;
            const int align = ps | seg_t;
            c.run = min(align & -align, G::RUN);
            c.first = seg_first;
            c.last = seg_t + rows >= seg_end;
            c.single = seg_single;
            c.slot = seg_slot;
            c.seg = seg_par;
        }
        seg_first = false;
        seg_t += rows;
        return true;
    };

    // -- the warp's own slots
    int issued = 0, used = 0, in_slot = 0, out_slot = 0, out_phase = 0;  // tiles started / finished; next slot of each
    bool dead = false;                                                   // a wait ran out: no more copies, no more waits
    Walk ahead;                                                          // the next tile to start, of chunk number ahead_no
    int ahead_no = 0, ahead_par = 0, ready_no = 0;                       // chunks up to ready_no are prepared
    ahead.left = 0;
    ahead.phase = 1;

    auto start_tile = [&](const Chunk& c, const Walk& w, int par) {
        const int row0 = w.j * G::TR, rows = min(G::TR, c.rows - row0);
        const Segment& sg = sm.seg[c.seg];
        const int plane = w.phase == 0 ? sg.id[w.p] : sg.head[w.p];
        const int planes = w.phase == 0 ? a.k : a.H;
        const uint32_t slot = smem_addr(sm.slot[warp][in_slot]), bar = smem_addr(&sm.full[warp][in_slot]);
        if (lane == 0) {
            const uint32_t bytes = rows * G::ROW + (G::FP8 ? ((rows + 3) & ~3) * 4 : 0);
            asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
        }
        __syncwarp();
        const int r0 = lane * c.run;
        if (r0 < rows) {
            const int n = min(c.run, rows - r0);
            const int2 at = sm.at[par][(row0 + r0) / kQuantum];
            const size_t stride = w.phase == 0 ? a.pool.k_page_stride : a.pool.v_page_stride;
            const size_t elem = (size_t)at.x * stride + ((size_t)plane * ps + at.y) * D;
            const char* src = static_cast<const char*>(w.phase == 0 ? a.k_pages : a.v_pages) + elem * sizeof(T);
            const uint32_t dst = slot + (G::FP8 ? (r0 / G::RUN) * G::RUN_STRIDE + (r0 % G::RUN) * G::ROW : r0 * G::ROW);
            copy_rows(dst, src, n * G::ROW, bar);
            if constexpr (G::FP8) {
                const float* scales = (w.phase == 0 ? a.k_scales : a.v_scales) + ((size_t)at.x * planes + plane) * ps + at.y;
                copy_rows(slot + G::DATA + r0 * 4, scales, ((n + 3) & ~3) * 4, bar);
            }
        }
        in_slot = in_slot + 1 == G::STAGES ? 0 : in_slot + 1;
        ++issued;
    };
    auto fill = [&]() {
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
            const Chunk& c = sm.chunk[ahead_par];
            start_tile(c, ahead, ahead_par);
            ahead.step(c.tiles);
        }
    };
    // Waits for the warp's next tile; false if the wait ran out, now or earlier.
    auto take = [&](uint32_t* tile) -> bool {
        if (dead) return false;
        if (!bar_wait(smem_addr(&sm.full[warp][out_slot]), out_phase, a.wait_limit)) dead = true;
        dead = __any_sync(0xffffffffu, dead);
        if (dead) {
            if (lane == 0) sm.err = CHAI_ERR_TIMEOUT;
            return false;
        }
        *tile = smem_addr(sm.slot[warp][out_slot]);
        return true;
    };
    auto release = [&]() {
        ++used;
        if (++out_slot == G::STAGES) {
            out_slot = 0;
            out_phase ^= 1;
        }
        __syncwarp();  // every lane has read the tile before a copy overwrites it
        fill();
    };

    // -- chunk by chunk
    int no = 0, par = 1;
    bool more = prepare(0);
    __syncthreads();
    if (more) ready_no = 1, ahead_par = 1;
    fill();
    while (more) {
        ++no;
        par ^= 1;
        const Chunk c = sm.chunk[par];
        const Segment& sg = sm.seg[c.seg];

        // K: scores of the warp's tiles, in powers of two
        {
            Walk w;
            w.start(0, c, warp);
            int have = -1;
            float factor = 1.f;
            constexpr int QN = G::FP8 ? 1 : 16 / (int)sizeof(T);
            float qf[QN];
            uint32_t qb[G::FP8 ? D / 8 : 1];  // e4m3: the fp16 fragments, column 0 the leading and column 1 the trailing half
            (void)qf;
            (void)qb;
            for (; w.left > 0; w.step(c.tiles)) {
                if (w.p != have) {
                    have = w.p;
                    const TQ* q = static_cast<const TQ*>(a.q) + ((size_t)c.b * a.H + sg.rep[w.p]) * D;
                    if constexpr (!G::FP8) {
                        Vec16<T>::unpack(*reinterpret_cast<const uint4*>(q + (lane % G::LPR) * QN), qf);
#pragma unroll
                        for (int e = 0; e < QN; ++e) qf[e] *= a.scale_log2;
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
                            const float u = x[2 * i] * f, v = x[2 * i + 1] * f;
                            const uint32_t hi = half_pair(u, v);
                            const float2 h = half_floats(hi);
                            const uint32_t lo = half_pair(u - h.x, v - h.y);
                            qb[i] = lane < 4 ? hi : (lane < 8 ? lo : 0u);
                        }
                    }
                }
                const int row0 = w.j * G::TR, rows = min(G::TR, c.rows - row0);
                uint32_t tile;
                if (!take(&tile)) break;
                float* score = sm.score + w.p * c.stride + row0;
                if constexpr (!G::FP8) {
                    // lanes of a group hold 16 bytes each of rows group * IT + i; a butterfly turns 16 partial sums a
                    // lane into whole sums, halving the rows a lane answers for at every step
                    const uint32_t base = tile + (lane / G::LPR) * G::IT * G::ROW + (lane % G::LPR) * 16;
                    float s[G::IT];
#pragma unroll
                    for (int i = 0; i < G::IT; ++i) {
                        float kf[QN];
                        Vec16<T>::unpack(lds16(base + i * G::ROW), kf);
                        s[i] = qf[0] * kf[0];
#pragma unroll
                        for (int e = 1; e < QN; ++e) s[i] = fmaf(qf[e], kf[e], s[i]);
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
                        if (row + i < rows && lane % SAME == 0) score[row + i] = s[i];
                } else {
                    // 16 keys are the rows of A, 16 columns of them a step; B holds the query (leading and trailing half)
                    const int g = lane >> 2, t = lane & 3;
                    const uint32_t scales = tile + G::DATA;
#pragma unroll
                    for (int m = 0; m < 4; ++m) {
                        if (16 * m < rows) {
                            const uint32_t base = tile + m * G::RUN_STRIDE + g * G::ROW + t * 16;
                            float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                            for (int j = 0; j < D / 64; ++j) {
                                const uint4 x = lds16(base + j * 64), y = lds16(base + j * 64 + 8 * G::ROW);
                                const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                                for (int i = 0; i < 4; ++i)
                                    mma16816(acc, e4m3_pair(xs[i] & 0xffffu), e4m3_pair(ys[i] & 0xffffu), e4m3_pair(xs[i] >> 16),
                                             e4m3_pair(ys[i] >> 16), qb[8 * j + 2 * i], qb[8 * j + 2 * i + 1]);
                            }
                            if (t == 0) {
                                const int r = 16 * m + g;
                                float ks;
                                if (r < rows) {
                                    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(ks) : "r"(scales + 4 * r));
                                    score[r] = (acc[0] + acc[1]) * (ks * factor);
                                }
                                if (r + 8 < rows) {
                                    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(ks) : "r"(scales + 4 * (r + 8)));
                                    score[r + 8] = (acc[2] + acc[3]) * (ks * factor);
                                }
                            }
                        }
                    }
                }
                release();
            }
        }
        __syncthreads();

        // S: running maximum and sum of every cluster, probabilities relative to the new maximum
        for (int cl = warp; cl < c.clusters; cl += kWarps) {
            float* score = sm.score + cl * c.stride;
            float top = -INFINITY, old = c.first ? -INFINITY : sm.top[cl], sum = 0.f;
            for (int r = lane; r < c.rows; r += 32) top = fmaxf(top, score[r]);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            top = fmaxf(top, old);
            const float ref = top == -INFINITY ? 0.f : top;  // scores of -inf leave their rows out
            for (int r = lane; r < c.rows; r += 32) {
                const float p = exp2_approx(score[r] - ref);
                score[r] = p;
                sum += p;
            }
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
        __syncthreads();
        if (more) ready_no = no + 1;
        fill();

        // V: sums of the warp's share
        float acc[G::VPL];
#pragma unroll
        for (int e = 0; e < G::VPL; ++e) acc[e] = 0.f;
        int open = -1;  // a head whose first rows are in acc and whose last rows another warp has
        // Writes the finished sums of a head.
        auto emit = [&](int p) {
            const int h = sg.head[p], cl = sg.cluster[p];
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
                    TQ* dst = static_cast<TQ*>(a.out) + ((size_t)c.b * a.H + h) * D + G::col(lane);
#pragma unroll
                    for (int e = 0; e < G::VPL; ++e) dst[e] = from_float<TQ>(bad_so_far ? 0.f : acc[e] / sum);
                } else {
#pragma unroll
                    for (int e = 0; e < G::VPL; e += 4)
                        *reinterpret_cast<float4*>(o + e) = make_float4(acc[e], acc[e + 1], acc[e + 2], acc[e + 3]);
                }
            }
            if (c.last && !c.single && lane == 0) a.ws.ml[(size_t)c.slot * a.H + h] = make_float2(sm.top[cl], sm.sum[cl]);
        };
        {
            Walk w;
            w.start(1, c, warp);
            bool from_start = w.j == 0;
            while (w.left > 0) {
                const int row0 = w.j * G::TR, rows = min(G::TR, c.rows - row0);
                uint32_t tile;
                if (!take(&tile)) break;
                const float* prob = sm.score + sg.cluster[w.p] * c.stride + row0;
                if constexpr (!G::FP8) {
                    const int first = (lane / G::LPR) * G::IT;
                    const uint32_t base = tile + first * G::ROW + (lane % G::LPR) * 16;
                    if (rows == G::TR) {
                        uint64_t sum[G::VPL / 2];
#pragma unroll
                        for (int e = 0; e < G::VPL / 2; ++e) sum[e] = pack2(acc[2 * e], acc[2 * e + 1]);
#pragma unroll
                        for (int i = 0; i < G::IT; i += 4) {
                            const float4 p4 = *reinterpret_cast<const float4*>(prob + first + i);
                            const float pr[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
                            for (int u = 0; u < 4; ++u) {
                                float vf[G::VPL];
                                Vec16<T>::unpack(lds16(base + (i + u) * G::ROW), vf);
                                const uint64_t pp = pack2(pr[u], pr[u]);
#pragma unroll
                                for (int e = 0; e < G::VPL / 2; ++e) sum[e] = fma2(pp, pack2(vf[2 * e], vf[2 * e + 1]), sum[e]);
                            }
                        }
#pragma unroll
                        for (int e = 0; e < G::VPL / 2; ++e) {
                            const float2 x = unpack2(sum[e]);
                            acc[2 * e] = x.x;
                            acc[2 * e + 1] = x.y;
                        }
                    } else {  // rows behind the last are not touched: they may hold anything
                        const int n = min(G::IT, rows - first);
                        for (int i = 0; i < n; ++i) {
                            float vf[G::VPL];
                            Vec16<T>::unpack(lds16(base + i * G::ROW), vf);
                            const float p = prob[first + i];
#pragma unroll
                            for (int e = 0; e < G::VPL; ++e) acc[e] = fmaf(p, vf[e], acc[e]);
                        }
                    }
                } else {
                    // 16 columns are the rows of A, 16 cache rows a step (four of each run); B holds the probabilities
                    // times the rows' scales, brought below 2 by a power of two and split into two fp16 numbers
                    const int g = lane >> 2, t = lane & 3;
                    const uint32_t scales = tile + G::DATA + 64 * t;
                    const bool whole = rows == G::TR;
                    float4 vs[4];
                    float top = 0.f, f, inv;
#pragma unroll
                    for (int s = 0; s < 4; ++s) {
                        const uint4 x = lds16(scales + 16 * s);
                        vs[s] = make_float4(__uint_as_float(x.x), __uint_as_float(x.y), __uint_as_float(x.z), __uint_as_float(x.w));
                        if (!whole) {
                            const int r = 16 * t + 4 * s;
                            vs[s].x = r < rows ? vs[s].x : 0.f;
                            vs[s].y = r + 1 < rows ? vs[s].y : 0.f;
                            vs[s].z = r + 2 < rows ? vs[s].z : 0.f;
                            vs[s].w = r + 3 < rows ? vs[s].w : 0.f;
                        }
                        top = fmaxf(top, fmaxf(fmaxf(fabsf(vs[s].x), fabsf(vs[s].y)), fmaxf(fabsf(vs[s].z), fabsf(vs[s].w))));
                    }
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                    normaliser(top, &f, &inv);
                    float part[D / 16][4];
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) part[i][0] = part[i][1] = part[i][2] = part[i][3] = 0.f;
#pragma unroll
                    for (int s = 0; s < 4; ++s) {
                        const int r = 16 * t + 4 * s;
                        float4 pr = make_float4(0.f, 0.f, 0.f, 0.f);
                        if (whole) {
                            pr = *reinterpret_cast<const float4*>(prob + r);
                        } else {
                            if (r < rows) pr.x = prob[r];
                            if (r + 1 < rows) pr.y = prob[r + 1];
                            if (r + 2 < rows) pr.z = prob[r + 2];
                            if (r + 3 < rows) pr.w = prob[r + 3];
                        }
                        const float x0 = pr.x * (vs[s].x * f), x1 = pr.y * (vs[s].y * f), x2 = pr.z * (vs[s].z * f), x3 = pr.w * (vs[s].w * f);
                        const uint32_t h0 = half_pair(x0, x1), h1 = half_pair(x2, x3);
                        const float2 y0 = half_floats(h0), y1 = half_floats(h1);
                        const uint32_t l0 = half_pair(x0 - y0.x, x1 - y0.y), l1 = half_pair(x2 - y1.x, x3 - y1.y);
                        const uint32_t b0 = g == 0 ? h0 : (g == 1 ? l0 : 0u), b1 = g == 0 ? h1 : (g == 1 ? l1 : 0u);
                        constexpr int WORDS = D / 32;  // 32-bit words a lane holds of a row
                        uint32_t v[4][WORDS];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t at = tile + t * G::RUN_STRIDE + (4 * s + i) * G::ROW + g * (4 * WORDS);
                            const bool there = whole || r + i < rows;
                            if constexpr (WORDS == 4) {
                                const uint4 x = there ? lds16(at) : make_uint4(0, 0, 0, 0);
                                v[i][0] = x.x; v[i][1] = x.y; v[i][2] = x.z; v[i][3] = x.w;
                            } else {
                                const uint2 x = there ? lds8(at) : make_uint2(0, 0);
                                v[i][0] = x.x; v[i][1] = x.y;
                            }
                        }
#pragma unroll
                        for (int wd = 0; wd < WORDS; ++wd) {
                            // columns 4 wd .. + 3 of two rows each, side by side
                            const uint32_t lo0 = __byte_perm(v[0][wd], v[1][wd], 0x5140), hi0 = __byte_perm(v[0][wd], v[1][wd], 0x7362);
                            const uint32_t lo1 = __byte_perm(v[2][wd], v[3][wd], 0x5140), hi1 = __byte_perm(v[2][wd], v[3][wd], 0x7362);
                            mma16816(part[2 * wd], e4m3_pair(lo0 & 0xffffu), e4m3_pair(lo0 >> 16), e4m3_pair(lo1 & 0xffffu),
                                     e4m3_pair(lo1 >> 16), b0, b1);
                            mma16816(part[2 * wd + 1], e4m3_pair(hi0 & 0xffffu), e4m3_pair(hi0 >> 16), e4m3_pair(hi1 & 0xffffu),
                                     e4m3_pair(hi1 >> 16), b0, b1);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) {
                        acc[2 * i] = fmaf(part[i][0] + part[i][1], inv, acc[2 * i]);
                        acc[2 * i + 1] = fmaf(part[i][2] + part[i][3], inv, acc[2 * i + 1]);
                    }
                }
                release();
                const int p = w.p;
                const bool ends = w.j + 1 == c.tiles;
                w.step(c.tiles);
                if (!ends && w.left > 0) continue;
                if constexpr (!G::FP8) {
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
                    break;
                }
#pragma unroll
                for (int e = 0; e < G::VPL; ++e) acc[e] = 0.f;
                from_start = true;
            }
        }
        __syncthreads();
        if (open >= 0) {
            const int n = c.heads * c.tiles, stop = (open + 1) * c.tiles;
            for (int w = warp + 1; w < kWarps; ++w) {
                const int lo = n * w / kWarps;
                if (lo >= stop) break;
                if (lo == n * (w + 1) / kWarps) continue;  // a warp without tiles
                if (G::own(lane))
#pragma unroll
                    for (int e = 0; e < G::VPL; ++e) acc[e] += sm.part[w][G::col(lane) + e];
            }
            emit(open);
        }
        if (c.last && tid == 0) {
            if (!c.single && group == 0) a.ws.slot_bad[c.slot] = bad_so_far;
            if (bad_so_far && atomicCAS(&sm.err, CHAI_OK, CHAI_ERR_BAD_PAGE) == CHAI_OK) sm.err_b = c.b;
        }
    }
    if (dead)  // copies in flight end before the shared memory goes
        for (int i = used; i < issued; ++i) {
            bar_wait(smem_addr(&sm.full[warp][out_slot]), out_phase, kDefaultWaitLimitCycles);
            if (++out_slot == G::STAGES) {
                out_slot = 0;
                out_phase ^= 1;
            }
        }
    if (!by_request && group == 0 && piece < pieces && !opened_span && tid == 0) a.ws.desc[piece] = make_int4(-1, 0, 0, 0);
    __syncthreads();
    if (tid == 0) {
        a.ws.err[blockIdx.x] = sm.err;
        a.ws.err_b[blockIdx.x] = sm.err_b;
    }
}

// ---- joining the pieces of a request ----------------------------------------------------------------------------

// grid (H, descriptions): out[b][h] from the partial results of consecutive pieces.
template <typename TQ, int D>
__global__ void __launch_bounds__(kJoinThreads) paged_join_kernel(const DecodeArgs a, int n_ctas) {
    constexpr int WARPS = kJoinThreads / 32, E = D / 32;
    __shared__ float s_w[kMaxCtas], s_top[WARPS], s_sum[WARPS], s_o[WARPS][D];
    dependent_grid_sync();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, h = blockIdx.x;
    if (blockIdx.x == 0 && blockIdx.y == 0 && warp == 0) {  // the call's status
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
    const int4 d = a.ws.desc[blockIdx.y];
    if (d.x < 0) return;
    const int b = d.x, first = d.y, n = d.z;
    float2 ml = make_float2(-INFINITY, 0.f);
    bool bad = false;
    if (tid < n) {
        ml = a.ws.ml[(size_t)(first + tid) * a.H + h];
        bad = a.ws.slot_bad[first + tid] != 0;
    }
    if (__syncthreads_or(tid == 0 && ml.y == -1.f)) return;  // an unknown head: zeros are written already
    float top = ml.x;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (lane == 0) s_top[warp] = top;
    const bool zero = __syncthreads_or(bad);
    for (int w = 0; w < WARPS; ++w) top = fmaxf(top, s_top[w]);
    const float ref = top == -INFINITY ? 0.f : top;
    const float weight = tid < n ? exp2_approx(ml.x - ref) : 0.f;
    if (tid < n) s_w[tid] = weight;
    float sum = tid < n ? weight * ml.y : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) s_sum[warp] = sum;
    __syncthreads();
    float o[E];
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.f;
    const float* src = a.ws.o + ((size_t)first * a.H + h) * D + lane * E;
    const size_t apart = (size_t)a.H * D;
#pragma unroll 8
    for (int i = warp; i < n; i += WARPS) {
        const float w = s_w[i];
        if constexpr (E == 4) {
            const float4 x = *reinterpret_cast<const float4*>(src + i * apart);
            o[0] = fmaf(w, x.x, o[0]);
            o[1] = fmaf(w, x.y, o[1]);
            o[2] = fmaf(w, x.z, o[2]);
            o[3] = fmaf(w, x.w, o[3]);
        } else {
            const float2 x = *reinterpret_cast<const float2*>(src + i * apart);
            o[0] = fmaf(w, x.x, o[0]);
            o[1] = fmaf(w, x.y, o[1]);
        }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) s_o[warp][lane * E + e] = o[e];
    __syncthreads();
    if (tid < D) {
        float l = 0.f, x = 0.f;
        for (int w = 0; w < WARPS; ++w) {
            l += s_sum[w];
            x += s_o[w][tid];
        }
        static_cast<TQ*>(a.out)[((size_t)b * a.H + h) * D + tid] = from_float<TQ>(zero ? 0.f : x / l);
    }
}

// ---- host -------------------------------------------------------------------------------------------------------

template <typename T, typename TQ, int D>
int launch_decode(const DecodeArgs& args, cudaStream_t s) {
    using G = Geom<T, D>;
    constexpr size_t smem = sizeof(Smem<G::SLOT, G::STAGES, D>);
    static_assert(smem <= 227 * 1024, "one CTA's shared memory");
    static_assert(G::DATA % 16 == 0 && G::SLOT % 16 == 0 && (G::FP8 || G::IT == 16), "tile geometry");
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
    CHAI_LAUNCH_DEPENDENT("paged_decode_kernel launch", (paged_decode_kernel<T, TQ, D>), dim3(n_ctas), dim3(kThreads), smem, s, a);
    CHAI_LAUNCH_DEPENDENT("paged_join_kernel launch", (paged_join_kernel<TQ, D>), dim3(a.H, a.n_desc), dim3(kJoinThreads), 0, s,
                          a, n_ctas);
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
    CHAI_REQUIRE((long long)B * a.pool.capacity < (1ll << 34), CHAI_ERR_UNSUPPORTED,
                 "%s: B * max_pages * page_size must be below 2^34", fn);
    const size_t need = chai_decode_paged_workspace_bytes(B, H, D);
    CHAI_REQUIRE(workspace_bytes >= need, CHAI_ERR_WORKSPACE, "%s: workspace has %zu bytes, %zu needed", fn, workspace_bytes,
                 need);
    decode_ws(static_cast<char*>(workspace), B, H, D, &a.ws);
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
