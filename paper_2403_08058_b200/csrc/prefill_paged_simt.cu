// Clustered attention of packed tokens over a paged cache on the CUDA cores: 32-bit queries and outputs, caches of fp32 or
// e4m3 rows.  (bf16 runs on the tensor cores, prefill_paged.cu.)
//
// One pass over the keys with a running maximum m and sum l per row; S = scale Q K^T, P = exp(S - m), O = O exp(m_old - m) + P V
// for up to 256 / D members of a cluster, whose probabilities are the same.  All in fp32.
// Many rows are bound by the FMA pipe (two products an instruction, fma.rn.f32x2), few by the copies and what stands in a row
// for a tile: keys there, S, the rows' maximum and sum, values there, O.  So two blocks of 256 threads stand on an SM, one busy
// while the other waits.  A block takes 16 RPT query rows and 32 or 64 keys, a thread RPT rows x 2 or 4 keys of S and RPT rows
// x 16 columns (of all members together, per member D / 16) of O.  RPT = 1, 2 or 4 by the tokens per request, since rows that a
// request does not have are computed all the same.  Every member has a buffer of its own: keys and values of the next tile are
// copied as soon as this tile's are done with, and where the rows lie is looked up a tile ahead.
// Measured (fp32): 5 requests of up to 93 rows over up to 700 positions, 12 heads of 64: 50 us (one block of 128 rows an SM, the
// pieces joined a vector at a time: 118); of 2 rows over up to 4096, 32 heads of 128: 180 us, 1.1 TB/s; of up to 400 rows over
// 2048: 857 us.
#include "prefill_paged.cuh"
#include "tc_ptx.cuh"

namespace chai {
namespace {

using tcx::fma2;
using tcx::pack2;
using tcx::unpack2;

constexpr int kThreads = 256;
// Keys of a tile: what lets two blocks stand on an SM.
constexpr int keys_of(int D, int rpt) { return rpt > 2 || (D == 128 && rpt > 1) ? 32 : 64; }

template <int D, int RPT>
struct Smem {
    static_assert(16 * RPT * kPagedMaxPieces <= 16 * RPT * (D + 4), "the joined pieces' shares fit where the queries were");
    static constexpr int BQ = 16 * RPT, BK = keys_of(D, RPT), STRIDE = D + 4, PSTRIDE = BK + 4;
    static constexpr int Q = 0, K = Q + BQ * STRIDE, V = K + BK * STRIDE, P = V + 256 / D * BK * STRIDE, M = P + BQ * PSTRIDE,
                         L = M + BQ, C = L + BQ, ROWS = C + BQ, FLOATS = ROWS + 2 * 2 * BK;
    static constexpr int BYTES = FLOATS * 4 + 16;
    static_assert(2 * (BYTES + 1024) <= 228 * 1024, "two blocks to an SM");
};

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
    const int bytes = there ? 16 : 0;  // 0: the destination is zeroed
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

// Where a key tile's rows are: (page, row in the page), page -1 where there is none.
template <int BK>
__device__ __forceinline__ void find_rows(const PagedCall& a, int b, int pos0, int kv, int2* rows) {
    const int r = threadIdx.x;
    if (r >= BK) return;
    const int pos = pos0 + r;
    int page = -1, row = 0;
    if (pos < kv) {
        const int pi = (int)a.pool.by_page.div((unsigned)pos);
        row = pos - pi * a.pool.page_size;
        page = a.pool.block_table[(size_t)b * a.pool.max_pages + pi];
        if (page < 0 || page >= a.pool.n_pages) page = -1;  // (the planner has looked; another stream may write the table)
    }
    rows[r] = make_int2(page, row);
}
// The rows of plane `plane` of the keys or values; those of no page are zero.
template <typename TC, int D, int BK>
__device__ __forceinline__ void load_tile(const PagedCall& a, bool key, int plane, const int2* rows, float* dst) {
    constexpr int STRIDE = D + 4;
    const size_t stride = key ? a.pool.k_page_stride : a.pool.v_page_stride;
    const char* pages = static_cast<const char*>(key ? a.k_pages : a.v_pages);
    constexpr int VPR = D * (int)sizeof(TC) / 16, EPV = 16 / (int)sizeof(TC);  // 16-byte vectors of a cached row
#pragma unroll
    for (int i = threadIdx.x; i < BK * VPR; i += kThreads) {
        const int r = i / VPR, x = i % VPR;
        const int2 where = rows[r];
        const size_t at = where.x < 0 ? 0 : (size_t)where.x * stride + ((size_t)plane * a.pool.page_size + where.y) * D + x * EPV;
        float* to = dst + r * STRIDE + x * EPV;
        if constexpr (sizeof(TC) == 4) {
            copy16(tcx::smem_u32(to), pages + at * 4, where.x >= 0);
        } else {
            float f[16];
            uint4 raw = make_uint4(0, 0, 0, 0);
            float s = 0.f;
            if (where.x >= 0) {
                raw = __ldcs(reinterpret_cast<const uint4*>(pages + at));
                s = __ldg((key ? a.k_scales : a.v_scales) + ((size_t)where.x * (key ? a.k : a.H) + plane) * a.pool.page_size + where.y);
            }
            Vec16<Fp8E4M3>::unpack(raw, f);
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *reinterpret_cast<float4*>(to + e) = make_float4(f[e] * s, f[e + 1] * s, f[e + 2] * s, f[e + 3] * s);
        }
    }
}

template <typename TC, int D, int RPT>
__global__ void __launch_bounds__(kThreads, 2) prefill_paged_simt_kernel(const __grid_constant__ PagedCall a) {
    using S = Smem<D, RPT>;
    constexpr int BQ = S::BQ, BK = S::BK, STRIDE = S::STRIDE, PSTRIDE = S::PSTRIDE, GM = 256 / D, CPT = D / 16, KPT = BK / 16;
    extern __shared__ __align__(16) float smem[];
    float *Qs = smem + S::Q, *Ks = smem + S::K, *Vs = smem + S::V, *Ps = smem + S::P, *Ms = smem + S::M, *Ls = smem + S::L, *Cs = smem + S::C;
    int2* s_rows = reinterpret_cast<int2*>(smem + S::ROWS);  // of an even and an odd tile
    int* s_id = reinterpret_cast<int*>(smem + S::FLOATS);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rg = (warp & 3) * 4 + (lane >> 3), cg = (warp >> 2) * 8 + (lane & 7);  // rows i * 16 + rg, keys j * 16 + cg
    dependent_grid_sync();
    PagedWalk walk;
    walk.begin(a, lane);  // (every warp does)
    PagedItem it;
    PagedGroup e;
    while (walk.next(a, it, e)) {
        __syncthreads();  // (the shared arrays are still read by the item before)
        const int members = min(e.n, GM);
        float* out = static_cast<float*>(a.out);
        if (it.count == 0) {
            for (int i = tid; i < it.rows * D * members; i += kThreads) {
                const int g = i / (it.rows * D), r = i / D % it.rows;
                int h = e.heads[0];
#pragma unroll
                for (int x = 1; x < GM; ++x)
                    if (g == x) h = e.heads[x];
                out[((size_t)(it.q0 + r) * a.H + h) * D + i % D] = 0.f;
            }
            continue;
        }
        // row t of the request sees positions below kv - n + t + 1 (causal)
        auto sees = [&](int r) { return a.causal ? min(it.kv, it.kv - it.n + it.t0 + r + 1) : it.kv; };
        auto pos0 = [&](int j) { return (it.first + j < it.tiles ? it.first + j : it.first + j - it.tiles) * BK; };
        const float* q = static_cast<const float*>(a.q) + (long long)it.q0 * a.q_stride + (long long)e.rep * D;
        for (int i = tid; i < BQ * (D / 4); i += kThreads) {
            const int r = i / (D / 4), x = i % (D / 4);
            copy16(tcx::smem_u32(Qs + r * STRIDE + x * 4), q + (r < it.rows ? (long long)r * a.q_stride + x * 4 : 0), r < it.rows);
        }
        if (tid < BQ) Ms[tid] = -INFINITY, Ls[tid] = 0.f;
        auto commit = [] { asm volatile("cp.async.commit_group;" ::: "memory"); };
        auto find = [&](int j) {
            if (j < it.count) find_rows<BK>(a, it.b, pos0(j), it.kv, s_rows + (j & 1) * BK);
        };
        auto load_k = [&](int j) {
            if (j < it.count) load_tile<TC, D, BK>(a, true, e.cluster, s_rows + (j & 1) * BK, Ks);
            commit();
        };
        auto load_v = [&](int j, int g) {  // (a buffer a member)
            if (j < it.count && g < members) {
                int h = e.heads[0];
#pragma unroll
                for (int x = 1; x < GM; ++x)
                    if (g == x) h = e.heads[x];
                load_tile<TC, D, BK>(a, false, h, s_rows + (j & 1) * BK, Vs + g * BK * STRIDE);
            }
            commit();
        };
        find(0);
        __syncthreads();
        load_k(0);  // (with the queries)
#pragma unroll
        for (int g = 0; g < GM - 1; ++g) load_v(0, g);
        float acc[GM][RPT][CPT];
#pragma unroll
        for (int g = 0; g < GM; ++g)
#pragma unroll
            for (int i = 0; i < RPT; ++i)
#pragma unroll
                for (int c = 0; c < CPT; ++c) acc[g][i][c] = 0.f;

        for (int j = 0; j < it.count; ++j) {
            // in order: keys of j, values of j but the last member's | those, keys of j + 1, values of j + 1 ...
            asm volatile("cp.async.wait_group %0;" ::"n"(GM - 1) : "memory");
            __syncthreads();
            load_v(j, GM - 1);
            find(j + 1);
            {
                uint64_t s2[RPT][KPT];  // sums over even and over odd columns
#pragma unroll
                for (int i = 0; i < RPT; ++i)
#pragma unroll
                    for (int c = 0; c < KPT; ++c) s2[i][c] = 0ull;
#pragma unroll 2
                for (int d = 0; d < D; d += 4) {
                    ulonglong2 kk[KPT];
#pragma unroll
                    for (int c = 0; c < KPT; ++c) kk[c] = *reinterpret_cast<const ulonglong2*>(Ks + (c * 16 + cg) * STRIDE + d);
#pragma unroll
                    for (int i = 0; i < RPT; ++i) {
                        const ulonglong2 qq = *reinterpret_cast<const ulonglong2*>(Qs + (i * 16 + rg) * STRIDE + d);
#pragma unroll
                        for (int c = 0; c < KPT; ++c) s2[i][c] = fma2(qq.y, kk[c].y, fma2(qq.x, kk[c].x, s2[i][c]));
                    }
                }
                const int col0 = pos0(j);
#pragma unroll
                for (int i = 0; i < RPT; ++i) {
                    const int r = i * 16 + rg, end = sees(r);
#pragma unroll
                    for (int c = 0; c < KPT; ++c) {
                        float x, y;
                        unpack2(s2[i][c], x, y);
                        Ps[r * PSTRIDE + c * 16 + cg] = col0 + c * 16 + cg < end ? (x + y) * a.scale : -INFINITY;
                    }
                }
            }
            __syncthreads();
            load_k(j + 1);
            {  // rows: maximum, probabilities, sum; kThreads / BQ threads a row
                constexpr int TPR = kThreads / BQ, N = BK / TPR;
                const int r = tid / TPR, part = tid % TPR;
                float* row = Ps + r * PSTRIDE + part;
                float mx = -INFINITY;
#pragma unroll
                for (int c = 0; c < N; ++c) mx = fmaxf(mx, row[c * TPR]);
#pragma unroll
                for (int o = TPR / 2; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
                const float m_old = Ms[r], m_new = fmaxf(m_old, mx), ref = m_new == -INFINITY ? 0.f : m_new;
                float sum = 0.f;
#pragma unroll
                for (int c = 0; c < N; ++c) {
                    const float p = expf(row[c * TPR] - ref);
                    row[c * TPR] = p;
                    sum += p;
                }
#pragma unroll
                for (int o = TPR / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                __syncwarp();
                if (part == 0) {
                    const float corr = expf(m_old - ref);  // (nothing so far: 0)
                    Ms[r] = m_new;
                    Ls[r] = Ls[r] * corr + sum;
                    Cs[r] = corr;
                }
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < RPT; ++i) {
                const float c = Cs[i * 16 + rg];
#pragma unroll
                for (int g = 0; g < GM; ++g)
#pragma unroll
                    for (int x = 0; x < CPT; ++x) acc[g][i][x] *= c;
            }
#pragma unroll
            for (int g = 0; g < GM; ++g) {
                if (g == 0) asm volatile("cp.async.wait_group %0;" ::"n"(GM) : "memory");
                else asm volatile("cp.async.wait_group %0;" ::"n"(GM - 1) : "memory");
                if (g <= members) __syncthreads();
                if (g > 0) load_v(j + 1, g - 1);  // (the member before is done with its buffer)
                if (g >= members) continue;
                const float* v = Vs + g * BK * STRIDE;
#pragma unroll 1
                for (int t = 0; t < BK; t += 4) {
                    float4 p[RPT];
#pragma unroll
                    for (int i = 0; i < RPT; ++i) p[i] = *reinterpret_cast<const float4*>(Ps + (i * 16 + rg) * PSTRIDE + t);
#pragma unroll
                    for (int tt = 0; tt < 4; ++tt) {
#pragma unroll
                        for (int x = 0; x < CPT; x += 4) {
                            const ulonglong2 vv = *reinterpret_cast<const ulonglong2*>(v + (t + tt) * STRIDE + x * 16 + cg * 4);
#pragma unroll
                            for (int i = 0; i < RPT; ++i) {
                                const float pi = tt == 0 ? p[i].x : tt == 1 ? p[i].y : tt == 2 ? p[i].z : p[i].w;
                                const uint64_t pp = pack2(pi, pi);
                                float* o = &acc[g][i][x];
                                unpack2(fma2(pp, vv.x, pack2(o[0], o[1])), o[0], o[1]);
                                unpack2(fma2(pp, vv.y, pack2(o[2], o[3])), o[2], o[3]);
                            }
                        }
                    }
                }
            }
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();
        // O[row][x * 16 + cg * 4 ..] of each member
        if (it.pieces == 1) {
#pragma unroll
            for (int i = 0; i < RPT; ++i) {
                const int r = i * 16 + rg;
                if (r >= it.rows) continue;
                const float l = Ls[r], inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
                for (int g = 0; g < GM; ++g) {
                    if (g >= members) break;
                    float* o = out + ((size_t)(it.q0 + r) * a.H + e.heads[g]) * D;
#pragma unroll
                    for (int x = 0; x < CPT; x += 4)
                        *reinterpret_cast<float4*>(o + x * 16 + cg * 4) =
                            make_float4(acc[g][i][x] * inv, acc[g][i][x + 1] * inv, acc[g][i][x + 2] * inv, acc[g][i][x + 3] * inv);
                }
            }
            continue;
        }
        // A piece: [member][row][D], then (reference, sum) of every row.
        const size_t slot_bytes = (size_t)a.slot_rows * kSlotRowBytes;
        auto slot = [&](int piece) { return a.slots + (size_t)piece_slot(it.owner, piece) * slot_bytes; };
        const size_t stats = (size_t)a.slot_rows * 1024;
        {
            float* o = reinterpret_cast<float*>(slot(it.piece));
#pragma unroll
            for (int i = 0; i < RPT; ++i) {
                const int r = i * 16 + rg;
                if (r >= it.rows) continue;
#pragma unroll
                for (int g = 0; g < GM; ++g) {
                    if (g >= members) break;
#pragma unroll
                    for (int x = 0; x < CPT; x += 4)
                        *reinterpret_cast<float4*>(o + ((size_t)g * a.slot_rows + r) * D + x * 16 + cg * 4) =
                            make_float4(acc[g][i][x], acc[g][i][x + 1], acc[g][i][x + 2], acc[g][i][x + 3]);
                }
            }
            if (tid < it.rows && tid < BQ)
                reinterpret_cast<float2*>(slot(it.piece) + stats)[tid] = make_float2(Ms[tid], Ls[tid]);
        }
        __threadfence();
        __syncthreads();
        if (tid == 0) {
            *s_id = atomicAdd(&a.done[it.owner], 1);
            __threadfence();
        }
        __syncthreads();
        if (*s_id != it.pieces - 1) continue;
        // The last one joins them, in order of the pieces: first every piece's share of every row, then four vectors at a time, whose
        // loads are on their way together.
        float* share = smem + S::Q;  // [row][piece]
        for (int r = tid; r < it.rows; r += kThreads) {
            float m = -INFINITY, l = 0.f;
            for (int p = 0; p < it.pieces; ++p) {
                const float2 ml = __ldcg(reinterpret_cast<const float2*>(slot(p) + stats) + r);
                share[r * kPagedMaxPieces + p] = ml.y == 0.f ? -INFINITY : ml.x;  // (nothing that the row may see)
                if (ml.y != 0.f) m = fmaxf(m, ml.x);
            }
            const float ref = m == -INFINITY ? 0.f : m;
            for (int p = 0; p < it.pieces; ++p) {
                const float w = expf(share[r * kPagedMaxPieces + p] - ref);
                share[r * kPagedMaxPieces + p] = w;
                l += w * __ldcg(reinterpret_cast<const float2*>(slot(p) + stats) + r).y;
            }
            const float inv = l == 0.f ? 0.f : 1.f / l;
            for (int p = 0; p < it.pieces; ++p) share[r * kPagedMaxPieces + p] *= inv;
        }
        __syncthreads();
        const int vectors = it.rows * members * (D / 4);
        constexpr int U = 4;
        for (int i0 = tid; i0 < vectors; i0 += U * kThreads) {
            size_t at[U];
            int row[U], to[U];
            float4 o[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = min(i0 + u * kThreads, vectors - 1), x = i % (D / 4), r = i / (D / 4) % it.rows, g = i / (D / 4) / it.rows;
                int h = e.heads[0];
#pragma unroll
                for (int y = 1; y < GM; ++y)
                    if (g == y) h = e.heads[y];
                at[u] = (((size_t)g * a.slot_rows + r) * D + x * 4) * 4;
                row[u] = r * kPagedMaxPieces;
                to[u] = h * D + x * 4;
                o[u] = make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll 4
            for (int p = 0; p < it.pieces; ++p) {
                const char* from = slot(p);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const float w = share[row[u] + p];
                    const float4 v = __ldcg(reinterpret_cast<const float4*>(from + at[u]));
                    if (w != 0.f) {
                        o[u].x += w * v.x;
                        o[u].y += w * v.y;
                        o[u].z += w * v.z;
                        o[u].w += w * v.w;
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i0 + u * kThreads < vectors)
                    *reinterpret_cast<float4*>(out + ((size_t)it.q0 + row[u] / kPagedMaxPieces) * a.H * D + to[u]) = o[u];
        }
    }
}

template <typename TC, int D, int RPT>
int launch(const PagedCall& a, cudaStream_t s) {
    using S = Smem<D, RPT>;
    static PerDeviceOnce once;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return cuda_fail(e, "prefill_paged_simt_kernel set-up");
    const int rc = once.run(dev, [&]() -> int {
        const cudaError_t f = cudaFuncSetAttribute(prefill_paged_simt_kernel<TC, D, RPT>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::BYTES);
        return f == cudaSuccess ? CHAI_OK : cuda_fail(f, "prefill_paged_simt_kernel set-up");
    });
    if (rc != CHAI_OK) return rc;
    CHAI_LAUNCH_DEPENDENT("prefill_paged_simt_kernel launch", (prefill_paged_simt_kernel<TC, D, RPT>), dim3(a.ctas), dim3(kThreads),
                          S::BYTES, s, a);
    return CHAI_OK;
}

}  // namespace

// Rows and keys of a tile: requests of few tokens take fewer rows.
void prefill_paged_simt_tile(int B, int n_tokens, int D, int* rows, int* keys) {
    const long long per = ((long long)n_tokens + B - 1) / B;
    const int rpt = per <= 16 ? 1 : per <= 48 ? 2 : 4;
    *rows = 16 * rpt;
    *keys = keys_of(D, rpt);
}

int prefill_paged_simt(const PagedCall& a, int D, bool fp8, cudaStream_t s) {
    if (D == 128) {
        if (a.bq == 16) return fp8 ? launch<Fp8E4M3, 128, 1>(a, s) : launch<float, 128, 1>(a, s);
        if (a.bq == 32) return fp8 ? launch<Fp8E4M3, 128, 2>(a, s) : launch<float, 128, 2>(a, s);
        return fp8 ? launch<Fp8E4M3, 128, 4>(a, s) : launch<float, 128, 4>(a, s);
    }
    if (a.bq == 16) return fp8 ? launch<Fp8E4M3, 64, 1>(a, s) : launch<float, 64, 1>(a, s);
    if (a.bq == 32) return fp8 ? launch<Fp8E4M3, 64, 2>(a, s) : launch<float, 64, 2>(a, s);
    return fp8 ? launch<Fp8E4M3, 64, 4>(a, s) : launch<float, 64, 4>(a, s);
}

}  // namespace chai
