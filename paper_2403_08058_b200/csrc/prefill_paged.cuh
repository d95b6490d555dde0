// Work division of clustered attention of packed tokens over a paged cache, shared by its kernels.
//
// The work is one line: requests, their member groups, the groups' query tiles, the key tiles of each.  Every key tile counts 1
// and every (group, query tile) kPagedItemCost more.  The line is cut into equal shares, one per CTA, wherever the cuts fall:
// neither ragged lengths nor uneven clusters nor a batch with few tiles unbalance it.  A planning kernel (a block a request,
// since the host knows no lengths) builds the member groups, looks the pages over and counts a request's tiles; one warp of
// each CTA then finds its share.  What lies on both sides of a cut leaves unnormalised partial results, at most two a
// CTA, which whoever finishes last joins in order: results follow from the lengths and memberships alone.
// (Tiles of one member and of two count alike: the softmax, which they share, takes most of a tile's time, and where
// copies do, a CTA that is done early leaves its bandwidth to the others.)
// CTAs that walk the same keys for different query tiles should meet them at the same time, while they are in L2: a CTA
// that has done t tiles begins a whole query tile at key tile t modulo its count and wraps around, and of a divided one the
// share that begins it, late in that CTA's time, takes the last key tiles.
// All of this stands in front of the first tile, mostly as code that runs once and has to be fetched: it is kept short (a share is
// found by one warp, without block-wide barriers, in 32-bit distances from its beginning).
#pragma once

#include "paged.cuh"

namespace chai {

// Up to 256 / head_dim heads of one cluster.
struct PagedGroup {
    int cluster;  // -1: heads of no usable cluster
    int rep;      // representative head
    int n;
    int pad;
    int heads[4];
};
static_assert(sizeof(PagedGroup) == 32, "PagedGroup is 32 bytes");

struct PagedRequest {
    int start, n, kv;      // first row, rows, cached positions (0 where a page is bad)
    int n_groups;
    int cost;              // of a group: its key tiles over all query tiles, and kPagedItemCost for each query tile
    int longest;           // key tiles of the last query tile
    int code;              // chai_status_t
    int pad;
};
static_assert(sizeof(PagedRequest) == 32, "PagedRequest is 32 bytes");

constexpr int kPagedItemCost = 1;
constexpr int kSlotRowBytes = 256 * 4 + 8;     // members x head_dim = 256 numbers and (reference, sum), per row
static_assert(2 * kSlotRowBytes % 16 == 0, "slots have an even number of rows");
constexpr size_t kSlotBytesPerToken = 640000;  // see chai_prefill_paged_workspace_bytes
constexpr int kPagedMaxCtas = 300;             // (two partial results each)
static_assert(2 * kPagedMaxCtas * kSlotRowBytes <= kSlotBytesPerToken, "partial results fit");
constexpr int kPagedMaxPieces = 32;
constexpr int kPagedJoinBytes = 64;            // what a CTA has to know of a query tile whose pieces it joins

struct PagedLayout {
    size_t off_done, off_joins, off_req, off_groups, off_slots, total;
};
inline PagedLayout paged_layout(int B, int H, int n_tokens) {
    PagedLayout L;
    L.off_done = sizeof(WsHeader);
    L.off_joins = round_up(L.off_done + sizeof(int) * kPagedMaxCtas, 256);
    L.off_req = round_up(L.off_joins + 2 * kPagedJoinBytes * (size_t)kPagedMaxCtas, 256);
    L.off_groups = round_up(L.off_req + sizeof(PagedRequest) * (size_t)B, 256);
    L.off_slots = round_up(L.off_groups + sizeof(PagedGroup) * (size_t)B * H, 256);
    L.total = L.off_slots + 2 * (size_t)kPagedMaxCtas * kSlotRowBytes * ((n_tokens < 128 ? n_tokens + 1 : 128) & ~1);
    return L;
}

// One call, as the planner and the attention kernels see it.
struct PagedCall {
    const void *q, *k_pages, *v_pages;
    const float *k_scales, *v_scales;
    const int32_t *membership, *reps, *kv_lens, *token_start;
    void* out;
    PagePool pool;
    WsHeader* hdr;
    int* done;              // [ctas] pieces that are finished of the query tile that a CTA's share ends in
    char* joins;            // [ctas][2] query tiles whose last piece the CTA finished (tensor cores)
    PagedRequest* req;
    PagedGroup* groups;
    char* slots;            // [2 ctas] partial results
    long long q_stride;
    float scale;
    int B, H, k, n_tokens, causal;
    int gmax, bq, bk;       // members per group, rows and keys per tile
    int slot_rows;
    int ctas;               // that share the work
};

// Key tiles that query tile qt needs.
__device__ __forceinline__ int key_tiles(const PagedCall& a, int n, int kv, int qt) {
    const int end = a.causal ? max(min(kv, kv - n + min(n, (qt + 1) * a.bq)), 0) : kv;
    return (end + a.bk - 1) / a.bk;
}

// Shared memory of the planner: membership, and of every cluster and the heads of none the representative, members, first group and
// member mask.
inline size_t prefill_paged_plan_smem(int H, int k) { return sizeof(int) * ((size_t)H + ((size_t)k + 1) * (3 + (H + 31) / 32)); }

// Grid B.  A head a thread, but for the clusters' sums, which the first warp makes while the others look the pages over.
// (One warp for all of it took 3 us for 32 heads, 10 for 72.)
constexpr int kPagedPlanThreads = 256;
static __global__ void __launch_bounds__(kPagedPlanThreads) prefill_paged_plan_kernel(const PagedCall a) {
    extern __shared__ __align__(16) int s_plan[];
    __shared__ int s_in[3];
    dependent_grid_sync();
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, H = a.H, k = a.k, W = (H + 31) >> 5;
    int* mem = s_plan;
    int* rep = mem + H;           // (k: the heads of no usable cluster)
    int* members = rep + k + 1;
    int* slot = members + k + 1;
    unsigned* mask = reinterpret_cast<unsigned*>(slot + k + 1);
    int x = 0;
    if (tid < 3) x = tid == 2 ? a.kv_lens[b] : a.token_start[b + tid];
    for (int h = tid; h < H; h += kPagedPlanThreads) mem[h] = a.membership[(size_t)b * H + h];
    for (int c = tid; c <= k; c += kPagedPlanThreads) rep[c] = c < k ? a.reps[(size_t)b * k + c] : -1;
    for (int i = tid; i < (k + 1) * W; i += kPagedPlanThreads) mask[i] = 0u;
    if (b == 0)
        for (int i = tid; i < a.ctas; i += kPagedPlanThreads) a.done[i] = 0;
    if (tid < 3) s_in[tid] = min(max(x, 0), tid == 2 ? a.pool.capacity : a.n_tokens);
    __syncthreads();
    const int start = s_in[0], n = max(s_in[1] - start, 0);
    int kv = s_in[2], n_groups = 0;
    bool bad_page = false;
    if (n > 0) {
        // a cluster is usable if its representative is one of its heads
        auto row_of = [&](int h) {
            const int c = mem[h];
            if (c < 0 || c >= k) return k;
            const int r = rep[c];
            return r >= 0 && r < H && mem[r] == c ? c : k;
        };
        for (int h = tid; h < H; h += kPagedPlanThreads) atomicOr(&mask[row_of(h) * W + (h >> 5)], 1u << (h & 31));
        __syncthreads();
        if (tid < 32) {  // first group of each cluster
            for (int c0 = 0; c0 <= k; c0 += 32) {
                const int c = c0 + lane;
                int count = 0;
                if (c <= k)
                    for (int w = 0; w < W; ++w) count += __popc(mask[c * W + w]);
                const int groups = (count + a.gmax - 1) / a.gmax;
                int incl = groups;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int y = __shfl_up_sync(0xffffffffu, incl, o);
                    if (lane >= o) incl += y;
                }
                if (c <= k) {
                    members[c] = count;
                    slot[c] = n_groups + incl - groups;
                }
                n_groups += __shfl_sync(0xffffffffu, incl, 31);
            }
        } else {
            const int32_t* table = a.pool.block_table + (size_t)b * a.pool.max_pages;
            const int pages = (kv + a.pool.page_size - 1) / a.pool.page_size;
#pragma unroll 4
            for (int p = tid - 32; p < pages; p += kPagedPlanThreads - 32) bad_page |= (unsigned)table[p] >= (unsigned)a.pool.n_pages;
        }
        __syncthreads();
        for (int h = tid; h < H; h += kPagedPlanThreads) {  // every head finds its group: sizes as even as possible, the larger ones first
            const int c = row_of(h), w = h >> 5, all = members[c];
            int rank = __popc(mask[c * W + w] & ((1u << (h & 31)) - 1u));
            for (int v = 0; v < w; ++v) rank += __popc(mask[c * W + v]);
            const int groups = (all + a.gmax - 1) / a.gmax, size = all / groups, larger = all - size * groups, cut = larger * (size + 1);
            const int g = rank < cut ? rank / (size + 1) : larger + (rank - cut) / size;
            const int first = g <= larger ? g * (size + 1) : cut + (g - larger) * size;
            PagedGroup* e = a.groups + (size_t)b * H + slot[c] + g;
            e->heads[rank - first] = h;
            if (rank == first) *reinterpret_cast<int4*>(e) = make_int4(c < k ? c : -1, rep[c], g < larger ? size + 1 : size, 0);
        }
    }
    const bool bad_head = n > 0 && members[k] > 0;  // (the first warp's own writing)
    bad_page = __syncthreads_or(bad_page);
    if (tid >= 32) return;
    if (bad_page) kv = 0;
    const int n_qt = (n + a.bq - 1) / a.bq;
    int cost = 0;
    for (int qt = lane; qt < n_qt; qt += 32) cost += key_tiles(a, n, kv, qt) + kPagedItemCost;
    cost = __reduce_add_sync(0xffffffffu, cost);
    if (lane == 0) {
        int4* r = reinterpret_cast<int4*>(a.req + b);
        r[0] = make_int4(start, n, kv, n_groups);
        r[1] = make_int4(cost, n > 0 ? key_tiles(a, n, kv, n_qt - 1) : 0, n > 0 && bad_page ? CHAI_ERR_BAD_PAGE : bad_head ? CHAI_ERR_BAD_MEMBERSHIP : CHAI_OK, 0);
    }
}

// What a CTA does of one (group, query tile).  count 0: rows of zeros.
struct PagedItem {
    int b, q0, rows, t0;            // request; first row of the packed arrays, rows, their first among the request's tokens
    int kv, n;                      // of the request
    int tiles, first, count;        // key tiles first, first + 1, ... (modulo tiles), count of them
    int pieces, piece;              // of the query tile, and which one this is
    int owner;                      // CTA whose share it begins in: pieces lie in the slots 2 owner + 1, 2 (owner + 1), 2 (owner + 2), ...
};
__device__ __forceinline__ int piece_slot(int owner, int piece) { return piece == 0 ? 2 * owner + 1 : 2 * (owner + piece); }

// A CTA's walk along its share, by one warp (or the same in several).  Every field is the same in all lanes.
struct PagedWalk {
    int at, length, share;          // where the current (group, query tile) begins, from the share's beginning; the share
    int b, g, qt;
    int start, n, kv, n_groups, n_qt;
    int done_tiles;
    PagedGroup e;

    __device__ __forceinline__ void set_request(const PagedCall& a, const int4& r) {
        start = r.x;
        n = r.y;
        kv = r.z;
        n_groups = r.w;
        n_qt = (n + a.bq - 1) / a.bq;
    }
    __device__ __forceinline__ void load_group(const PagedCall& a) {
        const int4* src = reinterpret_cast<const int4*>(a.groups + (size_t)b * a.H + g);
        reinterpret_cast<int4*>(&e)[0] = __ldcg(src);
        reinterpret_cast<int4*>(&e)[1] = __ldcg(src + 1);
    }
    // Tiles of the query tile that begins at `at` which begin before `end`: tile 0 at `at`, tile i at at + kPagedItemCost + i.
    __device__ __forceinline__ int tiles_before(int end, int tiles) const {
        return end <= at ? 0 : max(min(end - at - kPagedItemCost, tiles), min(tiles, 1));
    }

    // Finds the share.
    __device__ __forceinline__ void begin(const PagedCall& a, int lane) {
        const int per = (a.B + 31) >> 5, first = min(a.B, lane * per), last = min(a.B, first + per);
        int4 r0 = make_int4(0, 0, 0, 0);
        int longest = 0, bad = 0x7fffffff, cost = 0;
        long long mine = 0;
        auto read = [&](int i) {
            r0 = __ldcg(reinterpret_cast<const int4*>(a.req + i));
            const int4 r1 = __ldcg(reinterpret_cast<const int4*>(a.req + i) + 1);
            cost = r1.x;
            if (r1.z != CHAI_OK) bad = min(bad, i);
            longest = max(longest, r1.y);
            return (long long)r0.w * r1.x;
        };
        for (int i = first; i < last; ++i) mine += read(i);
        long long incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long x = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += x;
        }
        const long long total = __shfl_sync(0xffffffffu, incl, 31);
        longest = (int)__reduce_max_sync(0xffffffffu, (unsigned)longest);
        if (blockIdx.x == 0) {
            bad = (int)__reduce_min_sync(0xffffffffu, (unsigned)bad);
            if (lane == 0) {
                reset_status(a.hdr);
                if (bad < a.B) {
                    a.hdr->status = __ldcg(&a.req[bad].code);
                    a.hdr->bad_b = bad;
                }
            }
        }
        // A share holds the beginning of a tile wherever it lies, and no query tile is cut into more than kPagedMaxPieces.
        const int even = total >> 32 == 0 ? (int)(((unsigned)total + a.ctas - 1) / a.ctas) : (int)((total + a.ctas - 1) / a.ctas);
        share = max(max(even, kPagedItemCost + 1), (longest + kPagedItemCost) / (kPagedMaxPieces - 1) + 1);
        const long long lo = (long long)share * (int)blockIdx.x;
        done_tiles = 0;
        at = length = 0;
        if (lo >= total) return;
        length = (int)min((long long)share, total - lo);
        long long before = incl - mine;
        const bool here = before <= lo && lo < incl;
        int i = last - 1;
        if (here && per > 1)
            for (i = first;; ++i) {
                const long long c = read(i);
                if (lo < before + c) break;
                before += c;
            }
        const int src = __ffs(__ballot_sync(0xffffffffu, here)) - 1;
        b = __shfl_sync(0xffffffffu, i, src);
        cost = __shfl_sync(0xffffffffu, cost, src);
        r0.x = __shfl_sync(0xffffffffu, r0.x, src);
        r0.y = __shfl_sync(0xffffffffu, r0.y, src);
        r0.z = __shfl_sync(0xffffffffu, r0.z, src);
        r0.w = __shfl_sync(0xffffffffu, r0.w, src);
        const long long x = lo - __shfl_sync(0xffffffffu, before, src);
        set_request(a, r0);
        g = x >> 32 == 0 ? (int)((unsigned)x / (unsigned)cost) : (int)(x / cost);
        load_group(a);
        at = -(int)(x - (long long)g * cost);  // (of the group)
        for (qt = n_qt - 1; qt > 0; qt -= 32) {  // query tiles from the last to the first, 32 at a time
            const int q = qt - lane, c = q >= 0 ? kPagedItemCost + key_tiles(a, n, kv, q) : 0;
            int sum = c;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, sum, o);
                if (lane >= o) sum += y;
            }
            const unsigned behind = __ballot_sync(0xffffffffu, at + sum > 0);
            const int w = behind != 0 ? __ffs(behind) - 1 : 31;
            const int upto = __shfl_sync(0xffffffffu, sum, w);
            if (behind != 0) {
                at += upto - __shfl_sync(0xffffffffu, c, w);
                qt -= w;
                break;
            }
            at += upto;
        }
    }
    // The next thing to do and its group; false: the share is done.
    __device__ __forceinline__ bool next(const PagedCall& a, PagedItem& it, PagedGroup& entry) {
        while (at < length) {
            const int tiles = key_tiles(a, n, kv, qt), end = at + kPagedItemCost + tiles;
            bool mine = at >= 0;
            it.tiles = it.first = it.count = 0;
            it.pieces = 1;
            it.piece = 0;
            it.owner = blockIdx.x;
            if (tiles > 0 && e.cluster >= 0) {
                it.tiles = tiles;
                if (at >= 0 && end <= length) {
                    it.count = tiles;
                    it.first = done_tiles % tiles;
                } else {
                    const int i0 = tiles_before(0, tiles), i1 = tiles_before(length, tiles), cta = blockIdx.x;
                    it.count = i1 - i0;
                    mine = i1 > i0;
                    if (it.count < tiles) {
                        if (at < 0) it.owner = cta - (share - 1 - at) / share;
                        const int last = tiles == 1 ? at : end - 1;  // where the last tile begins
                        it.pieces = (last < length ? cta : cta + last / share) - it.owner + 1;
                        it.piece = cta - it.owner;
                        const int x = tiles_before((it.owner + 1 - cta) * share, tiles);  // tiles of the first share
                        it.first = i0 < x ? i0 + tiles - x : i0 - x;
                    }
                }
            }
            it.b = b;
            it.t0 = qt * a.bq;
            it.q0 = start + it.t0;
            it.rows = min(a.bq, n - it.t0);
            it.n = n;
            it.kv = kv;
            entry = e;
            at = end;
            if (--qt < 0 && at < length) {
                if (++g == n_groups) {
                    g = 0;
                    int4 r;
                    do r = __ldcg(reinterpret_cast<const int4*>(a.req + ++b));
                    while (r.w == 0);  // (there is a request behind, for the share goes on)
                    set_request(a, r);
                }
                qt = n_qt - 1;
                load_group(a);
            }
            if (mine) {
                done_tiles += it.count;
                return true;
            }
        }
        return false;
    }
};

}  // namespace chai
