// Work division of clustered attention of packed tokens over a paged cache, shared by its kernels.
//
// A unit of work is (request, member group of a cluster, tile of bq query rows, piece of the key tiles).  Requests differ in new
// tokens and cached positions, and the host knows neither, so a planning kernel divides: its blocks (one a request) build the member
// groups and look the pages over; the last one to finish chooses how many key tiles a piece has and numbers the items.
// Pieces of one (group, query tile) leave unnormalised partial results, which whoever finishes last joins.
#pragma once

#include "paged.cuh"
#include "prefill_plan.cuh"

namespace chai {

struct PagedRequest {
    int start, n, kv;      // first row, rows, cached positions (0 where a page is bad)
    int n_groups;
    int item_base;         // number of the request's first item
    int pieces;            // pieces of its longest query tile
    int slot_base;         // first partial result of a request whose tiles are divided
    int code;              // chai_status_t
};
static_assert(sizeof(PagedRequest) == 32, "PagedRequest is 32 bytes");

// words of the workspace header
constexpr int kPagedCounter = 0, kPagedArrival = 1, kPagedItems = 3, kPagedPiece = 4;
static_assert((12 + 4 * kPagedArrival) % 8 == 0, "the arrival word is 8-byte aligned");

constexpr int kSlotRowBytes = 256 * 4 + 8;     // members x head_dim = 256 numbers and (reference, sum), per row
static_assert(2 * kSlotRowBytes % 16 == 0, "slots have an even number of rows");
constexpr size_t kSlotBytesPerToken = 640000;  // see chai_prefill_paged_workspace_bytes

struct PagedLayout {
    size_t off_req, off_groups, off_counters, off_slots, total;
};
// The counters are laid out for query tiles of 16 rows, the smallest.
inline PagedLayout paged_layout(int B, int H, int n_tokens) {
    PagedLayout L;
    L.off_req = sizeof(WsHeader);
    L.off_groups = round_up(L.off_req + sizeof(PagedRequest) * (size_t)B, 256);
    L.off_counters = round_up(L.off_groups + sizeof(GroupEntry) * (size_t)B * H, 256);
    L.off_slots = round_up(L.off_counters + sizeof(int) * (size_t)H * ((size_t)B + n_tokens / 16 + 1), 256);
    L.total = L.off_slots + kSlotBytesPerToken * (n_tokens < 128 ? n_tokens : 128);
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
    PagedRequest* req;
    GroupEntry* groups;
    int* counters;  // pieces that are done, per (query tile, group)
    char* slots;
    long long q_stride;
    float scale;
    int B, H, k, n_tokens, causal;
    int gmax, bq, bk;       // members per group, rows and keys per tile
    int slot_rows, max_slots;
    int ctas;               // that will work on the items
    unsigned token;         // of this launch
};

// Key tiles that query tile qt needs.
__device__ __forceinline__ int key_tiles(const PagedCall& a, int n, int kv, int qt) {
    const int end = a.causal ? max(min(kv, kv - n + min(n, (qt + 1) * a.bq)), 0) : kv;
    return (end + a.bk - 1) / a.bk;
}

// An item, resolved.  n_kv < 0: nothing to do; 0: rows of zeros.
struct PagedItem {
    int b, q0, rows, first_tile, n_kv, kv, n;
    int pieces, piece, slot, counter;
};
__device__ __forceinline__ PagedItem paged_item(const PagedCall& a, int id, GroupEntry* e) {
    int lo = 0, hi = a.B;  // the last request whose items begin at or before id
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (__ldcg(&a.req[mid].item_base) <= id) lo = mid; else hi = mid;
    }
    const int4 r0 = __ldcg(reinterpret_cast<const int4*>(a.req + lo)), r1 = __ldcg(reinterpret_cast<const int4*>(a.req + lo) + 1);
    PagedItem it;
    it.b = lo;
    const int start = r0.x, n = r0.y, kv = r0.z, pieces = r1.y, local = id - r1.x;
    const int n_qt = (n + a.bq - 1) / a.bq, per = n_qt * pieces;
    const int g = local / per, rem = local - g * per, qt = n_qt - 1 - rem / pieces;
    it.piece = rem % pieces;
    const int4* src = reinterpret_cast<const int4*>(a.groups + (size_t)lo * a.H + g);
    reinterpret_cast<int4*>(e)[0] = __ldcg(src);
    reinterpret_cast<int4*>(e)[1] = __ldcg(src + 1);
    const int C = __ldcg(&a.hdr->pad[kPagedPiece]);
    const int tiles = e->cluster < 0 ? 0 : key_tiles(a, n, kv, qt);
    it.pieces = tiles <= C ? 1 : (tiles + C - 1) / C;
    it.q0 = qt * a.bq;
    it.rows = min(a.bq, n - it.q0);
    it.n = n;
    it.kv = kv;
    it.first_tile = it.piece * C;
    it.n_kv = it.piece >= it.pieces ? -1 : min(tiles - it.first_tile, C);
    it.slot = r1.z + local - it.piece;  // of piece 0
    it.counter = (start / a.bq + lo + qt) * a.H + g;
    it.q0 += start;                     // (a row of the packed arrays from here on)
    return it;
}

// Grid B, 128 threads.
static __global__ void __launch_bounds__(128) prefill_paged_plan_kernel(const PagedCall a) {
    extern __shared__ __align__(16) int s_plan[];
    __shared__ int s_in[3], s_last;
    __shared__ float s_items[4][32], s_slots[4][32];
    __shared__ float s_work[4];
    __shared__ int s_most[4], s_scan[4][2], s_code[4];
    __shared__ int2 s_req[128];  // 128 requests at a time: (groups x query tiles, key tiles of the longest)
    dependent_grid_sync();
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
        const int start = min(max(a.token_start[b], 0), a.n_tokens);
        s_in[0] = start;
        s_in[1] = max(min(max(a.token_start[b + 1], 0), a.n_tokens) - start, 0);
        s_in[2] = min(max(a.kv_lens[b], 0), a.pool.capacity);
    }
    __syncthreads();
    const int start = s_in[0], n = s_in[1];
    int kv = s_in[2], n_groups = 0, code = CHAI_OK;
    if (n > 0) {
        int first_bad = a.H;
        plan_groups(a.membership + (size_t)b * a.H, a.reps + (size_t)b * a.k, a.groups + (size_t)b * a.H, s_plan, a.H, a.k, a.gmax,
                    &n_groups, &first_bad);
        const int32_t* table = a.pool.block_table + (size_t)b * a.pool.max_pages;
        const int pages = (kv + a.pool.page_size - 1) / a.pool.page_size;
        bool bad = false;
        for (int p = tid; p < pages; p += blockDim.x) bad |= table[p] < 0 || table[p] >= a.pool.n_pages;
        int* done = a.counters + (size_t)(start / a.bq + b) * a.H;
        const int n_done = (n + a.bq - 1) / a.bq * a.H;
        for (int i = tid; i < n_done; i += blockDim.x) done[i] = 0;
        if (__syncthreads_or(bad)) {
            code = CHAI_ERR_BAD_PAGE;
            kv = 0;
        } else if (first_bad < a.H) {  // (thread 0 knows)
            code = CHAI_ERR_BAD_MEMBERSHIP;
        }
    }
    __threadfence();
    __syncthreads();
    if (tid == 0) {
        int4* r = reinterpret_cast<int4*>(a.req + b);
        r[0] = make_int4(start, n, kv, n_groups);
        r[1] = make_int4(0, 1, 0, code);
        __threadfence();
        // Arrivals are counted under this launch's token, whatever the word held before; the last one clears it, so that a
        // replayed launch begins at none again.
        unsigned long long* word = reinterpret_cast<unsigned long long*>(&a.hdr->pad[kPagedArrival]);
        unsigned long long old = *reinterpret_cast<volatile unsigned long long*>(word), seen;
        unsigned count;
        do {
            seen = old;
            count = (unsigned)(seen >> 32) == a.token ? (unsigned)seen : 0u;
            const unsigned long long next = count + 1 == gridDim.x ? 0ull : ((unsigned long long)a.token << 32) | (count + 1);
            old = atomicCAS(word, seen, next);
        } while (old != seen);
        s_last = count + 1 == gridDim.x;
        __threadfence();
    }
    __syncthreads();
    if (!s_last) return;

    // The last block: how long a piece is.  Work is counted in key tiles of a group.
    float work = 0.f;
    int most = 1;
    auto measure = [&](int i) {
        const int4 r = __ldcg(reinterpret_cast<const int4*>(a.req + i));
        const int n_qt = (r.y + a.bq - 1) / a.bq;
        return make_int2(r.w * n_qt, r.w > 0 ? key_tiles(a, r.y, r.z, n_qt - 1) : 0);
    };
    for (int i = tid; i < a.B; i += 128) {
        const int4 r = __ldcg(reinterpret_cast<const int4*>(a.req + i));
        const int2 m = measure(i);
        s_req[tid] = m;  // (with at most 128 requests: all of them)
        if (m.x == 0) continue;
        work += (float)m.x * 0.5f * (max(m.y, 1) + max(key_tiles(a, r.y, r.z, 0), 1));
        most = max(most, m.y);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        work += __shfl_xor_sync(0xffffffffu, work, o);
        most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
    }
    if (lane == 0) s_work[warp] = work, s_most[warp] = most;
    __syncthreads();
    work = s_work[0] + s_work[1] + s_work[2] + s_work[3];
    most = max(max(s_most[0], s_most[1]), max(s_most[2], s_most[3]));
    // Lane l tries pieces of ceil(most / (l + 1)) tiles.
    int piece = (most + lane) / (lane + 1);
    float items = 0.f, slots = 0.f;
    for (int base = 0; base < a.B; base += 128) {
        if (a.B > 128) {  // (else they lie there already)
            __syncthreads();
            s_req[tid] = base + tid < a.B ? measure(base + tid) : make_int2(0, 0);
            __syncthreads();
        }
        for (int i = warp; i < min(128, a.B - base); i += 4) {
            const int2 r = s_req[i];
            const int p = max((r.y + piece - 1) / piece, 1);
            items += (float)r.x * p;
            if (p > 1) slots += (float)r.x * p;
        }
    }
    s_items[warp][lane] = items;
    s_slots[warp][lane] = slots;
    __syncthreads();
    items = s_items[0][lane] + s_items[1][lane] + s_items[2][lane] + s_items[3][lane];
    slots = s_slots[0][lane] + s_slots[1][lane] + s_slots[2][lane] + s_slots[3][lane];
    // Time in tiles: whole rounds of average items, or the work with half an item left over at the end, or one item.  An item
    // costs about a tile more than its tiles, a piece's partial result as much again.
    const float own = lane == 0 ? 1.f : 2.f;
    float time = INFINITY;
    if (slots <= (float)a.max_slots) {
        const float avg = work / fmaxf(items, 1.f) + own;
        time = fmaxf(fmaxf(ceilf(items / a.ctas) * avg, items * avg / a.ctas + 0.5f * piece), piece + own);
    }
    int best = lane;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float t = __shfl_xor_sync(0xffffffffu, time, o);
        const int l = __shfl_xor_sync(0xffffffffu, best, o);
        if (t < time || (t == time && l < best)) time = t, best = l;
    }
    piece = __shfl_sync(0xffffffffu, piece, best);

    // Numbers of the requests' items and slots: running sums, 128 requests at a time.
    int item_run = 0, slot_run = 0;
    for (int base = 0; base < a.B; base += 128) {
        const int i = base + tid;
        int count = 0, split = 0, p = 1;
        if (i < a.B) {
            const int2 r = a.B <= 128 ? s_req[tid] : measure(i);
            p = max((r.y + piece - 1) / piece, 1);
            count = r.x * p;
            split = p > 1 ? count : 0;
        }
        int c = count, s = split;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, c, o), y = __shfl_up_sync(0xffffffffu, s, o);
            if (lane >= o) c += x, s += y;
        }
        __syncthreads();
        if (lane == 31) s_scan[warp][0] = c, s_scan[warp][1] = s;
        __syncthreads();
        for (int w = 0; w < warp; ++w) c += s_scan[w][0], s += s_scan[w][1];
        if (i < a.B) {
            a.req[i].item_base = item_run + c - count;
            a.req[i].pieces = p;
            a.req[i].slot_base = slot_run + s - split;
        }
        for (int w = 0; w < 4; ++w) item_run += s_scan[w][0], slot_run += s_scan[w][1];
    }
    // The first request with something to report.
    int who = 0x7fffffff;
    for (int i = tid; i < a.B; i += 128)
        if (__ldcg(&a.req[i].code) != CHAI_OK) who = min(who, i);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) who = min(who, __shfl_xor_sync(0xffffffffu, who, o));
    if (lane == 0) s_code[warp] = who;
    __syncthreads();
    if (tid == 0) {
        who = min(min(s_code[0], s_code[1]), min(s_code[2], s_code[3]));
        reset_status(a.hdr);
        if (who < a.B) {
            a.hdr->status = __ldcg(&a.req[who].code);
            a.hdr->bad_b = who;
        }
        a.hdr->pad[kPagedCounter] = 0;
        a.hdr->pad[kPagedItems] = item_run;
        a.hdr->pad[kPagedPiece] = piece;
    }
}

}  // namespace chai
