// Pages for a step's new tokens, and the maps that the step's other calls read (Section 3.5: caches are per request, and
// requests of a batch are at different positions).
//
//   chai_plan_paged   lengths, wanted tokens, a stack of free pages -> block tables, token_start, and for every token its
//                     request, position and slot
//
// With pages of ps positions a request of s cached positions that gets n more needs ceil((s + n) / ps) - ceil(s / ps)
// pages.  Where its pages lie on the stack and its tokens in the packed arrays are exclusive prefix sums over the requests,
// which one block computes (two scans a tile of requests).  A token's page then follows from its request's sums
// alone -- an entry of the list that was there, or the stack's entry at a known depth -- so tokens are independent of one another
// and of the list's new entries, which the token in a page's first row writes.
// Bound by latency: a chain of loads (lengths -> sums -> tokens' pages) behind one launch while there are few tokens.  Up
// to kOneBlockTokens the block that scans also writes the tokens; above, a dependent grid does (4 tokens a thread, 16-byte
// stores).  Measured: 16 requests of a token 4.1 us, 300 mixed ones 10.6, 4 prompts of 327680 tokens in all 7.0.
#include "paged.cuh"

namespace chai {
namespace {

constexpr int kPlanThreads = 1024, kTokenThreads = 256, kTokensPerThread = 4;
constexpr int kOneBlockTokens = 4096;

struct PlanArgs {
    const int32_t *seq_lens, *new_lens;
    int32_t *block_table, *free_pages;
    const int32_t* free_count;
    int32_t *free_count_out, *kv_lens, *token_start, *token_request, *positions;
    int64_t* slots;
    WsHeader* hdr;
    int32_t *top, *page_start;  // workspace: depth of the stack before pages are taken, and [B] pages taken before each request
    int B, n_tokens, n_pages, page_size, max_pages, capacity;
    int step, n_starts;         // of the requests' beginnings, every step-th (n_starts and the end) goes to shared memory
    FastDiv by_page;
};

__device__ __forceinline__ int pages_for(const PlanArgs& a, int positions) {  // ceil(positions / page_size)
    return (int)a.by_page.div((unsigned)positions + (unsigned)a.page_size - 1u);
}

// Inclusive sums of two numbers over the block's threads, and their totals.
struct Two {
    long long x, y;
};
__device__ __forceinline__ Two block_scan(Two v, Two* s_warp, Two* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, v.x, o), y = __shfl_up_sync(0xffffffffu, v.y, o);
        if (lane >= o) v.x += x, v.y += y;
    }
    if (n_warps == 1) {
        *total = {__shfl_sync(0xffffffffu, v.x, 31), __shfl_sync(0xffffffffu, v.y, 31)};
        return v;
    }
    __syncthreads();  // (the array may still be read by the scan before)
    if (lane == 31) s_warp[warp] = v;
    __syncthreads();
    Two all = lane < n_warps ? s_warp[lane] : Two{0, 0}, own = all;  // (every warp scans the warps' sums)
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, all.x, o), y = __shfl_up_sync(0xffffffffu, all.y, o);
        if (lane >= o) all.x += x, all.y += y;
    }
    v.x += __shfl_sync(0xffffffffu, all.x - own.x, warp);
    v.y += __shfl_sync(0xffffffffu, all.y - own.y, warp);
    *total = {__shfl_sync(0xffffffffu, all.x, 31), __shfl_sync(0xffffffffu, all.y, 31)};
    return v;
}

// Where requests' tokens begin, in shared memory: all beginnings, or of many requests every step-th.
constexpr int kStarts = 1024;
__device__ __forceinline__ void load_starts(const PlanArgs& a, int* s_start) {
    const int step = a.step;
    for (int i = threadIdx.x; i * step <= a.B; i += blockDim.x) s_start[i] = a.token_start[i * step];
    __syncthreads();
}

// Tokens t0 .. t0 + kTokensPerThread - 1 of the packed arrays.
__device__ __forceinline__ void plan_tokens(const PlanArgs& a, const int* s_start, int t0, int top) {
    if (t0 >= a.n_tokens) return;
    // the largest request with token_start <= t0 (requests without tokens: the last of equals)
    const int step = a.step;
    int lo = 0, hi = a.n_starts;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s_start[mid] <= t0) lo = mid; else hi = mid;
    }
    if (step > 1) {
        hi = min((lo + 1) * step, a.B);
        lo *= step;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (a.token_start[mid] <= t0) lo = mid; else hi = mid;
        }
    }
    auto begins = [&](int i) { return step == 1 ? s_start[i] : a.token_start[i]; };
    int b = lo, start = begins(b), end = begins(b + 1), cur = -1, held = 0, seq = 0, first = 0;
    int request[kTokensPerThread], position[kTokensPerThread];
    long long slot[kTokensPerThread];
    bool bad = false;
#pragma unroll
    for (int i = 0; i < kTokensPerThread; ++i) {
        const int t = t0 + i;
        while (t >= end && b + 1 < a.B) {
            ++b;
            start = end;
            end = begins(b + 1);
        }
        request[i] = -1;
        position[i] = 0;
        slot[i] = -1;
        if (t >= end || t >= a.n_tokens) continue;
        if (cur != b) {
            cur = b;
            seq = a.kv_lens[b] - (end - start);
            held = pages_for(a, seq);
            first = a.page_start[b];
        }
        const int pos = seq + (t - start);
        const int pi = (int)a.by_page.div((unsigned)pos), row = pos - pi * a.page_size;
        request[i] = b;
        position[i] = pos;
        // (always true for the lengths that the sums were made of; another stream may write into the arrays meanwhile)
        if (pos < 0 || pi >= a.max_pages) continue;
        const int depth = top - 1 - (first + pi - held);
        int page = -1;
        int32_t* entry = a.block_table + (size_t)b * a.max_pages + pi;
        if (pi < held) {
            page = *entry;
        } else if (depth >= 0 && depth < a.n_pages) {
            page = a.free_pages[depth];
            if (row == 0) *entry = page;
        }
        if (page >= 0 && page < a.n_pages) slot[i] = (long long)page * a.page_size + row;
        else bad = true;
    }
    if (t0 + kTokensPerThread <= a.n_tokens) {  // (the arrays start on 16-byte boundaries)
        *reinterpret_cast<int4*>(a.token_request + t0) = make_int4(request[0], request[1], request[2], request[3]);
        *reinterpret_cast<int4*>(a.positions + t0) = make_int4(position[0], position[1], position[2], position[3]);
        reinterpret_cast<longlong2*>(a.slots + t0)[0] = make_longlong2(slot[0], slot[1]);
        reinterpret_cast<longlong2*>(a.slots + t0)[1] = make_longlong2(slot[2], slot[3]);
    } else {
        for (int i = 0; i < kTokensPerThread && t0 + i < a.n_tokens; ++i) {
            a.token_request[t0 + i] = request[i];
            a.positions[t0 + i] = position[i];
            a.slots[t0 + i] = slot[i];
        }
    }
    if (bad) atomicExch(&a.hdr->status, CHAI_ERR_BAD_PAGE);  // (whatever the requests' sums said: it comes first)
}

// One block.  TOKENS: writes the tokens too.
template <bool TOKENS>
__global__ void __launch_bounds__(kPlanThreads) plan_requests_kernel(const PlanArgs a) {
    __shared__ Two s_warp[32];
    __shared__ int s_held[kPlanThreads];
    __shared__ long long s_off[kPlanThreads];
    __shared__ int s_list[kPlanThreads], s_n, s_start[kStarts + 1];
    dependent_grid_sync();
    const int tid = threadIdx.x, nt = blockDim.x, lane = tid & 31, warp = tid >> 5, n_warps = nt >> 5;
    const int count = *a.free_count;
    int top = min(max(count, 0), a.n_pages);
    bool full = false, bad = count != top;
    Two total;

    // 1. Pages of requests that end go onto the stack, request by request.
    for (int base = 0; base < a.B; base += nt) {
        const int b = base + tid;
        int held = 0;
        if (b < a.B && a.new_lens[b] < 0) {
            const int s = a.seq_lens[b];
            if (s < 0 || s > a.capacity) full = true;  // (not a length of this list: nothing is given back)
            else held = pages_for(a, s);
        }
        if (tid == 0) s_n = 0;
        if (!__syncthreads_or(held > 0)) continue;
        s_held[tid] = held;
        if (held > 0) s_list[atomicAdd(&s_n, 1)] = tid;  // (in any order: where a list goes is a sum over the requests before)
        __syncthreads();
        const int n_ended = s_n;
        for (int e = warp; e < n_ended; e += n_warps) {  // a list with an entry that is no page is not given back
            const int i = s_list[e], h = s_held[i];
            const int32_t* list = a.block_table + (size_t)(base + i) * a.max_pages;
            bool odd = false;
            for (int j = lane; j < h; j += 32) odd |= list[j] < 0 || list[j] >= a.n_pages;
            if (__any_sync(0xffffffffu, odd)) {
                bad = true;
                if (lane == 0) s_held[i] = 0;
            }
        }
        __syncthreads();
        held = s_held[tid];
        s_off[tid] = block_scan({held, 0}, s_warp, &total).x - held;
        __syncthreads();
        for (int e = warp; e < n_ended; e += n_warps) {
            const int i = s_list[e], h = s_held[i];
            const int32_t* list = a.block_table + (size_t)(base + i) * a.max_pages;
            for (int j = lane; j < h; j += 32) {
                const long long at = (long long)top + s_off[i] + j;
                if (at < a.n_pages) a.free_pages[at] = list[j];
                else bad = true;  // more pages than there are: some were given back twice
            }
        }
        top = (int)min((long long)top + total.x, (long long)a.n_pages);
        __syncthreads();
    }

    // 2. Who gets tokens, their pages and their place in the packed arrays.
    long long need_before = 0, want_before = 0, given = 0, taken = 0;
    for (int base = 0; base < a.B; base += nt) {
        const int b = base + tid;
        int n = 0, s = 0;
        if (b < a.B) n = a.new_lens[b], s = a.seq_lens[b];
        const bool ends = n < 0;
        const bool fits = !ends && s >= 0 && s <= a.capacity && n <= a.capacity - s;
        const int held = fits ? pages_for(a, s) : 0;
        const int need = fits ? pages_for(a, s + n) - held : 0, want = fits ? n : 0;
        const Two sum = block_scan({need, want}, s_warp, &total);
        const long long pages = need_before + sum.x, tokens = want_before + sum.y;
        need_before += total.x;
        want_before += total.y;
        const bool ok = fits && (need == 0 || pages <= top) && (want == 0 || tokens <= a.n_tokens);
        full |= b < a.B && !ends && !ok;
        const int give = ok ? n : 0, use = ok ? need : 0;
        const Two got = block_scan({give, use}, s_warp, &total);
        if (b < a.B) {
            a.token_start[b + 1] = (int)(given + got.x);
            // (requests that need pages and get them are the first that do: everyone before them got theirs)
            a.page_start[b] = (int)(taken + got.y - use);
            a.kv_lens[b] = ends ? 0 : s + give;
        }
        given += total.x;
        taken += total.y;
    }
    full = __syncthreads_or(full);
    bad = __syncthreads_or(bad);
    if (tid == 0) {
        a.token_start[0] = 0;
        *a.free_count_out = top - (int)taken;
        *a.top = top;
        reset_status(a.hdr);
        a.hdr->status = bad ? CHAI_ERR_BAD_PAGE : full ? CHAI_ERR_CACHE_FULL : CHAI_OK;
    }
    if constexpr (TOKENS) {
        __syncthreads();
        load_starts(a, s_start);
        for (int t0 = tid * kTokensPerThread; t0 < a.n_tokens; t0 += nt * kTokensPerThread) plan_tokens(a, s_start, t0, top);
    }
}

__global__ void __launch_bounds__(kTokenThreads) plan_tokens_kernel(const PlanArgs a) {
    __shared__ int s_start[kStarts + 1];
    dependent_grid_sync();
    load_starts(a, s_start);
    plan_tokens(a, s_start, (int)(blockIdx.x * kTokenThreads + threadIdx.x) * kTokensPerThread, *a.top);
}

int plan(PlanArgs a, cudaStream_t s) {
    const char* fn = "chai_plan_paged";
    const void* all[] = {a.seq_lens, a.new_lens, a.block_table, a.free_pages, a.free_count, a.free_count_out, a.kv_lens,
                         a.token_start, a.token_request, a.positions, a.slots, a.hdr};
    for (const void* p : all) CHAI_REQUIRE(p != nullptr, CHAI_ERR_INVALID_ARG, "%s: null pointer", fn);
    for (const void* p : {(const void*)a.token_request, (const void*)a.positions, (const void*)a.slots, (const void*)a.hdr})
        CHAI_REQUIRE(aligned16(p), CHAI_ERR_INVALID_ARG, "%s: token_request, positions, slots and workspace must be 16-byte aligned", fn);
    for (const void* p : all)
        CHAI_REQUIRE((reinterpret_cast<uintptr_t>(p) & 3u) == 0, CHAI_ERR_INVALID_ARG, "%s: pointers must be 4-byte aligned", fn);
    CHAI_REQUIRE(a.B > 0 && a.n_tokens > 0 && a.n_pages > 0 && a.page_size > 0 && a.max_pages > 0, CHAI_ERR_INVALID_ARG,
                 "%s: sizes must be positive", fn);
    CHAI_REQUIRE(a.page_size % 8 == 0 && a.page_size <= 65536, CHAI_ERR_UNSUPPORTED,
                 "%s: page_size %d (a multiple of 8 up to 65536 supported)", fn, a.page_size);
    CHAI_REQUIRE(a.B <= 65535 && a.n_tokens <= (1 << 30), CHAI_ERR_UNSUPPORTED, "%s: B must be <= 65535 and n_tokens <= 2^30", fn);
    CHAI_REQUIRE((long long)a.max_pages * a.page_size < (1ll << 30), CHAI_ERR_UNSUPPORTED,
                 "%s: max_pages * page_size must be below 2^30", fn);
    a.capacity = a.max_pages * a.page_size;
    a.by_page = FastDiv((unsigned)a.page_size);
    a.step = (a.B + kStarts - 1) / kStarts;
    a.n_starts = (a.B + a.step - 1) / a.step;
    const bool one = a.n_tokens <= kOneBlockTokens;
    const int want = max(a.B, one ? (a.n_tokens + kTokensPerThread - 1) / kTokensPerThread : 1);
    const int threads = want >= kPlanThreads ? kPlanThreads : (want + 31) / 32 * 32;
    CHAI_LOG_CALL("%s: B=%d n_tokens=%d n_pages=%d page_size=%d max_pages=%d", fn, a.B, a.n_tokens, a.n_pages, a.page_size, a.max_pages);
    if (one) {
        CHAI_LAUNCH_DEPENDENT("plan_requests_kernel launch", plan_requests_kernel<true>, dim3(1), dim3(threads), 0, s, a);
        return CHAI_OK;
    }
    CHAI_LAUNCH_DEPENDENT("plan_requests_kernel launch", plan_requests_kernel<false>, dim3(1), dim3(threads), 0, s, a);
    const int per_block = kTokenThreads * kTokensPerThread;
    CHAI_LAUNCH_DEPENDENT("plan_tokens_kernel launch", plan_tokens_kernel, dim3((a.n_tokens + per_block - 1) / per_block),
                          dim3(kTokenThreads), 0, s, a);
    return CHAI_OK;
}

}  // namespace
}  // namespace chai

extern "C" {

size_t chai_plan_paged_workspace_bytes(int B) { return B > 0 ? 512 + sizeof(int32_t) * (size_t)B : 0; }

int chai_plan_paged(const int32_t* seq_lens, const int32_t* new_lens, int32_t* block_table, int32_t* free_pages,
                    const int32_t* free_count, int32_t* free_count_out, int32_t* kv_lens, int32_t* token_start,
                    int32_t* token_request, int32_t* positions, int64_t* slots, int B, int n_tokens, int n_pages, int page_size,
                    int max_pages, void* workspace, size_t workspace_bytes, void* stream) {
    chai::PlanArgs a = {};
    a.seq_lens = seq_lens;
    a.new_lens = new_lens;
    a.block_table = block_table;
    a.free_pages = free_pages;
    a.free_count = free_count;
    a.free_count_out = free_count_out;
    a.kv_lens = kv_lens;
    a.token_start = token_start;
    a.token_request = token_request;
    a.positions = positions;
    a.slots = slots;
    a.hdr = static_cast<chai::WsHeader*>(workspace);
    a.B = B;
    a.n_tokens = n_tokens;
    a.n_pages = n_pages;
    a.page_size = page_size;
    a.max_pages = max_pages;
    if (workspace != nullptr) {
        CHAI_REQUIRE(workspace_bytes >= chai_plan_paged_workspace_bytes(B), CHAI_ERR_WORKSPACE,
                     "chai_plan_paged: workspace has %zu bytes, %zu needed", workspace_bytes, chai_plan_paged_workspace_bytes(B));
        a.top = reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + 256);
        a.page_start = reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + 512);
    }
    return chai::plan(a, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
