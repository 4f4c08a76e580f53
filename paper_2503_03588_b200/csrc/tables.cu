// pa_build_block_tables: pages, slots and positions of a batch's new tokens from the sequences' lengths.
//
// Two prefix sums over the batch (new tokens, pages wanted), then one entry per token.  Every fresh block has exactly one first
// token, and it is this token's thread that writes the table entry; a token's own page comes from the table for blocks that the
// sequence had and from the stack for fresh ones, so no thread reads what another one writes.
//
// Bound by latency: a launch, the sums, then a chain from a token's sequence over its page to its slot.  Up to 1024 sequences every
// CTA takes the sums itself, which costs less than a kernel that has to wait for them.  A warp finds the sequences of its first and
// last token 32 at a time, and a lane the one of its own between them; a lane's pages are all on their way before it writes.
// Measured: a decoding step of 64 sequences 2.2 us; 500 prompts of up to 4000 tokens, 1.15 million in all, 8.0 us (sums and
// launch 3.6 of them; 12 bytes a token are written at 3.1 TB/s; in two kernels 10.8; with one set of four tokens a lane 11.2, and
// with four sets 9.4).  500 prompts of 2294 tokens with results in place, a second kernel: 15.5 (7.4 without).  2500 sequences of a
// token each, the sums by one CTA: 19.4; of 400 tokens each 17.7.
#include <limits.h>

#include "common.cuh"

namespace pa {

constexpr int kPageTokens = 64;
constexpr int kTableThreads = 256;
constexpr int kPerThread = 4;        // sequences of a thread in one turn of the sums
constexpr int kTurn = kTableThreads * kPerThread;  // up to this many sequences every CTA takes the sums itself
constexpr int kFillTokens = 4;       // tokens of a thread that stand together
constexpr int kSets = 2;             // times as many per thread and turn
constexpr int kWarpTokens = 32 * kFillTokens * kSets;
constexpr int kStepTokens = 1024;    // one CTA does it all up to this many places for tokens
constexpr int32_t kMost = 1 << 30;   // tokens and pages of a call; sums are held at INT32_MAX

// What the tokens of a sequence need to know.
struct Sequence {
    int32_t start;   // its first token
    int32_t cached;  // tokens it had
    int32_t first;   // its first fresh page's place below the top of the stack; -1: refused
    int32_t end;     // behind its last token
};

struct TableArgs {
    const int32_t *new_lens, *cache_lens, *free_pages, *free_count;
    int32_t *table, *cu, *positions, *lens_out, *free_left;
    int64_t *slots;
    Sequence *seqs;      // [batch]
    int32_t *count;      // the stack's height before the call
    int32_t batch, max_blocks, n_pages, max_tokens, free_capacity;
    bool vector;         // slots and positions start on 16-byte boundaries
};

__device__ __forceinline__ int32_t clamp31(int64_t x) { return x > INT32_MAX ? INT32_MAX : (int32_t)x; }
// Sum of two numbers in [0, 2^31), held below 2^31.
__device__ __forceinline__ int32_t add31(int32_t a, int32_t b) { return (int32_t)min((uint32_t)a + (uint32_t)b, (uint32_t)INT32_MAX); }

// The sum of x over the CTA's threads before this one (held below 2^31) and over all; `sums`: room for one number a warp.
__device__ __forceinline__ int32_t scan_cta(int32_t x, int32_t *sums, int32_t *total)
{
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    int32_t upto = x;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const int32_t up = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto = add31(upto, up);
    }
    int32_t before = __shfl_up_sync(0xffffffffu, upto, 1);
    if (lane == 0) before = 0;
    if (lane == 31) sums[wid] = upto;
    __syncthreads();
    int32_t all = 0;
#pragma unroll
    for (int w = 0; w < kTableThreads / 32; ++w) {
        if (w == wid) before = add31(before, all);
        all = add31(all, sums[w]);
    }
    *total = all;
    return before;
}

// The sequences' sums, by one CTA: seqs[] and the stack's height for the tokens; if `results`, cu, lens_out and free_left.
__device__ __forceinline__ void scan_sequences(const TableArgs &a, bool results, Sequence *seqs, int32_t *height)
{
    __shared__ int32_t sums[2][kTableThreads / 32];
    __shared__ int32_t most_taken;
    const int tid = threadIdx.x;
    int32_t stack = *a.free_count;
    stack = stack < 0 ? 0 : stack > a.free_capacity ? a.free_capacity : stack;
    if (tid == 0) most_taken = 0;
    int32_t tokens = 0, wanted = 0;  // of the sequences before this turn's
    for (int b0 = 0; b0 < a.batch; b0 += kTurn) {
        int32_t n[kPerThread], c[kPerThread], want[kPerThread], start[kPerThread], upto[kPerThread];
        bool fits[kPerThread];
        int32_t mine = 0;
#pragma unroll
        for (int x = 0; x < kPerThread; ++x) {
            const int b = b0 + tid * kPerThread + x;
            n[x] = b < a.batch ? a.new_lens[b] : 0;
            c[x] = b < a.batch ? a.cache_lens[b] : 0;
        }
#pragma unroll
        for (int x = 0; x < kPerThread; ++x) mine = add31(mine, max(n[x], 0));
        int32_t total_tokens, total_pages;
        int32_t sum = add31(tokens, scan_cta(mine, sums[0], &total_tokens)), pages = 0;
#pragma unroll
        for (int x = 0; x < kPerThread; ++x) {
            start[x] = sum;
            upto[x] = sum = add31(sum, max(n[x], 0));
            const int64_t behind = (int64_t)c[x] + n[x];
            // (a length held in int32 has to fit behind the call as well)
            fits[x] = n[x] >= 0 && c[x] >= 0 && sum <= a.max_tokens && behind <= min((int64_t)a.max_blocks * kPageTokens, (int64_t)INT32_MAX);
            want[x] = fits[x] ? (int32_t)((behind + kPageTokens - 1) / kPageTokens) - (c[x] / kPageTokens + (c[x] % kPageTokens != 0)) : 0;
            pages = add31(pages, want[x]);
        }
        int32_t before = add31(wanted, scan_cta(pages, sums[1], &total_pages));
#pragma unroll
        for (int x = 0; x < kPerThread; ++x) {
            const int b = b0 + tid * kPerThread + x;
            if (b >= a.batch) break;
            const int32_t taken = add31(before, want[x]);
            const bool served = fits[x] && (want[x] == 0 || taken <= stack);
            if (seqs) seqs[b] = Sequence{start[x], c[x], served ? before : -1, upto[x]};
            if (results) {
                a.cu[b + 1] = upto[x];
                if (b == 0) a.cu[0] = 0;
                a.lens_out[b] = served ? c[x] + n[x] : c[x];
                if (served && want[x] > 0) atomicMax(&most_taken, taken);
            }
            before = taken;
        }
        tokens = add31(tokens, total_tokens);
        wanted = add31(wanted, total_pages);
        __syncthreads();
    }
    if (tid == 0) {
        if (height) *height = stack;
        if (results) *a.free_left = stack - most_taken;
    }
}

// The first sequence of batch that ends behind token i, for a warp (all lanes the same i): 32 at a time.
__device__ __forceinline__ int find_sequence(const TableArgs &a, const Sequence *seqs, int32_t i)
{
    const int lane = threadIdx.x & 31;
    int from = 0, span = 1;
    while (span * 32 < a.batch) span *= 32;
    for (; span > 0; span /= 32) {  // (groups of `span` sequences: how many of the next 32 groups end at or before i?)
        const int last = from + (lane + 1) * span - 1;
        const bool done = last < a.batch && seqs[last].end <= i;
        from += __popc(__ballot_sync(0xffffffffu, done)) * span;
    }
    return from;
}

// Where the page of block j of a sequence that is served stands: in the table, for a fresh block on the stack.
struct Block {
    const int32_t *from;
    int32_t *fresh;  // the table entry to write; null: the sequence had the block
};
__device__ __forceinline__ Block block_of(const TableArgs &a, const Sequence &s, int b, int32_t j, int32_t height)
{
    int32_t *entry = a.table + (int64_t)b * a.max_blocks + j;
    const int32_t have = s.cached / kPageTokens + (s.cached % kPageTokens != 0);
    if (j < have) return {entry, nullptr};
    return {a.free_pages + (height - 1 - (s.first + (j - have))), entry};
}
__device__ __forceinline__ int64_t slot_in(const TableArgs &a, int32_t page, int32_t place)
{
    return page >= 0 && page < a.n_pages ? (int64_t)page * kPageTokens + place : -1;
}
// The slot of the token at `place` of block j, -1 without a page; writes a fresh block's table entry with its first token.
__device__ __forceinline__ int64_t page_of(const TableArgs &a, const Sequence &s, int b, int32_t j, int32_t place, int32_t height)
{
    const Block block = block_of(a, s, b, j, height);
    const int32_t page = *block.from;
    if (place == 0 && block.fresh) *block.fresh = page;
    return slot_in(a, page, place);
}

// kFillTokens tokens from i0 on, of any sequences from b on.  All pages are on their way before anything is written.
__device__ __forceinline__ void fill_any(const TableArgs &a, const Sequence *seqs, int32_t height, int32_t i0, int b)
{
    Sequence s = {};
    if (b < a.batch) s = seqs[b];
    int32_t page[kFillTokens];
    int64_t at[kFillTokens];
    int32_t *fresh[kFillTokens];
#pragma unroll
    for (int x = 0; x < kFillTokens; ++x) {
        const int32_t i = i0 + x;
        while (b < a.batch && i >= s.end)
            if (++b < a.batch) s = seqs[b];
        page[x] = -1;
        at[x] = -1;
        fresh[x] = nullptr;
        if (b >= a.batch || i >= a.max_tokens) continue;
        at[x] = (int64_t)s.cached + (i - s.start);
        if (s.first < 0) continue;
        const Block block = block_of(a, s, b, (int32_t)at[x] / kPageTokens, height);
        page[x] = *block.from;
        if (at[x] % kPageTokens == 0) fresh[x] = block.fresh;
    }
#pragma unroll
    for (int x = 0; x < kFillTokens; ++x) {
        if (fresh[x]) *fresh[x] = page[x];
        if (i0 + x >= a.max_tokens) continue;
        a.positions[i0 + x] = clamp31(at[x]);
        a.slots[i0 + x] = slot_in(a, page[x], (int32_t)at[x] % kPageTokens);
    }
}

// kWarpTokens tokens of a warp from w0 on: a lane has four in each of kSets sets, and the pages of all its sets are on their way
// before the first is written.
__device__ __forceinline__ void fill_tokens(const TableArgs &a, const Sequence *seqs, int32_t height, int32_t w0)
{
    // The lanes' sequences lie between those of the warp's first and last token.
    const int first = find_sequence(a, seqs, w0), last = find_sequence(a, seqs, w0 + kWarpTokens - 1);
    int b[kSets];
    int32_t at[kSets], page[kSets], next[kSets];
    int32_t *fresh[kSets], *fresh_next[kSets];
    bool four[kSets];  // four tokens of one sequence, in one page or two: all but a few
#pragma unroll
    for (int y = 0; y < kSets; ++y) {
        const int32_t i0 = w0 + (y * 32 + (int32_t)(threadIdx.x & 31)) * kFillTokens;
        int lo = first, hi = last;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (seqs[mid].end <= i0) lo = mid + 1;
            else hi = mid;
        }
        b[y] = lo;
        Sequence s = {};
        if (lo < a.batch) s = seqs[lo];
        // (or four behind the last sequence)
        four[y] = a.vector && i0 + kFillTokens <= a.max_tokens && (lo == a.batch || (i0 + kFillTokens <= s.end && s.first >= 0));
        fresh[y] = fresh_next[y] = nullptr;
        page[y] = next[y] = at[y] = -1;
        if (four[y] && lo < a.batch) {
            at[y] = s.cached + (i0 - s.start);
            const int32_t j = at[y] / kPageTokens, place = at[y] % kPageTokens;
            const Block block = block_of(a, s, lo, j, height);
            page[y] = *block.from;
            if (place == 0) fresh[y] = block.fresh;
            if (place > kPageTokens - kFillTokens) {
                const Block behind = block_of(a, s, lo, j + 1, height);
                next[y] = *behind.from;
                fresh_next[y] = behind.fresh;
            }
        }
    }
#pragma unroll
    for (int y = 0; y < kSets; ++y) {
        const int32_t i0 = w0 + (y * 32 + (int32_t)(threadIdx.x & 31)) * kFillTokens;
        if (!four[y]) {
            fill_any(a, seqs, height, i0, b[y]);
            continue;
        }
        if (fresh[y]) *fresh[y] = page[y];
        if (fresh_next[y]) *fresh_next[y] = next[y];
        const int32_t place = at[y] % kPageTokens;
        auto slot = [&](int x) { return place + x < kPageTokens ? slot_in(a, page[y], place + x) : slot_in(a, next[y], place + x - kPageTokens); };
        longlong2 *to = reinterpret_cast<longlong2 *>(a.slots + i0);
        to[0] = make_longlong2(slot(0), slot(1));
        to[1] = make_longlong2(slot(2), slot(3));
        *reinterpret_cast<int4 *>(a.positions + i0) = at[y] < 0 ? make_int4(-1, -1, -1, -1) : make_int4(at[y], at[y] + 1, at[y] + 2, at[y] + 3);
    }
}

// Each CTA takes the sums and then its share of the tokens.  The results that may lie over what the other CTAs still read are left
// to tables_results_kernel unless `results`.
__global__ void __launch_bounds__(kTableThreads) tables_kernel(const TableArgs a, bool results)
{
    __shared__ Sequence seqs[kTurn];
    __shared__ int32_t height;
    pdl_launch_next();
    pdl_wait();
    scan_sequences(a, results && blockIdx.x == 0, seqs, &height);
    __syncthreads();
    constexpr int kWarps = kTableThreads / 32;
    const int64_t step = (int64_t)gridDim.x * kWarps * kWarpTokens;
    for (int64_t w = ((int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5)) * kWarpTokens; w < a.max_tokens; w += step)
        fill_tokens(a, seqs, height, (int32_t)w);
}
__global__ void __launch_bounds__(kTableThreads) tables_results_kernel(const TableArgs a)
{
    pdl_launch_next();
    pdl_wait();
    scan_sequences(a, true, nullptr, nullptr);
}

// A decoding step, one CTA: a thread per sequence takes the sums and, where no sequence has more than kFew tokens, writes its tokens
// itself.
constexpr int kFew = 4;
__global__ void __launch_bounds__(kTurn) tables_step_kernel(const TableArgs a)
{
    __shared__ Sequence seqs[kTurn];
    __shared__ int32_t sums[2][32], most_taken;
    pdl_launch_next();
    const int b = threadIdx.x, lane = b & 31, wid = b >> 5, warps = blockDim.x >> 5;
    if (b == 0) most_taken = 0;
    pdl_wait();
    int32_t stack = *a.free_count;
    const int32_t n_raw = b < a.batch ? a.new_lens[b] : 0, c = b < a.batch ? a.cache_lens[b] : 0, n = max(n_raw, 0);
    stack = stack < 0 ? 0 : stack > a.free_capacity ? a.free_capacity : stack;
    auto scan = [&](int32_t x, int32_t *sum, int32_t &all) {  // the sum before this thread, and over all
        int32_t upto = x;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int32_t up = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto = add31(upto, up);
        }
        if (lane == 31) sum[wid] = upto;
        __syncthreads();
        int32_t before = 0;
        all = 0;
        for (int w = 0; w < warps; ++w) {
            if (w == wid) before = all;
            all = add31(all, sum[w]);
        }
        const int32_t mine = __shfl_up_sync(0xffffffffu, upto, 1);
        return add31(before, lane ? mine : 0);
    };
    int32_t tokens, pages;
    const int32_t start = scan(n, sums[0], tokens), end = add31(start, n);
    const int64_t behind = (int64_t)c + n;
    const bool fits = n_raw >= 0 && c >= 0 && end <= a.max_tokens && behind <= min((int64_t)a.max_blocks * kPageTokens, (int64_t)INT32_MAX);
    const int32_t have = c > 0 ? c / kPageTokens + (c % kPageTokens != 0) : 0;
    const int32_t want = fits ? (int32_t)((behind + kPageTokens - 1) / kPageTokens) - have : 0;
    const int32_t before = scan(want, sums[1], pages), taken = add31(before, want);
    const bool served = fits && (want == 0 || taken <= stack);
    const Sequence s = {start, c, served ? before : -1, end};
    if (b < a.batch) {
        a.cu[b + 1] = end;
        if (b == 0) a.cu[0] = 0;
        a.lens_out[b] = served ? c + n : c;
        if (served && want > 0) atomicMax(&most_taken, taken);
    }
    seqs[b] = s;
    if (__syncthreads_or(n > kFew)) {
        for (int32_t w = wid * kWarpTokens; w < a.max_tokens; w += warps * kWarpTokens) fill_tokens(a, seqs, stack, w);
    } else {
        for (int x = 0; x < n && start + x < a.max_tokens; ++x) {
            const int64_t at = (int64_t)c + x;
            a.positions[start + x] = clamp31(at);
            a.slots[start + x] = served ? page_of(a, s, b, (int32_t)at / kPageTokens, (int32_t)at % kPageTokens, stack) : -1;
        }
        for (int32_t i = add31(tokens, b); i < a.max_tokens; i += blockDim.x) {
            a.positions[i] = -1;
            a.slots[i] = -1;
        }
    }
    if (b == 0) *a.free_left = stack - most_taken;
}

// Large batches: the sums by one CTA, then the tokens.
__global__ void __launch_bounds__(kTableThreads) tables_scan_kernel(const TableArgs a)
{
    pdl_launch_next();
    pdl_wait();
    scan_sequences(a, true, a.seqs, a.count);
}
__global__ void __launch_bounds__(kTableThreads) tables_fill_kernel(const TableArgs a)
{
    pdl_launch_next();
    pdl_wait();
    const int64_t w = ((int64_t)blockIdx.x * (kTableThreads / 32) + (threadIdx.x >> 5)) * kWarpTokens;
    if (w < a.max_tokens) fill_tokens(a, a.seqs, *a.count, (int32_t)w);
}

static pa_status check_table_params(const pa_table_params *p)
{
    if (!p) return fail(PA_ERR_INVALID_ARG, "params must be non-null");
    if (p->batch < 1 || p->max_blocks_per_seq < 1 || p->n_pages < 1 || p->max_tokens < 1 || p->free_capacity < 0)
        return fail(PA_ERR_INVALID_ARG, "batch, max_blocks_per_seq, n_pages and max_tokens must be positive");
    if (p->block != kPageTokens) return fail(PA_ERR_SHAPE, "block must be 64");
    if (p->batch > 65535) return fail(PA_ERR_SHAPE, "batch must be <= 65535");
    if (p->max_tokens > kMost || p->free_capacity > kMost) return fail(PA_ERR_SHAPE, "max_tokens and free_capacity must be <= 2^30");
    return PA_OK;
}

}  // namespace pa

extern "C" size_t pa_build_block_tables_workspace_bytes(const pa_table_params *p)
{
    using namespace pa;
    if (check_table_params(p) != PA_OK) return 0;
    return 16 + (size_t)p->batch * sizeof(Sequence);
}

extern "C" pa_status pa_build_block_tables(const pa_table_params *p, const int32_t *new_lens, const int32_t *cache_lens,
                                           const int32_t *free_pages, const int32_t *free_count, int32_t *block_table,
                                           int32_t *cu_seqlens, int64_t *slot_map, int32_t *positions, int32_t *lens_out,
                                           int32_t *free_left, void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace pa;
    clear_error();
    if (pa_status s = check_table_params(p)) return s;
    if (!new_lens || !cache_lens || (!free_pages && p->free_capacity > 0) || !free_count || !block_table || !cu_seqlens ||
        !slot_map || !positions || !lens_out || !free_left)
        return fail(PA_ERR_INVALID_ARG, "every array must be non-null");
    if (reinterpret_cast<uintptr_t>(slot_map) & 7) return fail(PA_ERR_ALIGNMENT, "slot_map must be 8-byte aligned");
    if (!aligned4(new_lens, cache_lens, free_pages, free_count, block_table, cu_seqlens, positions, lens_out, free_left))
        return fail(PA_ERR_ALIGNMENT, "the int32 arrays must be 4-byte aligned");
    const size_t need = pa_build_block_tables_workspace_bytes(p);
    if (!workspace || workspace_bytes < need)
        return fail(PA_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, workspace_bytes);
    if (!aligned16(workspace)) return fail(PA_ERR_ALIGNMENT, "workspace must be 16-byte aligned");
    TableArgs a;
    a.new_lens = new_lens;
    a.cache_lens = cache_lens;
    a.free_pages = free_pages;
    a.free_count = free_count;
    a.table = block_table;
    a.cu = cu_seqlens;
    a.positions = positions;
    a.lens_out = lens_out;
    a.free_left = free_left;
    a.slots = slot_map;
    a.count = static_cast<int32_t *>(workspace);
    a.seqs = reinterpret_cast<Sequence *>(static_cast<uint8_t *>(workspace) + 16);
    a.batch = p->batch;
    a.max_blocks = p->max_blocks_per_seq;
    a.n_pages = p->n_pages;
    a.max_tokens = p->max_tokens;
    a.free_capacity = p->free_capacity;
    a.vector = aligned16(slot_map) && aligned16(positions);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    constexpr int64_t kCtaTokens = kTableThreads / 32 * kWarpTokens;
    const int64_t ctas = (p->max_tokens + kCtaTokens - 1) / kCtaTokens;
    if (p->batch <= kTurn && p->max_tokens <= kStepTokens) {
        PA_CUDA_OK(launch_pdl(tables_step_kernel, dim3(1), (unsigned)(p->batch + 31) / 32 * 32, 0, st, a));
        return PA_OK;
    }
    if (p->batch <= kTurn) {
        constexpr int64_t kAtOnce = 148 * 2;  // (the sums cost as much as some tokens a thread)
        const bool apart = lens_out != cache_lens && free_left != free_count;
        PA_CUDA_OK(launch_pdl(tables_kernel, dim3((unsigned)(ctas < kAtOnce ? ctas : kAtOnce)), kTableThreads, 0, st, a, apart));
        if (!apart) PA_CUDA_OK(launch_pdl(tables_results_kernel, dim3(1), kTableThreads, 0, st, a));
        return PA_OK;
    }
    PA_CUDA_OK(launch_pdl(tables_scan_kernel, dim3(1), kTableThreads, 0, st, a));
    PA_CUDA_OK(launch_pdl(tables_fill_kernel, dim3((unsigned)ctas), kTableThreads, 0, st, a));
    return PA_OK;
}
