// pa_build_block_tables: pages, slots and positions of a batch's new tokens from the sequences' lengths.
//
// Two prefix sums over the batch (new tokens, pages wanted), then one entry per token.  A thread looks up the sequence of its
// tokens by bisection over the sums.  Every fresh block has exactly one first token, and it is this token's thread that
// writes the table entry; a token's own page comes from the table for blocks that the sequence had and from the stack
// for fresh ones, so no thread reads what another one writes.
#include <limits.h>

#include "common.cuh"

namespace pa {

constexpr int kPageTokens = 64;
constexpr int kScanThreads = 1024;
constexpr int kSmallBatch = 1024;    // one CTA does it all up to this many sequences ...
constexpr int kSmallTokens = 4096;   // ... and this many places for tokens
constexpr int kFillThreads = 256;
constexpr int kFillTokens = 4;       // tokens per thread and turn

// What the tokens of a sequence need to know.
struct Sequence {
    int32_t start;   // its first token (held at INT32_MAX)
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

// Inclusive sums of a number over the CTA's threads; `sums`: room for one number a warp.
__device__ __forceinline__ int64_t scan_cta(int64_t x, int64_t *sums)
{
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, warps = blockDim.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const int64_t up = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += up;
    }
    if (lane == 31) sums[wid] = x;
    __syncthreads();
    int64_t before = lane < wid && lane < warps ? sums[lane] : 0;
#pragma unroll
    for (int o = 16; o > 0; o /= 2) before += __shfl_xor_sync(0xffffffffu, before, o);
    return x + before;
}

// The sequences' sums, by one CTA; writes cu, lens_out, free_left and, for the tokens, seqs[] and the stack's height.
__device__ __forceinline__ void scan_sequences(const TableArgs &a, Sequence *seqs, int32_t *height)
{
    __shared__ int64_t sums[2][32], total[2];
    __shared__ int32_t most_taken;
    const int tid = threadIdx.x, threads = blockDim.x;
    int32_t stack = *a.free_count;
    stack = stack < 0 ? 0 : stack > a.free_capacity ? a.free_capacity : stack;
    if (tid == 0) most_taken = 0;
    int64_t tokens = 0, wanted = 0;  // of the sequences before this turn's
    for (int b0 = 0; b0 < a.batch; b0 += threads) {
        const int b = b0 + tid;
        const bool in = b < a.batch;
        const int32_t n_raw = in ? a.new_lens[b] : 0, c = in ? a.cache_lens[b] : 0;
        const int64_t n = n_raw > 0 ? n_raw : 0, upto = tokens + scan_cta(n, sums[0]);
        const int64_t have = c > 0 ? ((int64_t)c + kPageTokens - 1) / kPageTokens : 0;
        const int64_t need = ((int64_t)c + n + kPageTokens - 1) / kPageTokens;
        // (a length held in int32 has to fit behind the call as well)
        const bool fits = in && c >= 0 && n_raw >= 0 && need <= a.max_blocks && upto <= a.max_tokens &&
                          (int64_t)c + n <= INT32_MAX;
        const int64_t want = fits ? need - have : 0, pages = wanted + scan_cta(want, sums[1]);
        const bool served = fits && (want == 0 || pages <= stack);
        if (in) {
            a.cu[b] = clamp31(upto - n);
            if (b == a.batch - 1) a.cu[a.batch] = clamp31(upto);
            a.lens_out[b] = served ? (int32_t)(c + n) : c;
            seqs[b] = Sequence{clamp31(upto - n), c, served ? (int32_t)(pages - want) : -1, clamp31(upto)};
            if (served && want > 0) atomicMax(&most_taken, (int32_t)pages);
        }
        if (tid == threads - 1) {
            total[0] = upto;
            total[1] = pages;
        }
        __syncthreads();
        tokens = total[0];
        wanted = total[1];
    }
    if (tid == 0) {
        *height = stack;
        *a.free_left = stack - most_taken;
    }
}

// kFillTokens tokens from i0 on.
__device__ __forceinline__ void fill_tokens(const TableArgs &a, const Sequence *seqs, int32_t height, int32_t i0)
{
    // The first sequence that ends behind token i0.
    int lo = 0, hi = a.batch;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (seqs[mid].end <= i0) lo = mid + 1;
        else hi = mid;
    }
    int b = lo;
    Sequence s = {};
    if (b < a.batch) s = seqs[b];
    int64_t slot[kFillTokens];
    int32_t position[kFillTokens];
    int32_t block = -1, page = -1;  // the block that `page` belongs to, of sequence b
#pragma unroll
    for (int x = 0; x < kFillTokens; ++x) {
        const int32_t i = i0 + x;
        while (b < a.batch && i >= s.end) {
            block = -1;
            if (++b < a.batch) s = seqs[b];
        }
        slot[x] = -1;
        position[x] = -1;
        if (b >= a.batch || i >= a.max_tokens) continue;
        const int64_t at = (int64_t)s.cached + (i - s.start);
        position[x] = clamp31(at);
        if (s.first < 0) continue;  // refused
        const int32_t j = (int32_t)(at / kPageTokens), place = (int32_t)(at % kPageTokens);
        if (j != block) {
            block = j;
            int32_t *entry = a.table + (int64_t)b * a.max_blocks + j;
            const int32_t have = s.cached / kPageTokens + (s.cached % kPageTokens != 0);
            if (j < have) {
                page = *entry;
            } else {
                page = a.free_pages[height - 1 - (s.first + (j - have))];
                if (place == 0) *entry = page;
            }
        }
        if (page >= 0 && page < a.n_pages) slot[x] = (int64_t)page * kPageTokens + place;
    }
    if (a.vector && i0 + kFillTokens <= a.max_tokens) {
        longlong2 *to = reinterpret_cast<longlong2 *>(a.slots + i0);
        to[0] = make_longlong2(slot[0], slot[1]);
        to[1] = make_longlong2(slot[2], slot[3]);
        *reinterpret_cast<int4 *>(a.positions + i0) = make_int4(position[0], position[1], position[2], position[3]);
    } else {
#pragma unroll
        for (int x = 0; x < kFillTokens; ++x)
            if (i0 + x < a.max_tokens) {
                a.slots[i0 + x] = slot[x];
                a.positions[i0 + x] = position[x];
            }
    }
}

// One CTA: sums and tokens.
__global__ void __launch_bounds__(kScanThreads) tables_small_kernel(const TableArgs a)
{
    __shared__ Sequence seqs[kSmallBatch];
    __shared__ int32_t height;
    pdl_launch_next();
    pdl_wait();
    scan_sequences(a, seqs, &height);
    __syncthreads();
    for (int32_t i = threadIdx.x * kFillTokens; i < a.max_tokens; i += blockDim.x * kFillTokens)
        fill_tokens(a, seqs, height, i);
}

__global__ void __launch_bounds__(kScanThreads) tables_scan_kernel(const TableArgs a)
{
    pdl_launch_next();
    pdl_wait();
    scan_sequences(a, a.seqs, a.count);
}

__global__ void __launch_bounds__(kFillThreads) tables_fill_kernel(const TableArgs a)
{
    pdl_launch_next();
    pdl_wait();
    const int64_t i = ((int64_t)blockIdx.x * kFillThreads + threadIdx.x) * kFillTokens;
    if (i < a.max_tokens) fill_tokens(a, a.seqs, *a.count, (int32_t)i);
}

static pa_status check_table_params(const pa_table_params *p)
{
    if (!p) return fail(PA_ERR_INVALID_ARG, "params must be non-null");
    if (p->batch < 1 || p->max_blocks_per_seq < 1 || p->n_pages < 1 || p->max_tokens < 1 || p->free_capacity < 0)
        return fail(PA_ERR_INVALID_ARG, "batch, max_blocks_per_seq, n_pages and max_tokens must be positive");
    if (p->block != kPageTokens) return fail(PA_ERR_SHAPE, "block must be 64");
    if (p->batch > 65535) return fail(PA_ERR_SHAPE, "batch must be <= 65535");
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
    auto threads_for = [](int64_t n) { return (unsigned)(n >= kScanThreads ? kScanThreads : (n + 31) / 32 * 32); };
    if (p->batch <= kSmallBatch && p->max_tokens <= kSmallTokens) {
        const int64_t quads = (p->max_tokens + kFillTokens - 1) / kFillTokens;
        PA_CUDA_OK(launch_pdl(tables_small_kernel, dim3(1), threads_for(p->batch > quads ? p->batch : quads), 0, st, a));
        return PA_OK;
    }
    PA_CUDA_OK(launch_pdl(tables_scan_kernel, dim3(1), threads_for(p->batch), 0, st, a));
    const int64_t per_cta = kFillThreads * kFillTokens;
    PA_CUDA_OK(launch_pdl(tables_fill_kernel, dim3((unsigned)((p->max_tokens + per_cta - 1) / per_cta)), kFillThreads, 0, st, a));
    return PA_OK;
}
