// pa_kv4_append, pa_kv4_read: tokens into and out of the 4-bit pages.
//
// Bound by memory: append reads 2 bytes a number and writes 9/16, read the other way round.  Instructions are next (the first form,
// eight and four features a thread, had three times as many and took 86 and 134 us for what is measured below), so a thread takes
// 16 or 8 features of a head, of K or of V, and of four tokens: what it has to work out about its place is shared, and the loads of
// four tokens are on their way at once.  The two threads of a group share its largest magnitude by a shuffle.
// Measured, 153600 tokens of 4 heads of 128 features: append 61 us, 6.6 TB/s; read as fp32 116 us, 6.2 TB/s, as bf16 89 us,
// 4.5 TB/s (chains from slot to page).  A token a thread where all threads run at once anyhow: 256 tokens, append and read, 3.1 us
// and with four tokens a thread 5.0; read alone, 4000 tokens 5.2 and 5.0, 8000 tokens 9.3 and 7.3.
// CTAs of 256 threads: append 64 us; two tokens a thread: the same within 3 %.
#include <limits.h>

#include "common.cuh"
#include "kv4.cuh"
#include "sm100_ptx.cuh"

namespace pa {

constexpr int kKv4Threads = 128;

struct Kv4CacheArgs {
    const __nv_bfloat16 *k, *v;        // append: by the strides below
    void *k_out, *v_out;               // read: contiguous
    uint8_t *pool;
    const int64_t *slots;
    int64_t page_stride, head_stride;  // bytes
    int64_t k_st, k_sh, v_st, v_sh;    // elements
    int64_t tokens, n_slots;
    int32_t Hkv;
};

// A thread's features: which of kPer parts of a head, the head, K or V, and its first token.
struct Kv4Place {
    int64_t token;
    int head, c;
    bool is_v;
};
template <int kPer, int kTokens>
__device__ __forceinline__ Kv4Place place_of(const Kv4CacheArgs &a)
{
    Kv4Place p;
    p.c = threadIdx.x % kPer;
    const uint32_t row = blockIdx.x * (kKv4Threads / kPer) + threadIdx.x / kPer;  // (below 2^32: checked on the host)
    const uint32_t group = row / (2u * (uint32_t)a.Hkv), rest = row - group * 2u * (uint32_t)a.Hkv;
    p.is_v = rest >= (uint32_t)a.Hkv;
    p.head = (int)(p.is_v ? rest - (uint32_t)a.Hkv : rest);
    p.token = (int64_t)group * kTokens;
    return p;
}
// K's or V's half of the record that holds a slot's token.
template <int D>
__device__ __forceinline__ uint8_t *half_record(const Kv4CacheArgs &a, const Kv4Place &p, int64_t slot)
{
    return a.pool + (int64_t)(uint32_t)((uint64_t)slot / kKv4Page) * a.page_stride + p.head * a.head_stride +
           (p.is_v ? Kv4Record<D>::kHalf : 0);
}
__device__ __forceinline__ uint32_t max_magnitude(uint32_t a, uint32_t b)  // of two pairs of bf16 without sign; NaN stays
{
    uint32_t d;
    asm("max.NaN.bf16x2 %0, %1, %2;\n" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

// A thread's features: half a group, j its number.  In K two words of their row, in V two halfwords each of the chunks of this group
// and of its neighbour, which a thread of the neighbour's has the other halfwords of.
template <int D, int kTokens>
__global__ void __launch_bounds__(kKv4Threads) kv4_append_kernel(const Kv4CacheArgs a)
{
    using R = Kv4Record<D>;
    constexpr int NG = R::kGroups;
    pdl_launch_next();
    const Kv4Place p = place_of<D / 16, kTokens>(a);  // (the threads of a head share its tokens)
    const int j = p.c >> 1, half = p.c & 1;
    const int64_t st = p.is_v ? a.v_st : a.k_st;
    const __nv_bfloat16 *src = (p.is_v ? a.v + p.head * a.v_sh : a.k + p.head * a.k_sh) + p.token * st + 16 * p.c;
    pdl_wait();
    int64_t slot[kTokens];
    uint4 raw[kTokens][2];
#pragma unroll
    for (int y = 0; y < kTokens; ++y) {
        const bool in = p.token + y < a.tokens;
        slot[y] = in ? a.slots[p.token + y] : -1;
#pragma unroll
        for (int x = 0; x < 2; ++x) raw[y][x] = in ? *reinterpret_cast<const uint4 *>(src + y * st + 8 * x) : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int y = 0; y < kTokens; ++y) {
        const uint32_t w[8] = {raw[y][0].x, raw[y][0].y, raw[y][0].z, raw[y][0].w, raw[y][1].x, raw[y][1].y, raw[y][1].z, raw[y][1].w};
        constexpr uint32_t kAbs = 0x7fff7fffu;
        uint32_t two = w[0] & kAbs;
#pragma unroll
        for (int i = 1; i < 8; ++i) two = max_magnitude(two, w[i] & kAbs);
        two = max_magnitude(two, __shfl_xor_sync(0xffffffffu, two, 1));
        const uint32_t top = max(two & 0xffffu, two >> 16);  // (patterns without sign are ordered as integers, NaN on top)
        // s = amax / 7 in bf16.  A quotient by 7 is never near enough to the middle of two bf16 numbers for the fp32 product to
        // round differently (it is 1/14 of a step away at least).
        const float amax = __uint_as_float(top << 16);
        const bool zero = amax < 0x1p-100f, wild = top >= 0x7f80u;
        const __nv_bfloat16 s = wild ? __ushort_as_bfloat16(0x7fc0) : __float2bfloat16_rn(zero ? 0.f : amax * (1.0f / 7.0f));
        // x / s with ties towards zero: the quotient of two 8-bit mantissas lies on a tie or at least 2^-10 from it, so the
        // nearest integer of x / s (1 - 2^-16) is the one.  Adding 1.5 x 2^23 + 8 leaves u in the low bits of a sum, and the
        // sums' patterns, 16 times each and added up, leave all nibbles but for a constant.  (A group of NaNs has any nibbles.)
        const float inv = zero || wild ? 0.f : __fdividef(1.0f - 0x1p-16f, __bfloat162float(s));
        constexpr float kMagic = 12582912.f + 8.f;
        constexpr uint32_t kPattern = 0x4b400000u, kAll = 0x11111111u;
        const uint64_t inv2 = ptx::pack_f32x2(inv, inv), magic2 = ptx::pack_f32x2(kMagic, kMagic);
        uint32_t word[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            word[x] = 0;
#pragma unroll
            for (int i = 3; i >= 0; --i) {
                const uint32_t z = w[4 * x + i];
                float n0, n1;
                ptx::unpack_f32x2(ptx::fma_f32x2(ptx::pack_f32x2(__uint_as_float(z << 16), __uint_as_float(z & 0xffff0000u)), inv2, magic2), n0, n1);
                word[x] = (word[x] * 16u + __float_as_uint(n1)) * 16u + __float_as_uint(n0);
            }
            word[x] -= kPattern * kAll;
        }
        // V: of the chunks 4 half + {0, 1}, {2, 3} the even groups' threads take the even ones, for two groups each.
        const uint32_t got = __shfl_xor_sync(0xffffffffu, __byte_perm(word[0], word[1], j & 1 ? 0x5410 : 0x7632), 2);
        if (p.is_v) {
            word[0] = __byte_perm(word[0], got, j & 1 ? 0x3254 : 0x5410);
            word[1] = __byte_perm(word[1], got, j & 1 ? 0x3276 : 0x7610);
        }
        if ((uint64_t)slot[y] >= (uint64_t)a.n_slots) continue;
        const int place = (int)((uint32_t)slot[y] % kKv4Page);
        uint8_t *record = half_record<D>(a, p, slot[y]);
        const int at = p.is_v ? (4 * (half ^ (place >> 1 & 1)) + (j & 1)) * (2 * NG) + 2 * (j & ~1) : 8 * NG * half + 4 * j;
        uint32_t *to = reinterpret_cast<uint32_t *>(record + place * R::kRow + at);
        to[0] = word[0];
        to[NG] = word[1];
        if (half == 0) *reinterpret_cast<__nv_bfloat16 *>(record + R::kScales + place * R::kScaleRow + 2 * j) = s;
    }
}

// A thread's features: 4 g + (0 .. 3) of two groups, 2 jj and 2 jj + 1, whose scales are a word, whose nibbles in V are one and in K halves
// of two.  Its stores are its neighbours' neighbours.
template <int D, bool kF32, int kTokens>
__global__ void __launch_bounds__(kKv4Threads) kv4_read_kernel(const Kv4CacheArgs a)
{
    using R = Kv4Record<D>;
    constexpr int NG = R::kGroups;
    pdl_launch_next();
    const Kv4Place p = place_of<D / 8, kTokens>(a);
    const int g = p.c & 7, jj = p.c >> 3;
    pdl_wait();
    int64_t slot[kTokens];
    uint32_t word[kTokens], scale[kTokens];
#pragma unroll
    for (int y = 0; y < kTokens; ++y) slot[y] = p.token + y < a.tokens ? a.slots[p.token + y] : -1;
#pragma unroll
    for (int y = 0; y < kTokens; ++y) {
        word[y] = 0x88888888u;
        scale[y] = 0u;
        if ((uint64_t)slot[y] < (uint64_t)a.n_slots) {
            const int place = (int)((uint32_t)slot[y] % kKv4Page);
            const uint8_t *record = half_record<D>(a, p, slot[y]), *row = record + place * R::kRow;
            scale[y] = *reinterpret_cast<const uint32_t *>(record + R::kScales + place * R::kScaleRow + 4 * jj);
            if (p.is_v) {
                word[y] = *reinterpret_cast<const uint32_t *>(row + (g ^ ((place & 2) << 1)) * (2 * NG) + 4 * jj);
            } else {
                const uint2 both = *reinterpret_cast<const uint2 *>(row + (g >> 1) * (4 * NG) + 8 * jj);
                word[y] = __byte_perm(both.x, both.y, g & 1 ? 0x7632 : 0x5410);
            }
        }
    }
    const int64_t to = (p.token * a.Hkv + p.head) * D + 64 * jj + 4 * g, step = (int64_t)a.Hkv * D;
    void *out = p.is_v ? a.v_out : a.k_out;
#pragma unroll
    for (int y = 0; y < kTokens; ++y) {
        if (p.token + y >= a.tokens) break;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const float s = __uint_as_float(x ? scale[y] & 0xffff0000u : scale[y] << 16);
            const uint64_t s2 = ptx::pack_f32x2(s, s), off2 = ptx::pack_f32x2(-8388616.f, -8388616.f);
            auto two = [&](int i) {  // (2^23 + u as a pattern)
                const uint32_t u = word[y] >> (16 * x + 4 * i);
                return ptx::mul_f32x2(s2, ptx::add_f32x2(ptx::pack_f32x2(__uint_as_float((u & 15u) | 0x4b000000u),
                                                                         __uint_as_float((u >> 4 & 15u) | 0x4b000000u)), off2));
            };
            float v0, v1, v2, v3;
            ptx::unpack_f32x2(two(0), v0, v1);
            ptx::unpack_f32x2(two(2), v2, v3);
            const int64_t at = to + y * step + 32 * x;
            if constexpr (kF32)
                *reinterpret_cast<float4 *>(static_cast<float *>(out) + at) = make_float4(v0, v1, v2, v3);
            else
                *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(out) + at) = make_uint2(ptx::cvt_bf16x2(v0, v1), ptx::cvt_bf16x2(v2, v3));
        }
    }
}

pa_status check_kv4_pool(const pa_kv4_pool &p)
{
    if (p.n_kv_heads < 1 || p.n_pages < 1) return fail(PA_ERR_INVALID_ARG, "n_kv_heads and n_pages must be positive");
    if (p.head_dim != 64 && p.head_dim != 128) return fail(PA_ERR_SHAPE, "head_dim must be 64 or 128");
    if (p.block != kKv4Page) return fail(PA_ERR_SHAPE, "block must be 64");
    if (p.n_kv_heads > 65535) return fail(PA_ERR_SHAPE, "head counts must be <= 65535");
    const int64_t record = 72ll * p.head_dim;
    if (p.head_stride < record && p.n_kv_heads > 1) return fail(PA_ERR_SHAPE, "the head stride must cover a record of %lld bytes", (long long)record);
    if (p.page_stride < record && p.n_pages > 1) return fail(PA_ERR_SHAPE, "the page stride must cover a record of %lld bytes", (long long)record);
    if ((p.page_stride % 16) || (p.head_stride % 16) || p.page_stride < 0 || p.head_stride < 0)
        return fail(PA_ERR_ALIGNMENT, "pool strides must be multiples of 16 bytes");
    if (p.n_kv_heads > 1 && p.n_pages > 1 && p.head_stride > (p.page_stride - record) / (p.n_kv_heads - 1) &&
        p.page_stride > (p.head_stride - record) / (p.n_pages - 1))
        return fail(PA_ERR_SHAPE, "the records of the pool overlap");
    return PA_OK;
}

// per: threads of a row.  *many: four tokens a thread.
static pa_status cache_args(const pa_kv4_pool *p, int per, bool *many, int64_t n_tokens, const void *kv_pool, const int64_t *slot_map, const void *k,
                            const void *v, Kv4CacheArgs *a, int64_t *ctas)
{
    if (!p) return fail(PA_ERR_INVALID_ARG, "the pool's description must be non-null");
    if (pa_status s = check_kv4_pool(*p)) return s;
    if (n_tokens < 0) return fail(PA_ERR_INVALID_ARG, "n_tokens must be >= 0");
    *ctas = 0;
    if (n_tokens == 0) return PA_OK;
    if (!kv_pool || !slot_map || !k || !v) return fail(PA_ERR_INVALID_ARG, "the pool, slot_map and the tensors must be non-null");
    if (!aligned16(kv_pool) || !aligned16(k) || !aligned16(v))
        return fail(PA_ERR_ALIGNMENT, "the pool and the tensors must be 16-byte aligned");
    if (reinterpret_cast<uintptr_t>(slot_map) & 7) return fail(PA_ERR_ALIGNMENT, "slot_map must be 8-byte aligned");
    *a = Kv4CacheArgs{};
    a->slots = slot_map;
    a->page_stride = p->page_stride;
    a->head_stride = p->head_stride;
    a->tokens = n_tokens;
    a->n_slots = (int64_t)p->n_pages * kKv4Page;
    a->Hkv = p->n_kv_heads;
    if (n_tokens > INT_MAX / p->n_kv_heads) return fail(PA_ERR_SHAPE, "too many tokens");
    *many = n_tokens * 2 * p->n_kv_heads * per > 148 * 2048;  // (measured on both sides: see above)
    const int tokens = *many ? 4 : 1;
    const int64_t rows = (n_tokens + tokens - 1) / tokens * 2 * p->n_kv_heads;
    *ctas = (rows * per + kKv4Threads - 1) / kKv4Threads;
    return PA_OK;
}

}  // namespace pa

extern "C" size_t pa_kv4_page_bytes(int32_t head_dim)
{
    return head_dim == 64 || head_dim == 128 ? (size_t)72 * head_dim : 0;
}

extern "C" pa_status pa_kv4_append(const pa_kv4_pool *pool, int64_t n_tokens, const void *k_new, const void *v_new,
                                   pa_strides k_strides, pa_strides v_strides, void *kv_pool, const int64_t *slot_map,
                                   void *stream)
{
    using namespace pa;
    clear_error();
    Kv4CacheArgs a;
    int64_t ctas;
    bool many;
    if (pa_status s = cache_args(pool, pool ? pool->head_dim / 16 : 0, &many, n_tokens, kv_pool, slot_map, k_new, v_new, &a, &ctas)) return s;
    for (const pa_strides &s : {k_strides, v_strides}) {
        if (s.seq < 0 || s.head < 0) return fail(PA_ERR_SHAPE, "strides must be >= 0");
        if ((s.seq % 8) || (s.head % 8)) return fail(PA_ERR_ALIGNMENT, "strides must be multiples of 8 elements (16 bytes)");
    }
    if (ctas == 0) return PA_OK;
    a.k = static_cast<const __nv_bfloat16 *>(k_new);
    a.v = static_cast<const __nv_bfloat16 *>(v_new);
    a.pool = static_cast<uint8_t *>(kv_pool);
    a.k_st = k_strides.seq;
    a.k_sh = k_strides.head;
    a.v_st = v_strides.seq;
    a.v_sh = v_strides.head;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    auto launch = [&](auto kernel) { return launch_pdl(kernel, dim3((unsigned)ctas), kKv4Threads, 0, st, a); };
    static void (*const kernels[2][2])(const Kv4CacheArgs) = {{kv4_append_kernel<64, 1>, kv4_append_kernel<64, 4>},
                                                              {kv4_append_kernel<128, 1>, kv4_append_kernel<128, 4>}};
    PA_CUDA_OK(launch(kernels[pool->head_dim == 128][many]));
    return PA_OK;
}

extern "C" pa_status pa_kv4_read(const pa_kv4_pool *pool, int64_t n_tokens, const void *kv_pool, const int64_t *slot_map,
                                 void *k_out, void *v_out, pa_dtype dtype, void *stream)
{
    using namespace pa;
    clear_error();
    Kv4CacheArgs a;
    int64_t ctas;
    bool many;
    if (dtype != PA_BF16 && dtype != PA_F32) return fail(PA_ERR_INVALID_ARG, "bad dtype");
    if (pa_status s = cache_args(pool, pool ? pool->head_dim / 8 : 0, &many, n_tokens, kv_pool, slot_map, k_out, v_out, &a, &ctas)) return s;
    if (ctas == 0) return PA_OK;
    a.pool = static_cast<uint8_t *>(const_cast<void *>(kv_pool));
    a.k_out = k_out;
    a.v_out = v_out;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    auto launch = [&](auto kernel) { return launch_pdl(kernel, dim3((unsigned)ctas), kKv4Threads, 0, st, a); };
    static void (*const kernels[2][2][2])(const Kv4CacheArgs) = {
        {{kv4_read_kernel<64, false, 1>, kv4_read_kernel<64, false, 4>}, {kv4_read_kernel<64, true, 1>, kv4_read_kernel<64, true, 4>}},
        {{kv4_read_kernel<128, false, 1>, kv4_read_kernel<128, false, 4>}, {kv4_read_kernel<128, true, 1>, kv4_read_kernel<128, true, 4>}}};
    PA_CUDA_OK(launch(kernels[pool->head_dim == 128][dtype == PA_F32][many]));
    return PA_OK;
}
