// pa_kv4_append, pa_kv4_read: tokens into and out of the 4-bit pages.
//
// Bound by memory: append reads 2 bytes a number and writes 9/16.  A thread takes eight features (16 bytes in, one 32-bit word of
// nibbles out); the four threads of a group share its largest magnitude by shuffles.
#include <limits.h>

#include "common.cuh"
#include "kv4.cuh"

namespace pa {

constexpr int kKv4Threads = 256;

struct Kv4CacheArgs {
    const __nv_bfloat16 *k, *v;        // append: by the strides below
    void *k_out, *v_out;               // read: contiguous
    uint8_t *pool;
    const int64_t *slots;
    int64_t page_stride, head_stride;  // bytes
    int64_t k_st, k_sh, v_st, v_sh;    // elements
    int64_t tokens, n_slots;
    int32_t Hkv, pieces;               // pieces of eight features of a token: 2 Hkv D / 8, K's then V's
};

struct Piece {
    int64_t token;
    int head, c;  // KV head, number of the piece in its row
    bool is_v;
};
template <int D>
__device__ __forceinline__ Piece piece_of(const Kv4CacheArgs &a, int64_t x)
{
    Piece p;
    p.token = x / a.pieces;
    int rest = (int)(x - p.token * a.pieces);
    p.is_v = rest >= a.pieces / 2;
    if (p.is_v) rest -= a.pieces / 2;
    p.head = rest / (D / 8);
    p.c = rest % (D / 8);
    return p;
}
// K's or V's half of the record that holds a slot's token.
template <int D>
__device__ __forceinline__ uint8_t *half_record(const Kv4CacheArgs &a, const Piece &p, int64_t slot)
{
    return a.pool + (slot / kKv4Page) * a.page_stride + p.head * a.head_stride + (p.is_v ? Kv4Record<D>::kHalf : 0);
}
// Byte in its row at which a K piece's word, or the halfwords of a V piece, stand.
template <int D>
__device__ __forceinline__ int k_byte(int c) { return ((c & 3) * Kv4Record<D>::kGroups + (c >> 2)) * 4; }
template <int D>
__device__ __forceinline__ int v_byte(int c, int place, int upper)
{
    const int chunk = (2 * (c & 3) + upper) ^ ((place & 2) << 1);
    return chunk * (2 * Kv4Record<D>::kGroups) + 2 * (c >> 2);
}

template <int D>
__global__ void __launch_bounds__(kKv4Threads) kv4_append_kernel(const Kv4CacheArgs a)
{
    using R = Kv4Record<D>;
    pdl_launch_next();
    const int64_t x = (int64_t)blockIdx.x * kKv4Threads + threadIdx.x;
    const bool in = x < a.tokens * a.pieces;  // (the four threads of a group are in or out together)
    const Piece p = piece_of<D>(a, in ? x : 0);
    pdl_wait();
    const int64_t slot = in ? a.slots[p.token] : -1;
    uint4 raw = make_uint4(0u, 0u, 0u, 0u);
    if (in) {
        const __nv_bfloat16 *src = p.is_v ? a.v + p.token * a.v_st + p.head * a.v_sh : a.k + p.token * a.k_st + p.head * a.k_sh;
        raw = *reinterpret_cast<const uint4 *>(src + 8 * p.c);
    }
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
    // The largest magnitude: bf16 patterns without their sign are ordered as integers (infinity and NaN on top).
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, max(w[i] & 0x7fffu, (w[i] >> 16) & 0x7fffu));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    if (slot < 0 || slot >= a.n_slots) return;
    // s = amax / 7 in bf16.  A quotient by 7 is never near enough to the middle of two bf16 numbers for the fp32 product to
    // round differently (it is 1/14 of a step away at least).
    const float amax = __uint_as_float(top << 16);
    const bool zero = amax < 7.8886090522101181e-31f;  // 2^-100
    __nv_bfloat16 s = __float2bfloat16_rn(zero ? 0.f : amax * (1.0f / 7.0f));
    const bool wild = top >= 0x7f80u;
    if (wild) s = __ushort_as_bfloat16(0x7fc0);
    // x / s with ties towards zero: the quotient of two 8-bit mantissas lies on a tie or at least 2^-10 from it, so the
    // nearest integer of x / s (1 - 2^-16) is the one.
    const float inv = zero || wild ? 0.f : (1.0f - 0x1p-16f) / __bfloat162float(s);
    uint32_t word = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        // (adding 1.5 x 2^23 leaves the nearest integer in the low bits; a wild or zero group has nibbles of 8)
        const float lo = __uint_as_float(w[i] << 16), hi = __uint_as_float(w[i] & 0xffff0000u);
        const uint32_t n0 = inv != 0.f ? __float_as_uint(fmaf(lo, inv, 12582912.f + 8.f)) : 8u;
        const uint32_t n1 = inv != 0.f ? __float_as_uint(fmaf(hi, inv, 12582912.f + 8.f)) : 8u;
        word |= (n0 & 15u) << (8 * i) | (n1 & 15u) << (8 * i + 4);
    }
    const int place = (int)(slot % kKv4Page);
    uint8_t *half = half_record<D>(a, p, slot), *row = half + place * R::kRow;
    if (p.is_v) {
        *reinterpret_cast<uint16_t *>(row + v_byte<D>(p.c, place, 0)) = (uint16_t)word;
        *reinterpret_cast<uint16_t *>(row + v_byte<D>(p.c, place, 1)) = (uint16_t)(word >> 16);
    } else {
        *reinterpret_cast<uint32_t *>(row + k_byte<D>(p.c)) = word;
    }
    if ((p.c & 3) == 0)
        *reinterpret_cast<__nv_bfloat16 *>(half + R::kScales + place * R::kScaleRow + 2 * (p.c >> 2)) = s;
}

template <int D, bool kF32>
__global__ void __launch_bounds__(kKv4Threads) kv4_read_kernel(const Kv4CacheArgs a)
{
    using R = Kv4Record<D>;
    pdl_launch_next();
    const int64_t x = (int64_t)blockIdx.x * kKv4Threads + threadIdx.x;
    if (x >= a.tokens * a.pieces) return;
    const Piece p = piece_of<D>(a, x);
    pdl_wait();
    const int64_t slot = a.slots[p.token];
    uint32_t word = 0x88888888u;
    float s = 0.f;
    if (slot >= 0 && slot < a.n_slots) {
        const int place = (int)(slot % kKv4Page);
        const uint8_t *half = half_record<D>(a, p, slot), *row = half + place * R::kRow;
        if (p.is_v)
            word = *reinterpret_cast<const uint16_t *>(row + v_byte<D>(p.c, place, 0)) |
                   (uint32_t)*reinterpret_cast<const uint16_t *>(row + v_byte<D>(p.c, place, 1)) << 16;
        else
            word = *reinterpret_cast<const uint32_t *>(row + k_byte<D>(p.c));
        s = __bfloat162float(*reinterpret_cast<const __nv_bfloat16 *>(half + R::kScales + place * R::kScaleRow + 2 * (p.c >> 2)));
    }
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = s * (float)((int)((word >> (4 * i)) & 15u) - 8);
    const int64_t at = ((p.token * a.Hkv + p.head) * (D / 8) + p.c) * 8;
    void *out = p.is_v ? a.v_out : a.k_out;
    if (kF32) {
        float4 *to = reinterpret_cast<float4 *>(static_cast<float *>(out) + at);
        to[0] = make_float4(y[0], y[1], y[2], y[3]);
        to[1] = make_float4(y[4], y[5], y[6], y[7]);
    } else {
        uint32_t h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(y[2 * i], y[2 * i + 1]);
            h[i] = *reinterpret_cast<const uint32_t *>(&b);
        }
        *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(out) + at) = make_uint4(h[0], h[1], h[2], h[3]);
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
    return PA_OK;
}

static pa_status cache_args(const pa_kv4_pool *p, int64_t n_tokens, const void *kv_pool, const int64_t *slot_map, const void *k,
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
    a->pieces = 2 * p->n_kv_heads * (p->head_dim / 8);
    if (n_tokens > ((int64_t)INT_MAX * kKv4Threads) / a->pieces) return fail(PA_ERR_SHAPE, "too many tokens");
    *ctas = (n_tokens * a->pieces + kKv4Threads - 1) / kKv4Threads;
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
    if (pa_status s = cache_args(pool, n_tokens, kv_pool, slot_map, k_new, v_new, &a, &ctas)) return s;
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
    PA_CUDA_OK(pool->head_dim == 128 ? launch(kv4_append_kernel<128>) : launch(kv4_append_kernel<64>));
    return PA_OK;
}

extern "C" pa_status pa_kv4_read(const pa_kv4_pool *pool, int64_t n_tokens, const void *kv_pool, const int64_t *slot_map,
                                 void *k_out, void *v_out, pa_dtype dtype, void *stream)
{
    using namespace pa;
    clear_error();
    Kv4CacheArgs a;
    int64_t ctas;
    if (dtype != PA_BF16 && dtype != PA_F32) return fail(PA_ERR_INVALID_ARG, "bad dtype");
    if (pa_status s = cache_args(pool, n_tokens, kv_pool, slot_map, k_out, v_out, &a, &ctas)) return s;
    if (ctas == 0) return PA_OK;
    a.pool = static_cast<uint8_t *>(const_cast<void *>(kv_pool));
    a.k_out = k_out;
    a.v_out = v_out;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    auto launch = [&](auto kernel) { return launch_pdl(kernel, dim3((unsigned)ctas), kKv4Threads, 0, st, a); };
    const bool f32 = dtype == PA_F32;
    PA_CUDA_OK(pool->head_dim == 128 ? (f32 ? launch(kv4_read_kernel<128, true>) : launch(kv4_read_kernel<128, false>))
                                     : (f32 ? launch(kv4_read_kernel<64, true>) : launch(kv4_read_kernel<64, false>)));
    return PA_OK;
}
