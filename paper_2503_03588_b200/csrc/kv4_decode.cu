// pa_decode_kv4: one query token per sequence against 4-bit pages (kv4.cuh) under the PowerAttention row of its position.
//
// The mathematics.  A key is k = s (u - 8) per group of 32 features, u its nibble, so a logit is
//   S = sum_j s_kj <q_j, u_kj - 8>   (j: the groups),
// with integer operands that 16 bits hold exactly: the products run on the tensor cores (m16n8k16, keys as the 16 rows, the
// query heads as the 8 columns) and each group's sum is scaled in fp32.  The output is
//   O = sum_k (p_k s_kj) (u_kj - 8),
// V's scales folded into the weights: one 16-bit weight per key and group.
//
// Logits take fp16 operands: q is bf16, and each head is multiplied by a power of two so that its largest entry lies in [2^10, 2^11)
// and fits (an entry is off by 2^-35 of the largest at most, which smaller entries than 2^-27 of it feel).  Weights are bf16,
// since V's scales may differ by any factor from key to key and from group to group, in two parts (one would be off by as much
// as the output's own rounding), for fp32 outputs in three.
//
// The nibbles become 16-bit numbers without conversions.  K: w & 0x000f000f is two fp16 subnormals, u 2^-24, and w & 0x00f000f0 is
// 16 times as much, for which the queries of the former are multiplied by 16; -8 sum_i q_i is what the accumulator starts
// with.  V: (w & 0x000f000f) | 0x4300 is 128 + u in bf16, and an addition of -136 leaves u - 8.  (Products of 128 + u from which others are
// taken off would be 20 times the values, and overflow where the values do not.)  K rows are stored so that
// a thread's 16 bytes hold its share of every group; V rows so that the same halfwords of two tokens, put side by side by a byte
// permutation, are the fragments' key pairs.  Shared memory is read without bank conflicts and without ldmatrix.
//
// Two kernels.  Few rows (sequence and KV head): kv4_cluster_kernel, a thread-block cluster per row, bound by latency.  Many, or
// long ones: kv4_range_kernel, every warp of the device an equal share of all rows' blocks, bound by instructions and memory.
// A key block is one page and KV head, 72 D contiguous bytes, copied to shared memory in bulk.
#include <cuda_fp16.h>
#include <math.h>

#include <mutex>
#include <type_traits>

#include "common.cuh"
#include "kv4.cuh"
#include "layout_rule.cuh"
#include "sm100_ptx.cuh"

namespace pa {

constexpr int kD4MaxGroup = 8;
constexpr size_t kD4StatusBytes = 256;
constexpr int kD4MaxSmem = 226 * 1024;  // (227 KB less some static shared memory)
constexpr long long kD4WaitCycles = 2000000000ll;  // ~1 s
// Weights are 2^(S - m).  m is set this far above the largest logit so far and moves once a logit exceeds it: no weight is above 1
// (values as large as fp32 holds are summed without overflow where the sum by the true weights has none), and sums are rescaled
// seldom.
constexpr float kD4Grow = 6.f;

struct Kv4Args {
    const __nv_bfloat16 *q;
    const uint8_t *pool;
    const int32_t *table, *lens;
    float *parts;    // (range kernel) [CTAs][2] results of rows that other CTAs have parts of
    int32_t *status;
    void *o;
    float *lse;
    int64_t page_stride, head_stride, max_len;
    int32_t table_stride, n_pages, batch, Hkv, G, W, S, R, stages, clear_status;
    int32_t whole_rows;  // (range kernel) ranges begin and end with rows
    float scale_log2;
    long long wait_cycles;
};

// D(16x8, fp32) = A(16x16, row-major) * B(16x8, column-major) + C, one warp.
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};\n"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The same with C = c0 in even columns and c1 in odd ones.
__device__ __forceinline__ void mma_f16_from(float (&d)[4], float c0, float c1, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                             uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %10, %11};\n"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1));
}
__device__ __forceinline__ void mma_b16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};\n"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// (a & b) | c in one instruction: left to itself the compiler takes two, each with a constant of its own.
__device__ __forceinline__ uint32_t and_or(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t d;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;\n" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
// The lowest nibble of each half of a word as fp16 u 2^-24, and the one above it as u 2^-20.
__device__ __forceinline__ uint32_t nib_lo(uint32_t w) { return w & 0x000f000fu; }
__device__ __forceinline__ uint32_t nib_hi(uint32_t w) { return w & 0x00f000f0u; }
// The lowest nibble of each half as bf16 u - 8: 128 + u, less 136.
__device__ __forceinline__ uint32_t nib_bf16(uint32_t w)
{
    uint32_t d;
    asm("add.rn.bf16x2 %0, %1, %2;\n" : "=r"(d) : "r"(and_or(w, 0x000f000fu, 0x43004300u)), "r"(0xc308c308u));
    return d;
}
__device__ __forceinline__ uint32_t bf2_mul(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("mul.rn.bf16x2 %0, %1, %2;\n" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
// a b + c and a b - c, two at a time, rounded once.
__device__ __forceinline__ uint32_t bf2_fma(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t d;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;\n" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
__device__ __forceinline__ uint32_t bf2_fms(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t d;
    asm("{\n\t.reg .b32 n;\n\tneg.bf16x2 n, %3;\n\tfma.rn.bf16x2 %0, %1, %2, n;\n\t}\n" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
__device__ __forceinline__ uint32_t cvt_f16x2(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;\n" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// The transpose of an 8 x 8 matrix of 16-bit elements; lane (g, t) holds elements 2t, 2t + 1 of row g.
__device__ __forceinline__ uint32_t transpose8(uint32_t a)
{
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
template <int kWords>
__device__ __forceinline__ void lds_words(uint32_t addr, uint32_t (&w)[kWords])
{
    if constexpr (kWords == 4)
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];\n" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(addr) : "memory");
    else if constexpr (kWords == 2)
        asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];\n" : "=r"(w[0]), "=r"(w[1]) : "r"(addr) : "memory");
    else
        asm volatile("ld.shared.u32 %0, [%1];\n" : "=r"(w[0]) : "r"(addr) : "memory");
}

// What a thread (g, t) = (lane / 4, lane % 4) reads of a tile of 16 keys.  Row r < 8 of the 16 x 16 fragments is key r ^ (r / 4)
// of the tile, row r + 8 that plus 8: a permutation under which a warp's reads of K rows and of V rows fall into different
// banks.
template <int D>
struct Kv4Lane {
    using R4 = Kv4Record<D>;
    int key;                         // rows g and g + 8 of S: this key and that plus 8
    uint32_t off_k, off_s;           // in K's half: its words, its scales
    int key0, key1;                  // columns 2t and 2t + 1 of P (and these plus 8 of 2t + 8, 2t + 9)
    uint32_t off_v0, off_v1;         // in V's half: these keys' chunks, their scales
    uint32_t off_s0, off_s1;
    __device__ __forceinline__ Kv4Lane(int lane)
    {
        const int g = lane >> 2, t = lane & 3;
        key = g ^ (g >> 2);
        off_k = (uint32_t)(key * R4::kRow + t * 4 * R4::kGroups);
        off_s = (uint32_t)(R4::kScales + key * R4::kScaleRow);
        key0 = (2 * t) ^ (t >> 1);
        key1 = (2 * t + 1) ^ (t >> 1);
        auto chunk = [&](int k) { return (uint32_t)(k * R4::kRow + (g ^ ((k & 2) << 1)) * 2 * R4::kGroups); };
        off_v0 = chunk(key0);
        off_v1 = chunk(key1);
        off_s0 = (uint32_t)(R4::kScales + key0 * R4::kScaleRow);
        off_s1 = (uint32_t)(R4::kScales + key1 * R4::kScaleRow);
    }
};

// A row's queries as the B operand: head g, features 32 j + 8 t + {0, 4}, {1, 5}, {2, 6}, {3, 7}.
template <int D>
struct Kv4Query {
    static constexpr int NG = D / 32;
    static constexpr uint32_t kMore = 1u << 31;  // (in `more` of every lane, if any head of the warp has some)
    uint32_t f[NG][4];
    float o0[NG], o1[NG];  // of heads 2t and 2t + 1: -8 times the sum of the group's features, as the products come (2^-20)
    float c0, c1;          // of the same heads: the powers of two, the softmax scale, log2 e
    uint32_t more;         // of the same heads (halves): exponents that c0, c1 have no room for; 0 but for heads from 2^117 on
    static __device__ __forceinline__ void load(const Kv4Args &a, uint32_t row, int lane, uint4 (&raw)[NG])
    {
        const int g = lane >> 2, t = lane & 3;
        const __nv_bfloat16 *q = a.q + ((int64_t)row * a.G + (g < a.G ? g : 0)) * D + 8 * t;
#pragma unroll
        for (int j = 0; j < NG; ++j) raw[j] = g < a.G ? *reinterpret_cast<const uint4 *>(q + 32 * j) : make_uint4(0u, 0u, 0u, 0u);
    }
    __device__ __forceinline__ void set(const uint4 (&raw)[NG], float scale_log2, int lane)
    {
        const int t = lane & 3;
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < NG; ++j)
            for (uint32_t x : {raw[j].x, raw[j].y, raw[j].z, raw[j].w}) top = max(top, max(x & 0x7fffu, (x >> 16) & 0x7fffu));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // f is q 2^10 / 2^e with 2^e <= max |q| < 2^(e + 1) (q 2^14 / 2^e where the nibbles come as u 2^-24): products are u q 2^(-10 - e).
        const uint32_t field = min(max(top >> 7, 27u), 254u), fits = min(field, 243u);  // e + 127 (heads below 2^-100 lose bits)
        const float down = __uint_as_float((264u - field) << 23), up = __uint_as_float((fits + 10u) << 23) * scale_log2;
        c0 = __shfl_sync(0xffffffffu, up, 8 * t);
        c1 = __shfl_sync(0xffffffffu, up, 8 * t + 4);
        more = __any_sync(0xffffffffu, field > fits) ? __byte_perm(__shfl_sync(0xffffffffu, field - fits, 8 * t),
                                                                   __shfl_sync(0xffffffffu, field - fits, 8 * t + 4), 0x5410) | kMore : 0u;
#pragma unroll
        for (int j = 0; j < NG; ++j) {
            f[j][0] = cvt_f16x2(bf16_lo(raw[j].x) * (16.f * down), bf16_lo(raw[j].z) * (16.f * down));
            f[j][1] = cvt_f16x2(bf16_hi(raw[j].x) * down, bf16_hi(raw[j].z) * down);
            f[j][2] = cvt_f16x2(bf16_lo(raw[j].y) * (16.f * down), bf16_lo(raw[j].w) * (16.f * down));
            f[j][3] = cvt_f16x2(bf16_hi(raw[j].y) * down, bf16_hi(raw[j].w) * down);
            float2 x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = __half22float2(*reinterpret_cast<const __half2 *>(&f[j][i]));
            float sum = ((x[0].x + x[0].y) + (x[2].x + x[2].y)) * 0.0625f + ((x[1].x + x[1].y) + (x[3].x + x[3].y));
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
            sum *= -8.f * 0x1p-20f;
            o0[j] = __shfl_sync(0xffffffffu, sum, 8 * t);
            o1[j] = __shfl_sync(0xffffffffu, sum, 8 * t + 4);
        }
    }
};

// S^T = K Q^T of a tile of the half at `half`: rows g and g + 8 of heads 2t, 2t + 1, in powers of two.  Rounded here, once: the
// largest logit of a row less itself is 0 then, however large (a fused product less the rounded maximum is off by half a step of
// the logit, which from 2^30 on is more than the exponents of fp32 hold).
template <int D>
__device__ __forceinline__ void kv4_logits(uint32_t half, int tile, const Kv4Lane<D> &at, const Kv4Query<D> &q, float (&sx)[4])
{
    using R4 = Kv4Record<D>;
    constexpr int NG = R4::kGroups, NW = NG / 2;
    const uint32_t k = half + (uint32_t)(tile * 16 * R4::kRow) + at.off_k, ks = half + (uint32_t)(tile * 16 * R4::kScaleRow) + at.off_s;
    uint32_t ka[NG], kb[NG], sa[NW], sb[NW];
    lds_words(k, ka);
    lds_words(k + 8 * R4::kRow, kb);
    lds_words(ks, sa);
    lds_words(ks + 8 * R4::kScaleRow, sb);
#pragma unroll
    for (int x = 0; x < 4; ++x) sx[x] = 0.f;
#pragma unroll
    for (int j = 0; j < NG; ++j) {
        float d[4];
        mma_f16_from(d, q.o0[j], q.o1[j], nib_lo(ka[j]), nib_lo(kb[j]), nib_hi(ka[j]), nib_hi(kb[j]), q.f[j][0], q.f[j][1]);
        const uint32_t u = ka[j] >> 8, v = kb[j] >> 8;
        mma_f16(d, nib_lo(u), nib_lo(v), nib_hi(u), nib_hi(v), q.f[j][2], q.f[j][3]);
        const float s0 = j & 1 ? bf16_hi(sa[j / 2]) : bf16_lo(sa[j / 2]);
        const float s1 = j & 1 ? bf16_hi(sb[j / 2]) : bf16_lo(sb[j / 2]);
        sx[0] = fmaf(s0, d[0], sx[0]);
        sx[1] = fmaf(s0, d[1], sx[1]);
        sx[2] = fmaf(s1, d[2], sx[2]);
        sx[3] = fmaf(s1, d[3], sx[3]);
    }
    if (q.more) {  // (all lanes or none)
        const float x0 = __uint_as_float((127u + (q.more & 0xffu)) << 23), x1 = __uint_as_float((127u + (q.more >> 16 & 0xffu)) << 23);
        sx[0] *= x0;
        sx[1] *= x1;
        sx[2] *= x0;
        sx[3] *= x1;
    }
    sx[0] = __fmul_rn(sx[0], q.c0);
    sx[1] = __fmul_rn(sx[1], q.c1);
    sx[2] = __fmul_rn(sx[2], q.c0);
    sx[3] = __fmul_rn(sx[3], q.c1);
}

// O^T += V^T P^T of the tile in V's half `half`: p are the weights of rows g, g + 8 and heads 2t, 2t + 1; of a partial block's
// tile `keys` exist.  acc[2 j + h]: features 32 j + 4 g + 2 h + {0, 1}, heads 2t, 2t + 1.
// Weights times scales come as two bf16 parts, so that they are off by 2^-14 at most (one part: 2^-7, more than the output's own
// rounding).  For bf16 outputs the weights' two parts are transposed into the B operand once and multiplied by the keys' scales
// there, two at a time: the first product is rounded, what that leaves is exact (8 x 8 bits less their upper 8) and goes into the
// second one.  That is a quarter of the conversions and transposes.  For fp32 outputs they are scaled in fp32, group by group, and
// all 24 bits of the products come in three parts.
template <int D, bool kF32>
__device__ __forceinline__ void kv4_values(uint32_t half, int tile, const Kv4Lane<D> &at, const float (&p)[4], bool partial, int keys,
                                           float (&acc)[D / 16][4])
{
    using R4 = Kv4Record<D>;
    constexpr int NG = R4::kGroups, NW = NG / 2;
    const uint32_t v = half + (uint32_t)(tile * 16 * R4::kRow), vs = half + (uint32_t)(tile * 16 * R4::kScaleRow);
    uint32_t wa[NW], wb[NW], wc[NW], wd[NW];  // the keys of columns 2t, 2t + 1, and these plus 8
    lds_words(v + at.off_v0, wa);
    lds_words(v + at.off_v1, wb);
    lds_words(v + at.off_v0 + 8 * R4::kRow, wc);
    lds_words(v + at.off_v1 + 8 * R4::kRow, wd);
    uint32_t sa[NW], sb[NW], sc[NW], sd[NW];  // their scales; kF32: sa, sb those of rows g and g + 8
    lds_words(vs + (kF32 ? at.off_s : at.off_s0), sa);
    lds_words(vs + (kF32 ? at.off_s + 8 * R4::kScaleRow : at.off_s1), sb);
    if (!kF32) {
        lds_words(vs + at.off_s0 + 8 * R4::kScaleRow, sc);
        lds_words(vs + at.off_s1 + 8 * R4::kScaleRow, sd);
    }
    if (partial) {  // (whatever the page holds there)
#pragma unroll
        for (int y = 0; y < NW; ++y) {
            if ((kF32 ? at.key : at.key0) >= keys) sa[y] = 0u;
            if ((kF32 ? at.key + 8 : at.key1) >= keys) sb[y] = 0u;
            if (!kF32 && at.key0 + 8 >= keys) sc[y] = 0u;
            if (!kF32 && at.key1 + 8 >= keys) sd[y] = 0u;
        }
    }
    uint32_t t0 = 0u, t1 = 0u, t2 = 0u, t3 = 0u;
    if (!kF32) {
        const uint32_t h0 = ptx::cvt_bf16x2(p[0], p[1]), h1 = ptx::cvt_bf16x2(p[2], p[3]);
        t0 = transpose8(h0);
        t1 = transpose8(h1);
        t2 = transpose8(ptx::cvt_bf16x2(p[0] - bf16_lo(h0), p[1] - bf16_hi(h0)));
        t3 = transpose8(ptx::cvt_bf16x2(p[2] - bf16_lo(h1), p[3] - bf16_hi(h1)));
    }
#pragma unroll
    for (int j = 0; j < NG; ++j) {
        const uint32_t sel = j & 1 ? 0x7632u : 0x5410u;
        uint32_t b0, b1, b2, b3, b4 = 0u, b5 = 0u;
        if (kF32) {
            const float s0 = j & 1 ? bf16_hi(sa[j / 2]) : bf16_lo(sa[j / 2]);
            const float s1 = j & 1 ? bf16_hi(sb[j / 2]) : bf16_lo(sb[j / 2]);
            auto parts = [](float x, float y, uint32_t &first, uint32_t &second, uint32_t &third) {  // each what the roundings before it left
                first = ptx::cvt_bf16x2(x, y);
                x -= bf16_lo(first);
                y -= bf16_hi(first);
                second = ptx::cvt_bf16x2(x, y);
                third = transpose8(ptx::cvt_bf16x2(x - bf16_lo(second), y - bf16_hi(second)));
                first = transpose8(first);
                second = transpose8(second);
            };
            parts(p[0] * s0, p[1] * s0, b0, b2, b4);
            parts(p[2] * s1, p[3] * s1, b1, b3, b5);
        } else {
            const uint32_t s0 = __byte_perm(sa[j / 2], sb[j / 2], sel), s1 = __byte_perm(sc[j / 2], sd[j / 2], sel);
            b0 = bf2_mul(t0, s0);
            b1 = bf2_mul(t1, s1);
            b2 = bf2_fma(t2, s0, bf2_fms(t0, s0, b0));
            b3 = bf2_fma(t3, s1, bf2_fms(t1, s1, b1));
        }
        uint32_t x = __byte_perm(wa[j / 2], wb[j / 2], sel), y = __byte_perm(wc[j / 2], wd[j / 2], sel);
#pragma unroll
        for (int h = 0; h < 2; ++h, x >>= 8, y >>= 8) {
            const uint32_t a0 = nib_bf16(x), a1 = nib_bf16(x >> 4), a2 = nib_bf16(y), a3 = nib_bf16(y >> 4);
            mma_b16(acc[2 * j + h], a0, a1, a2, a3, b0, b1);
            mma_b16(acc[2 * j + h], a0, a1, a2, a3, b2, b3);
            if (kF32) mma_b16(acc[2 * j + h], a0, a1, a2, a3, b4, b5);
        }
    }
}

// Of a partial block's tile the keys from `keys` on do not exist.
__device__ __forceinline__ void kv4_mask(float (&sx)[4], int key, bool partial, int keys)
{
    if (partial) {
        if (key >= keys) sx[0] = sx[1] = -INFINITY;
        if (key + 8 >= keys) sx[2] = sx[3] = -INFINITY;
    }
}

// What a warp knows of a row: of heads 2t and 2t + 1 what the weights are relative to (m, see kD4Grow; -inf before the first key), the
// sum of weights (this thread's keys) and the output.
template <int D>
struct Kv4State {
    float m0, m1, l0, l1;
    float acc[D / 16][4];
    __device__ __forceinline__ void clear()
    {
        m0 = m1 = -INFINITY;
        l0 = l1 = 0.f;
#pragma unroll
        for (int e = 0; e < D / 16; ++e) acc[e][0] = acc[e][1] = acc[e][2] = acc[e][3] = 0.f;
    }
    // New logits have maxima mx0, mx1 (this thread's).
    __device__ __forceinline__ void raise(float mx0, float mx1)
    {
#pragma unroll
        for (int o = 4; o < 32; o *= 2) {
            mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, o));
            mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, o));
        }
        const bool up0 = mx0 > m0, up1 = mx1 > m1;
        mx0 += kD4Grow;
        mx1 += kD4Grow;
        if (__any_sync(0xffffffffu, up0 || up1)) {
            const float al0 = up0 ? ptx::ex2(m0 - mx0) : 1.f, al1 = up1 ? ptx::ex2(m1 - mx1) : 1.f;
            m0 = up0 ? mx0 : m0;
            m1 = up1 ? mx1 : m1;
            l0 *= al0;
            l1 *= al1;
#pragma unroll
            for (int e = 0; e < D / 16; ++e) {
                acc[e][0] *= al0;
                acc[e][1] *= al1;
                acc[e][2] *= al0;
                acc[e][3] *= al1;
            }
        }
    }
    // The weights of logits sx, added to the sums; the tile's keys from `keys` on have none.
    __device__ __forceinline__ void weigh(const float (&sx)[4], int key, bool partial, int keys, float (&p)[4])
    {
        p[0] = ptx::ex2(sx[0] - m0);
        p[1] = ptx::ex2(sx[1] - m1);
        p[2] = ptx::ex2(sx[2] - m0);
        p[3] = ptx::ex2(sx[3] - m1);
        if (partial) {
            if (key >= keys) p[0] = p[1] = 0.f;
            if (key + 8 >= keys) p[2] = p[3] = 0.f;
        }
        l0 += p[0] + p[2];
        l1 += p[1] + p[3];
    }
    __device__ __forceinline__ void sum_up()
    {
#pragma unroll
        for (int o = 4; o < 32; o *= 2) {
            l0 += __shfl_xor_sync(0xffffffffu, l0, o);
            l1 += __shfl_xor_sync(0xffffffffu, l1, o);
        }
    }
    // Output, maximum and sum of head h (behind sum_up()) to rows of (D + 4) floats and pairs, h = 0 .. 7.
    __device__ __forceinline__ void store(uint32_t rows, uint32_t stats, int lane) const
    {
        const int g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int j = 0; j < D / 32; ++j)
#pragma unroll
            for (int x = 0; x < 2; ++x)
                ptx::st_shared_v4(rows + (uint32_t)(2 * t + x) * (D + 4) * 4u + 128u * j + 16u * g, __float_as_uint(acc[2 * j][x]),
                                  __float_as_uint(acc[2 * j][2 + x]), __float_as_uint(acc[2 * j + 1][x]),
                                  __float_as_uint(acc[2 * j + 1][2 + x]));
        if (g == 0)
            ptx::st_shared_v4(stats + 16u * t, __float_as_uint(m0), __float_as_uint(l0), __float_as_uint(m1), __float_as_uint(l1));
    }
};

__device__ __forceinline__ void add_part(float4 &o, const float4 &v, float w)
{
    o.x = fmaf(v.x, w, o.x);
    o.y = fmaf(v.y, w, o.y);
    o.z = fmaf(v.z, w, o.z);
    o.w = fmaf(v.w, w, o.w);
}
template <bool kF32>
__device__ __forceinline__ void write4(void *o, int64_t at, const float4 &v, float f)
{
    if (kF32)
        *reinterpret_cast<float4 *>(static_cast<float *>(o) + at) = make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
    else
        *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(o) + at) =
            make_uint2(ptx::cvt_bf16x2(v.x * f, v.y * f), ptx::cvt_bf16x2(v.z * f, v.w * f));
}
__device__ __forceinline__ float natural(float m, float l) { return (m + log2f(l)) * 0.6931471805599453f; }

// ------------------------------------------------------------------------------------------
// The cluster kernel.  A row's blocks are dealt to the R CTAs of a cluster.  A CTA is eight consumer warps, which work on two
// blocks at a time, 16 keys each and all features, with maximum, sum and output of their own, and a warp that fetches the
// blocks into a ring of stages.  The eight results are merged through shared memory and pushed to the CTA that merges a
// head (CTA h % R) by asynchronous stores that count their bytes on a barrier of that CTA.
// Bound by the chain (cycles, one sequence of 4001 tokens, 4 rows of 9 blocks in clusters of 8; logits and values are some 100 more
// since the weights come in two parts): length 600, page 1400, block landed 2300, logits and values 4100, pushed 4600, received
// 5300, done 6000; 4.5 us a call.  Eight sequences of 64K to 128K tokens, 32 rows in clusters of 8: 6.5 us.  24 sequences of 64
// features, rows of up to 45 blocks in clusters of 2, fp32 outputs: 15.2 us.
// ------------------------------------------------------------------------------------------
constexpr int kC4Consumers = 8;
constexpr int kC4Threads = 32 * (kC4Consumers + 1);
constexpr int kC4MaxStages = 8;
constexpr int kC4MaxCluster = 8;

template <int D>
struct Kv4ClusterSmem {
    static constexpr uint32_t kStage = Kv4Record<D>::kBytes;
    static constexpr uint32_t kRow = (D + 4) * 4;  // (the pad spreads the heads over the banks)
    static constexpr uint32_t kStat = kC4Consumers * kD4MaxGroup * kRow;
    static constexpr uint32_t kRecv = kStat + kC4Consumers * kD4MaxGroup * 8;
    static constexpr uint32_t kBars = kRecv + 14 * kRow;  // R senders x ceil(8 / R) heads: at most 14 (R = 7)
    static constexpr uint32_t kRest = kBars + (2 * kC4MaxStages + 2) * 8;
    static constexpr size_t bytes(int stages) { return 128 + (size_t)stages * kStage + kRest; }
};

template <int D, bool kF32>
__global__ void __launch_bounds__(kC4Threads, 2) kv4_cluster_kernel(const Kv4Args a)
{
    using SM = Kv4ClusterSmem<D>;
    using R4 = Kv4Record<D>;
    extern __shared__ __align__(128) uint8_t smem_raw[];
    const uint32_t smem = (ptx::smem_u32(smem_raw) + 127u) & ~127u;
    const int stages = a.stages;
    const uint32_t rest = smem + (uint32_t)stages * SM::kStage, bars = rest + SM::kBars;
    volatile int *abort_flag =
        reinterpret_cast<volatile int *>(smem_raw + (bars - ptx::smem_u32(smem_raw)) + (2 * kC4MaxStages + 1) * 8);
    auto bar_full = [&](int s) { return bars + (uint32_t)s * 8u; };
    auto bar_empty = [&](int s) { return bars + (uint32_t)(kC4MaxStages + s) * 8u; };
    const uint32_t bar_recv = bars + 2 * kC4MaxStages * 8;
    auto wait_bar = [&](uint32_t b_, uint32_t parity, int code) {
        return ptx::mbar_wait_bounded(b_, parity, abort_flag, a.status, code, a.wait_cycles, (int)PA_ERR_TIMEOUT);
    };

    const int R = a.R, G = a.G;
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const uint32_t row = blockIdx.x / (uint32_t)R;  // = b Hkv + hk
    const int r = (int)(blockIdx.x - row * (uint32_t)R);
    const uint32_t b = row / (uint32_t)a.Hkv, hk = row - b * (uint32_t)a.Hkv;
    const int heads_here = G > r ? (G - r + R - 1) / R : 0, heads_per_owner = (kD4MaxGroup + R - 1) / R;

    // Started before the kernel ahead is done: nothing of global memory is touched up to pdl_wait().
    pdl_launch_next();
    if (tid == 0) {
        for (int s = 0; s < stages; ++s) {
            ptx::mbar_init(bar_full(s), 1);
            ptx::mbar_init(bar_empty(s), 4);
        }
        ptx::mbar_init(bar_recv, 1);
        *abort_flag = 0;
        ptx::fence_barrier_init();
        ptx::fence_proxy_async_smem();
        ptx::mbar_expect_tx(bar_recv, (uint32_t)(heads_here * R) * (D + 2) * 4u);
    }
    __syncthreads();
    ptx::cluster_arrive();  // (peers may push here from now on)
    pdl_wait();
    const int32_t len_raw = a.lens[b];
    if (a.clear_status && blockIdx.x == 0 && tid == 0) a.status[0] = 0;  // a wait that gives up (much later) sets it

    const int32_t len = len_raw >= 1 && len_raw <= a.max_len ? len_raw : 0;
    const LayoutRowOf<int32_t> list = layout_row_of<int32_t>(len ? (len - 1) / kKv4Page : 0, a.W, a.S);
    const int32_t n = len ? list.n : 0, mine = n > r ? (n - r + R - 1) / R : 0;

    if (wid == kC4Consumers) {
        // ------------------------------------------------------------------ producer
        bool ok = true;
        auto issue = [&](int s, const uint8_t *src) {
            ptx::mbar_expect_tx(bar_full(s), SM::kStage);
            ptx::bulk_load(smem + (uint32_t)s * SM::kStage, src, SM::kStage, bar_full(s));
        };
        int s = 0;
        uint32_t parity = 1;
        for (int base = 0; base < mine; base += 32) {
            // Each lane finds one block: from the diagonal block (the list's last) backwards, every R-th.
            const uint8_t *src = a.pool;
            if (base + lane < mine) {
                const int32_t j = layout_entry<int32_t>(list, n - 1 - (r + (base + lane) * R));
                int32_t page = a.table[(int64_t)b * a.table_stride + j];
                page = page < 0 ? 0 : page >= a.n_pages ? a.n_pages - 1 : page;
                src = a.pool + (int64_t)page * a.page_stride + (int64_t)hk * a.head_stride;
            }
            const int count = min(32, mine - base);
            int x = 0;
            if (base == 0) {  // stages that nothing has been in yet: all at once
                x = min(count, stages);
                if (lane < x) issue(lane, src);
            }
            for (; x < count; ++x) {
                const uint64_t from = __shfl_sync(0xffffffffu, reinterpret_cast<uint64_t>(src), x);
                if (s == 0) parity ^= 1;
                if (lane == 0 && ok) {
                    ok = wait_bar(bar_empty(s), parity, 1);
                    if (ok) issue(s, reinterpret_cast<const uint8_t *>(from));
                }
                s = s + 1 == stages ? 0 : s + 1;
            }
            __syncwarp();
        }
        ptx::cluster_wait();
    } else {
        // ------------------------------------------------------------------ consumers
        Kv4Query<D> q;
        {
            uint4 raw[D / 32];
            Kv4Query<D>::load(a, row, lane, raw);
            q.set(raw, a.scale_log2, lane);
        }
        const Kv4Lane<D> at(lane);
        const int tile = wid & 3;
        Kv4State<D> st;
        st.clear();
        bool ok = true;
        int s = wid >> 2;
        uint32_t parity = 0;
        while (s >= stages) {  // (one stage: block 1 is its second phase)
            s -= stages;
            parity ^= 1;
        }
#pragma unroll 1
        for (int i = wid >> 2; i < mine && ok; i += 2) {
            const int n_keys = r == 0 && i == 0 ? (len - 1) % kKv4Page + 1 : kKv4Page;  // (the diagonal block is first)
            ok = wait_bar(bar_full(s), parity, 2);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            const bool partial = n_keys < kKv4Page;
            if (16 * tile < n_keys) {
                const uint32_t k_half = smem + (uint32_t)s * SM::kStage;
                float sx[4], p[4];
                kv4_logits<D>(k_half, tile, at, q, sx);
                kv4_mask(sx, at.key, partial, n_keys - 16 * tile);
                st.raise(fmaxf(sx[0], sx[2]), fmaxf(sx[1], sx[3]));
                st.weigh(sx, at.key, partial, n_keys - 16 * tile, p);
                kv4_values<D, kF32>(k_half + R4::kHalf, tile, at, p, partial, n_keys - 16 * tile, st.acc);
            }
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(bar_empty(s));
            s += 2;
            while (s >= stages) {
                s -= stages;
                parity ^= 1;
            }
        }

        // ---- The eight warps' results meet in shared memory.
        st.sum_up();
        st.store(rest + (uint32_t)(wid * kD4MaxGroup) * SM::kRow, rest + SM::kStat + (uint32_t)(wid * kD4MaxGroup) * 8u, lane);
        asm volatile("bar.sync 1, %0;\n" ::"n"(32 * kC4Consumers) : "memory");
        // Warp: a head; thread: features 4 lane + {0 .. 3} (64 features: half the threads).
        const int h = wid;
        const uint32_t f0 = 16u * lane;
        float m = -INFINITY, l = 0.f;
        float4 out = make_float4(0.f, 0.f, 0.f, 0.f);
        float mw[kC4Consumers], lw[kC4Consumers];
#pragma unroll
        for (int x = 0; x < kC4Consumers; ++x) {
            ptx::ld_shared_v2(rest + SM::kStat + (uint32_t)(x * kD4MaxGroup + h) * 8u, mw[x], lw[x]);
            m = fmaxf(m, mw[x]);
        }
#pragma unroll
        for (int x = 0; x < kC4Consumers; ++x) {
            const float w = mw[x] != -INFINITY ? ptx::ex2(mw[x] - m) : 0.f;
            l = fmaf(lw[x], w, l);
            if (4 * lane < D) {
                float4 v;
                ptx::ld_shared_v4(rest + (uint32_t)(x * kD4MaxGroup + h) * SM::kRow + f0, v.x, v.y, v.z, v.w);
                add_part(out, v, w);
            }
        }
        ptx::cluster_wait();  // every CTA of the row has set its barrier up
        if (h < G) {
            const uint32_t slot = (uint32_t)(h / R), owner = (uint32_t)(h - (int)slot * R);
            const uint32_t dst = ptx::map_shared(rest + SM::kRecv, owner) + ((uint32_t)r * (uint32_t)heads_per_owner + slot) * SM::kRow;
            const uint32_t their_bar = ptx::map_shared(bar_recv, owner);
            if (4 * lane < D) ptx::st_async_v4(dst + f0, out, their_bar);
            if (lane == 0) ptx::st_async_v2(dst + 4u * D, m, l, their_bar);
        }

        // ---- Heads r, r + R, ... of the row, a warp each.
        if (wid < heads_here) {
            if (!ptx::mbar_wait_bounded_cluster(bar_recv, 0, abort_flag, a.status, 3, a.wait_cycles, (int)PA_ERR_TIMEOUT)) {
                // This CTA's shared memory has to last until every peer's part is in it: a peer is there after a wait for each
                // of its blocks at most, so this is over before its own limit is.
                const long long t0 = clock64(), most = kv4_outlast_cycles(a.wait_cycles, n, R);
                while (!ptx::mbar_try_wait_cluster(bar_recv, 0) && clock64() - t0 < most) {
                }
            } else {
                const int slot = wid, hh = r + slot * R;
                float mr[kC4MaxCluster], lr[kC4MaxCluster];
                m = -INFINITY;
                l = 0.f;
                out = make_float4(0.f, 0.f, 0.f, 0.f);
                auto src = [&](int x) { return rest + SM::kRecv + (uint32_t)((x < R ? x : 0) * heads_per_owner + slot) * SM::kRow; };
#pragma unroll
                for (int x = 0; x < kC4MaxCluster; ++x) {
                    ptx::ld_shared_v2(src(x) + 4u * D, mr[x], lr[x]);
                    if (x < R) m = fmaxf(m, mr[x]);
                }
#pragma unroll
                for (int x = 0; x < kC4MaxCluster; ++x) {
                    const float w = x < R && mr[x] != -INFINITY ? ptx::ex2(mr[x] - m) : 0.f;
                    if (x < R) l = fmaf(lr[x], w, l);
                    if (x < R && 4 * lane < D) {
                        float4 v;
                        ptx::ld_shared_v4(src(x) + f0, v.x, v.y, v.z, v.w);
                        add_part(out, v, w);
                    }
                }
                const int64_t head = (int64_t)row * G + hh;
                if (4 * lane < D) write4<kF32>(a.o, head * D + 4 * lane, out, n > 0 ? 1.0f / l : 0.f);
                if (lane == 0) a.lse[head] = n > 0 ? natural(m, l) : -INFINITY;  // (n = 0: a length outside [1, max_len])
            }
        }
    }

    __syncthreads();
    if (*abort_flag && tid == 0) {
        // A wait gave up: copies that may still be in flight have a bounded time to land before the CTA's shared memory is
        // handed to another CTA.
        const long long t0 = clock64();
        while (clock64() - t0 < 2000000ll) {
        }
    }
}

// ------------------------------------------------------------------------------------------
// The range kernel.  All blocks of all rows, row after row, are cut into equal ranges, one for each CTA and in it one for
// each warp: no warp waits for another one before its range is done, and all are done at the same time whatever the lengths
// are.  A warp takes whole blocks, the halves (K, V) of which it copies into a ring of its own, the next ones as soon as
// one is free.  A row that lies in a warp's range from end to end is written from its registers; of the others it keeps
// the first in shared memory and the last in its registers, and behind a barrier the CTA's warps merge these.  A row that
// other CTAs have parts of goes to the workspace, where kv4_join_kernel merges it.
// Where no row is long, ranges are rounded to whole rows instead, and nothing is left for the second kernel.
// The ranges follow from the lengths, which are on the device: each CTA sums all sequences' blocks up (a thread takes
// batch / 384 of them), and each thread looks one block of the CTA's range up.
// Bound by instructions: a block of 64 keys, 128 features and up to eight heads takes about 1500 (260 of them for the weights' second
// part), half of the issue slots, and the pipe of masks, shifts and byte permutations is 40 % busy.  256 sequences of 4K to 16K
// tokens, 1024 rows, 99.5 MB: 34.5 us, 2.9 TB/s.  Of these the blocks take 24, the start 2.7, a CTA's wait for its last warp 2.3,
// the merge 2.4, unequal shares of whole rows 3.
// ------------------------------------------------------------------------------------------
constexpr int kR4Warps = 12;
constexpr int kR4Threads = 32 * kR4Warps;
constexpr int kR4Ctas = 148;         // CTAs, times a number that keeps every range at no more than a block per thread

template <int D>
struct Kv4RangeSmem {
    static constexpr int kHalves = D == 128 ? 2 : 4;                   // halves in a warp's ring
    static constexpr uint32_t kHalf = Kv4Record<D>::kHalf;
    static constexpr uint32_t kRing = kHalves * kHalf;                  // of a warp
    static constexpr uint32_t kRow = (D + 4) * 4;
    static constexpr uint32_t kPiece = kD4MaxGroup * kRow + kD4MaxGroup * 8;  // rows of eight heads, their maxima and sums
    static_assert(kPiece <= kRing, "the last pieces take the rings' place");
    static constexpr uint32_t kFirst = kR4Warps * kRing;                // first pieces
    static constexpr uint32_t kBars = kFirst + kR4Warps * kPiece;
    static constexpr uint32_t kDesc = (kBars + kR4Warps * kHalves * 8 + 15) & ~15u;
    static constexpr uint32_t kSums = kDesc + kR4Threads * 16;
    static constexpr uint32_t kIds = kSums + kR4Threads * 8;      // rows of the pieces, int32 [warps][2]; the abort flag
    static constexpr size_t bytes() { return 128 + kIds + 2 * kR4Warps * 4 + 16; }
};

// A row's result in the workspace: its number (-1: none; -2: the CTA has no blocks), then eight heads' maxima, sums and outputs.
template <int D>
struct Kv4Part {
    static constexpr int kFloats = 4 + 2 * kD4MaxGroup + kD4MaxGroup * D;
};

template <int D, bool kF32>
__global__ void __launch_bounds__(kR4Threads, 1) kv4_range_kernel(const Kv4Args a)
{
    using SM = Kv4RangeSmem<D>;
    constexpr int NH = SM::kHalves;
    extern __shared__ __align__(128) uint8_t smem_raw[];
    const uint32_t smem = (ptx::smem_u32(smem_raw) + 127u) & ~127u;
    uint8_t *base = smem_raw + (smem - ptx::smem_u32(smem_raw));
    // A block: where its record is (two words), its row, the blocks left in the row | keys - 1 << 24 | first in the row << 30
    int4 *desc = reinterpret_cast<int4 *>(base + SM::kDesc);
    int2 *sums = reinterpret_cast<int2 *>(base + SM::kSums);  // a thread's first block, and the length of its only sequence
    int32_t *ids = reinterpret_cast<int32_t *>(base + SM::kIds);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(ids + 2 * kR4Warps);
    __shared__ int32_t warp_sums[kR4Warps];

    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const uint32_t ring = smem + (uint32_t)wid * SM::kRing, bars = smem + SM::kBars + (uint32_t)(wid * NH) * 8u;
    const int G = a.G;

    pdl_launch_next();
    if (lane == 0) {
        for (int s = 0; s < NH; ++s) ptx::mbar_init(bars + 8u * s, 1);
        ids[2 * wid] = ids[2 * wid + 1] = -1;
        if (wid == 0) *abort_flag = 0;
        ptx::fence_barrier_init();
        ptx::fence_proxy_async_smem();
    }
    pdl_wait();
    if (a.clear_status && blockIdx.x == 0 && tid == 0) a.status[0] = 0;

    // ---- The sequences' blocks, summed up.  Thread: sequences tid per .. tid per + per - 1.
    const int per = (a.batch + kR4Threads - 1) / kR4Threads;
    auto row_of = [&](int32_t len) {
        LayoutRowOf<int32_t> r = layout_row_of<int32_t>(len ? (len - 1) / kKv4Page : 0, a.W, a.S);
        if (!len) r.n = 0;
        return r;
    };
    auto len_of = [&](int b) {
        const int32_t len = a.lens[b];
        return len >= 1 && len <= a.max_len ? len : 0;
    };
    int32_t mine = 0, my_len = 0;  // (the length of its only sequence)
    for (int x = 0; x < per; ++x) {
        const int b = tid * per + x;
        if (b < a.batch) {
            my_len = len_of(b);
            mine += row_of(my_len).n * a.Hkv;
        }
    }
    int32_t upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const int32_t u = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += u;
    }
    if (lane == 31) warp_sums[wid] = upto;
    __syncthreads();
    int32_t before = 0, total = 0;
#pragma unroll
    for (int x = 0; x < kR4Warps; ++x) {
        const int32_t v = warp_sums[x];
        before += x < wid ? v : 0;
        total += v;
    }
    sums[tid] = make_int2(before + upto - mine, my_len);
    const int32_t lo = (int32_t)((int64_t)total * blockIdx.x / gridDim.x), hi = (int32_t)((int64_t)total * (blockIdx.x + 1) / gridDim.x);
    __syncthreads();

    // ---- Thread: block lo + tid.  It belongs to the range if it lies in [lo, hi), or if its row begins there (whole_rows).
    bool inside = false, earlier = false;
    int4 found = make_int4(0, 0, 0, 0);
    if (lo + tid < (a.whole_rows ? total : hi)) {
        int k = 0, end = kR4Threads;  // the last k whose sequences begin at or before this block
        while (end - k > 1) {
            const int mid = (k + end) >> 1;
            if (sums[mid].x <= lo + tid) k = mid;
            else end = mid;
        }
        int32_t at = lo + tid - sums[k].x, len = per == 1 ? sums[k].y : len_of(k * per);
        int b = k * per;
        LayoutRowOf<int32_t> r = row_of(len);
        while (at >= r.n * a.Hkv) {
            at -= r.n * a.Hkv;
            len = len_of(++b);
            r = row_of(len);
        }
        const int32_t hk = at / r.n, i = at - hk * r.n, begin = lo + tid - i;
        earlier = a.whole_rows && begin < lo;
        inside = !a.whole_rows || (begin >= lo && begin < hi);
        if (inside) {
            int32_t page = a.table[(int64_t)b * a.table_stride + layout_entry<int32_t>(r, i)];
            page = page < 0 ? 0 : page >= a.n_pages ? a.n_pages - 1 : page;
            const int32_t keys = i == r.n - 1 ? (len - 1) % kKv4Page + 1 : kKv4Page;
            const int64_t src = (int64_t)page * a.page_stride + (int64_t)hk * a.head_stride;
            found = make_int4((int)(uint32_t)src, (int)(src >> 32), b * a.Hkv + hk, (r.n - i) | (keys - 1) << 24 | (i == 0) << 30);
        }
    }
    const int skipped = a.whole_rows ? __syncthreads_count(earlier) : 0;  // (the first ones)
    if (inside) desc[tid - skipped] = found;
    const int count = __syncthreads_count(inside);  // (at most a block per thread: see the launch)

    // ---- Warp: blocks first .. last - 1 of the range.
    const int first = count * wid / kR4Warps, last = count * (wid + 1) / kR4Warps;
    auto issue = [&](int x, int half, uint32_t slot) {  // (one lane)
        const uint8_t *src = a.pool + *reinterpret_cast<const int64_t *>(&desc[x]) + (half ? SM::kHalf : 0);
        ptx::mbar_expect_tx(bars + 8u * slot, SM::kHalf);
        ptx::bulk_load(ring + slot * SM::kHalf, src, SM::kHalf, bars + 8u * slot);
    };
    const int halves = 2 * (last - first);
    if (lane == 0 && halves) issue(first, 0, 0);  // (the others behind it, so that all warps' first K come first)

    const Kv4Lane<D> at(lane);
    Kv4Query<D> q;
    Kv4State<D> st;
    st.clear();
    bool ok = true;
    uint32_t slot = 0, parity = 0;
    auto next_slot = [&] {
        if (++slot == (uint32_t)NH) {
            slot = 0;
            parity ^= 1;
        }
    };
    // The half in `slot` has been read by all lanes: half number `x` of the range takes its place.
    auto refill = [&](int x) {
        __syncwarp();
        if (lane == 0 && x < halves) issue(first + (x >> 1), x & 1, slot);
    };
    auto wait_half = [&](int code) {
        ok = ptx::mbar_wait_bounded(bars + 8u * slot, parity, abort_flag, a.status, code, a.wait_cycles, (int)PA_ERR_TIMEOUT);
        ok = __all_sync(0xffffffffu, ok);
    };
    bool row_start = true;  // the next block is its row's first one in this range
    bool whole = false;     // ... and in the row
#pragma unroll 1
    for (int x = first; x < last; ++x) {
        const int32_t row = desc[x].z, w = desc[x].w, left = w & 0xffffff, n_keys = (w >> 24 & 63) + 1;
        if (row_start) {
            uint4 raw[D / 32];
            Kv4Query<D>::load(a, (uint32_t)row, lane, raw);
            q.set(raw, a.scale_log2, lane);
            whole = w >> 30;
            row_start = false;
            if (x == first) {
                if (lane > 0 && lane < NH && lane < halves) issue(first + (lane >> 1), lane & 1, (uint32_t)lane);
                __syncwarp();
            }
        }
        wait_half(1);
        if (!ok) break;
        const bool partial = n_keys < kKv4Page;
        float sx[4][4];
        const uint32_t k_half = ring + slot * SM::kHalf;
#pragma unroll
        for (int tile = 0; tile < 4; ++tile) {
            if (!partial || 16 * tile < n_keys) {
                kv4_logits<D>(k_half, tile, at, q, sx[tile]);
                kv4_mask(sx[tile], at.key, partial, n_keys - 16 * tile);
            } else {
                sx[tile][0] = sx[tile][1] = sx[tile][2] = sx[tile][3] = -INFINITY;
            }
        }
        refill(2 * (x - first) + NH);
        next_slot();
        float mx0 = -INFINITY, mx1 = -INFINITY;
#pragma unroll
        for (int tile = 0; tile < 4; ++tile) {
            mx0 = fmaxf(mx0, fmaxf(sx[tile][0], sx[tile][2]));
            mx1 = fmaxf(mx1, fmaxf(sx[tile][1], sx[tile][3]));
        }
        st.raise(mx0, mx1);
        wait_half(2);
        if (!ok) break;
        const uint32_t v_half = ring + slot * SM::kHalf;
#pragma unroll
        for (int tile = 0; tile < 4; ++tile)
            if (!partial || 16 * tile < n_keys) {
                float p[4];
                st.weigh(sx[tile], at.key, partial, n_keys - 16 * tile, p);
                kv4_values<D, kF32>(v_half, tile, at, p, partial, n_keys - 16 * tile, st.acc);
            }
        refill(2 * (x - first) + 1 + NH);
        next_slot();
        if (left == 1 && x + 1 < last) {  // the row ends, the range goes on
            st.sum_up();
            if (whole) {
                const int g = lane >> 2, t = lane & 3;
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const int h = 2 * t + y;
                    if (h < G) {
                        const int64_t head = (int64_t)row * G + h;
                        const float m = y ? st.m1 : st.m0, l = y ? st.l1 : st.l0, inv = 1.0f / l;
#pragma unroll
                        for (int j = 0; j < D / 32; ++j)
                            write4<kF32>(a.o, head * D + 32 * j + 4 * g,
                                         make_float4(st.acc[2 * j][y], st.acc[2 * j][2 + y], st.acc[2 * j + 1][y], st.acc[2 * j + 1][2 + y]), inv);
                        if (g == 0) a.lse[head] = natural(m, l);
                    }
                }
            } else {  // (only the range's first row can be this)
                const uint32_t piece = smem + SM::kFirst + (uint32_t)wid * SM::kPiece;
                st.store(piece, piece + kD4MaxGroup * SM::kRow, lane);
                if (lane == 0) ids[2 * wid] = row;
            }
            st.clear();
            row_start = true;
        }
    }
    // ---- The last row's piece stays in the ring's place (nothing is on its way to it any more, unless a wait gave up).
    __syncthreads();
    if (first < last && ok) {
        st.sum_up();
        st.store(ring, ring + kD4MaxGroup * SM::kRow, lane);
        if (lane == 0) ids[2 * wid + 1] = desc[last - 1].z;
    }
    __syncthreads();
    if (*abort_flag) {
        if (tid < 2 && !a.whole_rows) reinterpret_cast<int32_t *>(a.parts + ((int64_t)blockIdx.x * 2 + tid) * Kv4Part<D>::kFloats)[0] = -1;
        if (tid == 0) {  // copies that may still be in flight have a bounded time to land
            const long long t0 = clock64();
            while (clock64() - t0 < 2000000ll) {
            }
        }
        return;
    }

    // ---- Pieces of the same row follow one another: a run of them.  Warp: a run, or where there are few, some heads of one.
    float *parts = a.parts + (int64_t)blockIdx.x * 2 * Kv4Part<D>::kFloats;
    const int32_t row_first = count ? desc[0].z : -1, row_last = count ? desc[count - 1].z : -1;
    const bool open_first = count && !(desc[0].w >> 30), open_last = count && (desc[count - 1].w & 0xffffff) != 1;
    static_assert(2 * kR4Warps <= 32, "a lane per piece");
    const int32_t id = lane < 2 * kR4Warps ? ids[lane] : -1;
    const uint32_t valid = __ballot_sync(0xffffffffu, id >= 0), below = valid & ((1u << lane) - 1u);
    const int32_t id_before = __shfl_sync(0xffffffffu, id, below ? 31 - __clz(below) : 0);
    const uint32_t starts = __ballot_sync(0xffffffffu, id >= 0 && (below == 0 || id_before != id));
    auto merge = [&](auto heads_of, int unit, int split) {  // heads unit % split, + split, ... of run unit / split
        constexpr int NHd = decltype(heads_of)::value;
        uint32_t rest = starts;
        for (int run = unit / split; run > 0; --run) rest &= rest - 1;
        const int h0 = unit % split, from = __ffs(rest) - 1;
        const uint32_t more = rest & (rest - 1);
        const uint32_t mask = valid & ~((1u << from) - 1u) & (more ? (1u << (__ffs(more) - 1)) - 1u : 0xffffffffu);
        const int32_t row = __shfl_sync(0xffffffffu, id, from);
        auto piece = [&](int y) { return y & 1 ? smem + (uint32_t)(y >> 1) * SM::kRing : smem + SM::kFirst + (uint32_t)(y >> 1) * SM::kPiece; };
        // Lane: one piece's maxima and sums, then its weights.
        const bool have = mask >> lane & 1u;
        float m[NHd], l[NHd], w[NHd];
        float4 out[NHd];
#pragma unroll
        for (int y = 0; y < NHd; ++y) {
            m[y] = -INFINITY;
            l[y] = 0.f;
            if (have && h0 + split * y < kD4MaxGroup) ptx::ld_shared_v2(piece(lane) + kD4MaxGroup * SM::kRow + 8u * (h0 + split * y), m[y], l[y]);
            w[y] = m[y];
            out[y] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int o = 16; o > 0; o /= 2)
#pragma unroll
            for (int y = 0; y < NHd; ++y) m[y] = fmaxf(m[y], __shfl_xor_sync(0xffffffffu, m[y], o));
#pragma unroll
        for (int y = 0; y < NHd; ++y) {
            w[y] = w[y] != -INFINITY ? ptx::ex2(w[y] - m[y]) : 0.f;
            l[y] *= w[y];
        }
#pragma unroll
        for (int o = 16; o > 0; o /= 2)
#pragma unroll
            for (int y = 0; y < NHd; ++y) l[y] += __shfl_xor_sync(0xffffffffu, l[y], o);
        for (uint32_t left = mask; left; left &= left - 1) {
            const int p = __ffs(left) - 1;
#pragma unroll
            for (int y = 0; y < NHd; ++y) {
                const float wy = __shfl_sync(0xffffffffu, w[y], p);
                if (4 * lane < D && h0 + split * y < G) {
                    float4 v;
                    ptx::ld_shared_v4(piece(p) + (uint32_t)(h0 + split * y) * SM::kRow + 16u * lane, v.x, v.y, v.z, v.w);
                    add_part(out[y], v, wy);
                }
            }
        }
        // A row that began in an earlier CTA is part 0, one that goes on in the next CTA part 1 (part 0 if both).
        const bool from_before = open_first && row == row_first, goes_on = open_last && row == row_last;
        float *part = parts + (from_before ? 0 : Kv4Part<D>::kFloats);
#pragma unroll
        for (int y = 0; y < NHd; ++y) {
            const int h = h0 + split * y;
            if (h >= G) break;
            if (from_before || goes_on) {
                if (4 * lane < D) *reinterpret_cast<float4 *>(part + 4 + 2 * kD4MaxGroup + h * D + 4 * lane) = out[y];
                if (lane == 0) *reinterpret_cast<float2 *>(part + 4 + 2 * h) = make_float2(m[y], l[y]);
            } else {
                const int64_t head = (int64_t)row * G + h;
                if (4 * lane < D) write4<kF32>(a.o, head * D + 4 * lane, out[y], 1.0f / l[y]);
                if (lane == 0) a.lse[head] = natural(m[y], l[y]);
            }
        }
    };
    const int runs = __popc(starts);
    if (4 * runs > kR4Warps)
        for (int unit = wid; unit < runs; unit += kR4Warps) merge(std::integral_constant<int, kD4MaxGroup>(), unit, 1);
    else if (wid < 4 * runs)
        merge(std::integral_constant<int, 2>(), wid, 4);
    if (tid < 2 && !a.whole_rows) {
        const bool there = tid == 0 ? open_first : open_last && !(open_first && row_first == row_last);
        reinterpret_cast<int32_t *>(parts + tid * Kv4Part<D>::kFloats)[0] = there ? (tid == 0 ? row_first : row_last) : count ? -1 : -2;
    }

    // ---- Sequences without a key (a length outside [1, max_len]): zeros.
    for (int b = blockIdx.x; b < a.batch; b += gridDim.x) {
        if (len_of(b)) continue;
        const int heads = a.Hkv * G;
        for (int x = tid; x < heads * D / 4; x += kR4Threads) write4<kF32>(a.o, (int64_t)b * heads * D + 4 * x, make_float4(0.f, 0.f, 0.f, 0.f), 0.f);
        for (int x = tid; x < heads; x += kR4Threads) a.lse[(int64_t)b * heads + x] = -INFINITY;
    }
}

// Rows that more than one CTA of kv4_range_kernel has a part of: the CTA whose last row goes on in the next ones.  Warp: heads h
// and h + 4; lane: four features.  Small, so that its CTAs wait beside those of the range kernel.
constexpr int kJ4Threads = 128;

template <int D, bool kF32>
__global__ void __launch_bounds__(kJ4Threads) kv4_join_kernel(const Kv4Args a)
{
    constexpr int64_t kStep = 2 * Kv4Part<D>::kFloats;  // from one CTA's parts to the next one's
    const int lane = threadIdx.x & 31;
    const unsigned c0 = blockIdx.x;
    const float *part = a.parts + (int64_t)c0 * kStep + Kv4Part<D>::kFloats, *next = a.parts + (int64_t)(c0 + 1) * kStep;
    pdl_launch_next();
    pdl_wait();
    const int32_t row = *reinterpret_cast<const int32_t *>(part);
    // Its other parts are part 0 of the next CTAs that have blocks.  Lane: one of these CTAs.
    unsigned first = 0;
    auto look = [&](uint32_t &mask) {  // which of the next 32 have a part; whether the row ends among them
        const unsigned c = c0 + 1 + first + lane;
        const int32_t id = c < gridDim.x ? *reinterpret_cast<const int32_t *>(next + (int64_t)(first + lane) * kStep) : -1;
        const uint32_t others = __ballot_sync(0xffffffffu, id != row && id != -2);
        const uint32_t until = others ? (1u << (__ffs(others) - 1)) - 1u : 0xffffffffu;
        mask = __ballot_sync(0xffffffffu, id == row) & until;
        return others != 0;
    };
    uint32_t mask;
    bool ends = look(mask);
    if (row < 0) return;
    for (int h = threadIdx.x >> 5; h < a.G; h += kJ4Threads / 32) {
        float m = part[4 + 2 * h], l = part[5 + 2 * h];
        float4 out = make_float4(0.f, 0.f, 0.f, 0.f);
        if (4 * lane < D) out = *reinterpret_cast<const float4 *>(part + 4 + 2 * kD4MaxGroup + h * D + 4 * lane);
        while (true) {
            const float *mine = next + (int64_t)(first + lane) * kStep;
            float mp = -INFINITY, lp = 0.f;
            if (mask >> lane & 1u) {
                mp = mine[4 + 2 * h];
                lp = mine[5 + 2 * h];
            }
            float top = mp;
#pragma unroll
            for (int o = 16; o > 0; o /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            top = fmaxf(top, m);
            const float w0 = m != -INFINITY ? ptx::ex2(m - top) : 0.f, w = mp != -INFINITY ? ptx::ex2(mp - top) : 0.f;
            lp *= w;
#pragma unroll
            for (int o = 16; o > 0; o /= 2) lp += __shfl_xor_sync(0xffffffffu, lp, o);
            l = fmaf(l, w0, lp);
            m = top;
            out = make_float4(out.x * w0, out.y * w0, out.z * w0, out.w * w0);
            for (uint32_t left = mask; left; left &= left - 1) {
                const int p = __ffs(left) - 1;
                const float wp = __shfl_sync(0xffffffffu, w, p);
                if (4 * lane < D)
                    add_part(out, *reinterpret_cast<const float4 *>(next + (int64_t)(first + p) * kStep + 4 + 2 * kD4MaxGroup + h * D + 4 * lane), wp);
            }
            if (ends) break;
            first += 32;
            ends = look(mask);
        }
        const int64_t head = (int64_t)row * a.G + h;
        if (4 * lane < D) write4<kF32>(a.o, head * D + 4 * lane, out, 1.0f / l);
        if (lane == 0) a.lse[head] = natural(m, l);
        if (first) {  // (a row of more than 33 CTAs: the next head begins with the first ones again)
            first = 0;
            ends = look(mask);
        }
    }
}

// ------------------------------------------------------------------------------------------ host
// Blocks of the longest row, at most.
static int kv4_most_blocks(const pa_kv4_params *p)
{
    const int64_t rows = p->max_blocks_per_seq, w = p->window_blocks > 1 ? p->window_blocks : 1;
    int64_t n = w + p->sink_blocks;
    for (int64_t pw = 1; pw < rows; pw *= 2) n += pw >= w;
    return (int)(n < rows ? n : rows);
}
static pa_status check_kv4(const pa_kv4_params *p)
{
    if (!p) return fail(PA_ERR_INVALID_ARG, "params must be non-null");
    if (pa_status s = check_kv4_pool(p->pool)) return s;
    if (p->batch < 1 || p->n_q_heads < 1 || p->max_blocks_per_seq < 1)
        return fail(PA_ERR_INVALID_ARG, "batch, head counts and max_blocks_per_seq must be positive");
    if (p->window_blocks < 0 || p->sink_blocks < 0)
        return fail(PA_ERR_INVALID_ARG, "window_blocks and sink_blocks must be >= 0");
    if (p->o_dtype != PA_BF16 && p->o_dtype != PA_F32) return fail(PA_ERR_INVALID_ARG, "bad o_dtype");
    if (!(p->softmax_scale >= 0.f) || isinf(p->softmax_scale))
        return fail(PA_ERR_INVALID_ARG, "softmax_scale must be finite and >= 0 (0 = default)");
    if (p->n_q_heads % p->pool.n_kv_heads) return fail(PA_ERR_SHAPE, "n_q_heads must be a multiple of n_kv_heads");
    if (p->n_q_heads / p->pool.n_kv_heads > kD4MaxGroup)
        return fail(PA_ERR_SHAPE, "at most %d query heads per KV head", kD4MaxGroup);
    if ((int64_t)p->max_blocks_per_seq * kKv4Page > ((int64_t)1 << 30))
        return fail(PA_ERR_SHAPE, "max_blocks_per_seq too large (limit 2^30 tokens)");
    if (p->batch > 65535 || p->n_q_heads > 65535) return fail(PA_ERR_SHAPE, "batch and head counts must be <= 65535");
    if (p->window_blocks > 4096 || p->sink_blocks > 4096)
        return fail(PA_ERR_SHAPE, "window_blocks and sink_blocks must be <= 4096");
    if ((int64_t)p->batch * p->pool.n_kv_heads * kv4_most_blocks(p) > INT32_MAX)
        return fail(PA_ERR_SHAPE, "more than 2^31 blocks in one call");
    return PA_OK;
}

// Whether ranges are rounded to whole rows: where a row is worth less than the second kernel, and CTAs have many.
static bool kv4_whole_rows(const pa_kv4_params *p)
{
    return kv4_most_blocks(p) <= 24 && (int64_t)p->batch * p->pool.n_kv_heads >= 2 * kR4Ctas;
}
// CTAs of the range kernel: no range, rounded or not, is longer than a block per thread, whatever the lengths are.
static int64_t kv4_range_ctas(const pa_kv4_params *p)
{
    const int64_t most = kv4_most_blocks(p), blocks = (int64_t)p->batch * p->pool.n_kv_heads * most;
    const int64_t room = kv4_whole_rows(p) ? kR4Threads - 2 * most : kR4Threads;
    const int64_t turns = (blocks + kR4Ctas * room - 1) / (kR4Ctas * room);
    return turns * kR4Ctas;
}

using Kv4Kernel = void (*)(const Kv4Args);
// 0: cluster, 1: range, 2: join
static Kv4Kernel kv4_kernel(int head_dim, bool f32, int which)
{
    static const Kv4Kernel kernels[2][2][3] = {
        {{kv4_cluster_kernel<64, false>, kv4_range_kernel<64, false>, kv4_join_kernel<64, false>},
         {kv4_cluster_kernel<64, true>, kv4_range_kernel<64, true>, kv4_join_kernel<64, true>}},
        {{kv4_cluster_kernel<128, false>, kv4_range_kernel<128, false>, kv4_join_kernel<128, false>},
         {kv4_cluster_kernel<128, true>, kv4_range_kernel<128, true>, kv4_join_kernel<128, true>}}};
    return kernels[head_dim == 128][f32][which];
}
static size_t kv4_cluster_smem(int head_dim, int stages)
{
    return head_dim == 128 ? Kv4ClusterSmem<128>::bytes(stages) : Kv4ClusterSmem<64>::bytes(stages);
}

// How many clusters of R CTAs the device holds at once.  Asked once per device and kind of launch.
static pa_status kv4_resident_clusters(int device, int head_dim, bool f32, int stages, int R, int *out)
{
    static std::mutex mu;
    static int known[kMaxDevices][2][2][kC4MaxStages + 1][kC4MaxCluster + 1];  // the number plus one; 0: not asked yet
    std::lock_guard<std::mutex> lock(mu);
    int &n = known[device][head_dim == 128][f32][stages][R];
    if (n == 0) {
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = (unsigned)R;
        attr.val.clusterDim.y = 1;
        attr.val.clusterDim.z = 1;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)R, 1, 1);
        cfg.blockDim = dim3(kC4Threads, 1, 1);
        cfg.dynamicSmemBytes = kv4_cluster_smem(head_dim, stages);
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        int found = 0;
        PA_CUDA_OK(cudaOccupancyMaxActiveClusters(&found, kv4_kernel(head_dim, f32, 0), &cfg));
        n = found + 1;
    }
    *out = n - 1;
    return PA_OK;
}

}  // namespace pa

extern "C" size_t pa_decode_kv4_workspace_bytes(const pa_kv4_params *p)
{
    using namespace pa;
    if (check_kv4(p) != PA_OK) return 0;
    const size_t part = sizeof(float) * (p->pool.head_dim == 128 ? Kv4Part<128>::kFloats : Kv4Part<64>::kFloats);
    return kD4StatusBytes + (size_t)kv4_range_ctas(p) * 2 * part;
}

extern "C" pa_status pa_decode_kv4(const pa_kv4_params *p, const void *q, const void *kv_pool, const int32_t *block_table,
                                   const int32_t *cache_lens, void *o, float *lse, void *workspace, size_t workspace_bytes,
                                   void *stream)
{
    using namespace pa;
    clear_error();
    if (pa_status s = check_kv4(p)) return s;
    if (!q || !kv_pool || !block_table || !cache_lens || !o || !lse)
        return fail(PA_ERR_INVALID_ARG, "q, the pool, block_table, cache_lens, o and lse must be non-null");
    if (!aligned16(q) || !aligned16(kv_pool) || !aligned16(o))
        return fail(PA_ERR_ALIGNMENT, "q, the pool and o must be 16-byte aligned");
    if (!aligned4(block_table, cache_lens, lse)) return fail(PA_ERR_ALIGNMENT, "block_table, cache_lens and lse must be 4-byte aligned");
    const size_t need = pa_decode_kv4_workspace_bytes(p);
    if (!workspace || workspace_bytes < need)
        return fail(PA_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, workspace_bytes);
    if (!aligned16(workspace)) return fail(PA_ERR_ALIGNMENT, "workspace must be 16-byte aligned");
    DeviceInfo dev;
    if (pa_status s = current_sm100_device(&dev)) return s;

    const int D = p->pool.head_dim;
    const bool f32 = p->o_dtype == PA_F32;
    Kv4Args a;
    a.q = static_cast<const __nv_bfloat16 *>(q);
    a.pool = static_cast<const uint8_t *>(kv_pool);
    a.table = block_table;
    a.lens = cache_lens;
    a.status = static_cast<int32_t *>(workspace);
    a.parts = reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) + kD4StatusBytes);
    a.o = o;
    a.lse = lse;
    a.page_stride = p->pool.page_stride;
    a.head_stride = p->pool.head_stride;
    a.max_len = (int64_t)p->max_blocks_per_seq * kKv4Page;
    a.table_stride = p->max_blocks_per_seq;
    a.n_pages = p->pool.n_pages;
    a.batch = p->batch;
    a.Hkv = p->pool.n_kv_heads;
    a.G = p->n_q_heads / p->pool.n_kv_heads;
    a.W = p->window_blocks;
    a.S = p->sink_blocks;
    const float scale = p->softmax_scale != 0.f ? p->softmax_scale : 1.0f / sqrtf((float)D);
    a.scale_log2 = scale * 1.4426950408889634f;
    const long long wait_cycles = wait_limit_cycles();
    a.wait_cycles = wait_cycles > 0 ? wait_cycles : kD4WaitCycles;
    a.clear_status = wait_cycles <= 0;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (!a.clear_status) PA_CUDA_OK(cudaMemsetAsync(a.status, 0, sizeof(int32_t), st));
    if (pa_status s = device_once(dev.device, ONCE_KV4_ATTR, [] {
            cudaError_t e = cudaSuccess;
            for (int i = 0; i < 8; ++i)
                e = first_error(e, cudaFuncSetAttribute(kv4_kernel(i & 1 ? 128 : 64, i & 2, i >> 2),
                                                        cudaFuncAttributeMaxDynamicSharedMemorySize, kD4MaxSmem));
            return e;
        }))
        return s;

    const EnvSwitches env = env_switches();
    const int most = kv4_most_blocks(p);
    const int64_t rows = (int64_t)a.batch * a.Hkv;
    // A cluster per row, as many CTAs as run all at once (two per SM), where that is faster than ranges.  Measured with 128 features,
    // G = 7 (us): a cluster's CTA takes 4 + 0.72 per block, ranges take 14 + 0.26 per block of an SM's share, 9 where they are of
    // whole rows; with 64 features all of it times 0.6.  Clusters and ranges, rows of 95 blocks: 144 rows 41.2 and 43.1 (ranges are
    // taken), 192 rows (one CTA each, which leaves a third of the places empty) 75.8 and 54.0; rows of 46 blocks: 96 rows 20.8 and
    // 22.1, 192 rows 37.5 and 31.0, 296 rows 38.9 and 36.6 (clusters are taken); rows of 11 blocks: 192 rows 12.1 and 18.7, 296 rows
    // 12.6 and 13.3.  64 features: rows of 46 blocks, 96 rows 13.7 and 17.7, 192 rows 23.6 and 22.4, 296 rows 23.9 and 25.6.
    int R = 0;
    auto stages_of = [&](int r) {
        // (Each four warps wait for every other block: if stages are used again their number is even, so that a stage is
        // always the same four warps', which see each of its phases.)
        const int n = (most + r - 1) / r, room = env.decode_stages ? env.decode_stages : D == 128 ? 6 : 8;
        return n <= room ? n : room < 2 ? 2 : room & ~1;
    };
    if (env.decode_path != 3) {
        const int64_t fit = (int64_t)dev.sms * 2 / rows;
        R = env.decode_cluster ? env.decode_cluster : fit < kC4MaxCluster ? (int)fit : kC4MaxCluster;
        if (R > most) R = most;
        if (env.decode_path == 2 && R < 1) R = 1;
        for (; R > 1 && !env.decode_cluster; --R) {
            int found = 0;
            if (pa_status s = kv4_resident_clusters(dev.device, D, f32, stages_of(R), R, &found)) return s;
            if (rows <= found) break;
        }
        const int64_t ranges = (kv4_whole_rows(p) ? 500 : 1000) + 26 * rows * most / kR4Ctas;
        if (env.decode_path != 2 && (R < 1 || 72 * ((most + R - 1) / R) > ranges)) R = 0;
    }
    if (R > 0) {
        a.R = R;
        a.stages = stages_of(R);
        cudaLaunchAttribute attr[2];
        attr[0] = pdl_attribute();
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = (unsigned)R;
        attr[1].val.clusterDim.y = 1;
        attr[1].val.clusterDim.z = 1;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)(rows * R), 1, 1);
        cfg.blockDim = dim3(kC4Threads, 1, 1);
        cfg.dynamicSmemBytes = kv4_cluster_smem(D, a.stages);
        cfg.stream = st;
        cfg.attrs = attr;
        cfg.numAttrs = 2;
        PA_CUDA_OK(cudaLaunchKernelEx(&cfg, kv4_kernel(D, f32, 0), a));
        return PA_OK;
    }
    a.R = 1;
    a.stages = 0;
    a.whole_rows = kv4_whole_rows(p);
    const unsigned ctas = (unsigned)kv4_range_ctas(p);
    const size_t smem = D == 128 ? Kv4RangeSmem<128>::bytes() : Kv4RangeSmem<64>::bytes();
    PA_CUDA_OK(launch_pdl(kv4_kernel(D, f32, 1), dim3(ctas), kR4Threads, smem, st, a));
    if (!a.whole_rows) PA_CUDA_OK(launch_pdl(kv4_kernel(D, f32, 2), dim3(ctas), kJ4Threads, 0, st, a));
    return PA_OK;
}
