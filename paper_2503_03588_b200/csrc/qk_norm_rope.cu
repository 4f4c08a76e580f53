// pa_qk_norm_rope and its backward pass: root-mean-square norm of every query and key head and rotation by the
// token's position, in one pass over both tensors.
//
// With r = 1 / sqrt(mean x^2 + eps), x^ = x r: out = R(pos) (x^ w).  Back: g = R(pos)^T d_out, dw = sum g x^, h = g w,
// dx = r (h - x^ mean(h x^)).  Sums, means and products in fp32, one rounding at the end.
//
// Bound by memory: a head is read and written once (backward: the head, its output's gradient, its gradient).  D / 8 or D / 16 lanes
// share a head, each with pairs that belong together under the rotation, so that nothing but the norm's sums crosses lanes;
// arithmetic goes two numbers an instruction, and what a token's heads share stays in registers.
// Measured in a graph, 28 and 4 heads of 128 features, 32768 tokens: forward 90 us (554 MB, 0.94 of a copy's rate), backward with fp32
// gradients 172 us (1074 MB, 0.95); 8 tokens forward 2.0 us; 3406 tokens of 16 and 4 heads of 64 features forward 8.2 us, backward
// 11.1 us (two kernels).
#include <cuda_bf16.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "sm100_ptx.cuh"

namespace pa {

constexpr int kRopeThreads = 128;
constexpr int kRopeWarps = kRopeThreads / 32;
constexpr int kBackThreads = 256;
constexpr int kBackWarps = kBackThreads / 32;

struct RopeArgs {
    const __nv_bfloat16 *q, *k;
    __nv_bfloat16 *q_out, *k_out;           // backward: the gradients of q and k, contiguous
    const void *d_q, *d_k;                  // backward: the gradients of the outputs
    const void *q_weight, *k_weight;
    const float *cos_sin;
    const int32_t *positions;
    float *parts;                           // backward: [CTAs][2][D] sums of the weights' gradients
    pa_strides sq, sk, sqo, sko;            // (backward: sqo, sko are those of d_q, d_k)
    int64_t tokens, seq;                    // of all batch entries, of one
    int32_t Hq, Hkv, half, max_positions;   // half: pairs that are rotated
    int32_t w_f32, chunks;
    float eps;
};

using ptx::add_f32x2;
using ptx::fma_f32x2;
using ptx::mul_f32x2;
using ptx::pack_f32x2;

// Eight numbers of a lane as four pairs: [0], [1] hold the first numbers of its four rotated pairs, [2], [3] the second ones.
struct Eight {
    uint64_t v[4];
};
__device__ __forceinline__ uint64_t both(float x) { return pack_f32x2(x, x); }
__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
// A lane's pieces of four features, a and b, in that order and back.  In neighbouring pairs (kPairs) the pieces hold first and
// second numbers in turns, else piece a the first and piece b the second ones.
template <bool kPairs>
__device__ __forceinline__ Eight in_order(float a0, float a1, float a2, float a3, float b0, float b1, float b2, float b3)
{
    if (kPairs) return {{pack_f32x2(a0, a2), pack_f32x2(b0, b2), pack_f32x2(a1, a3), pack_f32x2(b1, b3)}};
    return {{pack_f32x2(a0, a1), pack_f32x2(a2, a3), pack_f32x2(b0, b1), pack_f32x2(b2, b3)}};
}
template <bool kPairs>
__device__ __forceinline__ Eight from_bf16(const uint2 &a, const uint2 &b)
{
    return in_order<kPairs>(bf_lo(a.x), bf_hi(a.x), bf_lo(a.y), bf_hi(a.y), bf_lo(b.x), bf_hi(b.x), bf_lo(b.y), bf_hi(b.y));
}
template <bool kPairs>
__device__ __forceinline__ void pieces(const Eight &e, float (&x)[8])
{
    float f0, f1, f2, f3, s0, s1, s2, s3;
    ptx::unpack_f32x2(e.v[0], f0, f1);
    ptx::unpack_f32x2(e.v[1], f2, f3);
    ptx::unpack_f32x2(e.v[2], s0, s1);
    ptx::unpack_f32x2(e.v[3], s2, s3);
    if (kPairs) {
        x[0] = f0; x[1] = s0; x[2] = f1; x[3] = s1;
        x[4] = f2; x[5] = s2; x[6] = f3; x[7] = s3;
    } else {
        x[0] = f0; x[1] = f1; x[2] = f2; x[3] = f3;
        x[4] = s0; x[5] = s1; x[6] = s2; x[7] = s3;
    }
}
template <bool kPairs>
__device__ __forceinline__ void write_bf16(const Eight &e, __nv_bfloat16 *a, __nv_bfloat16 *b)
{
    float x[8];
    pieces<kPairs>(e, x);
    *reinterpret_cast<uint2 *>(a) = make_uint2(ptx::cvt_bf16x2(x[0], x[1]), ptx::cvt_bf16x2(x[2], x[3]));
    *reinterpret_cast<uint2 *>(b) = make_uint2(ptx::cvt_bf16x2(x[4], x[5]), ptx::cvt_bf16x2(x[6], x[7]));
}
__device__ __forceinline__ uint2 ld8(const void *p) { return *reinterpret_cast<const uint2 *>(p); }

// Where a lane's two pieces of four features stand in a head, which of its pairs [0] and [1] are rotated, and the first of their
// angles.  Neighbours' pieces are neighbours, so that a load or a store of a warp fills its sectors.
struct Pieces {
    int a, b, angle[2];
    bool turn[2];
};
// Lane l of kLanes: pieces of kWide features, of them the four from 4 part on.  Rotated features in halves: the lane's first numbers
// in piece a, their partners half a rotated part further on; the rest of the head is shared out behind them.  In neighbouring
// pairs: one piece of each half of the head.
template <int D, bool kPairs, int kWide>
__device__ __forceinline__ Pieces pieces_of(int l, int half, int part = 0)
{
    Pieces p;
    if (kPairs) {
        p.a = kWide * l + 4 * part;
        p.b = D / 2 + p.a;
        p.turn[0] = p.a < 2 * half;
        p.turn[1] = p.b < 2 * half;
        p.angle[0] = p.a / 2;
        p.angle[1] = p.b / 2;
    } else {
        const bool turn = kWide * l < half;
        p.a = (turn ? 0 : half) + kWide * l + 4 * part;
        p.b = p.a + (turn ? half : D / 2 - half);
        p.turn[0] = p.turn[1] = turn;
        p.angle[0] = p.a;
        p.angle[1] = p.a + 2;
    }
    return p;
}
template <bool kPairs, typename T>
__device__ __forceinline__ Eight load_eight(const T *src, const Pieces &p)
{
    if constexpr (sizeof(T) == 4) {
        const float4 a = *reinterpret_cast<const float4 *>(src + p.a), b = *reinterpret_cast<const float4 *>(src + p.b);
        return in_order<kPairs>(a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w);
    } else {
        return from_bf16<kPairs>(ld8(src + p.a), ld8(src + p.b));
    }
}
template <bool kPairs>
__device__ __forceinline__ Eight load_weights(const void *w, bool f32, const Pieces &p)
{
    return f32 ? load_eight<kPairs>(static_cast<const float *>(w), p) : load_eight<kPairs>(static_cast<const __nv_bfloat16 *>(w), p);
}
// The cosines and sines of a token's four pairs (not rotated: 1 and 0).
struct Angles {
    uint64_t c[2], s[2];
};
template <bool kPairs>
__device__ __forceinline__ Angles load_angles(const RopeArgs &a, const Pieces &p, int32_t pos)
{
    Angles t = {{both(1.f), both(1.f)}, {0, 0}};
    const float *row = a.cos_sin + (int64_t)pos * (2 * a.half);
    if (kPairs) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (p.turn[i]) {
                const float2 u = *reinterpret_cast<const float2 *>(row + p.angle[i]);
                const float2 v = *reinterpret_cast<const float2 *>(row + a.half + p.angle[i]);
                t.c[i] = pack_f32x2(u.x, u.y);
                t.s[i] = pack_f32x2(v.x, v.y);
            }
    } else if (p.turn[0]) {
        const float4 u = *reinterpret_cast<const float4 *>(row + p.angle[0]);
        const float4 v = *reinterpret_cast<const float4 *>(row + a.half + p.angle[0]);
        t = {{pack_f32x2(u.x, u.y), pack_f32x2(u.z, u.w)}, {pack_f32x2(v.x, v.y), pack_f32x2(v.z, v.w)}};
    }
    return t;
}
template <int kLanes>
__device__ __forceinline__ float sum_lanes(float x)
{
#pragma unroll
    for (int o = kLanes / 2; o > 0; o /= 2) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
__device__ __forceinline__ float sum_pairs(uint64_t x)
{
    float lo, hi;
    ptx::unpack_f32x2(x, lo, hi);
    return lo + hi;
}
__device__ __forceinline__ uint64_t negative(uint64_t x) { return x ^ 0x8000000080000000ull; }

// What a lane multiplies a head's numbers by, weights, cosines and sines once for all heads of a token:
// out_first = r (first w c - second w s), out_second = r (second w c + first w s)
struct Factors {
    uint64_t fc[2], sc[2], fs[2], ss[2];
};
__device__ __forceinline__ Factors factors(const Eight &w, const Angles &t)
{
    Factors f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        f.fc[i] = mul_f32x2(w.v[i], t.c[i]);
        f.sc[i] = mul_f32x2(w.v[2 + i], t.c[i]);
        f.fs[i] = mul_f32x2(w.v[i], t.s[i]);
        f.ss[i] = negative(mul_f32x2(w.v[2 + i], t.s[i]));
    }
    return f;
}
// Numbers times r, multiplied and rotated.
__device__ __forceinline__ Eight turned(const Eight &v, uint64_t r, const Factors &k, const Pieces &p)
{
    Eight o;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint64_t f = mul_f32x2(v.v[i], r), g = mul_f32x2(v.v[2 + i], r);
        if (p.turn[i]) {
            o.v[i] = fma_f32x2(f, k.fc[i], mul_f32x2(g, k.ss[i]));
            o.v[2 + i] = fma_f32x2(g, k.sc[i], mul_f32x2(f, k.fs[i]));
        } else {
            o.v[i] = mul_f32x2(f, k.fc[i]);
            o.v[2 + i] = mul_f32x2(g, k.sc[i]);
        }
    }
    return o;
}

// Forward, few tokens: a warp takes 256 / D heads of a token, so that the call is as short as one chain of loads.
template <int D, bool kPairs>
__global__ void __launch_bounds__(kRopeThreads) rope_few_kernel(const RopeArgs a)
{
    constexpr int kLanes = D / 8, kHeads = 32 / kLanes;
    pdl_launch_next();
    const int lane = threadIdx.x & 31, l = lane % kLanes, mine = lane / kLanes;
    const Pieces p = pieces_of<D, kPairs, 4>(l, a.half);
    const int64_t item = (int64_t)blockIdx.x * kRopeWarps + (threadIdx.x >> 5), token = item / a.chunks;
    const int h0 = (int)(item - token * a.chunks) * kHeads + mine, q_chunks = (a.Hq + kHeads - 1) / kHeads * kHeads;
    const bool is_k = h0 - mine >= q_chunks;
    const int h = is_k ? h0 - q_chunks : h0;
    pdl_wait();
    if (token >= a.tokens) return;
    const int32_t pos = a.positions[token];
    const int64_t b = token / a.seq, n = token - b * a.seq;
    const pa_strides &sx = is_k ? a.sk : a.sq, &so = is_k ? a.sko : a.sqo;
    const bool in = h < (is_k ? a.Hkv : a.Hq);
    const __nv_bfloat16 *x = (is_k ? a.k : a.q) + b * sx.batch + n * sx.seq + (in ? h : 0) * sx.head;
    const uint2 ra = ld8(x + p.a), rb = ld8(x + p.b);
    const Eight w = load_weights<kPairs>(is_k ? a.k_weight : a.q_weight, a.w_f32, p);
    if (pos < 0 || pos >= a.max_positions) return;
    __nv_bfloat16 *out = (is_k ? a.k_out : a.q_out) + b * so.batch + n * so.seq + (in ? h : 0) * so.head;
    const Eight v = from_bf16<kPairs>(ra, rb);
    uint64_t sq = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) sq = fma_f32x2(v.v[i], v.v[i], sq);
    const uint64_t r = both(rsqrtf(sum_lanes<kLanes>(sum_pairs(sq)) * (1.0f / D) + a.eps));
    if (in) write_bf16<kPairs>(turned(v, r, factors(w, load_angles<kPairs>(a, p, pos)), p), out + p.a, out + p.b);
}

__device__ __forceinline__ void copy16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;\n" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;\n" ::"n"(kLeft) : "memory"); }

// Forward.  Warps stride over the tokens, 512 / D heads at a time, queries, then keys.  A lane has sixteen features here, two times
// eight numbers as above: half the instructions a head.  What a lane will need of the next kRopeAhead turns is on its way to
// places of its own in shared memory (nobody else reads them, so there is nothing to wait for but its own copies).
// (32768 tokens of 28 and 4 heads of 128: 90 us; with the next heads in registers 104, with a warp per few heads 100.)
constexpr int kRopeAhead = 8;
constexpr int kRopeTurn = 32 * 32;  // bytes of a turn: 32 of a lane

template <int D, bool kPairs>
__global__ void __launch_bounds__(kBackThreads, 2) rope_kernel(const RopeArgs a)
{
    constexpr int kLanes = D / 16, kHeads = 32 / kLanes;
    extern __shared__ __align__(16) uint8_t rope_smem[];
    pdl_launch_next();
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, l = lane % kLanes, mine = lane / kLanes;
    const Pieces p[2] = {pieces_of<D, kPairs, 8>(l, a.half, 0), pieces_of<D, kPairs, 8>(l, a.half, 1)};
    const uint8_t *ring = rope_smem + wid * (kRopeAhead * kRopeTurn) + lane * 16;
    const int64_t step = (int64_t)gridDim.x * kBackWarps;
    const int turns_q = (a.Hq + kHeads - 1) / kHeads, turns = turns_q + (a.Hkv + kHeads - 1) / kHeads;
    pdl_wait();
    auto position = [&](int64_t token) {  // -1: none
        const int32_t pos = token < a.tokens ? a.positions[token] : -1;
        return pos < a.max_positions ? pos : -1;
    };
    auto place = [&](int64_t token, const pa_strides &s) {
        const int64_t b = a.seq >= a.tokens ? 0 : token / a.seq;
        return b * s.batch + (token - b * a.seq) * s.seq + mine * s.head;
    };
    // What is fetched next.
    int64_t f_token = (int64_t)blockIdx.x * kBackWarps + wid;
    int f_turn = 0, f_left = 0, f_slot = 0;  // heads left from this lane's one on
    const __nv_bfloat16 *x = nullptr;
    int64_t x_step = 0;
    auto fetch = [&] {
        if (f_token < a.tokens) {
            if (f_turn == 0) {
                x = a.q + place(f_token, a.sq);
                x_step = kHeads * a.sq.head;
                f_left = a.Hq - mine;
            } else if (f_turn == turns_q) {
                x = a.k + place(f_token, a.sk);
                x_step = kHeads * a.sk.head;
                f_left = a.Hkv - mine;
            }
            if (f_left > 0) {
                const uint32_t at = ptx::smem_u32(ring) + f_slot * kRopeTurn;
                copy16(at, x + p[0].a);
                copy16(at + 512, x + p[0].b);
            }
            x += x_step;
            f_left -= kHeads;
            if (++f_turn == turns) {
                f_turn = 0;
                f_token += step;
            }
        }
        copies_commit();
        f_slot = (f_slot + 1) % kRopeAhead;
    };
    for (int y = 0; y < kRopeAhead; ++y) fetch();
    int slot = 0;
    int64_t token = (int64_t)blockIdx.x * kBackWarps + wid;
    int32_t pos = position(token), pos_next = position(token + step);
    for (; token < a.tokens; token += step) {
        const int32_t pos_after = position(token + 2 * step);
#pragma unroll 1
        for (int which = 0; which < 2; ++which) {
            const int H = which ? a.Hkv : a.Hq;
            const pa_strides &so = which ? a.sko : a.sqo;
            const int64_t out_step = kHeads * so.head;
            __nv_bfloat16 *out = (which ? a.k_out : a.q_out) + place(token, so);
            Factors f[2];
#pragma unroll
            for (int e = 0; e < 2; ++e)
                f[e] = factors(load_weights<kPairs>(which ? a.k_weight : a.q_weight, a.w_f32, p[e]), load_angles<kPairs>(a, p[e], pos < 0 ? 0 : pos));
            for (int h = mine; h - mine < H; h += kHeads) {
                copies_wait<kRopeAhead - 1>();
                const uint4 va = *reinterpret_cast<const uint4 *>(ring + slot * kRopeTurn);
                const uint4 vb = *reinterpret_cast<const uint4 *>(ring + slot * kRopeTurn + 512);
                slot = (slot + 1) % kRopeAhead;
                const Eight v[2] = {from_bf16<kPairs>(make_uint2(va.x, va.y), make_uint2(vb.x, vb.y)),
                                    from_bf16<kPairs>(make_uint2(va.z, va.w), make_uint2(vb.z, vb.w))};
                uint64_t sq[2] = {0, 0};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    sq[0] = fma_f32x2(v[0].v[i], v[0].v[i], sq[0]);
                    sq[1] = fma_f32x2(v[1].v[i], v[1].v[i], sq[1]);
                }
                const uint64_t r = both(rsqrtf(sum_lanes<kLanes>(sum_pairs(add_f32x2(sq[0], sq[1]))) * (1.0f / D) + a.eps));
                fetch();  // (behind the last use of what was in its place)
                float o[2][8];
#pragma unroll
                for (int e = 0; e < 2; ++e) pieces<kPairs>(turned(v[e], r, f[e], p[e]), o[e]);
                if (pos >= 0 && h < H) {
                    auto four = [&](int i) {
                        return make_uint4(ptx::cvt_bf16x2(o[0][i], o[0][i + 1]), ptx::cvt_bf16x2(o[0][i + 2], o[0][i + 3]),
                                          ptx::cvt_bf16x2(o[1][i], o[1][i + 1]), ptx::cvt_bf16x2(o[1][i + 2], o[1][i + 3]));
                    };
                    *reinterpret_cast<uint4 *>(out + p[0].a) = four(0);
                    *reinterpret_cast<uint4 *>(out + p[0].b) = four(4);
                }
                out += out_step;
            }
        }
        pos = pos_next;
        pos_next = pos_after;
    }
    copies_wait<0>();
}

// Backward.  Warps stride over the tokens and keep the weights' gradients in registers, and the next heads' numbers; at the end a CTA
// adds its warps' up, in their order, and leaves the sums for rope_weights_kernel.  Two CTAs of 128 registers a thread an SM (172 us
// for the call above; smaller CTAs that keep less on its way 200 to 250).
// kSplit: a token's heads, kBatch x 256 / D at a time, are dealt to a.chunks warps.
constexpr int kBatch = 2;
template <int D, bool kPairs, typename T, bool kSplit>
__global__ void __launch_bounds__(kBackThreads, 2) rope_backward_kernel(const RopeArgs a)
{
    constexpr int kLanes = D / 8, kHeads = 32 / kLanes;
    __shared__ float sums[kBackWarps * kHeads][2][D];
    pdl_launch_next();
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, l = lane % kLanes, mine = lane / kLanes;
    const Pieces p = pieces_of<D, kPairs, 4>(l, a.half);
    Eight dw[2] = {};
    pdl_wait();
    const int parts = kSplit ? a.chunks : 1, stride = parts * kBatch * kHeads;
    const int64_t items = kSplit ? a.tokens * parts : a.tokens;
    for (int64_t item = (int64_t)blockIdx.x * kBackWarps + wid; item < items; item += (int64_t)gridDim.x * kBackWarps) {
        const int64_t token = kSplit ? (int64_t)((uint32_t)item / (uint32_t)parts) : item;  // (few items: see the launch)
        const int part = kSplit ? (int)(item - token * parts) : 0;
        const int32_t pos = a.positions[token];
        const bool there = pos >= 0 && pos < a.max_positions;
        const int64_t b = token / a.seq, n = token - b * a.seq;
        Angles t = {};
        bool looked_up = false;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const int H = which ? a.Hkv : a.Hq;
            const pa_strides &sx = which ? a.sk : a.sq, &sd = which ? a.sko : a.sqo;
            // The first heads of this part: the keys' follow the queries' in turn.
            int first = 0;
            if (kSplit) first = kBatch * kHeads * (which ? (part + parts - (a.Hq + kBatch * kHeads - 1) / (kBatch * kHeads) % parts) % parts : part);
            if (kSplit && first >= H) continue;
            const __nv_bfloat16 *x = (which ? a.k : a.q) + b * sx.batch + n * sx.seq + (first + mine) * sx.head;
            const T *d = static_cast<const T *>(which ? a.d_k : a.d_q) + b * sd.batch + n * sd.seq + (first + mine) * sd.head;
            __nv_bfloat16 *out = (which ? a.k_out : a.q_out) + (token * H + first + mine) * D;
            uint2 ra[kBatch], rb[kBatch];
            uint4 da[kBatch], db[kBatch];
            auto load = [&](int h) {
#pragma unroll
                for (int y = 0; y < kBatch; ++y) {
                    ra[y] = rb[y] = make_uint2(0u, 0u);
                    da[y] = db[y] = make_uint4(0u, 0u, 0u, 0u);
                    if (there && h + y * kHeads + mine < H) {
                        const __nv_bfloat16 *src = x + y * kHeads * sx.head;
                        const T *grad = d + y * kHeads * sd.head;
                        ra[y] = ld8(src + p.a);
                        rb[y] = ld8(src + p.b);
                        if constexpr (sizeof(T) == 4) {
                            da[y] = *reinterpret_cast<const uint4 *>(grad + p.a);
                            db[y] = *reinterpret_cast<const uint4 *>(grad + p.b);
                        } else {
                            const uint2 u = ld8(grad + p.a), v = ld8(grad + p.b);
                            da[y] = make_uint4(u.x, u.y, 0u, 0u);
                            db[y] = make_uint4(v.x, v.y, 0u, 0u);
                        }
                    }
                }
                x += stride * sx.head;
                d += stride * sd.head;
            };
            load(first);
            // (A token without a position has weights and angles of zero: what these are, finite or not, is nothing to it.)
            Eight w = {};
            if (there) w = load_weights<kPairs>(which ? a.k_weight : a.q_weight, a.w_f32, p);
            if (there && !looked_up) {
                t = load_angles<kPairs>(a, p, pos);
                looked_up = true;
            }
            for (int h = first; h < H; h += stride) {
                Eight v[kBatch], g[kBatch];
#pragma unroll
                for (int y = 0; y < kBatch; ++y) {
                    v[y] = from_bf16<kPairs>(ra[y], rb[y]);
                    if constexpr (sizeof(T) == 4)
                        g[y] = in_order<kPairs>(__uint_as_float(da[y].x), __uint_as_float(da[y].y), __uint_as_float(da[y].z),
                                                __uint_as_float(da[y].w), __uint_as_float(db[y].x), __uint_as_float(db[y].y),
                                                __uint_as_float(db[y].z), __uint_as_float(db[y].w));
                    else
                        g[y] = from_bf16<kPairs>(make_uint2(da[y].x, da[y].y), make_uint2(db[y].x, db[y].y));
                }
                if (h + stride < H) load(h + stride);
#pragma unroll
                for (int y = 0; y < kBatch; ++y) {
                    const bool in = h + y * kHeads + mine < H;
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        if (p.turn[i]) {  // back by the angle
                            const uint64_t f = g[y].v[i], s = g[y].v[2 + i];
                            g[y].v[i] = fma_f32x2(f, t.c[i], mul_f32x2(s, t.s[i]));
                            g[y].v[2 + i] = fma_f32x2(s, t.c[i], negative(mul_f32x2(f, t.s[i])));
                        }
                    // dx = r (h - x^ mean(h x^)), h = g w, x^ = x r;  dw = sum g x^
                    Eight gw;
                    uint64_t sq = 0, along = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        gw.v[i] = mul_f32x2(g[y].v[i], w.v[i]);
                        sq = fma_f32x2(v[y].v[i], v[y].v[i], sq);
                        along = fma_f32x2(gw.v[i], v[y].v[i], along);
                    }
                    const float sum_sq = sum_lanes<kLanes>(sum_pairs(sq)), sum_along = sum_lanes<kLanes>(sum_pairs(along));
                    // (no head, no gradient, whatever eps is)
                    const float r = in && there ? rsqrtf(sum_sq * (1.0f / D) + a.eps) : 0.f;
                    const uint64_t r2 = both(r), mean = both(-sum_along * (1.0f / D) * r);
                    Eight dx;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint64_t xn = mul_f32x2(v[y].v[i], r2);
                        dw[which].v[i] = fma_f32x2(g[y].v[i], xn, dw[which].v[i]);
                        dx.v[i] = mul_f32x2(r2, fma_f32x2(xn, mean, gw.v[i]));
                    }
                    if (in) write_bf16<kPairs>(dx, out + p.a, out + p.b);
                    out += kHeads * D;
                }
                if (kSplit) out += (stride - kBatch * kHeads) * D;
            }
        }
    }
    float(*row)[D] = sums[wid * kHeads + mine];
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float x[8];
        pieces<kPairs>(dw[which], x);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            row[which][p.a + i] = x[i];
            row[which][p.b + i] = x[4 + i];
        }
    }
    __syncthreads();
    for (int f = threadIdx.x; f < 2 * D; f += kBackThreads) {
        float t = 0.f;
        for (int y = 0; y < kBackWarps * kHeads; ++y) t += sums[y][f / D][f % D];
        a.parts[(int64_t)blockIdx.x * 2 * D + f] = t;
    }
}

// Sums over the CTAs of rope_backward_kernel: 8 columns a CTA, a sector of each of 128 rows at a time, added up in a fixed order.
constexpr int kSumThreads = 1024;
__global__ void __launch_bounds__(kSumThreads) rope_weights_kernel(const float *parts, int n, int D, float *dq_weight, float *dk_weight)
{
    __shared__ float sums[kSumThreads / 32][8];
    pdl_launch_next();
    const int x = threadIdx.x & 7, y = threadIdx.x >> 3, f = blockIdx.x * 8 + x;
    pdl_wait();
    float t = 0.f;
#pragma unroll 4
    for (int i = y; i < n; i += kSumThreads / 8) t += parts[(int64_t)i * 2 * D + f];
    t += __shfl_xor_sync(0xffffffffu, t, 8);
    t += __shfl_xor_sync(0xffffffffu, t, 16);
    if ((threadIdx.x & 31) < 8) sums[threadIdx.x >> 5][x] = t;
    __syncthreads();
    if (threadIdx.x < 32) {  // lane: column x, rows lane / 8, lane / 8 + 4, ...
        t = 0.f;
#pragma unroll
        for (int i = 0; i < kSumThreads / 32; i += 4) t += sums[i + (threadIdx.x >> 3)][x];
        t += __shfl_xor_sync(0xffffffffu, t, 8);
        t += __shfl_xor_sync(0xffffffffu, t, 16);
        if (threadIdx.x < 8) (f < D ? dq_weight : dk_weight)[f % D] = t;
    }
}

static pa_status check_rope(const pa_rope_params *p)
{
    if (!p) return fail(PA_ERR_INVALID_ARG, "params must be non-null");
    if (p->batch < 1 || p->n_q_heads < 1 || p->n_kv_heads < 1 || p->seq_len < 1 || p->max_positions < 1)
        return fail(PA_ERR_INVALID_ARG, "batch, head counts, seq_len and max_positions must be positive");
    if (p->head_dim != 64 && p->head_dim != 128) return fail(PA_ERR_SHAPE, "head_dim must be 64 or 128");
    if (p->rotary_dim < 0 || p->rotary_dim > p->head_dim || p->rotary_dim % 16)
        return fail(PA_ERR_SHAPE, "rotary_dim must be a multiple of 16 between 0 and head_dim");
    if (!(p->eps >= 0.f) || isinf(p->eps)) return fail(PA_ERR_INVALID_ARG, "eps must be finite and >= 0");
    if (p->w_dtype != PA_BF16 && p->w_dtype != PA_F32) return fail(PA_ERR_INVALID_ARG, "bad w_dtype");
    if (p->n_q_heads > 65535 || p->n_kv_heads > 65535) return fail(PA_ERR_SHAPE, "head counts must be <= 65535");
    if (p->seq_len > ((int64_t)1 << 31) / p->batch) return fail(PA_ERR_SHAPE, "batch x seq_len must be <= 2^31");
    const pa_strides *st[4] = {&p->q, &p->k, &p->q_out, &p->k_out};
    for (auto s : st) {
        if (s->seq < 0 || s->head < 0 || s->batch < 0) return fail(PA_ERR_SHAPE, "strides must be >= 0");
        if ((s->seq % 8) || (s->head % 8) || (s->batch % 8))
            return fail(PA_ERR_ALIGNMENT, "strides must be multiples of 8 elements (16 bytes)");
    }
    return PA_OK;
}

// Whether two heads of a tensor share a number.  Axes of one entry have no part in it.
static bool rows_overlap(const pa_strides &st, const int64_t (&sizes)[3], int64_t D)
{
    struct Axis {
        int64_t size, stride;
    } x[3];
    int n = 0;
    for (int i = 0; i < 3; ++i)
        if (sizes[i] > 1) x[n++] = {sizes[i], i == 0 ? st.batch : i == 1 ? st.seq : st.head};
    // No, if each axis steps over all that the axes of smaller strides cover: nearly every tensor.
    std::sort(x, x + n, [](const Axis &a, const Axis &b) { return a.stride < b.stride; });
    bool nested = true;
    int64_t covered = D;
    for (int i = 0; i < n && nested; ++i) {
        nested = x[i].stride >= covered && x[i].stride <= (INT64_MAX - covered) / x[i].size;
        covered += x[i].stride * (nested ? x[i].size - 1 : 0);
    }
    if (nested) return false;
    for (int i = 0; i < n; ++i)
        if (x[i].stride < D || x[i].stride > INT64_MAX / 4 / x[i].size) return true;  // (the latter: beyond any memory)
    // Else heads overlap where steps a and b along two axes lie less than a head from a step c along the third: all a and b of the
    // two shorter axes are tried.  (Where these are more than 2^16, the tensor is refused.)
    std::sort(x, x + n, [](const Axis &a, const Axis &b) { return a.size < b.size; });
    while (n < 3) x[n++] = {1, 0};
    std::sort(x, x + n, [](const Axis &a, const Axis &b) { return a.size < b.size; });
    if (x[0].size > (1 << 16) / x[1].size) return true;
    for (int64_t a = 0; a < x[0].size; ++a)
        for (int64_t b = a ? 1 - x[1].size : 0; b < x[1].size; ++b) {
            const int64_t at = a * x[0].stride + b * x[1].stride, away = at < 0 ? -at : at;
            const int64_t c = away / x[2].stride;  // (c and c + 1 steps are the nearest ones)
            for (int64_t y = c; y <= c + 1 && y < x[2].size; ++y) {
                const int64_t d = away - y * x[2].stride;
                if ((a || b || y) && d < D && -d < D) return true;
            }
        }
    return false;
}

// Rows that are written must not lie over one another.
static pa_status check_written(const pa_rope_params *p)
{
    const int64_t q[3] = {p->batch, p->seq_len, p->n_q_heads}, k[3] = {p->batch, p->seq_len, p->n_kv_heads};
    if (rows_overlap(p->q_out, q, p->head_dim) || rows_overlap(p->k_out, k, p->head_dim))
        return fail(PA_ERR_SHAPE, "rows of the outputs overlap");
    return PA_OK;
}

static pa_status rope_args(const pa_rope_params *p, const void *q, const void *k, const void *q_weight, const void *k_weight,
                           const float *cos_sin, const int32_t *positions, const void *more0, const void *more1, const void *more2,
                           const void *more3, RopeArgs *a)
{
    if (!q || !k || !q_weight || !k_weight || (!cos_sin && p->rotary_dim > 0) || !positions || !more0 || !more1 || !more2 || !more3)
        return fail(PA_ERR_INVALID_ARG, "every array must be non-null");
    if (!aligned16(q) || !aligned16(k) || !aligned16(q_weight) || !aligned16(k_weight) || !aligned16(cos_sin) || !aligned16(more0) ||
        !aligned16(more1) || !aligned16(more2) || !aligned16(more3))
        return fail(PA_ERR_ALIGNMENT, "the tensors, weights and the table must be 16-byte aligned");
    if (!aligned4(positions)) return fail(PA_ERR_ALIGNMENT, "positions must be 4-byte aligned");
    *a = RopeArgs{};
    a->q = static_cast<const __nv_bfloat16 *>(q);
    a->k = static_cast<const __nv_bfloat16 *>(k);
    a->q_weight = q_weight;
    a->k_weight = k_weight;
    a->cos_sin = cos_sin;
    a->positions = positions;
    a->sq = p->q;
    a->sk = p->k;
    a->sqo = p->q_out;
    a->sko = p->k_out;
    a->tokens = (int64_t)p->batch * p->seq_len;
    a->seq = p->seq_len;
    a->Hq = p->n_q_heads;
    a->Hkv = p->n_kv_heads;
    a->half = p->rotary_dim / 2;
    a->max_positions = p->max_positions;
    a->w_f32 = p->w_dtype == PA_F32;
    a->eps = p->eps;
    return PA_OK;
}

// CTAs of the kernels that stride over the tokens, a warp a token: two per SM (the workspace holds a part for each).
constexpr int64_t kRopeCtas = 148 * 2;
static int64_t token_ctas(const pa_rope_params *p, int64_t per_token = 1)
{
    const int64_t need = ((int64_t)p->batch * p->seq_len * per_token + kBackWarps - 1) / kBackWarps;
    return need < kRopeCtas ? need : kRopeCtas;
}
// Backward: the warps that a token's heads are dealt to, as many as leave every warp one item.  Measured (us, backward alone, dealt and
// not): 28 and 4 heads of 128 features, 7 tokens 4.6 and 8.7, 300 tokens 6.7 and 9.2, 1100 tokens 9.8 and 12.4; 16 and 4 heads of 64,
// 64 tokens 4.2 and 5.1, 1100 tokens 6.4 and 7.0.
static int64_t backward_parts(const pa_rope_params *p)
{
    const int64_t tokens = (int64_t)p->batch * p->seq_len, at_once = kBatch * 256 / p->head_dim;
    const int64_t most = (p->n_q_heads + at_once - 1) / at_once + (p->n_kv_heads + at_once - 1) / at_once;
    const int64_t room = kRopeCtas * kBackWarps / tokens;
    return room < 1 ? 1 : room < most ? room : most;
}
// Up to this many warps of one piece each, else the persistent ones that ring.  Measured (us, one piece a warp and persistent):
// 28 and 4 heads of 128 features, 600 tokens 4.6 and 6.5, 1200 tokens 7.5 and 7.3, 2500 tokens 14.1 and 10.6; 16 and 4 heads of
// 64, 1200 tokens 3.4 and 4.5, 3500 tokens (17500 warps) 6.8 and 7.5, 4736 tokens 8.7 and 7.6.  The two cross near 18000 warps with 128
// features and near 20000 with 64; from the line to there the persistent form is up to a tenth the slower one.
constexpr int64_t kRopeFewWarps = 148 * 112;

}  // namespace pa

extern "C" pa_status pa_qk_norm_rope(const pa_rope_params *p, const void *q, const void *k, const void *q_weight,
                                     const void *k_weight, const float *cos_sin, const int32_t *positions, void *q_out,
                                     void *k_out, void *stream)
{
    using namespace pa;
    clear_error();
    if (pa_status s = check_rope(p)) return s;
    if (pa_status s = check_written(p)) return s;
    RopeArgs a;
    if (pa_status s = rope_args(p, q, k, q_weight, k_weight, cos_sin, positions, q_out, k_out, q_out, k_out, &a)) return s;
    a.q_out = static_cast<__nv_bfloat16 *>(q_out);
    a.k_out = static_cast<__nv_bfloat16 *>(k_out);
    const int at_once = 256 / p->head_dim;
    a.chunks = (p->n_q_heads + at_once - 1) / at_once + (p->n_kv_heads + at_once - 1) / at_once;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    static void (*const few[2][2])(const RopeArgs) = {{rope_few_kernel<64, false>, rope_few_kernel<64, true>},
                                                      {rope_few_kernel<128, false>, rope_few_kernel<128, true>}};
    static void (*const many[2][2])(const RopeArgs) = {{rope_kernel<64, false>, rope_kernel<64, true>},
                                                       {rope_kernel<128, false>, rope_kernel<128, true>}};
    const int64_t warps = a.tokens * a.chunks;
    DeviceInfo dev;
    if (pa_status s = current_sm100_device(&dev)) return s;
    if (pa_status s = device_once(dev.device, ONCE_ROPE_ATTR, [] {
            cudaError_t e = cudaSuccess;
            for (int i = 0; i < 4; ++i)
                e = first_error(e, cudaFuncSetAttribute(many[i >> 1][i & 1], cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                        kBackWarps * kRopeAhead * kRopeTurn));
            return e;
        }))
        return s;
    if (warps <= kRopeFewWarps)
        PA_CUDA_OK(launch_pdl(few[p->head_dim == 128][p->interleaved != 0], dim3((unsigned)((warps + kRopeWarps - 1) / kRopeWarps)),
                              kRopeThreads, 0, st, a));
    else
        PA_CUDA_OK(launch_pdl(many[p->head_dim == 128][p->interleaved != 0], dim3((unsigned)token_ctas(p)), kBackThreads,
                              kBackWarps * kRopeAhead * kRopeTurn, st, a));
    return PA_OK;
}

extern "C" size_t pa_qk_norm_rope_backward_workspace_bytes(const pa_rope_params *p)
{
    using namespace pa;
    if (check_rope(p) != PA_OK) return 0;
    return (size_t)token_ctas(p, backward_parts(p)) * 2 * p->head_dim * sizeof(float);
}

extern "C" pa_status pa_qk_norm_rope_backward(const pa_rope_params *p, const void *q, const void *k, const void *q_weight,
                                              const void *k_weight, const float *cos_sin, const int32_t *positions,
                                              const void *d_q_out, const void *d_k_out, pa_dtype d_dtype, void *dq, void *dk,
                                              float *dq_weight, float *dk_weight, void *workspace, size_t workspace_bytes,
                                              void *stream)
{
    using namespace pa;
    clear_error();
    if (pa_status s = check_rope(p)) return s;
    if (d_dtype != PA_BF16 && d_dtype != PA_F32) return fail(PA_ERR_INVALID_ARG, "bad d_dtype");
    RopeArgs a;
    if (pa_status s = rope_args(p, q, k, q_weight, k_weight, cos_sin, positions, d_q_out, d_k_out, dq, dk, &a)) return s;
    if (!dq_weight || !dk_weight) return fail(PA_ERR_INVALID_ARG, "every array must be non-null");
    if (!aligned4(dq_weight, dk_weight)) return fail(PA_ERR_ALIGNMENT, "the weights' gradients must be 4-byte aligned");
    const size_t need = pa_qk_norm_rope_backward_workspace_bytes(p);
    if (!workspace || workspace_bytes < need)
        return fail(PA_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, workspace_bytes);
    if (!aligned16(workspace)) return fail(PA_ERR_ALIGNMENT, "workspace must be 16-byte aligned");
    a.q_out = static_cast<__nv_bfloat16 *>(dq);
    a.k_out = static_cast<__nv_bfloat16 *>(dk);
    a.d_q = d_q_out;
    a.d_k = d_k_out;
    a.parts = static_cast<float *>(workspace);
    const int64_t parts = backward_parts(p), ctas = token_ctas(p, parts);
    a.chunks = (int32_t)parts;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    auto launch = [&](auto split) {
        constexpr bool S = decltype(split)::value;
        using bf16 = __nv_bfloat16;
        static void (*const kernels[2][2][2])(const RopeArgs) = {
            {{rope_backward_kernel<64, false, bf16, S>, rope_backward_kernel<64, false, float, S>},
             {rope_backward_kernel<64, true, bf16, S>, rope_backward_kernel<64, true, float, S>}},
            {{rope_backward_kernel<128, false, bf16, S>, rope_backward_kernel<128, false, float, S>},
             {rope_backward_kernel<128, true, bf16, S>, rope_backward_kernel<128, true, float, S>}}};
        return launch_pdl(kernels[p->head_dim == 128][p->interleaved != 0][d_dtype == PA_F32], dim3((unsigned)ctas), kBackThreads, 0, st, a);
    };
    PA_CUDA_OK(parts > 1 ? launch(std::true_type()) : launch(std::false_type()));
    PA_CUDA_OK(launch_pdl(rope_weights_kernel, dim3((unsigned)(2 * p->head_dim / 8)), kSumThreads, 0, st,
                          static_cast<const float *>(a.parts), (int)ctas, (int)p->head_dim, dq_weight, dk_weight));
    return PA_OK;
}
