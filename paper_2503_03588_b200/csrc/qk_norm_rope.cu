// pa_qk_norm_rope and its backward pass: root-mean-square norm of every query and key head and rotation by the
// token's position, in one pass over both tensors.
//
// Bound by memory: a head is read and written once (backward: the head, its output's gradient, its gradient).  D / 8 lanes
// share a head, eight features each, as two pieces of four that belong together under the rotation, so that nothing but the
// norm's sums crosses lanes.  A warp works on 256 / D heads of one token at a time and keeps the token's cosines and sines and
// the weights in registers over all of the token's heads.
#include <cuda_bf16.h>
#include <math.h>

#include "common.cuh"

namespace pa {

constexpr int kRopeThreads = 256;
constexpr int kRopeWarps = kRopeThreads / 32;

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
    int32_t interleaved, w_f32, chunks, heads_per_chunk;
    float eps;
};

__device__ __forceinline__ uint2 ld8(const void *p) { return *reinterpret_cast<const uint2 *>(p); }
__device__ __forceinline__ void unpack4(const uint2 &u, float *x)
{
    x[0] = __uint_as_float(u.x << 16);
    x[1] = __uint_as_float(u.x & 0xffff0000u);
    x[2] = __uint_as_float(u.y << 16);
    x[3] = __uint_as_float(u.y & 0xffff0000u);
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ uint2 pack4(const float *x) { return make_uint2(pack2(x[0], x[1]), pack2(x[2], x[3])); }

// Where a lane's two pieces of four features stand in a head, and the first of its four angles.
struct Pieces {
    int a, b, angle;
    bool rotated;
};
__device__ __forceinline__ Pieces pieces_of(int l, int half, bool interleaved)
{
    Pieces p;
    p.angle = 4 * l;
    p.rotated = 4 * l < half;
    // (behind the rotated features, 2 half + 8 (l - half / 4) = 8 l)
    p.a = !interleaved && p.rotated ? 4 * l : 8 * l;
    p.b = !interleaved && p.rotated ? half + 4 * l : 8 * l + 4;
    return p;
}
// x[0..3] is piece a, x[4..7] piece b.
__device__ __forceinline__ void rotate(float *x, const float *c, const float *s, bool interleaved)
{
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float u = x[2 * i], v = x[2 * i + 1];
            x[2 * i] = u * c[i] - v * s[i];
            x[2 * i + 1] = v * c[i] + u * s[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float u = x[i], v = x[4 + i];
            x[i] = u * c[i] - v * s[i];
            x[4 + i] = v * c[i] + u * s[i];
        }
    }
}
__device__ __forceinline__ void load_weights(const void *w, bool f32, const Pieces &p, float *out)
{
    if (f32) {
        const float4 a = *reinterpret_cast<const float4 *>(static_cast<const float *>(w) + p.a);
        const float4 b = *reinterpret_cast<const float4 *>(static_cast<const float *>(w) + p.b);
        out[0] = a.x; out[1] = a.y; out[2] = a.z; out[3] = a.w;
        out[4] = b.x; out[5] = b.y; out[6] = b.z; out[7] = b.w;
    } else {
        unpack4(ld8(static_cast<const __nv_bfloat16 *>(w) + p.a), out);
        unpack4(ld8(static_cast<const __nv_bfloat16 *>(w) + p.b), out + 4);
    }
}
// The four angles of a token.
__device__ __forceinline__ void load_angles(const RopeArgs &a, const Pieces &p, int32_t pos, float *c, float *s)
{
    float4 u = make_float4(0.f, 0.f, 0.f, 0.f), v = u;
    if (p.rotated) {
        const float *row = a.cos_sin + (int64_t)pos * (2 * a.half) + p.angle;
        u = *reinterpret_cast<const float4 *>(row);
        v = *reinterpret_cast<const float4 *>(row + a.half);
    }
    c[0] = u.x; c[1] = u.y; c[2] = u.z; c[3] = u.w;
    s[0] = v.x; s[1] = v.y; s[2] = v.z; s[3] = v.w;
}
template <int kLanes>
__device__ __forceinline__ float sum_lanes(float x)
{
#pragma unroll
    for (int o = kLanes / 2; o > 0; o /= 2) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// A warp takes heads_per_chunk heads of a token, kBatch times 256 / D of them at a time.
template <int D, int kBatch>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const RopeArgs a)
{
    constexpr int kLanes = D / 8, kHeads = 32 / kLanes;
    pdl_launch_next();
    const int lane = threadIdx.x & 31, l = lane % kLanes, mine = lane / kLanes;
    const Pieces p = pieces_of(l, a.half, a.interleaved);
    const int64_t item = (int64_t)blockIdx.x * kRopeWarps + (threadIdx.x >> 5);
    const int64_t token = item / a.chunks;
    const int chunk = (int)(item - token * a.chunks);
    pdl_wait();
    if (token >= a.tokens) return;
    const int32_t pos = a.positions[token];
    if (pos < 0 || pos >= a.max_positions) return;
    const int64_t b = token / a.seq, n = token - b * a.seq;
    const __nv_bfloat16 *q = a.q + b * a.sq.batch + n * a.sq.seq, *k = a.k + b * a.sk.batch + n * a.sk.seq;
    __nv_bfloat16 *q_out = a.q_out + b * a.sqo.batch + n * a.sqo.seq, *k_out = a.k_out + b * a.sko.batch + n * a.sko.seq;
    float c[4], s[4], wq[8], wk[8];
    load_angles(a, p, pos, c, s);
    load_weights(a.q_weight, a.w_f32, p, wq);
    load_weights(a.k_weight, a.w_f32, p, wk);
    const int H = a.Hq + a.Hkv, first = chunk * a.heads_per_chunk;
    const int end = first + a.heads_per_chunk < H ? first + a.heads_per_chunk : H;
    for (int h0 = first; h0 < end; h0 += kBatch * kHeads) {
        uint2 ra[kBatch], rb[kBatch];
#pragma unroll
        for (int x = 0; x < kBatch; ++x) {
            const int h = h0 + x * kHeads + mine;
            if (h < end) {
                const __nv_bfloat16 *src = h < a.Hq ? q + h * a.sq.head : k + (h - a.Hq) * a.sk.head;
                ra[x] = ld8(src + p.a);
                rb[x] = ld8(src + p.b);
            } else {
                ra[x] = rb[x] = make_uint2(0u, 0u);
            }
        }
#pragma unroll
        for (int x = 0; x < kBatch; ++x) {
            const int h = h0 + x * kHeads + mine;
            float v[8];
            unpack4(ra[x], v);
            unpack4(rb[x], v + 4);
            float sq = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) sq = fmaf(v[i], v[i], sq);
            const float r = rsqrtf(sum_lanes<kLanes>(sq) * (1.0f / D) + a.eps);
            const bool is_q = h < a.Hq;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= r * (is_q ? wq[i] : wk[i]);
            if (p.rotated) rotate(v, c, s, a.interleaved);
            if (h < end) {
                __nv_bfloat16 *dst = is_q ? q_out + h * a.sqo.head : k_out + (h - a.Hq) * a.sko.head;
                *reinterpret_cast<uint2 *>(dst + p.a) = pack4(v);
                *reinterpret_cast<uint2 *>(dst + p.b) = pack4(v + 4);
            }
        }
    }
}

template <typename T>
__device__ __forceinline__ void load_gradient(const T *src, const Pieces &p, float *g)
{
    if constexpr (sizeof(T) == 4) {
        const float4 a = *reinterpret_cast<const float4 *>(src + p.a), b = *reinterpret_cast<const float4 *>(src + p.b);
        g[0] = a.x; g[1] = a.y; g[2] = a.z; g[3] = a.w;
        g[4] = b.x; g[5] = b.y; g[6] = b.z; g[7] = b.w;
    } else {
        unpack4(ld8(src + p.a), g);
        unpack4(ld8(src + p.b), g + 4);
    }
}

// Warps stride over the tokens and keep the weights' gradients in registers; at the end a CTA adds its warps' up, in their
// order, and leaves the sums for rope_weights_kernel.
template <int D, typename T>
__global__ void __launch_bounds__(kRopeThreads) rope_backward_kernel(const RopeArgs a)
{
    constexpr int kLanes = D / 8, kHeads = 32 / kLanes, kBatch = 2;
    __shared__ float sums[kRopeWarps * kHeads][2][D];
    pdl_launch_next();
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, l = lane % kLanes, mine = lane / kLanes;
    const Pieces p = pieces_of(l, a.half, a.interleaved);
    float dw[2][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[0][i] = dw[1][i] = 0.f;
    pdl_wait();
    for (int64_t token = (int64_t)blockIdx.x * kRopeWarps + wid; token < a.tokens; token += (int64_t)gridDim.x * kRopeWarps) {
        const int32_t pos = a.positions[token];
        const bool there = pos >= 0 && pos < a.max_positions;
        const int64_t b = token / a.seq, n = token - b * a.seq;
        float c[4], s[4];
        load_angles(a, p, there ? pos : 0, c, s);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = -s[i];
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const int H = which ? a.Hkv : a.Hq;
            const pa_strides &sx = which ? a.sk : a.sq, &sd = which ? a.sko : a.sqo;
            const __nv_bfloat16 *x_row = (which ? a.k : a.q) + b * sx.batch + n * sx.seq;
            const T *d_row = static_cast<const T *>(which ? a.d_k : a.d_q) + b * sd.batch + n * sd.seq;
            __nv_bfloat16 *out = (which ? a.k_out : a.q_out) + token * H * D;
            float w[8];
            load_weights(which ? a.k_weight : a.q_weight, a.w_f32, p, w);
            for (int h0 = 0; h0 < H; h0 += kBatch * kHeads) {
                uint2 ra[kBatch], rb[kBatch];
                float g[kBatch][8];
#pragma unroll
                for (int y = 0; y < kBatch; ++y) {
                    const int h = h0 + y * kHeads + mine;
                    ra[y] = rb[y] = make_uint2(0u, 0u);
#pragma unroll
                    for (int i = 0; i < 8; ++i) g[y][i] = 0.f;
                    if (h < H && there) {
                        ra[y] = ld8(x_row + h * sx.head + p.a);
                        rb[y] = ld8(x_row + h * sx.head + p.b);
                        load_gradient(d_row + h * sd.head, p, g[y]);
                    }
                }
#pragma unroll
                for (int y = 0; y < kBatch; ++y) {
                    const int h = h0 + y * kHeads + mine;
                    float v[8];
                    unpack4(ra[y], v);
                    unpack4(rb[y], v + 4);
                    if (p.rotated) rotate(g[y], c, s, a.interleaved);
                    float sq = 0.f, along = 0.f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        sq = fmaf(v[i], v[i], sq);
                        along = fmaf(g[y][i] * w[i], v[i], along);
                    }
                    sq = sum_lanes<kLanes>(sq);
                    along = sum_lanes<kLanes>(along);
                    // dx = r (h - x r^2 mean(h x)), h = g w
                    // (no head, no gradient, whatever eps is)
                    const float r = h < H && there ? rsqrtf(sq * (1.0f / D) + a.eps) : 0.f, t = along * (1.0f / D) * r * r;
                    float dx[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        dx[i] = r * (g[y][i] * w[i] - v[i] * t);
                        dw[which][i] = fmaf(g[y][i], v[i] * r, dw[which][i]);
                    }
                    if (h < H) {
                        *reinterpret_cast<uint2 *>(out + h * D + p.a) = pack4(dx);
                        *reinterpret_cast<uint2 *>(out + h * D + p.b) = pack4(dx + 4);
                    }
                }
            }
        }
    }
    float(*row)[D] = sums[wid * kHeads + mine];
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            row[which][p.a + i] = dw[which][i];
            row[which][p.b + i] = dw[which][4 + i];
        }
    __syncthreads();
    for (int f = threadIdx.x; f < 2 * D; f += kRopeThreads) {
        float t = 0.f;
        for (int y = 0; y < kRopeWarps * kHeads; ++y) t += sums[y][f / D][f % D];
        a.parts[(int64_t)blockIdx.x * 2 * D + f] = t;
    }
}

// Sums over the CTAs of rope_backward_kernel: 32 columns a CTA, 32 rows at a time.
__global__ void __launch_bounds__(1024) rope_weights_kernel(const float *parts, int n, int D, float *dq_weight, float *dk_weight)
{
    __shared__ float sums[32][33];
    pdl_launch_next();
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, f = blockIdx.x * 32 + x;
    pdl_wait();
    float t = 0.f;
    for (int i = y; i < n; i += 32) t += parts[(int64_t)i * 2 * D + f];
    sums[y][x] = t;
    __syncthreads();
    if (y == 0) {
        t = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) t += sums[i][x];
        (f < D ? dq_weight : dk_weight)[f % D] = t;
    }
}

static pa_status check_rope(const pa_rope_params *p)
{
    if (!p) return fail(PA_ERR_INVALID_ARG, "params must be non-null");
    if (p->batch < 1 || p->n_q_heads < 1 || p->n_kv_heads < 1 || p->seq_len < 1 || p->max_positions < 1)
        return fail(PA_ERR_INVALID_ARG, "batch, head counts, seq_len and max_positions must be positive");
    if (p->head_dim != 64 && p->head_dim != 128) return fail(PA_ERR_SHAPE, "head_dim must be 64 or 128");
    if (p->rotary_dim < 0 || p->rotary_dim > p->head_dim || p->rotary_dim % 8)
        return fail(PA_ERR_SHAPE, "rotary_dim must be a multiple of 8 between 0 and head_dim");
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

// Writing through a stride of 0, or one below a head, would have rows overlap.
static pa_status check_written(const pa_rope_params *p)
{
    const pa_strides *st[2] = {&p->q_out, &p->k_out};
    const int32_t heads[2] = {p->n_q_heads, p->n_kv_heads};
    for (int i = 0; i < 2; ++i) {
        if ((heads[i] > 1 && st[i]->head < p->head_dim) || (p->seq_len > 1 && st[i]->seq < p->head_dim) ||
            (p->batch > 1 && st[i]->batch < p->head_dim))
            return fail(PA_ERR_SHAPE, "rows of the outputs overlap");
    }
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
    a->interleaved = p->interleaved != 0;
    a->w_f32 = p->w_dtype == PA_F32;
    a->eps = p->eps;
    return PA_OK;
}

// CTAs of rope_backward_kernel, for the workspace and the launch alike.
constexpr int64_t kRopeBackwardCtas = 148 * 4;
static int64_t backward_ctas(const pa_rope_params *p)
{
    const int64_t need = ((int64_t)p->batch * p->seq_len + kRopeWarps - 1) / kRopeWarps;
    return need < kRopeBackwardCtas ? need : kRopeBackwardCtas;
}

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
    const int heads = p->n_q_heads + p->n_kv_heads, at_once = 256 / p->head_dim;
    // Few tokens: one batch of heads a warp, so that the call is as short as a warp's chain of loads.
    const bool few = a.tokens * heads <= 148 * 64 * at_once;
    a.heads_per_chunk = few ? at_once : heads;
    a.chunks = (heads + a.heads_per_chunk - 1) / a.heads_per_chunk;
    const int64_t ctas = (a.tokens * a.chunks + kRopeWarps - 1) / kRopeWarps;
    if (ctas > INT32_MAX) return fail(PA_ERR_SHAPE, "too many tokens");
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    auto launch = [&](auto kernel) { return launch_pdl(kernel, dim3((unsigned)ctas), kRopeThreads, 0, st, a); };
    PA_CUDA_OK(p->head_dim == 128 ? (few ? launch(rope_kernel<128, 1>) : launch(rope_kernel<128, 4>))
                                  : (few ? launch(rope_kernel<64, 1>) : launch(rope_kernel<64, 4>)));
    return PA_OK;
}

extern "C" size_t pa_qk_norm_rope_backward_workspace_bytes(const pa_rope_params *p)
{
    using namespace pa;
    if (check_rope(p) != PA_OK) return 0;
    return (size_t)backward_ctas(p) * 2 * p->head_dim * sizeof(float);
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
    const int64_t ctas = backward_ctas(p);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    auto launch = [&](auto kernel) { return launch_pdl(kernel, dim3((unsigned)ctas), kRopeThreads, 0, st, a); };
    const bool f32 = d_dtype == PA_F32;
    PA_CUDA_OK(p->head_dim == 128 ? (f32 ? launch(rope_backward_kernel<128, float>) : launch(rope_backward_kernel<128, __nv_bfloat16>))
                                  : (f32 ? launch(rope_backward_kernel<64, float>) : launch(rope_backward_kernel<64, __nv_bfloat16>)));
    PA_CUDA_OK(launch_pdl(rope_weights_kernel, dim3((unsigned)(2 * p->head_dim / 32)), 1024, 0, st,
                          static_cast<const float *>(a.parts), (int)ctas, (int)p->head_dim, dq_weight, dk_weight));
    return PA_OK;
}
