// pa_decode_kv4: one query token per sequence against 4-bit pages (kv4.cuh) under the PowerAttention row of its position.
//
// The mathematics.  A key is k = s (u - 8) per group of 32 features, u its nibble, so a logit is
//   S = sum_j s_kj <q_j, u_kj - 8>   (j: the groups),
// with integer operands that 16 bits hold exactly: the products run on the tensor cores (m16n8k16, keys as the 16 rows, the
// query heads as the 8 columns) and each group's sum is scaled in fp32.  The output is
//   O = sum_k (p_k s_kj) (u_kj - 8),
// V's scales folded into the weights: one 16-bit weight per key and group.
//
// Logits take fp16 operands: q is bf16, and each head is divided by a power of two so that its largest entry lies in [1, 2) and
// fits (entries below 2^-14 of it lose bits that are below 2^-24 of it).  Weights are bf16, since V's scales may differ by any
// factor from key to key and from group to group: rounded once, half a step 2^-8 as the output's own rounding; for fp32
// outputs they come in two parts.
//
// The nibbles become 16-bit numbers without conversions: in fp16 (w & 0x000f000f) | 0x6400 is 1024 + u in both halves and
// (w & 0x00f000f0) | 0x6400 is 1024 + 16 u, in bf16 (w & 0x000f000f) | 0x4300 is 128 + u; one instruction takes u - 8 from
// each, exactly.  K rows are stored so that a thread's 16 bytes hold its share of every group; V rows so that the same
// halfwords of two tokens, put side by side by a byte permutation, are the fragments' key pairs.  Shared memory is read without
// bank conflicts and without ldmatrix.
//
// A CTA is four consumer warps and a producer.  A key block (one page and KV head: 72 D contiguous bytes) is one bulk copy into
// a ring of stages; warp w takes keys 16 w .. 16 w + 15 of every block and all features, with a maximum, sum and output of
// its own, and the four are merged at the end of the row.
#include <cuda_fp16.h>
#include <math.h>

#include <mutex>

#include "common.cuh"
#include "kv4.cuh"
#include "layout_rule.cuh"
#include "sm100_ptx.cuh"

namespace pa {

constexpr int kD4Consumers = 4;
constexpr int kD4Threads = 32 * (kD4Consumers + 1);
constexpr int kD4MaxGroup = 8;
constexpr int kD4MaxStages = 8;
constexpr int kD4MaxCluster = 8;
constexpr size_t kD4StatusBytes = 256;
constexpr int kD4MaxSmem = 227 * 1024;
constexpr long long kD4WaitCycles = 2000000000ll;  // ~1 s
constexpr float kD4Grow = 6.f;  // the maximum moves once it is exceeded by more than this (weights up to 2^6)

enum Kv4Form { KV4_ROWS = 0, KV4_CLUSTER = 1, KV4_PARTS = 2 };

struct Kv4Args {
    const __nv_bfloat16 *q;
    const uint8_t *pool;
    const int32_t *table, *lens;
    float *partial;  // [rows G][R][D + 2]
    int32_t *status;
    void *o;
    float *lse;
    int64_t page_stride, head_stride, max_len;
    int32_t table_stride, n_pages, batch, Hkv, G, W, S, R, stages, clear_status, o_is_f32;
    uint32_t items;
    float scale_log2;
    long long wait_cycles;
};

template <int D>
struct Kv4Smem {
    static constexpr uint32_t kStage = Kv4Record<D>::kBytes;
    static constexpr uint32_t kPartRow = (D + 4) * 4;  // (the pad spreads the heads over the banks)
    static constexpr uint32_t kPart = kD4Consumers * kD4MaxGroup * kPartRow;
    static constexpr uint32_t kStat = kD4Consumers * kD4MaxGroup * 8 + 16;  // maximum and sum; whether a warp got there
    static constexpr uint32_t kRecvRow = (D + 4) * 4;                  // o[D], m, l
    static constexpr uint32_t kRecv = 14 * kRecvRow;  // R senders x ceil(8 / R) heads
    static constexpr uint32_t kBars = (2 * kD4MaxStages + 2) * 8;
    static constexpr size_t bytes(int stages, bool cluster)
    {
        return 128 + (size_t)stages * kStage + kPart + kStat + (cluster ? kRecv : 0) + kBars;
    }
};

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};\n"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_b16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};\n"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t h2_fma(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t d;
    asm("fma.rn.f16x2 %0, %1, %2, %3;\n" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
__device__ __forceinline__ uint32_t h2_add(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("add.rn.f16x2 %0, %1, %2;\n" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
// The lowest nibble of each half of a word, or the one above it, as fp16 u - 8.
__device__ __forceinline__ uint32_t nib_lo(uint32_t w) { return h2_add((w & 0x000f000fu) | 0x64006400u, 0xe408e408u); }  // - 1032
__device__ __forceinline__ uint32_t nib_hi(uint32_t w)
{
    return h2_fma((w & 0x00f000f0u) | 0x64006400u, 0x2c002c00u, 0xd480d480u);  // / 16 - 72
}
// The lowest nibble of each half as bf16 u - 8.
__device__ __forceinline__ uint32_t nib_bf16(uint32_t w)
{
    uint32_t d;
    asm("add.rn.bf16x2 %0, %1, %2;\n" : "=r"(d) : "r"((w & 0x000f000fu) | 0x43004300u), "r"(0xc308c308u));  // - 136
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
// kForm KV4_ROWS: a persistent grid over the rows (sequence and KV head), results written at once.  KV4_CLUSTER: a row's blocks
// are dealt to the R CTAs of a cluster, which push their results to the CTA that merges a head (CTA h % R) by asynchronous
// stores.  KV4_PARTS: dealt to R CTAs anywhere, whose results go to the workspace for kv4_merge_kernel.
template <int D, bool kF32, int kForm>
__global__ void __launch_bounds__(kD4Threads, 3) kv4_decode_kernel(const Kv4Args a)
{
    using SM = Kv4Smem<D>;
    using R4 = Kv4Record<D>;
    constexpr int NG = R4::kGroups, NW = NG / 2;  // groups; words of a token's scales, or of a V chunk
    extern __shared__ __align__(128) uint8_t smem_raw[];
    const uint32_t smem = (ptx::smem_u32(smem_raw) + 127u) & ~127u;
    const int stages = a.stages;
    const uint32_t s_part = smem + (uint32_t)stages * SM::kStage, s_stat = s_part + SM::kPart;
    const uint32_t s_recv = s_stat + SM::kStat, bars = s_recv + (kForm == KV4_CLUSTER ? SM::kRecv : 0);
    volatile int *abort_flag =
        reinterpret_cast<volatile int *>(smem_raw + (bars - ptx::smem_u32(smem_raw)) + (2 * kD4MaxStages + 1) * 8);
    auto bar_full = [&](int s) { return bars + (uint32_t)s * 8u; };
    auto bar_empty = [&](int s) { return bars + (uint32_t)(kD4MaxStages + s) * 8u; };
    const uint32_t bar_recv = bars + 2 * kD4MaxStages * 8;
    auto wait_bar = [&](uint32_t b_, uint32_t parity, int code) {
        return ptx::mbar_wait_bounded(b_, parity, abort_flag, a.status, code, a.wait_cycles, (int)PA_ERR_TIMEOUT);
    };

    const int R = kForm == KV4_ROWS ? 1 : a.R, G = a.G;
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const int g = lane >> 2, t = lane & 3;
    const int my_r = kForm == KV4_CLUSTER ? (int)(blockIdx.x % (uint32_t)R) : 0;
    const int heads_here = G > my_r ? (G - my_r + R - 1) / R : 0, heads_per_owner = (kD4MaxGroup + R - 1) / R;

    // Started before the kernel ahead is done: nothing of global memory is touched up to pdl_wait().
    pdl_launch_next();
    if (tid == 0) {
        for (int s = 0; s < stages; ++s) {
            ptx::mbar_init(bar_full(s), 1);
            ptx::mbar_init(bar_empty(s), kD4Consumers);
        }
        if (kForm == KV4_CLUSTER) ptx::mbar_init(bar_recv, 1);
        *abort_flag = 0;
        ptx::fence_barrier_init();
        ptx::fence_proxy_async_smem();
        if (kForm == KV4_CLUSTER) ptx::mbar_expect_tx(bar_recv, (uint32_t)(heads_here * R) * (D + 2) * 4u);
    }
    __syncthreads();
    if (kForm == KV4_CLUSTER) ptx::cluster_arrive();  // (peers may push here from now on)
    pdl_wait();
    if (a.clear_status && blockIdx.x == 0 && tid == 0) a.status[0] = 0;

    const uint32_t it0 = blockIdx.x, it_step = gridDim.x;
    auto item_len = [&](uint32_t it) -> int32_t { return it < a.items ? a.lens[(it / (uint32_t)R) / (uint32_t)a.Hkv] : 0; };
    struct Item {
        uint32_t row;     // sequence x KV heads + KV head
        int32_t r, len;   // chunk; cache length, 0: invalid
        int32_t mine;     // blocks of the chunk
        LayoutRow list;
    };
    auto make_item = [&](uint32_t it, int32_t len) {
        Item w;
        w.row = it / (uint32_t)R;
        w.r = (int32_t)(it - w.row * (uint32_t)R);
        w.len = len >= 1 && len <= a.max_len ? len : 0;
        w.list = layout_row(w.len ? (w.len - 1) / kKv4Page : 0, a.W, a.S);
        const int32_t n = w.len ? (int32_t)w.list.n : 0;
        w.mine = n > w.r ? (n - w.r + R - 1) / R : 0;
        return w;
    };
    int32_t len_next = item_len(it0);

    if (wid == kD4Consumers) {
        // ------------------------------------------------------------------ producer
        bool ok = true;
        uint32_t ci = 0;  // blocks issued so far
        for (uint32_t it = it0; it < a.items; it += it_step) {
            const Item w = make_item(it, len_next);
            len_next = item_len(it + it_step);
            const uint32_t b = w.row / (uint32_t)a.Hkv, hk = w.row - b * (uint32_t)a.Hkv;
            auto issue = [&](uint32_t at, const uint8_t *src) {
                const int s = (int)(at % (uint32_t)stages);
                ptx::mbar_expect_tx(bar_full(s), SM::kStage);
                ptx::bulk_load(smem + (uint32_t)s * SM::kStage, src, SM::kStage, bar_full(s));
            };
            for (int base = 0; base < w.mine; base += 32) {
                // Each lane finds one block: from the diagonal block (the list's last) backwards, every R-th.
                const uint8_t *src = a.pool;
                if (base + lane < w.mine) {
                    const int32_t j = (int32_t)layout_entry(w.list, w.list.n - 1 - (w.r + (int64_t)(base + lane) * R));
                    int32_t page = a.table[(int64_t)b * a.table_stride + j];
                    page = page < 0 ? 0 : page >= a.n_pages ? a.n_pages - 1 : page;
                    src = a.pool + (int64_t)page * a.page_stride + (int64_t)hk * a.head_stride;
                }
                const int count = min(32, w.mine - base);
                int x = 0;
                if (ci < (uint32_t)stages) {  // stages that nothing has been in yet: all at once
                    x = min(count, stages - (int)ci);
                    if (lane < x) issue(ci + lane, src);
                }
                for (; x < count; ++x) {
                    const uint64_t from = __shfl_sync(0xffffffffu, reinterpret_cast<uint64_t>(src), x);
                    if (lane == 0 && ok) {
                        const uint32_t at = ci + x;
                        ok = wait_bar(bar_empty((int)(at % (uint32_t)stages)), (at / (uint32_t)stages - 1) & 1, 1);
                        if (ok) issue(at, reinterpret_cast<const uint8_t *>(from));
                    }
                }
                __syncwarp();
                ci += count;
            }
        }
        if (kForm == KV4_CLUSTER) ptx::cluster_wait();
    } else {
        // ------------------------------------------------------------------ consumers
        // Row r of the 16 x 16 fragments, r < 8, is key r ^ (r / 4) of the warp's (r >= 8: that plus 8): a permutation
        // under which the threads' reads of K rows and of V rows fall into different banks.
        const int key_a = 16 * wid + (g ^ (g >> 2));                                      // rows g (and g + 8) of S
        const int v0 = 16 * wid + ((2 * t) ^ (t >> 1)), v1 = 16 * wid + ((2 * t + 1) ^ (t >> 1));  // columns 2t, 2t + 1
        const uint32_t off_k = (uint32_t)key_a * R4::kRow + (uint32_t)t * 4u * NG;
        const uint32_t off_ks = R4::kScales + (uint32_t)key_a * R4::kScaleRow;
        auto off_v = [&](int key) { return (uint32_t)(R4::kHalf + key * R4::kRow + (g ^ ((key & 2) << 1)) * 2 * NG); };
        const uint32_t off_v0 = off_v(v0), off_v1 = off_v(v1);

        uint4 raw[NG];
        auto load_q = [&](uint32_t it) {
            const bool in = it < a.items && g < G;
            const __nv_bfloat16 *qb = a.q + ((int64_t)(in ? it / (uint32_t)R : 0) * G + (in ? g : 0)) * D + 8 * t;
#pragma unroll
            for (int j = 0; j < NG; ++j)
                raw[j] = in ? *reinterpret_cast<const uint4 *>(qb + 32 * j) : make_uint4(0u, 0u, 0u, 0u);
        };
        load_q(it0);
        bool ok = true;
        uint32_t ci = 0;
        for (uint32_t it = it0; it < a.items && ok; it += it_step) {
            const Item w = make_item(it, len_next);
            len_next = item_len(it + it_step);
            // ---- Q as the B operand: head g, features 32 j + 8 t + {0, 4}, {1, 5}, {2, 6}, {3, 7}
            uint32_t qf[NG][4];
            float c0, c1;  // factors of heads 2t and 2t + 1: the power of two, the softmax scale, log2 e
            {
                uint32_t top = 0;
#pragma unroll
                for (int j = 0; j < NG; ++j)
                    for (uint32_t x : {raw[j].x, raw[j].y, raw[j].z, raw[j].w}) top = max(top, max(x & 0x7fffu, (x >> 16) & 0x7fffu));
                top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
                const uint32_t field = min(max(top >> 7, 1u), 253u);
                const float down = __uint_as_float((254u - field) << 23), up = __uint_as_float(field << 23) * a.scale_log2;
                c0 = __shfl_sync(0xffffffffu, up, 8 * t);
                c1 = __shfl_sync(0xffffffffu, up, 8 * t + 4);
#pragma unroll
                for (int j = 0; j < NG; ++j) {
                    qf[j][0] = cvt_f16x2(bf16_lo(raw[j].x) * down, bf16_lo(raw[j].z) * down);
                    qf[j][1] = cvt_f16x2(bf16_hi(raw[j].x) * down, bf16_hi(raw[j].z) * down);
                    qf[j][2] = cvt_f16x2(bf16_lo(raw[j].y) * down, bf16_lo(raw[j].w) * down);
                    qf[j][3] = cvt_f16x2(bf16_hi(raw[j].y) * down, bf16_hi(raw[j].w) * down);
                }
            }
            float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;  // of heads 2t, 2t + 1 (the sums: this thread's keys)
            float acc[2 * NG][4];  // O^T: tile 2 j + h, rows 32 j + 4 g + 2 h + {0, 1}, heads 2t, 2t + 1
#pragma unroll
            for (int e = 0; e < 2 * NG; ++e) acc[e][0] = acc[e][1] = acc[e][2] = acc[e][3] = 0.f;
#pragma unroll 1
            for (int i = 0; i < w.mine && ok; ++i, ++ci) {
                const int s = (int)(ci % (uint32_t)stages);
                const int n_keys = w.r == 0 && i == 0 ? (w.len - 1) % kKv4Page + 1 : kKv4Page;  // (the diagonal block is first)
                ok = wait_bar(bar_full(s), (ci / (uint32_t)stages) & 1, 2);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                if (16 * wid < n_keys) {
                    const uint32_t st = smem + (uint32_t)s * SM::kStage;
                    uint32_t ka[NG], kb[NG], sa[NW], sb[NW], va[NW], vb[NW];
                    lds_words(st + off_k, ka);
                    lds_words(st + off_k + 8 * R4::kRow, kb);
                    lds_words(st + off_ks, sa);
                    lds_words(st + off_ks + 8 * R4::kScaleRow, sb);
                    lds_words(st + R4::kHalf + off_ks, va);
                    lds_words(st + R4::kHalf + off_ks + 8 * R4::kScaleRow, vb);
                    // ---- S^T = K Q^T: keys x heads, group by group
                    float sx[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int j = 0; j < NG; ++j) {
                        float d[4] = {0.f, 0.f, 0.f, 0.f};
                        mma_f16(d, nib_lo(ka[j]), nib_lo(kb[j]), nib_hi(ka[j]), nib_hi(kb[j]), qf[j][0], qf[j][1]);
                        const uint32_t u = ka[j] >> 8, v = kb[j] >> 8;
                        mma_f16(d, nib_lo(u), nib_lo(v), nib_hi(u), nib_hi(v), qf[j][2], qf[j][3]);
                        const float s0 = j & 1 ? bf16_hi(sa[j / 2]) : bf16_lo(sa[j / 2]);
                        const float s1 = j & 1 ? bf16_hi(sb[j / 2]) : bf16_lo(sb[j / 2]);
                        sx[0] = fmaf(s0, d[0], sx[0]);
                        sx[1] = fmaf(s0, d[1], sx[1]);
                        sx[2] = fmaf(s1, d[2], sx[2]);
                        sx[3] = fmaf(s1, d[3], sx[3]);
                    }
                    uint32_t wa[NW], wb[NW], wc[NW], wd[NW];  // V: keys v0, v1, v0 + 8, v1 + 8
                    lds_words(st + off_v0, wa);
                    lds_words(st + off_v1, wb);
                    lds_words(st + off_v0 + 8 * R4::kRow, wc);
                    lds_words(st + off_v1 + 8 * R4::kRow, wd);
                    sx[0] *= c0;
                    sx[1] *= c1;
                    sx[2] *= c0;
                    sx[3] *= c1;
                    // Keys that do not exist: no weight, whatever the page holds there.
                    if (n_keys < kKv4Page) {
                        if (key_a >= n_keys) {
                            sx[0] = sx[1] = -INFINITY;
#pragma unroll
                            for (int y = 0; y < NW; ++y) va[y] = 0u;
                        }
                        if (key_a + 8 >= n_keys) {
                            sx[2] = sx[3] = -INFINITY;
#pragma unroll
                            for (int y = 0; y < NW; ++y) vb[y] = 0u;
                        }
                    }
                    float mx0 = fmaxf(sx[0], sx[2]), mx1 = fmaxf(sx[1], sx[3]);
#pragma unroll
                    for (int o = 4; o < 32; o *= 2) {
                        mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, o));
                        mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, o));
                    }
                    // The maximum is moved only where it is exceeded by far: the weights stay below 2^6.
                    const bool up0 = mx0 > m0 + kD4Grow, up1 = mx1 > m1 + kD4Grow;
                    if (__any_sync(0xffffffffu, up0 || up1)) {
                        const float al0 = up0 ? ptx::ex2(m0 - mx0) : 1.f, al1 = up1 ? ptx::ex2(m1 - mx1) : 1.f;
                        m0 = up0 ? mx0 : m0;
                        m1 = up1 ? mx1 : m1;
                        l0 *= al0;
                        l1 *= al1;
#pragma unroll
                        for (int e = 0; e < 2 * NG; ++e) {
                            acc[e][0] *= al0;
                            acc[e][1] *= al1;
                            acc[e][2] *= al0;
                            acc[e][3] *= al1;
                        }
                    }
                    const bool none_a = key_a >= n_keys, none_b = key_a + 8 >= n_keys;
                    const float p0 = none_a ? 0.f : ptx::ex2(sx[0] - m0), p1 = none_a ? 0.f : ptx::ex2(sx[1] - m1);
                    const float p2 = none_b ? 0.f : ptx::ex2(sx[2] - m0), p3 = none_b ? 0.f : ptx::ex2(sx[3] - m1);
                    l0 += p0 + p2;
                    l1 += p1 + p3;
                    // ---- O^T += V^T P^T, group by group: the weights times the keys' scales, transposed into the B operand
#pragma unroll
                    for (int j = 0; j < NG; ++j) {
                        const float s0 = j & 1 ? bf16_hi(va[j / 2]) : bf16_lo(va[j / 2]);
                        const float s1 = j & 1 ? bf16_hi(vb[j / 2]) : bf16_lo(vb[j / 2]);
                        const float w0 = p0 * s0, w1 = p1 * s0, w2 = p2 * s1, w3 = p3 * s1;
                        const uint32_t h0 = ptx::cvt_bf16x2(w0, w1), h1 = ptx::cvt_bf16x2(w2, w3);
                        const uint32_t b0 = transpose8(h0), b1 = transpose8(h1);
                        uint32_t b2 = 0u, b3 = 0u;
                        if (kF32) {  // what the rounding left
                            b2 = transpose8(ptx::cvt_bf16x2(w0 - bf16_lo(h0), w1 - bf16_hi(h0)));
                            b3 = transpose8(ptx::cvt_bf16x2(w2 - bf16_lo(h1), w3 - bf16_hi(h1)));
                        }
                        const uint32_t sel = j & 1 ? 0x7632u : 0x5410u;
                        uint32_t x = __byte_perm(wa[j / 2], wb[j / 2], sel), y = __byte_perm(wc[j / 2], wd[j / 2], sel);
#pragma unroll
                        for (int h = 0; h < 2; ++h, x >>= 8, y >>= 8) {
                            const uint32_t a0 = nib_bf16(x), a1 = nib_bf16(x >> 4), a2 = nib_bf16(y), a3 = nib_bf16(y >> 4);
                            mma_b16(acc[2 * j + h], a0, a1, a2, a3, b0, b1);
                            if (kF32) mma_b16(acc[2 * j + h], a0, a1, a2, a3, b2, b3);
                        }
                    }
                }
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(bar_empty(s));
            }
            load_q(it + it_step);

            // ---- The four warps' results meet in shared memory.
#pragma unroll
            for (int o = 4; o < 32; o *= 2) {
                l0 += __shfl_xor_sync(0xffffffffu, l0, o);
                l1 += __shfl_xor_sync(0xffffffffu, l1, o);
            }
            {
                const uint32_t row0 = s_part + (uint32_t)(wid * kD4MaxGroup + 2 * t) * SM::kPartRow + 16u * g;
#pragma unroll
                for (int j = 0; j < NG; ++j)
#pragma unroll
                    for (int x = 0; x < 2; ++x)
                        ptx::st_shared_v4(row0 + x * SM::kPartRow + 128u * j, __float_as_uint(acc[2 * j][x]), __float_as_uint(acc[2 * j][2 + x]),
                                          __float_as_uint(acc[2 * j + 1][x]), __float_as_uint(acc[2 * j + 1][2 + x]));
                if (lane == 0) ptx::st_shared(s_stat + kD4Consumers * kD4MaxGroup * 8u + 4u * wid, ok ? 1u : 0u);
                if (g == 0) {
                    const uint32_t at = s_stat + (uint32_t)(wid * kD4MaxGroup + 2 * t) * 8u;
                    ptx::st_shared_v4(at, __float_as_uint(m0), __float_as_uint(l0), __float_as_uint(m1), __float_as_uint(l1));
                }
            }
            asm volatile("bar.sync 1, %0;\n" ::"n"(32 * kD4Consumers) : "memory");
            // (A wait that gave up ends the loop for all four, or those that go on would wait for the others for good.)
#pragma unroll
            for (int x = 0; x < kD4Consumers; ++x)
                ok = ok && ptx::ld_shared(s_stat + kD4Consumers * kD4MaxGroup * 8u + 4u * x) != 0u;
            // Thread: head tid / 16, features 4 (tid % 16) + {0 .. 3} (and 64 more).
            const int h = tid >> 4, f0 = 4 * (tid & 15);
            float m = -INFINITY, l = 0.f;
            float4 out[D / 64];
            {
                float mw[kD4Consumers], lw[kD4Consumers];
#pragma unroll
                for (int x = 0; x < kD4Consumers; ++x) {
                    ptx::ld_shared_v2(s_stat + (uint32_t)(x * kD4MaxGroup + h) * 8u, mw[x], lw[x]);
                    m = fmaxf(m, mw[x]);
                }
#pragma unroll
                for (int y = 0; y < D / 64; ++y) out[y] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int x = 0; x < kD4Consumers; ++x) {
                    const float wgt = mw[x] != -INFINITY ? ptx::ex2(mw[x] - m) : 0.f;
                    l = fmaf(lw[x], wgt, l);
#pragma unroll
                    for (int y = 0; y < D / 64; ++y) {
                        float4 v;
                        ptx::ld_shared_v4(s_part + (uint32_t)(x * kD4MaxGroup + h) * SM::kPartRow + 4u * (f0 + 64 * y), v.x, v.y, v.z, v.w);
                        out[y].x = fmaf(v.x, wgt, out[y].x);
                        out[y].y = fmaf(v.y, wgt, out[y].y);
                        out[y].z = fmaf(v.z, wgt, out[y].z);
                        out[y].w = fmaf(v.w, wgt, out[y].w);
                    }
                }
            }
            if (kForm == KV4_CLUSTER) {
                ptx::cluster_wait();  // every CTA of the row has set its barrier up
                if (h < G) {
                    const uint32_t slot = (uint32_t)(h / R), owner = (uint32_t)(h - (int)slot * R);
                    const uint32_t dst = ptx::map_shared(s_recv, owner) + ((uint32_t)w.r * (uint32_t)heads_per_owner + slot) * SM::kRecvRow;
                    const uint32_t their_bar = ptx::map_shared(bar_recv, owner);
#pragma unroll
                    for (int y = 0; y < D / 64; ++y) ptx::st_async_v4(dst + 4u * (f0 + 64 * y), out[y], their_bar);
                    if ((tid & 15) == 0) ptx::st_async_v2(dst + 4u * D, m, l, their_bar);
                }
            } else if (h < G) {
                const int64_t head = (int64_t)w.row * G + h;
                if (kForm == KV4_PARTS) {
                    float *dst = a.partial + (head * R + w.r) * (D + 2);
#pragma unroll
                    for (int y = 0; y < D / 64; ++y) {
                        *reinterpret_cast<float2 *>(dst + f0 + 64 * y) = make_float2(out[y].x, out[y].y);
                        *reinterpret_cast<float2 *>(dst + f0 + 64 * y + 2) = make_float2(out[y].z, out[y].w);
                    }
                    if ((tid & 15) == 0) *reinterpret_cast<float2 *>(dst + D) = make_float2(m, l);
                } else {
                    const float inv = w.mine > 0 ? 1.0f / l : 0.f;
#pragma unroll
                    for (int y = 0; y < D / 64; ++y) {
                        const int64_t at = head * D + f0 + 64 * y;
                        const float4 v = make_float4(out[y].x * inv, out[y].y * inv, out[y].z * inv, out[y].w * inv);
                        if (kF32)
                            *reinterpret_cast<float4 *>(static_cast<float *>(a.o) + at) = v;
                        else
                            *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(a.o) + at) =
                                make_uint2(ptx::cvt_bf16x2(v.x, v.y), ptx::cvt_bf16x2(v.z, v.w));
                    }
                    if ((tid & 15) == 0) a.lse[head] = w.mine > 0 ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
                }
            }
            // The area is written again only after every warp has read it.
            if (kForm != KV4_CLUSTER) asm volatile("bar.sync 1, %0;\n" ::"n"(32 * kD4Consumers) : "memory");
        }

        if (kForm == KV4_CLUSTER && heads_here > 0) {
            // ---- Heads r, r + R, ... of the row: D threads a head.
            if (!ptx::mbar_wait_bounded_cluster(bar_recv, 0, abort_flag, a.status, 3, a.wait_cycles, (int)PA_ERR_TIMEOUT)) {
                // This CTA's shared memory has to last until every peer's part is in it: a peer is there after a wait for each of
                // its blocks at most, so this is over before its own limit is.
                const long long t0 = clock64(), most = 4 * (a.wait_cycles + 2000000ll) * (2 + (int64_t)a.table_stride / R);
                while (!ptx::mbar_try_wait_cluster(bar_recv, 0) && clock64() - t0 < most) {
                }
            } else {
                const uint32_t row = it0 / (uint32_t)R;
                constexpr int kPer = 32 * kD4Consumers / D;  // heads at a time
                for (int slot = tid / D; slot < heads_here; slot += kPer) {
                    const int d = tid % D, hh = my_r + slot * R;
                    float m = -INFINITY, l = 0.f, o = 0.f;
                    float mr[kD4MaxCluster], lr[kD4MaxCluster], orr[kD4MaxCluster];
#pragma unroll
                    for (int x = 0; x < kD4MaxCluster; ++x) {
                        const uint32_t src = s_recv + (uint32_t)((x < R ? x : 0) * heads_per_owner + slot) * SM::kRecvRow;
                        ptx::ld_shared_v2(src + 4u * D, mr[x], lr[x]);
                        orr[x] = __uint_as_float(ptx::ld_shared(src + 4u * d));
                    }
#pragma unroll
                    for (int x = 0; x < kD4MaxCluster; ++x)
                        if (x < R) m = fmaxf(m, mr[x]);
#pragma unroll
                    for (int x = 0; x < kD4MaxCluster; ++x) {
                        const float wgt = mr[x] != -INFINITY ? ptx::ex2(mr[x] - m) : 0.f;
                        if (x < R) {
                            l = fmaf(lr[x], wgt, l);
                            o = fmaf(orr[x], wgt, o);
                        }
                    }
                    const bool any = l != 0.f;  // (no key: a length outside [1, max_len])
                    const float res = any ? o / l : 0.f;
                    const int64_t head = (int64_t)row * G + hh;
                    if (kF32)
                        static_cast<float *>(a.o)[head * D + d] = res;
                    else
                        static_cast<__nv_bfloat16 *>(a.o)[head * D + d] = __float2bfloat16_rn(res);
                    if (d == 0) a.lse[head] = any ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
                }
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

// The parts of a row's chunks, merged: a CTA per sequence and query head, a thread per feature.
template <int D, bool kF32>
__global__ void __launch_bounds__(D) kv4_merge_kernel(const Kv4Args a)
{
    __shared__ float s_max[D / 32];
    const int d = threadIdx.x;
    const int64_t head = blockIdx.x;
    pdl_launch_next();
    pdl_wait();
    const float *src = a.partial + head * a.R * (D + 2);
    float m = -INFINITY;
    for (int c = d; c < a.R; c += D) m = fmaxf(m, src[(int64_t)c * (D + 2) + D]);
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if ((d & 31) == 0) s_max[d >> 5] = m;
    __syncthreads();
#pragma unroll
    for (int x = 0; x < D / 32; ++x) m = fmaxf(m, s_max[x]);
    float l = 0.f, o = 0.f;
#pragma unroll 8
    for (int c = 0; c < a.R; ++c) {
        const float *p = src + (int64_t)c * (D + 2);
        const float mc = p[D], wgt = mc != -INFINITY ? ptx::ex2(mc - m) : 0.f;
        l = fmaf(p[D + 1], wgt, l);
        o = fmaf(p[d], wgt, o);
    }
    const bool any = l != 0.f;
    const float res = any ? o / l : 0.f;
    if (kF32)
        static_cast<float *>(a.o)[head * D + d] = res;
    else
        static_cast<__nv_bfloat16 *>(a.o)[head * D + d] = __float2bfloat16_rn(res);
    if (d == 0) a.lse[head] = any ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

// ------------------------------------------------------------------------------------------ host
constexpr int kD4MaxParts = 64;  // chunks per row in the KV4_PARTS form

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
    return PA_OK;
}

static int kv4_stages(int head_dim, int most)
{
    const int n = head_dim == 128 ? 6 : 8;
    return most < n ? most : n;
}
static int kv4_most_blocks(const pa_kv4_params *p)
{
    const int64_t rows = p->max_blocks_per_seq, w = p->window_blocks > 1 ? p->window_blocks : 1;
    int64_t n = w + p->sink_blocks;
    for (int64_t pw = 1; pw < rows; pw *= 2) n += pw >= w;
    return (int)(n < rows ? n : rows);
}
static size_t kv4_smem(int head_dim, int stages, bool cluster)
{
    return head_dim == 128 ? Kv4Smem<128>::bytes(stages, cluster) : Kv4Smem<64>::bytes(stages, cluster);
}
// Parts per row, at most: two CTAs a row of 148 x 3 places would be too few otherwise.
static int kv4_parts(int64_t rows, int most)
{
    int64_t R = (148 * 3) / rows;
    if (R > most / 4) R = most / 4;
    if (R > kD4MaxParts) R = kD4MaxParts;
    return R < 1 ? 1 : (int)R;
}

using Kv4Kernel = void (*)(const Kv4Args);
static Kv4Kernel kv4_kernel(int head_dim, bool f32, int form)
{
    static const Kv4Kernel kernels[2][2][3] = {
        {{kv4_decode_kernel<64, false, 0>, kv4_decode_kernel<64, false, 1>, kv4_decode_kernel<64, false, 2>},
         {kv4_decode_kernel<64, true, 0>, kv4_decode_kernel<64, true, 1>, kv4_decode_kernel<64, true, 2>}},
        {{kv4_decode_kernel<128, false, 0>, kv4_decode_kernel<128, false, 1>, kv4_decode_kernel<128, false, 2>},
         {kv4_decode_kernel<128, true, 0>, kv4_decode_kernel<128, true, 1>, kv4_decode_kernel<128, true, 2>}}};
    return kernels[head_dim == 128][f32][form];
}

}  // namespace pa

extern "C" size_t pa_decode_kv4_workspace_bytes(const pa_kv4_params *p)
{
    using namespace pa;
    if (check_kv4(p) != PA_OK) return 0;
    const int most = kv4_most_blocks(p), parts = kD4MaxParts < most ? kD4MaxParts : most;
    return kD4StatusBytes + (size_t)p->batch * p->n_q_heads * parts * (p->pool.head_dim + 2) * sizeof(float);
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
    Kv4Args a;
    a.q = static_cast<const __nv_bfloat16 *>(q);
    a.pool = static_cast<const uint8_t *>(kv_pool);
    a.table = block_table;
    a.lens = cache_lens;
    a.status = static_cast<int32_t *>(workspace);
    a.partial = reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) + kD4StatusBytes);
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
    a.o_is_f32 = p->o_dtype == PA_F32;
    const float scale = p->softmax_scale != 0.f ? p->softmax_scale : 1.0f / sqrtf((float)D);
    a.scale_log2 = scale * 1.4426950408889634f;
    const long long wait_cycles = wait_limit_cycles();
    a.wait_cycles = wait_cycles > 0 ? wait_cycles : kD4WaitCycles;
    a.clear_status = wait_cycles <= 0;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (!a.clear_status) PA_CUDA_OK(cudaMemsetAsync(a.status, 0, sizeof(int32_t), st));

    const EnvSwitches env = env_switches();
    const bool f32 = p->o_dtype == PA_F32;
    const int most = kv4_most_blocks(p);
    const int64_t rows = (int64_t)a.batch * a.Hkv, places = (int64_t)dev.sms * 3;
    if (rows > 0x3fffffff / kD4MaxParts) return fail(PA_ERR_SHAPE, "too many rows (%lld)", (long long)rows);
    int form = rows * 2 <= places ? KV4_CLUSTER : KV4_ROWS, R = 1;
    if (form == KV4_CLUSTER && kv4_parts(rows, most) > kD4MaxCluster) form = KV4_PARTS;
    if (env.decode_path == 1) form = KV4_PARTS;
    if (env.decode_path == 2) form = KV4_CLUSTER;
    if (env.decode_path == 3) form = KV4_ROWS;
    if (form != KV4_ROWS) {
        R = form == KV4_PARTS ? kv4_parts(rows, most) : (int)(places / rows < kD4MaxCluster ? places / rows : kD4MaxCluster);
        if (env.decode_cluster) R = env.decode_cluster;
        if (R > most) R = most;
        if (R < 1) R = 1;
        if (R == 1 && env.decode_path != 2 && env.decode_path != 1) form = KV4_ROWS;
    }
    a.R = R;
    a.items = (uint32_t)(rows * R);
    a.stages = env.decode_stages ? env.decode_stages : kv4_stages(D, (most + R - 1) / R);

    if (pa_status s = device_once(dev.device, ONCE_KV4_ATTR, [] {
            cudaError_t e = cudaSuccess;
            for (int i = 0; i < 12; ++i)
                e = first_error(e, cudaFuncSetAttribute(kv4_kernel(i & 1 ? 128 : 64, i & 2, i / 4),
                                                        cudaFuncAttributeMaxDynamicSharedMemorySize, kD4MaxSmem));
            return e;
        }))
        return s;
    const bool cluster = form == KV4_CLUSTER;
    cudaLaunchAttribute attr[2];
    attr[0] = pdl_attribute();
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)R;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(cluster || (int64_t)a.items < places ? a.items : places), 1, 1);
    cfg.blockDim = dim3(kD4Threads, 1, 1);
    cfg.dynamicSmemBytes = kv4_smem(D, a.stages, cluster);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = cluster ? 2 : 1;
    PA_CUDA_OK(cudaLaunchKernelEx(&cfg, kv4_kernel(D, f32, form), a));
    if (form != KV4_PARTS) return PA_OK;
    const dim3 heads((unsigned)((int64_t)a.batch * p->n_q_heads));
    if (D == 128)
        PA_CUDA_OK(f32 ? launch_pdl(kv4_merge_kernel<128, true>, heads, 128, 0, st, a) : launch_pdl(kv4_merge_kernel<128, false>, heads, 128, 0, st, a));
    else
        PA_CUDA_OK(f32 ? launch_pdl(kv4_merge_kernel<64, true>, heads, 64, 0, st, a) : launch_pdl(kv4_merge_kernel<64, false>, heads, 64, 0, st, a));
    return PA_OK;
}
