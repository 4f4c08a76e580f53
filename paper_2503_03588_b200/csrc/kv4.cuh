// The 4-bit page format (described at pa_kv4_pool in powerattn.h): where a token's bytes stand.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

#include "powerattn.h"

namespace pa {

constexpr int kKv4Page = 64;    // tokens of a page
constexpr int kKv4Group = 32;   // features that share a scale

template <int D>
struct Kv4Record {  // of a page and KV head, in bytes
    static constexpr int kGroups = D / kKv4Group;
    static constexpr int kRow = D / 2;                     // a token's nibbles
    static constexpr int kScaleRow = 2 * kGroups;          // a token's scales
    static constexpr int kScales = kKv4Page * kRow;        // where K's (or V's) scales start
    static constexpr int kHalf = kScales + kKv4Page * kScaleRow;  // K's part; V's follows
    static constexpr int kBytes = 2 * kHalf;               // 72 D
};

// How long a CTA of a cluster outlives a wait of its own that ran out, at most (in cycles): until each of its R peers has pushed its
// part of a row of `blocks` blocks, which takes a peer a wait of up to `limit` for each of its blocks and one more for the barrier of
// the cluster.  (Two million cycles a wait for the work itself.)  The table's length has no part in it.
__host__ __device__ inline long long kv4_outlast_cycles(long long limit, int32_t blocks, int32_t R)
{
    return (limit + 2000000ll) * (2 + (blocks + R - 1) / R);
}

// Checks of a pool's description, shared by the entry points.
pa_status check_kv4_pool(const pa_kv4_pool &p);

}  // namespace pa
