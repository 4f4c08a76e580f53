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

// Checks of a pool's description, shared by the entry points.
pa_status check_kv4_pool(const pa_kv4_pool &p);

}  // namespace pa
