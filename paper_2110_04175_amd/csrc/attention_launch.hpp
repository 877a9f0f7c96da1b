// What the attention calls and the kernels of each type share.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#define RELAYSUM_HIDDEN __attribute__((visibility("hidden")))

namespace attention {

// Heads of n workers: entry k of head h of row t of worker i is entry
// i * ws + t * rs + h * hs + k.
struct Heads {
    char *data;
    int64_t ws, rs, hs;
};

struct AttentionArgs {
    Heads q, k, v, out;
    Heads dout, dq, dk, dv;
    float *lse;                // [n][heads][tokens]
    float2 *stats;             // [pairs][rows]: lse in powers of two, dout . out
    int4 *bounds;              // [n or 1][ceil(rows / 32)]: least and most lo, least and most hi
    int32_t *marks, *key_marks;   // of each workgroup: what it has done is to be done once more
    int32_t *order;            // [n or 1][ceil(keys / 128)]: worker * tiles + tile, or NULL
    const int2 *ranges;
    float *part_out;           // [pairs][rows][parts][width]; backward: [pairs][keys][parts][2 * width], dk and dv
    float2 *part_soft;         // [pairs][rows][parts]
    int64_t range_stride;      // rows between workers' ranges; 0: all have the same
    int64_t bound_stride;
    int32_t tokens, keys, heads, kv, group, width, rows;   // rows = tokens * group
    int32_t causal, tiles, parts, span;
    uint32_t pairs;            // n * kv
    uint32_t group_factor, group_shift;   // row / group = (mulhi(row, factor) + row) >> shift
    float scale, dot_scale;    // dot_scale = scale * log2(e)
};

// The heads' width that kernels are made for.
constexpr int padded_width(int64_t width) { return width <= 64 ? 64 : width <= 128 ? 128 : 256; }

// Waves of a workgroup that has few rows: as many as LDS holds the sums of.
constexpr int split_waves(int bytes, int padded) {
    const int own = 32 * padded * 4 + 16 * 32 * bytes + 256;
    return own * 8 <= 160 << 10 ? 8 : own * 4 <= 160 << 10 ? 4 : 2;
}

// Tiles of the forward pass, or the parts that the keys are split into.
struct ForwardPlan {
    int64_t blocks;
    int32_t tiles, parts, span;
    bool split;
    size_t workspace;
};

// Queue the kernels of a call; T is float, __bf16 or _Float16.
template <typename T>
RELAYSUM_HIDDEN void launch_attention(const AttentionArgs &a, const ForwardPlan &p, hipStream_t st);
template <typename T>
RELAYSUM_HIDDEN void launch_attention_backward(AttentionArgs a, int32_t n, hipStream_t st);

}  // namespace attention
