// Attention: the C calls (relaysum.h), and the ranges of packed sequences.  The
// kernels are in attention_kernels.hpp.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "attention_launch.hpp"
#include "layer_call.hpp"

namespace {

using namespace attention;

constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kMaxHeadWidth = 256;

// ---- ranges of packed sequences --------------------------------------------------------

struct RangeArgs {
    const int32_t *starts, *key_starts;
    int64_t starts_stride, key_starts_stride, ranges_stride;
    int2 *ranges;
    int64_t tokens, total;
    int32_t keys, count, causal;
};

__global__ __launch_bounds__(256) void attention_ranges_kernel(RangeArgs a) {
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= a.total) return;
    const int64_t worker = at / a.tokens;
    const int t = (int)(at - worker * a.tokens);
    const int32_t *s = a.starts + worker * a.starts_stride, *ks = a.key_starts + worker * a.key_starts_stride;
    // The last sequence that starts at or before t.
    int low = 0, high = a.count + 1;
    while (low < high) {
        const int mid = (low + high) / 2;
        if (s[mid] <= t) low = mid + 1;
        else high = mid;
    }
    int2 r = {0, 0};
    if (low > 0 && low <= a.count) {
        const int lo = ks[low - 1], hi = ks[low], left = s[low] - 1 - t;
        r.x = max(0, min(lo, a.keys));
        r.y = (int)max((int64_t)r.x, min((int64_t)a.keys, a.causal ? (int64_t)hi - left : (int64_t)hi));
    }
    a.ranges[worker * a.ranges_stride + t] = r;
}

// ---- host side -------------------------------------------------------------------------

Heads heads_of(const relaysum_heads *h, int32_t n, int64_t rows, int32_t heads) {
    if (!h) return Heads{nullptr, 0, 0, 0};
    return Heads{static_cast<char *>(h->data), n > 1 ? h->worker_stride : 0, rows > 1 ? h->row_stride : 0,
                 heads > 1 ? h->head_stride : 0};
}

struct AttentionCall : Call {
    bool shape(int32_t n, int64_t tokens, int64_t keys, int32_t heads, int32_t kv, int64_t width) {
        if (!sizes(n, tokens, 1, "tokens")) return false;
        if (keys < 0 || keys > (int64_t)1 << 30 || tokens > (int64_t)1 << 30)
            fail(refuse("tokens and keys must be in 0..2^30"));
        else if (heads < 1 || kv < 1 || heads % kv)
            fail(refuse("heads must be a multiple of kv_heads, both at least 1"));
        else if (width < 1 || width > kMaxHeadWidth)
            fail(refuse("the heads' width must be in 1..%d", kMaxHeadWidth));
        else if (heads > 65536 || (__int128)tokens * heads > ((__int128)1 << 30))
            fail(refuse("tokens * heads is more than 2^30"));
        else if ((__int128)n * (tokens + keys) * heads * width > ((__int128)1 << 50))
            fail(refuse("n * (tokens + keys) * heads * width is more than 2^50"));
        return code == RELAYSUM_OK;
    }

    void heads(const char *name, const relaysum_heads *h, int32_t type, int32_t n, int64_t rows, int32_t heads,
               int64_t width, bool out) {
        if (code != RELAYSUM_OK) return;
        if (!h) return fail(refuse("%s must not be NULL", name));
        if (h->type < RELAYSUM_FLOAT || h->type > RELAYSUM_HALF) return fail(refuse("%s: unknown type %d", name, h->type));
        if (h->type != type) return fail(refuse("%s is not of q's type", name));
        const Heads s = heads_of(h, n, rows, heads);
        const int64_t most = (int64_t)1 << 44;
        if (s.ws < 0 || s.rs < 0 || s.hs < 0 || s.ws > most / n || (rows && s.rs > most / rows) || s.hs > most / heads)
            return fail(refuse("%s: a stride is negative or reaches past 2^44 entries", name));
        if (!rows) return;
        // Outputs' rows must not share entries: each axis steps over all of the
        // smaller ones.
        int64_t step[3] = {s.ws, s.rs, s.hs}, times[3] = {n, rows, heads};
        for (int i = 0; i < 3; ++i)
            for (int j = i + 1; j < 3; ++j)
                if (step[j] < step[i]) std::swap(step[i], step[j]), std::swap(times[i], times[j]);
        int64_t extent = width;
        for (int i = 0; i < 3; ++i) {
            if (times[i] == 1) continue;
            if (out && step[i] < extent) return fail(refuse("%s: its rows overlap", name));
            extent += (times[i] - 1) * step[i];
        }
        const int64_t b = (int64_t)type_bytes(type);
        Span span{name, static_cast<const char *>(h->data), (size_t)(extent * b), out, true, width * b, s.ws * b, s.rs * b, n, rows};
        span.hs = s.hs * b;
        span.heads = heads;
        add(span, type_bytes(type));
    }

    void ranges(const int32_t *r, int64_t stride, int32_t n, int64_t tokens, bool out) {
        if (code != RELAYSUM_OK || (!r && !out)) return;
        if (n == 1) stride = 0;
        if (stride < 0 || (stride > 0 && stride < tokens) || stride > ((int64_t)1 << 40) / n)
            return fail(refuse("ranges_stride must be 0 or at least tokens"));
        if (out && n > 1 && stride < tokens) return fail(refuse("ranges_stride must be at least tokens"));
        span("ranges", r, (size_t)((n - 1) * stride + tokens) * 8, 8, out);
    }
};

ForwardPlan plan_forward(int32_t n, int64_t tokens, int64_t keys, int32_t heads, int32_t kv, int64_t width, int32_t type) {
    const int64_t pairs = (int64_t)n * kv, rows = tokens * (heads / kv);
    ForwardPlan p{};
    p.tiles = (int32_t)tiles(rows, 128);
    p.blocks = pairs * p.tiles;
    p.workspace = (size_t)p.blocks * 4;
    // Tiles of 128 rows, whose waves share keys in LDS, where they are full and occupy
    // a quarter of the CUs.  Causal prompts in bfloat16, us in tiles and in parts, heads
    // of 64 | 128:
    //   114 tiles,  777 keys, 3 workers   19,  24 |  27,  52
    //    64 tiles, 2048 keys, 4 on 4      37,  53 |  54,  90
    //    64 tiles, 1024 keys, 8 on 8      23,  16 |  33,  34
    //    32 tiles, 4096 keys, 1 on 1      66,  43 |  97,  77
    //    32 tiles,  512 keys, 8 on 8      15,  12 |  22,  25
    //    32 tiles,  256 keys, 16 on 16    12,  10 |  16,  22
    //    64 tiles of 96 rows, 1024 keys   22,  18 |  33,  40
    // So the border is not sharp: full tiles of short prompts lose by a third at heads
    // of 64 (of floats by half), parts below it by up to a third at heads of 128.
    if (p.blocks >= kCus || (rows >= 128 && p.blocks >= kCus / 4)) return p;
    p.split = true;
    const int64_t waves = split_waves((int)type_bytes(type), padded_width(width));
    p.tiles = (int32_t)tiles(rows, 32);
    const int64_t base = pairs * p.tiles;
    // Up to four steps of each wave need no parts, which cost a second kernel.  A row's
    // three heads on each key head of 64 bfloat16 entries, us with parts from 2, 4 and
    // 8 steps on: 16 key heads and 1024 keys 11.9, 12.8, 12.8, 2048 keys 11.9, 13.3, 18.9;
    // 256 key heads 26, 17, 17 and 35, 35, 27.
    const int64_t want = keys <= 4 * 32 * waves ? 1 : std::min<int64_t>(tiles(keys, 64 * waves), tiles(2 * kCus, std::max<int64_t>(1, base)));
    p.span = (int32_t)std::max<int64_t>(32, tiles(tiles(keys, want), 32) * 32);
    p.parts = (int32_t)std::max<int64_t>(1, tiles(keys, p.span));
    p.blocks = base * p.parts;
    p.workspace = p.parts > 1 ? (size_t)pairs * rows * p.parts * (width + 2) * 4 : 0;
    return p;
}

struct BackwardPlan {
    int32_t parts;
    size_t stats, bounds, order, marks, key_marks, sums;   // offsets
    size_t workspace;
};

BackwardPlan plan_backward(int32_t n, int64_t tokens, int64_t keys, int32_t heads, int32_t kv, int64_t width) {
    BackwardPlan p{};
    const int64_t rows = tokens * heads, pairs = (int64_t)n * kv, blocks = pairs * tiles(keys, 128);
    // Rows of a key head are split over workgroups where there are few of them, at
    // least four tiles each; without keys there is nothing to split.
    p.parts = 1;
    const int64_t enough = width > 128 ? 3 * kCus / 2 : 3 * kCus;   // one or two run on a CU
    while (blocks && p.parts < 32 && blocks * p.parts < enough && 8 * p.parts * 64 <= tokens * (heads / kv)) p.parts *= 2;
    size_t at = 0;
    p.stats = at, at += tiles((size_t)n * rows * 8, 16) * 16;
    p.bounds = at, at += (size_t)n * tiles(tokens * (heads / kv), 32) * 16;
    p.order = at, at += tiles((size_t)n * tiles(keys, 128) * 4, 16) * 16;
    p.marks = at, at += tiles((size_t)pairs * tiles(tokens * (heads / kv), 128) * 4, 16) * 16;
    p.key_marks = at, at += tiles((size_t)blocks * p.parts * 4, 16) * 16;
    p.sums = at, at += p.parts > 1 ? (size_t)pairs * keys * p.parts * 2 * width * 4 : 0;
    p.workspace = at;
    return p;
}

AttentionArgs attention_args(int32_t n, int64_t tokens, int64_t keys, int32_t heads, int32_t kv, int64_t width,
                             const relaysum_heads *q, const relaysum_heads *k, const relaysum_heads *v,
                             const int32_t *ranges, int64_t ranges_stride, int32_t causal, float scale,
                             const relaysum_heads *out, float *lse) {
    AttentionArgs a{};
    a.q = heads_of(q, n, tokens, heads);
    a.k = heads_of(k, n, keys, kv);
    a.v = heads_of(v, n, keys, kv);
    a.out = heads_of(out, n, tokens, heads);
    a.lse = lse;
    a.ranges = reinterpret_cast<const int2 *>(ranges);
    a.range_stride = n > 1 ? ranges_stride : 0;
    a.tokens = (int32_t)tokens, a.keys = (int32_t)keys, a.heads = heads, a.kv = kv, a.group = heads / kv;
    a.width = (int32_t)width, a.rows = (int32_t)(tokens * a.group), a.causal = causal != 0;
    a.pairs = (uint32_t)n * kv;
    while ((int64_t)1 << a.group_shift < a.group) ++a.group_shift;
    a.group_factor = (uint32_t)(((((uint64_t)1 << a.group_shift) - a.group) << 32) / a.group + 1);
    a.scale = scale, a.dot_scale = scale * kLog2e;
    return a;
}

}  // namespace

extern "C" {

int relaysum_attention_ranges(int32_t n, int64_t tokens, int64_t keys, int32_t count, const int32_t *starts,
                              int64_t starts_stride, const int32_t *key_starts, int64_t key_starts_stride,
                              int32_t causal, int32_t *ranges, int64_t ranges_stride, void *hip_stream) {
    AttentionCall c;
    if (c.shape(n, tokens, keys, 1, 1, 1)) {
        if (count < 1 || count > 1 << 30) c.fail(refuse("count must be in 1..2^30"));
        if (c.code == RELAYSUM_OK && n > 1 && (starts_stride < 0 || key_starts_stride < 0 ||
                                               starts_stride > ((int64_t)1 << 40) / n || key_starts_stride > ((int64_t)1 << 40) / n))
            c.fail(refuse("a stride of starts is negative or reaches past 2^40 entries"));
        if (n == 1) starts_stride = key_starts_stride = 0;
        c.span("starts", starts, (size_t)((n - 1) * starts_stride + count + 1) * 4, 4, false);
        c.span("key_starts", key_starts, (size_t)((n - 1) * key_starts_stride + count + 1) * 4, 4, false);
        if (tokens) c.ranges(ranges, ranges_stride, n, tokens, true);
        if (c.code == RELAYSUM_OK && (n * tokens + 255) / 256 > kMaxBlocks) c.fail(refuse("n * tokens is too large"));
    }
    if (!c.ready()) return c.code;
    if (tokens == 0) return done("relaysum_attention_ranges");
    const RangeArgs a{starts, key_starts, starts_stride, key_starts_stride, ranges_stride,
                      reinterpret_cast<int2 *>(ranges), tokens, n * tokens, (int32_t)keys, count, causal != 0};
    hipLaunchKernelGGL(attention_ranges_kernel, dim3((unsigned)((a.total + 255) / 256)), dim3(256), 0,
                       (hipStream_t)hip_stream, a);
    return done("relaysum_attention_ranges");
}

int64_t relaysum_attention_workspace(int32_t n, int64_t tokens, int64_t keys, int32_t heads, int32_t kv_heads,
                                     int64_t width) {
    AttentionCall c;
    if (!c.shape(n, tokens, keys, heads, kv_heads, width)) return -1;
    g_error[0] = '\0';
    if (!tokens) return 0;
    return (int64_t)std::max(plan_forward(n, tokens, keys, heads, kv_heads, width, RELAYSUM_FLOAT).workspace,
                             plan_forward(n, tokens, keys, heads, kv_heads, width, RELAYSUM_HALF).workspace);
}

int relaysum_attention(int32_t n, int64_t tokens, int64_t keys, int32_t heads, int32_t kv_heads, int64_t width,
                       const relaysum_heads *q, const relaysum_heads *k, const relaysum_heads *v,
                       const int32_t *ranges, int64_t ranges_stride, int32_t causal, float scale,
                       const relaysum_heads *out, float *lse, void *workspace, size_t workspace_bytes,
                       void *hip_stream) {
    AttentionCall c;
    ForwardPlan p{};
    if (c.shape(n, tokens, keys, heads, kv_heads, width)) {
        const int32_t type = q ? q->type : 0;
        c.heads("q", q, type, n, tokens, heads, width, false);
        c.heads("k", k, type, n, keys, kv_heads, width, false);
        c.heads("v", v, type, n, keys, kv_heads, width, false);
        c.heads("out", out, type, n, tokens, heads, width, true);
        if (tokens) c.ranges(ranges, ranges_stride, n, tokens, false);
        if (lse) c.span("lse", lse, (size_t)n * heads * tokens * 4, 4, true);
        if (!(scale > 0.0f && scale <= 0x1p126f)) c.fail(refuse("scale must be positive, and at most 2^126"));
        if (c.code == RELAYSUM_OK && tokens) {
            p = plan_forward(n, tokens, keys, heads, kv_heads, width, type);
            c.product_launch(p, workspace, workspace_bytes);
        }
    }
    if (!c.ready()) return c.code;
    if (tokens == 0) return done("relaysum_attention");
    AttentionArgs a = attention_args(n, tokens, keys, heads, kv_heads, width, q, k, v, ranges, ranges_stride, causal,
                                     scale, out, lse);
    a.tiles = p.tiles, a.parts = p.parts, a.span = p.span;
    a.marks = static_cast<int32_t *>(workspace);
    a.part_soft = static_cast<float2 *>(workspace);
    a.part_out = static_cast<float *>(workspace) + (size_t)a.pairs * a.rows * p.parts * 2;
    const hipStream_t st = (hipStream_t)hip_stream;
    with_type(q->type, [&](auto zero) { launch_attention<decltype(zero)>(a, p, st); });
    return done("relaysum_attention");
}

int64_t relaysum_attention_backward_workspace(int32_t n, int64_t tokens, int64_t keys, int32_t heads, int32_t kv_heads,
                                              int64_t width, int32_t type) {
    AttentionCall c;
    if (!c.shape(n, tokens, keys, heads, kv_heads, width)) return -1;
    if (type < RELAYSUM_FLOAT || type > RELAYSUM_HALF) {
        refuse("unknown type %d", type);
        return -1;
    }
    g_error[0] = '\0';
    return (int64_t)plan_backward(n, tokens, keys, heads, kv_heads, width).workspace;
}

int relaysum_attention_backward(int32_t n, int64_t tokens, int64_t keys, int32_t heads, int32_t kv_heads,
                                int64_t width, const relaysum_heads *dout, const relaysum_heads *q,
                                const relaysum_heads *k, const relaysum_heads *v, const relaysum_heads *out,
                                const float *lse, const int32_t *ranges, int64_t ranges_stride, int32_t causal,
                                float scale, const relaysum_heads *dq, const relaysum_heads *dk,
                                const relaysum_heads *dv, void *workspace, size_t workspace_bytes, void *hip_stream) {
    AttentionCall c;
    BackwardPlan p{};
    if (c.shape(n, tokens, keys, heads, kv_heads, width)) {
        const int32_t type = q ? q->type : 0;
        c.heads("q", q, type, n, tokens, heads, width, false);
        c.heads("dout", dout, type, n, tokens, heads, width, false);
        c.heads("k", k, type, n, keys, kv_heads, width, false);
        c.heads("v", v, type, n, keys, kv_heads, width, false);
        c.heads("out", out, type, n, tokens, heads, width, false);
        c.span("lse", lse, (size_t)n * heads * tokens * 4, 4, false);
        if (tokens) c.ranges(ranges, ranges_stride, n, tokens, false);
        c.heads("dq", dq, type, n, tokens, heads, width, true);
        c.heads("dk", dk, type, n, keys, kv_heads, width, true);
        c.heads("dv", dv, type, n, keys, kv_heads, width, true);
        if (!(scale > 0.0f && scale <= 0x1p126f)) c.fail(refuse("scale must be positive, and at most 2^126"));
        if (c.code == RELAYSUM_OK) {
            p = plan_backward(n, tokens, keys, heads, kv_heads, width);
            const int64_t pairs = (int64_t)n * kv_heads;
            if (pairs * tiles(tokens * (heads / kv_heads), 128) > kMaxBlocks || pairs * tiles(keys, 128) * p.parts > kMaxBlocks)
                c.fail(refuse("n * kv_heads is too large"));
            if (p.workspace > workspace_bytes)
                c.fail(refuse("the workspace has %zu bytes, %zu are needed", workspace_bytes, p.workspace));
            c.span("workspace", workspace, p.workspace, 16, true);
        }
    }
    if (!c.ready()) return c.code;
    AttentionArgs a = attention_args(n, tokens, keys, heads, kv_heads, width, q, k, v, ranges, ranges_stride, causal,
                                     scale, out, const_cast<float *>(lse));
    a.dout = heads_of(dout, n, tokens, heads);
    a.dq = heads_of(dq, n, tokens, heads);
    a.dk = heads_of(dk, n, keys, kv_heads);
    a.dv = heads_of(dv, n, keys, kv_heads);
    char *ws = static_cast<char *>(workspace);
    a.stats = reinterpret_cast<float2 *>(ws + p.stats);
    a.bounds = reinterpret_cast<int4 *>(ws + p.bounds);
    a.marks = reinterpret_cast<int32_t *>(ws + p.marks);
    a.key_marks = reinterpret_cast<int32_t *>(ws + p.key_marks);
    a.order = reinterpret_cast<int32_t *>(ws + p.order);
    a.part_out = reinterpret_cast<float *>(ws + p.sums);
    a.parts = p.parts;
    a.bound_stride = a.range_stride ? tiles(a.rows, 32) : 0;
    const hipStream_t st = (hipStream_t)hip_stream;
    with_type(q->type, [&](auto zero) { launch_attention_backward<decltype(zero)>(a, n, st); });
    return done("relaysum_attention_backward");
}

}  // extern "C"
