// Attention of n workers' packed sequences, and its gradients, on CDNA4
// (gfx950); the C ABI is in relaysum.h.
//
//   s_j = scale * q . k_j for the keys lo <= j < hi that a row sees,
//   p_j = exp(s_j) / sum exp(s),  out = sum p_j v_j,  lse = log sum exp(s)
//   dv_j = sum p_j dout,  ds_j = p_j (dout . v_j - dout . out),
//   dq = scale * sum ds_j k_j,  dk_j = scale * sum ds_j q
//
// The query heads that share a key head are rows of one matrix: row
// t * group + g is token t of the group's head g.  Their keys and values are
// then read once, and the gradients of k and v sum over the group within a
// workgroup, without atomics.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "attention_tiles.hpp"
#include "layer_call.hpp"

namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr int kMaxHeadWidth = 256;

// Weights of binary16 are held times 2^7 (forward, where they reach 2^8 times
// their largest) and 2^15 (backward, where they are at most 1): below 2^-14 it
// loses bits.
template <typename T>
constexpr float kForwardShift = std::is_same<T, _Float16>::value ? 7.0f : 0.0f;
template <typename T>
constexpr float kBackwardShift = std::is_same<T, _Float16>::value ? 15.0f : 0.0f;

struct AttentionArgs {
    Heads q, k, v, out;
    Heads dout, dq, dk, dv;
    float *lse;                // [n][heads][tokens]
    float *delta;              // [n][heads][tokens]: dout . out
    float2 *largest;           // [n][parts]: squared norms of rows of dout and v
    int4 *bounds;              // [n or 1][ceil(rows / 32)]: least and most lo, least and most hi
    const int2 *ranges;
    float *part_out;           // [pairs][rows][parts][width]
    float2 *part_soft;         // [pairs][rows][parts]
    int64_t range_stride;      // rows between workers' ranges; 0: all have the same
    int64_t bound_stride;
    int32_t tokens, keys, heads, kv, group, width, rows;   // rows = tokens * group
    int32_t causal, tiles, parts, span;
    uint32_t pairs;            // n * kv
    float scale, dot_scale;    // dot_scale = scale * log2(e)
};

// The keys that a token sees.
__device__ __forceinline__ int2 seen(const AttentionArgs &a, int64_t worker, int t) {
    if (a.ranges) {
        const int2 r = a.ranges[worker * a.range_stride + t];
        return int2{max(r.x, 0), min(r.y, a.keys)};
    }
    const int64_t last = (int64_t)t + 1 + a.keys - a.tokens;
    return int2{0, a.causal ? (int)max((int64_t)0, min(last, (int64_t)a.keys)) : a.keys};
}

// Which workers' key head and which tile of it a workgroup has.  Tiles of one
// key head are put on one XCD, whose L2 then holds its keys; the last tiles,
// which see the most keys of a causal sequence, go first.
__device__ __forceinline__ void place(const AttentionArgs &a, unsigned block, unsigned &pair, int &tile) {
    if (a.pairs % 8 == 0) {
        const unsigned i = block / 8;
        pair = block % 8 + i / a.tiles * 8;
        tile = a.tiles - 1 - (int)(i % a.tiles);
    } else {
        pair = block % a.pairs;
        tile = a.tiles - 1 - (int)(block / a.pairs);
    }
}

template <typename T>
__device__ __forceinline__ T *head_at(const Heads &h, int64_t worker, int64_t t, int head) {
    return reinterpret_cast<T *>(h.data) + worker * h.ws + t * h.rs + head * h.hs;
}

// Over the 32 columns that a wave's lanes have twice.
template <typename F>
__device__ __forceinline__ int column_reduce(int v, F f) {
#pragma unroll
    for (int m = 1; m < 32; m *= 2) v = f(v, __shfl_xor(v, m));
    return __builtin_amdgcn_readfirstlane(v);
}

// What a wave's columns see: whether a stretch of keys is seen by all, by some.
struct Sight {
    int least_lo, most_lo, least_hi, most_hi;
    __device__ __forceinline__ bool whole(int j, int count) const { return most_lo <= j && j + count <= least_hi; }
    __device__ __forceinline__ bool any(int j, int count) const { return least_lo < j + count && j < most_hi; }
};

__device__ __forceinline__ Sight sight_of(int lo, int hi, bool valid) {
    const bool some = valid && lo < hi;
    Sight s;
    s.least_lo = column_reduce(some ? lo : INT_MAX, [](int x, int y) { return min(x, y); });
    s.most_hi = column_reduce(some ? hi : 0, [](int x, int y) { return max(x, y); });
    s.most_lo = column_reduce(valid ? (some ? lo : INT_MAX) : 0, [](int x, int y) { return max(x, y); });
    s.least_hi = column_reduce(valid ? hi : INT_MAX, [](int x, int y) { return min(x, y); });
    return s;
}

// ---- forward -----------------------------------------------------------------------
//
// One pass over the keys: `off` is the column's reference (a maximum of its
// scores so far, in powers of two), l this lane's sum of the weights
// 2^(s - off), acc the sum of weighted values.  The reference moves, and acc
// with it, only when a score passes it by more than 2^8.
template <typename T, int DP>
struct Softmax {
    typedef Tile<T, DP> L;
    u4_t q[L::kOwn];
    f16_t acc[L::kBlocks];
    float m, off, l;

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int b = 0; b < L::kBlocks; ++b) acc[b] = f16_t{0};
        m = -INFINITY;
        off = l = 0.0f;
    }

    // 32 * NB keys from j on.
    template <int NB>
    __device__ __forceinline__ void step(const AttentionArgs &a, const char *kt, const char *vt, int j, int lo, int hi,
                                         bool whole, bool apart, char *room, int lane) {
        const int h = lane / 32;
        float p[NB][16];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const f16_t s = dots<T, DP>(kt, 32 * b, q, lane);
#pragma unroll
            for (int i = 0; i < 16; ++i) p[b][i] = s[i];
        }
        if (!whole) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int key = j + 32 * b + 8 * (i / 4) + 4 * h + i % 4;
                    p[b][i] = key >= lo && key < hi ? p[b][i] : -INFINITY;
                }
        }
        float top = p[0][0];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, p[b][i]);
        top = fmaxf(top, other_half(top));
        if (__ballot(top > m + 8.0f / a.dot_scale)) {
            const float to = fmaxf(m, top);
            const float moved = to == -INFINITY ? 0.0f : to * a.dot_scale - kForwardShift<T>;
            const float f = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(off - moved);
            l *= f;
#pragma unroll
            for (int b = 0; b < L::kBlocks; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[b][i] *= f;
            m = to;
            off = moved;
        }
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                p[b][i] = __builtin_amdgcn_exp2f(fmaf(p[b][i], a.dot_scale, -off));
                l += p[b][i];
            }
        if (apart && !whole) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
                add_rows_apart<T, DP>(acc, vt, 32 * b, p[b], room, lane, [&](int row) {
                    const int key = j + 32 * b + row;
                    return key >= lo && key < hi;
                });
        } else {
#pragma unroll
            for (int b = 0; b < NB; ++b) add_rows<T, DP>(acc, vt, 32 * b, Weights<T>(p[b]), lane);
        }
    }
};

template <typename T, int DP>
constexpr int kKeyTile = sizeof(T) == 4 && DP >= 128 ? 32 : 64;

template <typename T, int DP>
__global__ __launch_bounds__(256) void attention_kernel(AttentionArgs a) {
    typedef Tile<T, DP> L;
    constexpr int BN = kKeyTile<T, DP>;
    __shared__ __align__(16) char lds[2][2][BN * L::kRowBytes];
    __shared__ __align__(16) char room[4][kApartBytes<T>];
    __shared__ int most[4][2];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    unsigned pair;
    int tile;
    place(a, blockIdx.x, pair, tile);
    const int64_t worker = pair / a.kv;
    const int kvh = (int)(pair % a.kv);
    const int row = tile * 128 + wave * 32 + lane % 32;
    const bool valid = row < a.rows;
    const int t = valid ? row / a.group : 0, head = kvh * a.group + (valid ? row % a.group : 0);
    const int2 range = valid ? seen(a, worker, t) : int2{0, INT_MAX};
    const int lo = range.x, hi = range.y;
    const Sight sight = sight_of(lo, hi, valid);
    if (lane == 0) most[wave][0] = sight.least_lo, most[wave][1] = sight.most_hi;
    __syncthreads();
    const int first = min(min(most[0][0], most[1][0]), min(most[2][0], most[3][0]));
    const int end = max(max(most[0][1], most[1][1]), max(most[2][1], most[3][1]));

    Softmax<T, DP> st;
    const T *qrow = head_at<const T>(a.q, worker, t, head);
#pragma unroll
    for (int i = 0; i < L::kOwn; ++i) st.q[i] = load_chunk<T>(qrow, (2 * i + lane / 32) * L::E, a.width, valid);
    const T *kbase = head_at<const T>(a.k, worker, 0, kvh), *vbase = head_at<const T>(a.v, worker, 0, kvh);
    Stage<T, DP, BN, 256> ks, vs;
    const int begin = first / BN * BN;

    float sum;
    for (int pass = 0;; ++pass) {
        st.clear();
        const auto fetch = [&](int j) {
            ks.load(a.width, threadIdx.x, [&](int r) { return j + r < a.keys ? kbase + (int64_t)(j + r) * a.k.rs : nullptr; });
            vs.load(a.width, threadIdx.x, [&](int r) { return j + r < a.keys ? vbase + (int64_t)(j + r) * a.v.rs : nullptr; });
        };
        if (first < end) {
            fetch(begin);
            ks.store(lds[0][0], threadIdx.x);
            vs.store(lds[0][1], threadIdx.x);
        }
        int half = 0;
        for (int j = begin; j < end; j += BN, half ^= 1) {
            __syncthreads();
            const bool more = j + BN < end;
            if (more) fetch(j + BN);
            if (sight.any(j, BN))
                st.template step<BN / 32>(a, lds[half][0], lds[half][1], j, lo, hi, sight.whole(j, BN), pass > 0,
                                          room[wave], lane);
            if (more) {
                ks.store(lds[half ^ 1][0], threadIdx.x);
                vs.store(lds[half ^ 1][1], threadIdx.x);
            }
        }
        sum = st.l + other_half(st.l);
        // Infinities and NaN of rows that a column does not see may be in it: once
        // more, with those kept out.
        if (pass || !__syncthreads_or(valid && (not_finite(st.acc) || !(fabsf(sum) < INFINITY)))) break;
    }
    if (!valid) return;
    const bool empty = lo >= hi;
    store_column<T>(head_at<T>(a.out, worker, t, head), a.width, st.acc, empty ? 0.0f : 1.0f / sum, lane);
    if (a.lse && lane < 32)
        a.lse[(worker * a.heads + head) * a.tokens + t] =
            empty ? -INFINITY : kLn2 * (st.off + __builtin_amdgcn_logf(sum));
}

// Few rows: the keys are split over workgroups (parts) and their waves, each of
// which walks through its own keys; waves join through LDS, parts in a second
// kernel.
template <typename T, int DP>
constexpr int kSplitWaves = sizeof(T) == 4 && DP == 256 ? 2 : 4;   // whose tiles fit LDS

template <typename T, int DP>
__global__ __launch_bounds__((64 * kSplitWaves<T, DP>)) void attention_split_kernel(AttentionArgs a) {
    typedef Tile<T, DP> L;
    constexpr int W = kSplitWaves<T, DP>;
    constexpr int kTile = 32 * L::kRowBytes;
    // A wave's keys and values, and later its sums.
    constexpr int kOwnBytes = 2 * kTile > 32 * DP * 4 ? 2 * kTile : 32 * DP * 4;
    __shared__ __align__(16) char lds[W][kOwnBytes];
    __shared__ __align__(16) char room[W][kApartBytes<T>];
    __shared__ float soft[W][2][32];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const unsigned part = blockIdx.x % a.parts, at = blockIdx.x / a.parts;
    const unsigned pair = at / a.tiles;
    const int tile = (int)(at % a.tiles);
    const int64_t worker = pair / a.kv;
    const int kvh = (int)(pair % a.kv);
    const int row = tile * 32 + lane % 32;
    const bool valid = row < a.rows;
    const int t = valid ? row / a.group : 0, head = kvh * a.group + (valid ? row % a.group : 0);
    const int2 range = valid ? seen(a, worker, t) : int2{0, INT_MAX};
    const int lo = range.x, hi = range.y;
    const Sight sight = sight_of(lo, hi, valid);

    Softmax<T, DP> st;
    const T *qrow = head_at<const T>(a.q, worker, t, head);
#pragma unroll
    for (int i = 0; i < L::kOwn; ++i) st.q[i] = load_chunk<T>(qrow, (2 * i + lane / 32) * L::E, a.width, valid);
    const T *kbase = head_at<const T>(a.k, worker, 0, kvh), *vbase = head_at<const T>(a.v, worker, 0, kvh);
    // Keys of this part, 32 at a time in turn.
    const int64_t from = (int64_t)part * a.span, to = min(from + a.span, (int64_t)sight.most_hi);
    char *kt = lds[wave], *vt = kt + kTile;
    Stage<T, DP, 32, 64> ks, vs;
    float sum;
    for (int pass = 0;; ++pass) {
        st.clear();
        const auto fetch = [&](int j) {
            ks.load(a.width, lane, [&](int r) { return j + r < a.keys ? kbase + (int64_t)(j + r) * a.k.rs : nullptr; });
            vs.load(a.width, lane, [&](int r) { return j + r < a.keys ? vbase + (int64_t)(j + r) * a.v.rs : nullptr; });
        };
        int64_t j = from + 32 * wave;
        while (j < to && !sight.any((int)j, 32)) j += 32 * W;
        if (j < to) fetch((int)j);
        while (j < to) {
            ks.store(kt, lane);
            vs.store(vt, lane);
            wave_fence();
            int64_t next = j + 32 * W;
            while (next < to && !sight.any((int)next, 32)) next += 32 * W;
            if (next < to) fetch((int)next);
            st.template step<1>(a, kt, vt, (int)j, lo, hi, sight.whole((int)j, 32), pass > 0, room[wave], lane);
            wave_fence();
            j = next;
        }
        sum = st.l + other_half(st.l);
        if (pass || !__ballot(valid && (not_finite(st.acc) || !(fabsf(sum) < INFINITY)))) break;
    }
    // Waves join: every wave's sums [entry][column], times what brings them to
    // the largest reference.  A wave without keys has none.
    if (lane < 32) {
        soft[wave][0][lane] = st.m == -INFINITY ? -INFINITY : st.off;
        soft[wave][1][lane] = sum;
    }
    float *sums = reinterpret_cast<float *>(lds[wave]);
    wave_fence();
#pragma unroll
    for (int b = 0; b < L::kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i)
            sums[(32 * b + 8 * (i / 4) + 4 * (lane / 32) + i % 4) * 32 + lane % 32] = st.acc[b][i];
    __syncthreads();
    const int col = threadIdx.x / (2 * W);
    const int r = tile * 32 + col;
    if (r >= a.rows) return;
    float top = -INFINITY, all = 0.0f, f[W];
#pragma unroll
    for (int w = 0; w < W; ++w) top = fmaxf(top, soft[w][0][col]);
#pragma unroll
    for (int w = 0; w < W; ++w) {
        f[w] = soft[w][0][col] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(soft[w][0][col] - top);
        all += soft[w][1][col] * (soft[w][0][col] == -INFINITY ? 1.0f : f[w]);
    }
    const int rt = r / a.group, rh = kvh * a.group + r % a.group;
    const int2 rr = seen(a, worker, rt);
    const bool empty = rr.x >= rr.y;
    const float inv = a.parts > 1 ? 1.0f : empty ? 0.0f : 1.0f / all;
    const int64_t slot = ((int64_t)pair * a.rows + r) * a.parts + part;
    for (int k = threadIdx.x % (2 * W); k < a.width; k += 2 * W) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w)
            if (soft[w][0][col] != -INFINITY) v += reinterpret_cast<const float *>(lds[w])[k * 32 + col] * f[w];
        // All of its scores are -infinity: 0 / 0.
        if (a.parts > 1) a.part_out[slot * a.width + k] = v;
        else head_at<T>(a.out, worker, rt, rh)[k] = (T)(empty ? 0.0f : v * inv);
    }
    if (threadIdx.x % (2 * W)) return;
    if (a.parts > 1) a.part_soft[slot] = float2{top, all};
    else if (a.lse)
        a.lse[(worker * a.heads + rh) * a.tokens + rt] =
            empty ? -INFINITY : kLn2 * ((top == -INFINITY ? 0.0f : top) + __builtin_amdgcn_logf(all));
}

// Parts of a row join: a wave each.
template <typename T>
__global__ __launch_bounds__(256) void attention_join_kernel(AttentionArgs a) {
    const int lane = threadIdx.x % kWave;
    const int64_t at = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
    if (at >= (int64_t)a.pairs * a.rows) return;
    const int64_t pair = at / a.rows, worker = pair / a.kv;
    const int r = (int)(at % a.rows), t = r / a.group, head = (int)(pair % a.kv) * a.group + r % a.group;
    const int2 range = seen(a, worker, t);
    const bool empty = range.x >= range.y;
    const float2 *soft = a.part_soft + at * a.parts;
    float top = -INFINITY, all = 0.0f;
    for (int p = lane; p < a.parts; p += kWave) top = fmaxf(top, soft[p].x);
#pragma unroll
    for (int m = 1; m < kWave; m *= 2) top = fmaxf(top, __shfl_xor(top, m));
    for (int p = lane; p < a.parts; p += kWave)
        all += soft[p].y * (soft[p].x == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(soft[p].x - top));
#pragma unroll
    for (int m = 1; m < kWave; m *= 2) all += __shfl_xor(all, m);
    const float inv = 1.0f / all;
    T *out = head_at<T>(a.out, worker, t, head);
    for (int k = lane; k < a.width; k += kWave) {
        float v = 0.0f;
        for (int p = 0; p < a.parts; ++p)
            if (soft[p].x != -INFINITY)
                v += a.part_out[(at * a.parts + p) * a.width + k] * __builtin_amdgcn_exp2f(soft[p].x - top);
        out[k] = (T)(empty ? 0.0f : v * inv);
    }
    if (a.lse && lane == 0)
        a.lse[(worker * a.heads + head) * a.tokens + t] =
            empty ? -INFINITY : kLn2 * ((top == -INFINITY ? 0.0f : top) + __builtin_amdgcn_logf(all));
}

// ---- backward ----------------------------------------------------------------------

// delta = dout . out of every row, 16 lanes each; for binary16 also the largest
// squared norms of the rows of dout that see something and of v's.
template <typename T>
__global__ __launch_bounds__(256) void attention_delta_kernel(AttentionArgs a) {
    __shared__ float red[2][16];
    const int64_t worker = blockIdx.x / a.parts;
    const int part = (int)(blockIdx.x % a.parts), lane = threadIdx.x % 16, slot = threadIdx.x / 16;
    float most_dout = 0.0f, most_v = 0.0f;
    const int64_t rows = (int64_t)a.tokens * a.heads;
    for (int64_t r = (int64_t)part * 16 + slot; r < rows; r += (int64_t)a.parts * 16) {
        const int t = (int)(r / a.heads), head = (int)(r % a.heads);
        const T *x = head_at<const T>(a.dout, worker, t, head), *y = head_at<const T>(a.out, worker, t, head);
        float dot = 0.0f, norm = 0.0f;
        for (int k = lane * 8; k < a.width; k += 128) {
            float u[8], v[8];
            load8(x + k, a.width - k, u);
            load8(y + k, a.width - k, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) dot = fmaf(u[i], v[i], dot), norm = fmaf(u[i], u[i], norm);
        }
        dot = row_reduce<16, float, pick_sum>(dot, nullptr);
        if (lane == 0) a.delta[(worker * a.heads + head) * a.tokens + t] = dot;
        if (std::is_same<T, _Float16>::value) {
            norm = row_reduce<16, float, pick_sum>(norm, nullptr);
            const int2 s = seen(a, worker, t);
            if (s.x < s.y && norm < INFINITY) most_dout = fmaxf(most_dout, norm);
        }
    }
    if (std::is_same<T, _Float16>::value) {
        const int64_t vrows = (int64_t)a.keys * a.kv;
        for (int64_t r = (int64_t)part * 16 + slot; r < vrows; r += (int64_t)a.parts * 16) {
            const T *x = head_at<const T>(a.v, worker, r / a.kv, (int)(r % a.kv));
            float norm = 0.0f;
            for (int k = lane * 8; k < a.width; k += 128) {
                float u[8];
                load8(x + k, a.width - k, u);
#pragma unroll
                for (int i = 0; i < 8; ++i) norm = fmaf(u[i], u[i], norm);
            }
            norm = row_reduce<16, float, pick_sum>(norm, nullptr);
            if (norm < INFINITY) most_v = fmaxf(most_v, norm);
        }
        if (lane == 0) red[0][slot] = most_dout, red[1][slot] = most_v;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int i = 1; i < 16; ++i) most_dout = fmaxf(most_dout, red[0][i]), most_v = fmaxf(most_v, red[1][i]);
            a.largest[blockIdx.x] = float2{most_dout, most_v};
        }
    }
}

// What blocks of 32 rows see.
__global__ __launch_bounds__(256) void attention_bounds_kernel(AttentionArgs a, int64_t total) {
    const int64_t at = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
    if (at >= total) return;
    const int64_t per = (a.rows + 31) / 32, worker = at / per;
    const int row = (int)(at % per) * 32 + threadIdx.x % 32;
    int2 s = row < a.rows ? seen(a, worker, row / a.group) : int2{INT_MAX, 0};
    int4 b = {row < a.rows ? s.x : INT_MAX, row < a.rows ? s.x : 0, row < a.rows ? s.y : 0, s.y};
#pragma unroll
    for (int m = 1; m < 32; m *= 2) {
        b.x = min(b.x, __shfl_xor(b.x, m));
        b.y = max(b.y, __shfl_xor(b.y, m));
        b.z = min(b.z, __shfl_xor(b.z, m));
        b.w = max(b.w, __shfl_xor(b.w, m));
    }
    if (threadIdx.x % 32 == 0) a.bounds[at] = b;
}

// Least and most lo, least and most hi of 32 rows; rows behind the last see nothing.
__device__ __forceinline__ Sight block_sight(const AttentionArgs &a, int64_t worker, int block) {
    if (a.ranges) {
        const int4 b = a.bounds[worker * a.bound_stride + block];
        return Sight{b.x, b.y, b.z, b.w};
    }
    const int last = min(block * 32 + 31, a.rows - 1);
    return Sight{0, 0, block * 32 + 32 > a.rows ? 0 : seen(a, worker, block * 32 / a.group).y,
                 seen(a, worker, last / a.group).y};
}

// The power of two that ds is held times in binary16, so that its largest is
// below 2^15: |ds| <= 2 |dout| |v|.  Every thread of the workgroup takes part.
template <typename T>
__device__ __forceinline__ float gradient_scale(const AttentionArgs &a, int64_t worker, float2 *red) {
    if (!std::is_same<T, _Float16>::value) return 1.0f;
    float2 m = {0.0f, 0.0f};
    for (int p = threadIdx.x; p < a.parts; p += 256) {
        const float2 v = a.largest[worker * a.parts + p];
        m.x = fmaxf(m.x, v.x), m.y = fmaxf(m.y, v.y);
    }
#pragma unroll
    for (int s = 1; s < kWave; s *= 2) m.x = fmaxf(m.x, __shfl_xor(m.x, s)), m.y = fmaxf(m.y, __shfl_xor(m.y, s));
    if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = m;
    __syncthreads();
    for (int w = 0; w < 4; ++w) m.x = fmaxf(m.x, red[w].x), m.y = fmaxf(m.y, red[w].y);
    const float bound = 2.0f * sqrtf(m.x) * sqrtf(m.y);
    if (!(bound > 0.0f)) return 1.0f;
    return ldexpf(1.0f, 13 - max(-80, min(80, ilogbf(bound))));
}

// The gradient of q: as forward, with the weights known from lse.
template <typename T, int DP>
__global__ __launch_bounds__(256) void attention_dq_kernel(AttentionArgs a) {
    typedef Tile<T, DP> L;
    constexpr int BN = kKeyTile<T, DP>;
    __shared__ __align__(16) char lds[2][2][BN * L::kRowBytes];
    __shared__ __align__(16) char room[4][kApartBytes<T>];
    __shared__ int most[4][2];
    __shared__ float2 red[4];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    unsigned pair;
    int tile;
    place(a, blockIdx.x, pair, tile);
    const int64_t worker = pair / a.kv;
    const int kvh = (int)(pair % a.kv);
    const int row = tile * 128 + wave * 32 + lane % 32;
    const bool valid = row < a.rows;
    const int t = valid ? row / a.group : 0, head = kvh * a.group + (valid ? row % a.group : 0);
    const int2 range = valid ? seen(a, worker, t) : int2{0, INT_MAX};
    const int lo = range.x, hi = range.y;
    const Sight sight = sight_of(lo, hi, valid);
    if (lane == 0) most[wave][0] = sight.least_lo, most[wave][1] = sight.most_hi;
    const float up = gradient_scale<T>(a, worker, red);
    __syncthreads();
    const int first = min(min(most[0][0], most[1][0]), min(most[2][0], most[3][0]));
    const int end = max(max(most[0][1], most[1][1]), max(most[2][1], most[3][1]));

    u4_t q[L::kOwn], dout[L::kOwn];
    const T *qrow = head_at<const T>(a.q, worker, t, head), *drow = head_at<const T>(a.dout, worker, t, head);
#pragma unroll
    for (int i = 0; i < L::kOwn; ++i) {
        q[i] = load_chunk<T>(qrow, (2 * i + lane / 32) * L::E, a.width, valid);
        dout[i] = load_chunk<T>(drow, (2 * i + lane / 32) * L::E, a.width, valid);
    }
    const int64_t stat = (worker * a.heads + head) * a.tokens + t;
    const float off = valid ? a.lse[stat] * kLog2e : 0.0f, delta = valid ? a.delta[stat] : 0.0f;
    const T *kbase = head_at<const T>(a.k, worker, 0, kvh), *vbase = head_at<const T>(a.v, worker, 0, kvh);
    Stage<T, DP, BN, 256> ks, vs;
    const int begin = first / BN * BN;
    f16_t acc[L::kBlocks];
    for (int pass = 0;; ++pass) {
#pragma unroll
        for (int b = 0; b < L::kBlocks; ++b) acc[b] = f16_t{0};
        const auto fetch = [&](int j) {
            ks.load(a.width, threadIdx.x, [&](int r) { return j + r < a.keys ? kbase + (int64_t)(j + r) * a.k.rs : nullptr; });
            vs.load(a.width, threadIdx.x, [&](int r) { return j + r < a.keys ? vbase + (int64_t)(j + r) * a.v.rs : nullptr; });
        };
        if (first < end) {
            fetch(begin);
            ks.store(lds[0][0], threadIdx.x);
            vs.store(lds[0][1], threadIdx.x);
        }
        int half = 0;
        for (int j0 = begin; j0 < end; j0 += BN, half ^= 1) {
            __syncthreads();
            const bool more = j0 + BN < end;
            if (more) fetch(j0 + BN);
#pragma unroll
            for (int b = 0; b < BN / 32; ++b) {
                const int j = j0 + 32 * b;
                if (!sight.any(j, 32)) continue;
                const bool whole = sight.whole(j, 32);
                const f16_t s = dots<T, DP>(lds[half][0], 32 * b, q, lane);
                const f16_t dp = dots<T, DP>(lds[half][1], 32 * b, dout, lane);
                float ds[16];
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    ds[i] = __builtin_amdgcn_exp2f(fmaf(s[i], a.dot_scale, -off)) * up * (dp[i] - delta);
                if (!whole) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int key = j + 8 * (i / 4) + 4 * (lane / 32) + i % 4;
                        ds[i] = key >= lo && key < hi ? ds[i] : 0.0f;
                    }
                }
                if (pass && !whole)
                    add_rows_apart<T, DP>(acc, lds[half][0], 32 * b, ds, room[wave], lane,
                                          [&](int r) { return j + r >= lo && j + r < hi; });
                else
                    add_rows<T, DP>(acc, lds[half][0], 32 * b, Weights<T>(ds), lane);
            }
            if (more) {
                ks.store(lds[half ^ 1][0], threadIdx.x);
                vs.store(lds[half ^ 1][1], threadIdx.x);
            }
        }
        if (pass || !__syncthreads_or(valid && not_finite(acc))) break;
    }
    if (valid) store_column<T>(head_at<T>(a.dq, worker, t, head), a.width, acc, a.scale / up, lane);
}

// The gradients of k and v: columns are keys, rows the queries that see them.
template <typename T, int DP>
__global__ __launch_bounds__(256) void attention_dkv_kernel(AttentionArgs a) {
    typedef Tile<T, DP> L;
    constexpr int BR = 32;
    __shared__ __align__(16) char lds[2][2][BR * L::kRowBytes];
    __shared__ __align__(16) char room[4][kApartBytes<T>];
    __shared__ __align__(16) float stats[2][2][BR];   // lse in powers of two, delta
    __shared__ __align__(16) int2 sees[2][BR];
    __shared__ float2 red[4];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    unsigned pair;
    int tile;
    place(a, blockIdx.x, pair, tile);
    tile = a.tiles - 1 - tile;   // the first keys are seen by the most rows
    const int64_t worker = pair / a.kv;
    const int kvh = (int)(pair % a.kv);
    const int j0 = tile * 128, mine = j0 + wave * 32, key = mine + lane % 32;
    const bool valid = key < a.keys;
    const float up = gradient_scale<T>(a, worker, red);
    u4_t k[L::kOwn], v[L::kOwn];
    const T *krow = head_at<const T>(a.k, worker, valid ? key : 0, kvh), *vrow = head_at<const T>(a.v, worker, valid ? key : 0, kvh);
#pragma unroll
    for (int i = 0; i < L::kOwn; ++i) {
        k[i] = load_chunk<T>(krow, (2 * i + lane / 32) * L::E, a.width, valid);
        v[i] = load_chunk<T>(vrow, (2 * i + lane / 32) * L::E, a.width, valid);
    }
    const int blocks = (a.rows + BR - 1) / BR;
    // Without ranges the rows that see a key are all from one on.
    int begin = 0;
    if (!a.ranges && a.causal) begin = (int)(max((int64_t)0, (int64_t)j0 + a.tokens - a.keys) * a.group / BR);
    Stage<T, DP, BR, 256> qs, os;
    float2 stat = {0.0f, 0.0f};
    int2 range = {0, 0};
    f16_t dk[L::kBlocks], dv[L::kBlocks];
    const float shift = kBackwardShift<T>, factor = ldexpf(up, -(int)shift);
    for (int pass = 0;; ++pass) {
#pragma unroll
        for (int b = 0; b < L::kBlocks; ++b) dk[b] = dv[b] = f16_t{0};
        const auto next = [&](int block) {
            if (!a.ranges) return block;
            for (; block < blocks; block += kWave) {
                bool any = false;
                if (block + lane < blocks) any = block_sight(a, worker, block + lane).any(j0, 128);
                const unsigned long long m = __ballot(any);
                if (m) return block + __ffsll((long long)m) - 1;
            }
            return blocks;
        };
        const auto fetch = [&](int block) {
            const auto at = [&](const Heads &x, int r) -> const T * {
                const int row = block * BR + r;
                if (row >= a.rows) return nullptr;
                return head_at<const T>(x, worker, row / a.group, kvh * a.group + row % a.group);
            };
            qs.load(a.width, threadIdx.x, [&](int r) { return at(a.q, r); });
            os.load(a.width, threadIdx.x, [&](int r) { return at(a.dout, r); });
            if (threadIdx.x < BR) {
                const int row = block * BR + threadIdx.x;
                stat = float2{0.0f, 0.0f}, range = int2{0, 0};
                if (row < a.rows) {
                    const int t = row / a.group;
                    const int64_t s = (worker * a.heads + kvh * a.group + row % a.group) * a.tokens + t;
                    stat = float2{a.lse[s] * kLog2e - shift, a.delta[s]};
                    range = seen(a, worker, t);
                }
            }
        };
        const auto put = [&](int half) {
            qs.store(lds[half][0], threadIdx.x);
            os.store(lds[half][1], threadIdx.x);
            if (threadIdx.x < BR) {
                stats[half][0][threadIdx.x] = stat.x;
                stats[half][1][threadIdx.x] = stat.y;
                sees[half][threadIdx.x] = range;
            }
        };
        int block = next(begin), half = 0;
        if (block < blocks) {
            fetch(block);
            put(0);
        }
        while (block < blocks) {
            __syncthreads();
            const int then = next(block + 1);
            if (then < blocks) fetch(then);
            const Sight sight = block_sight(a, worker, block);
            if (sight.any(mine, 32)) {
                const bool whole = sight.whole(mine, 32);
                const f16_t s = dots<T, DP>(lds[half][0], 0, k, lane);
                const f16_t dp = dots<T, DP>(lds[half][1], 0, v, lane);
                float p[16], ds[16];
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f4_t off = *reinterpret_cast<const f4_t *>(&stats[half][0][8 * g + 4 * (lane / 32)]);
                    const f4_t delta = *reinterpret_cast<const f4_t *>(&stats[half][1][8 * g + 4 * (lane / 32)]);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int i = 4 * g + r;
                        p[i] = __builtin_amdgcn_exp2f(fmaf(s[i], a.dot_scale, -off[r]));
                        ds[i] = p[i] * factor * (dp[i] - delta[r]);
                    }
                }
                if (!whole) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int2 x = sees[half][8 * (i / 4) + 4 * (lane / 32) + i % 4];
                        const bool there = key >= x.x && key < x.y;
                        p[i] = there ? p[i] : 0.0f;
                        ds[i] = there ? ds[i] : 0.0f;
                    }
                }
                if (pass && !whole) {
                    const auto there = [&](int r) { return key >= sees[half][r].x && key < sees[half][r].y; };
                    add_rows_apart<T, DP>(dv, lds[half][1], 0, p, room[wave], lane, there);
                    add_rows_apart<T, DP>(dk, lds[half][0], 0, ds, room[wave], lane, there);
                } else {
                    add_rows<T, DP>(dv, lds[half][1], 0, Weights<T>(p), lane);
                    add_rows<T, DP>(dk, lds[half][0], 0, Weights<T>(ds), lane);
                }
            }
            half ^= 1;
            if (then < blocks) put(half);
            block = then;
        }
        if (pass || !__syncthreads_or(valid && (not_finite(dk) || not_finite(dv)))) break;
    }
    if (!valid) return;
    store_column<T>(head_at<T>(a.dk, worker, key, kvh), a.width, dk, a.scale / up, lane);
    store_column<T>(head_at<T>(a.dv, worker, key, kvh), a.width, dv, ldexpf(1.0f, -(int)shift), lane);
}

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

template <typename F>
void with_width(int64_t width, F f) {
    if (width <= 64) f(Int<64>());
    else if (width <= 128) f(Int<128>());
    else f(Int<256>());
}

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

// Tiles of the forward pass, or the parts that the keys are split into.
struct ForwardPlan {
    int64_t blocks;
    int32_t tiles, parts, span;
    bool split;
    size_t workspace;
};

ForwardPlan plan_forward(int32_t n, int64_t tokens, int64_t keys, int32_t heads, int32_t kv, int64_t width) {
    const int64_t pairs = (int64_t)n * kv, rows = tokens * (heads / kv);
    ForwardPlan p{};
    p.tiles = (int32_t)tiles(rows, 128);
    p.blocks = pairs * p.tiles;
    if (p.blocks >= kCus) return p;
    p.split = true;
    p.tiles = (int32_t)tiles(rows, 32);
    const int64_t base = pairs * p.tiles;
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>(tiles(keys, 128), tiles(2 * kCus, std::max<int64_t>(1, base))));
    p.span = (int32_t)std::max<int64_t>(32, tiles(tiles(keys, want), 32) * 32);
    p.parts = (int32_t)std::max<int64_t>(1, tiles(keys, p.span));
    p.blocks = base * p.parts;
    p.workspace = p.parts > 1 ? (size_t)pairs * rows * p.parts * (width + 2) * 4 : 0;
    return p;
}

struct BackwardPlan {
    int32_t parts;
    size_t delta, largest, bounds;   // offsets
    size_t workspace;
};

BackwardPlan plan_backward(int32_t n, int64_t tokens, int32_t heads, int32_t kv, int32_t type) {
    BackwardPlan p{};
    const int64_t rows = tokens * heads;
    p.parts = (int32_t)std::max<int64_t>(1, std::min<int64_t>(tiles(rows, 64), std::max<int64_t>(1, 8 * kCus / n)));
    p.parts = std::min(p.parts, 256);
    size_t at = 0;
    p.delta = at, at += tiles((size_t)n * rows * 4, 16) * 16;
    p.largest = at, at += type == RELAYSUM_HALF ? tiles((size_t)n * p.parts * 8, 16) * 16 : 0;
    p.bounds = at, at += (size_t)n * tiles(tokens * (heads / kv), 32) * 16;
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
    return tokens ? (int64_t)plan_forward(n, tokens, keys, heads, kv_heads, width).workspace : 0;
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
        if (!(scale > 0.0f && scale < INFINITY)) c.fail(refuse("scale must be positive"));
        if (c.code == RELAYSUM_OK && tokens) {
            p = plan_forward(n, tokens, keys, heads, kv_heads, width);
            c.product_launch(p, workspace, workspace_bytes);
        }
    }
    if (!c.ready()) return c.code;
    if (tokens == 0) return done("relaysum_attention");
    AttentionArgs a = attention_args(n, tokens, keys, heads, kv_heads, width, q, k, v, ranges, ranges_stride, causal,
                                     scale, out, lse);
    a.tiles = p.tiles, a.parts = p.parts, a.span = p.span;
    a.part_soft = static_cast<float2 *>(workspace);
    a.part_out = static_cast<float *>(workspace) + (size_t)a.pairs * a.rows * p.parts * 2;
    const hipStream_t st = (hipStream_t)hip_stream;
    with_type(q->type, [&](auto zero) {
        using T = decltype(zero);
        with_width(width, [&](auto dp) {
            constexpr int DP = decltype(dp)::value;
            if (p.split)
                hipLaunchKernelGGL(HIP_KERNEL_NAME(attention_split_kernel<T, DP>), dim3((unsigned)p.blocks),
                                   dim3(64 * kSplitWaves<T, DP>), 0, st, a);
            else
                hipLaunchKernelGGL(HIP_KERNEL_NAME(attention_kernel<T, DP>), dim3((unsigned)p.blocks), dim3(256), 0, st, a);
        });
        if (p.parts > 1)
            hipLaunchKernelGGL(attention_join_kernel<T>, dim3((unsigned)tiles((int64_t)a.pairs * a.rows, 4)), dim3(256), 0, st, a);
    });
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
    return (int64_t)plan_backward(n, tokens, heads, kv_heads, type).workspace;
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
        if (!(scale > 0.0f && scale < INFINITY)) c.fail(refuse("scale must be positive"));
        if (c.code == RELAYSUM_OK) {
            p = plan_backward(n, tokens, heads, kv_heads, type);
            const int64_t pairs = (int64_t)n * kv_heads;
            if (pairs * tiles(tokens * (heads / kv_heads), 128) > kMaxBlocks || pairs * tiles(keys, 128) > kMaxBlocks)
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
    a.delta = reinterpret_cast<float *>(ws + p.delta);
    a.largest = reinterpret_cast<float2 *>(ws + p.largest);
    a.bounds = reinterpret_cast<int4 *>(ws + p.bounds);
    a.parts = p.parts;
    const int64_t blocks = tiles(a.rows, 32);
    a.bound_stride = a.range_stride ? blocks : 0;
    const hipStream_t st = (hipStream_t)hip_stream;
    if (ranges && tokens) {
        const int64_t total = (a.range_stride ? n : 1) * blocks;
        hipLaunchKernelGGL(attention_bounds_kernel, dim3((unsigned)tiles(total, 8)), dim3(256), 0, st, a, total);
    }
    with_type(q->type, [&](auto zero) {
        using T = decltype(zero);
        if (tokens) hipLaunchKernelGGL(attention_delta_kernel<T>, dim3((unsigned)(n * p.parts)), dim3(256), 0, st, a);
        with_width(width, [&](auto dp) {
            constexpr int DP = decltype(dp)::value;
            a.tiles = (int32_t)tiles(keys, 128);
            if (keys)
                hipLaunchKernelGGL(HIP_KERNEL_NAME(attention_dkv_kernel<T, DP>), dim3((unsigned)(a.pairs * a.tiles)), dim3(256), 0, st, a);
            a.tiles = (int32_t)tiles(a.rows, 128);
            if (tokens)
                hipLaunchKernelGGL(HIP_KERNEL_NAME(attention_dq_kernel<T, DP>), dim3((unsigned)(a.pairs * a.tiles)), dim3(256), 0, st, a);
        });
    });
    return done("relaysum_attention_backward");
}

}  // extern "C"
