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
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "attention_launch.hpp"
#include "attention_tiles.hpp"
#include "layer_call.hpp"

namespace {

using namespace attention;

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// Weights of binary16 are held times 2^7 (forward, where they reach 2^8 times
// their largest) and 2^15 (backward, where they are at most 1): below 2^-14 it
// loses bits.
template <typename T>
constexpr float kForwardShift = std::is_same<T, _Float16>::value ? 7.0f : 0.0f;
template <typename T>
constexpr float kBackwardShift = std::is_same<T, _Float16>::value ? 15.0f : 0.0f;

// A kernel's arguments for what it does last.  They are read from memory there,
// not kept in scalar registers from its start on, which would run out of them and
// take a stack.  `a` is the kernel's first argument.
__device__ __forceinline__ const AttentionArgs &later_arguments() {
    typedef const __attribute__((address_space(4))) AttentionArgs *Place;
    Place p = (Place)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const AttentionArgs *)p;
}

// The token of a row.
__device__ __forceinline__ int token_of(const AttentionArgs &a, int row) {
    return (int)((__umulhi((unsigned)row, a.group_factor) + (unsigned)row) >> a.group_shift);
}

// The keys that a token sees.
__device__ __forceinline__ int2 seen(const AttentionArgs &a, int64_t worker, int t) {
    if (a.ranges) {
        const int2 r = a.ranges[worker * a.range_stride + t];
        return int2{max(r.x, 0), max(0, min(r.y, a.keys))};
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

// Whether a column that sees keys lo <= j < hi sees the one that is `far` and
// `more` behind lo.
__device__ __forceinline__ bool sees(int far, int more, int lo, int hi) {
    return (unsigned)(far + more) < (unsigned)max(hi - lo, 0);
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
// 128 rows a workgroup, tiles of 64 keys (of 128 floats or more 32) and their
// values by turns in two halves of LDS, which all four waves read.  Of heads of 64
// vector instructions bound it: for 32 x 64 scores 16 matrix instructions and some
// 155 others where nothing is masked, 32 of them exponentials; masks are 96 more, a
// reference that moves 68, and a quarter of all are in front of the loop and behind
// it.  At 16 x 2048 tokens in three texts, 16 heads on 4, bfloat16, vector units are
// busy 72%, matrix units 29% (92 us, the call 98: 545 TFLOP/s).  Of 128 matrix units
// are busy half of the time: one sequence of 16,384, 8 heads on 2: 580 us, 950 TFLOP/s.
// All reads of a product in front of it: 4% quicker with 64 entries, 10% slower
// with 128 (registers).
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

    // 32 * NB keys from j on.  APART: what a column does not see is kept out of it
    // also where it is not finite.
    template <int NB, bool APART>
    __device__ __forceinline__ void step(const AttentionArgs &a, const char *kt, const char *vt, int j, int lo, int hi,
                                         bool whole, char *room, int lane) {
        f16_t s[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) s[b] = dots<T, DP>(kt, 32 * b, q, lane);
        add<NB, APART>(a, s, vt, j, lo, hi, whole, room, lane);
    }

    // The same from their products with q.
    template <int NB, bool APART>
    __device__ __forceinline__ void add(const AttentionArgs &a, const f16_t (&s)[NB], const char *vt, int j, int lo, int hi,
                                        bool whole, char *room, int lane) {
        const int h = lane / 32;
        float p[NB][16];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) p[b][i] = s[b][i];
        if (!whole) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    p[b][i] = sees(j + 4 * h - lo, 32 * b + 8 * (i / 4) + i % 4, lo, hi) ? p[b][i] : -INFINITY;
                }
        }
        float top = p[0][0];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, p[b][i]);
        top = fmaxf(top, other_half(top));
        // Finite, so that the first score passes -infinity whatever the scale is.
        const bool past = top > m + fminf(8.0f / a.dot_scale, 3e38f);
        if (__ballot(past)) {
            // Others' references stay: what they do not see moves no rounding of theirs.
            const float to = past ? top : m;
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
        if (APART && !whole) {
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

// Waves of a SIMD that registers are given out for: as many as the loops leave
// room for.
template <typename T, int DP>
constexpr int kForwardWaves = sizeof(T) == 4 || DP > 128 ? 1 : DP > 64 ? 2 : 4;
template <typename T, int DP>
constexpr int kQueryWaves = sizeof(T) == 4 || DP > 128 ? 1 : DP > 64 ? 2 : 3;
template <typename T, int DP>
constexpr int kKeyWaves = sizeof(T) == 4 || DP > 128 ? 1 : 2;

// A workgroup's 128 rows, 32 of each wave, and the keys that they see.
struct RowTile {
    unsigned pair;
    int tile, wave, lane, kvh, row, t, head, lo, hi, first, end;
    int64_t worker;
    bool valid;
    Sight sight;

    __device__ __forceinline__ RowTile(const AttentionArgs &a, unsigned block, int (&most)[4][2]) {
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
        place(a, block, pair, tile);
        worker = pair / a.kv;
        kvh = (int)(pair % a.kv);
        row = tile * 128 + wave * 32 + lane % 32;
        valid = row < a.rows;
        t = valid ? token_of(a, row) : 0, head = kvh * a.group + (valid ? row - t * a.group : 0);
        const int2 range = valid ? seen(a, worker, t) : int2{0, INT_MAX};
        lo = range.x, hi = range.y;
        sight = sight_of(lo, hi, valid);
        if (lane == 0) most[wave][0] = sight.least_lo, most[wave][1] = sight.most_hi;
        __syncthreads();
        first = __builtin_amdgcn_readfirstlane(min(min(most[0][0], most[1][0]), min(most[2][0], most[3][0])));
        end = __builtin_amdgcn_readfirstlane(max(max(most[0][1], most[1][1]), max(most[2][1], most[3][1])));
    }
};

// Runs `step(tile, j)` over tiles of BN keys from `first` to `end`: keys at
// `tile` and the values behind them, the next tile's on their way meanwhile.
template <typename T, int DP, int BN, bool DIRECT, typename F>
__device__ __forceinline__ void over_keys(const AttentionArgs &a, const RowTile &r, char (&lds)[2][2 * BN * Tile<T, DP>::kRowBytes],
                                          F step) {
    constexpr int kTile = BN * Tile<T, DP>::kRowBytes;
    const int begin = r.first / BN * BN, end = r.end;
    if (r.first >= end) return;
    const char *kbase = reinterpret_cast<const char *>(head_at<const T>(a.k, r.worker, 0, r.kvh));
    const char *vbase = reinterpret_cast<const char *>(head_at<const T>(a.v, r.worker, 0, r.kvh));
    const int64_t kr = a.k.rs * (int64_t)sizeof(T), vr = a.v.rs * (int64_t)sizeof(T);
    Stage<T, DP, BN, 256, DIRECT> ks, vs;
    const auto kat = [&](int x) { return x * kr; };
    const auto vat = [&](int x) { return x * vr; };
    const auto fetch = [&](int j, char *to) __attribute__((always_inline)) {
        const int rows = min(BN, a.keys - j);
        ks.load(kbase + j * kr, to, a.width, rows, threadIdx.x, kat);
        vs.load(vbase + j * vr, to + kTile, a.width, rows, threadIdx.x, vat);
    };
    const auto put = [&](char *to) {
        ks.put(to, threadIdx.x);
        vs.put(to + kTile, threadIdx.x);
    };
    if (DIRECT && a.width < DP) {
#pragma unroll
        for (int i = 0; i < 4; ++i) ks.clear(lds[i / 2] + i % 2 * kTile, threadIdx.x);
        __syncthreads();
    }
    ks.places(threadIdx.x, kat);
    vs.places(threadIdx.x, vat);
    fetch(begin, lds[0]);
    put(lds[0]);
    int half = 0;
    for (int j = begin; j < end; j += BN, half ^= 1) {
        __syncthreads();
        const bool more = j + BN < end;
        if (more) fetch(j + BN, lds[half ^ 1]);
        step(lds[half], j);
        if (more) put(lds[half ^ 1]);
    }
}

// A column's own row in chunks.
template <typename T, int DP>
__device__ __forceinline__ void load_own(const T *row, u4_t (&own)[Tile<T, DP>::kOwn], int width, bool valid, int lane) {
#pragma unroll
    for (int i = 0; i < Tile<T, DP>::kOwn; ++i)
        own[i] = load_chunk<T>(row, (2 * i + lane / 32) * Tile<T, DP>::E, width, valid);
}

template <typename T, int DP>
__device__ __forceinline__ void store_rows(const AttentionArgs &a, const RowTile &r, const Softmax<T, DP> &st, float sum) {
    if (!r.valid) return;
    const bool empty = r.lo >= r.hi;
    store_column<T>(head_at<T>(a.out, r.worker, r.t, r.head), a.width, st.acc, empty ? 0.0f : 1.0f / sum, r.lane);
    if (a.lse && r.lane < 32)
        a.lse[(r.worker * a.heads + r.head) * a.tokens + r.t] =
            empty ? -INFINITY : kLn2 * (st.off + __builtin_amdgcn_logf(sum));
}

// Workgroups in whose sums something is not finite leave a mark in place of
// results, and a second kernel works on what is marked once more, with what a
// column does not see kept out of it.  In a kernel of its own, because it takes
// more registers, and called as a function it costs every wave of the first one
// a stack (16 x 2048 tokens, 16 heads on 4 of 64: 161 us for 109 us).
//
// Few workgroups look at the marks: there is seldom one, and with heads above 128
// entries these kernels do take a stack (11 to 24 us of 256 workgroups).
constexpr int kApartBlocks = kCus / 4;

template <typename F>
__device__ __forceinline__ void over_marks(const int32_t *marks, int64_t blocks, F f) {
    // 256 marks at a time, neighbours in other workgroups.
    const int64_t step = gridDim.x;
    for (int64_t first = blockIdx.x; first < blocks; first += 256 * step) {
        const int64_t own = first + threadIdx.x * step;
        if (!__syncthreads_or(own < blocks && marks[own])) continue;
        for (int64_t i = first; i < min(blocks, first + 256 * step); i += step) {
            if (!marks[i]) continue;
            __syncthreads();
            f((unsigned)i);
        }
    }
}

template <typename T, int DP>
__global__ __launch_bounds__(256) void attention_apart_kernel(AttentionArgs a, int64_t blocks) {
    constexpr int BN = kKeyTile<T, DP>, kRowBytes = Tile<T, DP>::kRowBytes;
    __shared__ __align__(16) char lds[2][2 * BN * kRowBytes];
    __shared__ __align__(16) char room[4][kApartBytes<T>];
    __shared__ int most[4][2];
    over_marks(a.marks, blocks, [&](unsigned block) {
        const RowTile r(a, block, most);
        Softmax<T, DP> st;
        load_own<T, DP>(head_at<const T>(a.q, r.worker, r.t, r.head), st.q, a.width, r.valid, r.lane);
        st.clear();
        over_keys<T, DP, BN, false>(a, r, lds, [&](const char *tile, int j) {
#pragma unroll 1
            for (int b = 0; b < BN; b += 32)
                if (r.sight.any(j + b, 32))
                    st.template step<1, true>(a, tile + b * kRowBytes, tile + (BN + b) * kRowBytes, j + b, r.lo, r.hi,
                                              r.sight.whole(j + b, 32), room[r.wave], r.lane);
        });
        store_rows(a, r, st, st.l + other_half(st.l));
    });
}

template <typename T, int DP, bool DIRECT>
__global__ __launch_bounds__(256, (kForwardWaves<T, DP>)) void attention_kernel(AttentionArgs a) {
    constexpr int BN = kKeyTile<T, DP>;
    __shared__ __align__(16) char lds[2][2 * BN * Tile<T, DP>::kRowBytes];
    __shared__ int most[4][2];
    const RowTile r(a, blockIdx.x, most);
    Softmax<T, DP> st;
    load_own<T, DP>(head_at<const T>(a.q, r.worker, r.t, r.head), st.q, a.width, r.valid, r.lane);
    st.clear();
    over_keys<T, DP, BN, DIRECT>(a, r, lds, [&](const char *tile, int j) __attribute__((always_inline)) {
        if (r.sight.any(j, BN))
            st.template step<BN / 32, false>(a, tile, tile + BN * Tile<T, DP>::kRowBytes, j, r.lo, r.hi,
                                             r.sight.whole(j, BN), nullptr, r.lane);
    });
    const float sum = st.l + other_half(st.l);
    const bool again = __syncthreads_or(r.valid && (not_finite(st.acc) || !(fabsf(sum) < INFINITY)));
    const AttentionArgs &later = later_arguments();
    if (threadIdx.x == 0) later.marks[blockIdx.x] = again;
    if (!again) store_rows(later, r, st, sum);
}

// Few rows: the keys are split over workgroups (parts) and their waves, each of
// which walks through its own keys, 32 at a time in turn; waves join through LDS,
// parts in a second kernel.  Keys go from memory to where the products take them.
// Bound by the latency of its loads, or by memory: 16 workers' row over 1024 keys,
// 12 heads on 4 of 64, bfloat16 14 us with the call; over 8192 keys 35 us, 3.9
// TB/s.  16 waves of 128 registers (and a stack) took 18 us for the first.
template <typename T, int DP>
__global__ __launch_bounds__(64 * split_waves(sizeof(T), DP)) void attention_split_kernel(AttentionArgs a) {
    typedef Tile<T, DP> L;
    constexpr int W = split_waves(sizeof(T), DP);
    // A wave's values, and later its sums.
    constexpr int kOwnBytes = std::max(32 * L::kRowBytes, 32 * DP * 4);
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
    const int t = valid ? token_of(a, row) : 0, head = kvh * a.group + (valid ? row - t * a.group : 0);
    const int2 range = valid ? seen(a, worker, t) : int2{0, INT_MAX};
    const int lo = range.x, hi = range.y;
    Softmax<T, DP> st;
    load_own<T, DP>(head_at<const T>(a.q, worker, t, head), st.q, a.width, valid, lane);
    const Sight sight = sight_of(lo, hi, valid);

    const T *kbase = head_at<const T>(a.k, worker, 0, kvh), *vbase = head_at<const T>(a.v, worker, 0, kvh);
    const int64_t from = (int64_t)part * a.span, to = min(from + a.span, (int64_t)sight.most_hi);
    char *vt = lds[wave];
    const auto next = [&](int64_t j) {
        while (j < to && !sight.any((int)j, 32)) j += 32 * W;
        return j;
    };
    u4_t keys[L::kOwn];
    Stage<T, DP, 32, 64, false> vs;
    const auto over = [&](auto apart) __attribute__((always_inline)) {
        constexpr bool kApart = decltype(apart)::value;
        const auto fetch = [&](int64_t j) {
            const int rows = (int)min((int64_t)32, a.keys - j);
            load_own<T, DP>(kbase + (j + min(lane % 32, rows - 1)) * a.k.rs, keys, a.width, lane % 32 < rows, lane);
            vs.load(reinterpret_cast<const char *>(vbase + j * a.v.rs), vt, a.width, rows, lane,
                    [&](int x) { return x * a.v.rs * (int64_t)sizeof(T); });
        };
        st.clear();
        int64_t j = next(from + 32 * wave);
        if (!kApart && j < to) fetch(j);
#pragma unroll 1
        while (j < to) {
            // Without registers for what comes next it needs no stack.
            if (kApart) fetch(j);
            f16_t s[1] = {};
#pragma unroll
            for (int i = 0; i < L::kOwn; ++i) s[0] = multiply(s[0], keys[i], st.q[i], (T)0.0f);
            vs.put(vt, lane);
            wave_fence();
            const int64_t then = next(j + 32 * W);
            if (!kApart && then < to) fetch(then);
            st.template add<1, kApart>(a, s, vt, (int)j, lo, hi, sight.whole((int)j, 32), room[wave], lane);
            wave_fence();
            j = then;
        }
    };
    over(std::false_type());
    float sum = st.l + other_half(st.l);
    if (__ballot(valid && (not_finite(st.acc) || !(fabsf(sum) < INFINITY)))) {
        over(std::true_type());
        sum = st.l + other_half(st.l);
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
    const int rt = token_of(a, r), rh = kvh * a.group + r - rt * a.group;
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

// Parts of a row join: a workgroup a row, whose waves share out the parts.
constexpr int kJoinWaves = 8;

template <typename T>
__global__ __launch_bounds__(64 * kJoinWaves) void attention_join_kernel(AttentionArgs a) {
    __shared__ float sums[kJoinWaves][256];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t at = blockIdx.x, pair = at / a.rows, worker = pair / a.kv;
    const int r = (int)(at % a.rows), t = token_of(a, r), head = (int)(pair % a.kv) * a.group + r - t * a.group;
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
    for (int k = lane; k < a.width; k += kWave) {
        const float *from = a.part_out + at * a.parts * a.width + k;
        float v = 0.0f;
#pragma unroll 8
        for (int p = wave; p < a.parts; p += kJoinWaves) {
            const float x = from[(int64_t)p * a.width], own = soft[p].x;
            v += own == -INFINITY ? 0.0f : x * __builtin_amdgcn_exp2f(own - top);
        }
        sums[wave][k] = v;
    }
    __syncthreads();
    const int k = threadIdx.x;
    if (k < a.width) {
        float v = sums[0][k];
#pragma unroll
        for (int w = 1; w < kJoinWaves; ++w) v += sums[w][k];
        // All of its scores are -infinity: 0 / 0.
        head_at<T>(a.out, worker, t, head)[k] = (T)(empty ? 0.0f : v * (1.0f / all));
    }
    if (a.lse && k == 0)
        a.lse[(worker * a.heads + head) * a.tokens + t] =
            empty ? -INFINITY : kLn2 * ((top == -INFINITY ? 0.0f : top) + __builtin_amdgcn_logf(all));
}

// ---- backward ----------------------------------------------------------------------

// What blocks of 32 rows see.
template <typename T>
__global__ __launch_bounds__(256) void attention_bounds_kernel(AttentionArgs a, int64_t total) {
    const int64_t at = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
    if (at >= total) return;
    const int64_t per = (a.rows + 31) / 32, worker = at / per;
    const int row = (int)(at % per) * 32 + threadIdx.x % 32;
    int2 s = row < a.rows ? seen(a, worker, token_of(a, row)) : int2{INT_MAX, 0};
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

// The tiles of 128 keys of every worker (of all, where they have the same ranges)
// in the order of how many blocks of rows see them, the most first: a device
// whose last workgroups have the least to do is done sooner (16 x 2048 tokens, 16
// heads on 4 of 64: 1024 workgroups, two for a CU at once).  By a workgroup of
// its own: each block opens and closes a run of tiles, sums give the counts, and
// a tile's place is the number of those that come before it.
constexpr int kMostOrdered = 2048;

template <typename T>
__global__ __launch_bounds__(1024) void attention_order_kernel(AttentionArgs a, int workers) {
    __shared__ int count[kMostOrdered + 1];
    const int all = workers * a.tiles, blocks = (a.rows + 31) / 32;
    for (int i = threadIdx.x; i < all; i += 1024) count[i] = 0;
    __syncthreads();
    for (int64_t i = threadIdx.x; i < (int64_t)workers * blocks; i += 1024) {
        const int4 b = a.bounds[i];
        if (b.x >= b.w || b.x >= a.keys) continue;
        const int worker = (int)(i / blocks), from = b.x / 128, to = (b.w - 1) / 128 + 1;
        atomicAdd(&count[worker * a.tiles + from], 1);
        if (to < a.tiles) atomicSub(&count[worker * a.tiles + to], 1);
    }
    __syncthreads();
    for (int w = threadIdx.x; w < workers; w += 1024)
        for (int i = 1; i < a.tiles; ++i) count[w * a.tiles + i] += count[w * a.tiles + i - 1];
    __syncthreads();
    for (int i = threadIdx.x; i < all; i += 1024) {
        int before = 0;
        for (int j = 0; j < all; ++j) before += count[j] > count[i] || (count[j] == count[i] && j < i);
        a.order[before] = i;
    }
}

// Least and most lo, least and most hi of 32 rows; rows behind the last see nothing.
__device__ __forceinline__ Sight block_sight(const AttentionArgs &a, int64_t worker, int block) {
    if (a.ranges) {
        const int4 b = a.bounds[worker * a.bound_stride + block];
        return Sight{b.x, b.y, b.z, b.w};
    }
    const int last = min(block * 32 + 31, a.rows - 1);
    return Sight{0, 0, block * 32 + 32 > a.rows ? 0 : seen(a, worker, token_of(a, block * 32)).y,
                 seen(a, worker, token_of(a, last)).y};
}

// What a column's ds is held times in binary16, which loses bits below 2^-14: a
// power of two that brings the largest that the column has had to 2^13 at least,
// and never past the type's largest number.  Where a larger one comes by, the sums
// so far follow, which are floats.  It is the column's own, because one of several
// columns, or from bounds of |dout| and |v|, leaves no bits to a column where
// another, or what it does not see, is large.
template <typename T>
struct Held {
    static constexpr bool kOn = std::is_same<T, _Float16>::value;
    float up;

    __device__ __forceinline__ void clear() { up = kOn ? 0x1p100f : 1.0f; }

    template <int B>
    __device__ __forceinline__ void hold(float (&ds)[16], f16_t (&sums)[B]) {
        if constexpr (kOn) {
            float top = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, fabsf(ds[i]));
            top = fmaxf(top, other_half(top));
            const bool more = top * up > 65504.0f && top < INFINITY;
            if (__ballot(more)) {
                const float to = more ? ldexpf(1.0f, 13 - ilogbf(top)) : up, f = to / up;
#pragma unroll
                for (int b = 0; b < B; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) sums[b][i] *= f;
                up = to;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) ds[i] *= up;
        }
    }
    // What the sums are to be multiplied by, with a factor of their own.  Finite:
    // sums of zero stay zero.
    __device__ __forceinline__ float down(float f) const { return fminf(f / up, 3e38f); }
};

// A column's own row in the gradients: in registers, or of more than 128 floats,
// two of which with a sum would pass the registers of a wave, in memory.
template <typename T, int DP>
struct OwnRow {
    static constexpr bool kFar = sizeof(T) == 4 && DP > 128;
    u4_t x[kFar ? 1 : Tile<T, DP>::kOwn];
    const T *row;
    bool valid;

    __device__ __forceinline__ void load(const T *from, int width, bool there, int lane) {
        row = from, valid = there;
        if constexpr (!kFar) load_own<T, DP>(from, x, width, there, lane);
    }
    __device__ __forceinline__ u4_t chunk(int i, int width, int lane) const {
        if constexpr (kFar) return load_chunk<T>(row, (2 * i + lane / 32) * Tile<T, DP>::E, width, valid);
        else return x[i];
    }
    // Of 32 rows of a tile from row0 on.
    __device__ __forceinline__ f16_t products(const char *tile, int row0, int width, int lane) const {
        if constexpr (kFar) return dots_in_memory<T, DP>(tile, row0, row, width, valid, lane);
        else return dots<T, DP>(tile, row0, x, lane);
    }
};

// The gradient of q: as forward, with the weights known from lse.  delta is
// dout . out of a row.  16 x 2048 tokens, 16 heads on 4 of 64, bfloat16 128 us; 16,384
// tokens, 8 heads on 2 of 128 800 us, 1030 TFLOP/s.
template <typename T, int DP>
struct QueryGradient {
    typedef Tile<T, DP> L;
    OwnRow<T, DP> q, dout;
    f16_t acc[L::kBlocks];
    float off, delta;
    Held<T> held;

    __device__ __forceinline__ void start(const AttentionArgs &a, const RowTile &r) {
        q.load(head_at<const T>(a.q, r.worker, r.t, r.head), a.width, r.valid, r.lane);
        dout.load(head_at<const T>(a.dout, r.worker, r.t, r.head), a.width, r.valid, r.lane);
        off = r.valid ? a.lse[(r.worker * a.heads + r.head) * a.tokens + r.t] * kLog2e : 0.0f;
        delta = 0.0f;
        constexpr int kAtOnce = OwnRow<T, DP>::kFar ? 4 : L::kOwn;
#pragma unroll kAtOnce
        for (int i = 0; i < L::kOwn; ++i)
            delta = chunk_dot<T>(dout.chunk(i, a.width, r.lane), load_chunk<T>(head_at<const T>(a.out, r.worker, r.t, r.head),
                                                        (2 * i + r.lane / 32) * L::E, a.width, r.valid), delta);
        delta += other_half(delta);
        held.clear();
#pragma unroll
        for (int b = 0; b < L::kBlocks; ++b) acc[b] = f16_t{0};
    }
    // For the gradients of k and v.
    __device__ __forceinline__ void keep(const AttentionArgs &a, const RowTile &r) const {
        if (r.valid && r.lane < 32) a.stats[(int64_t)r.pair * a.rows + r.row] = float2{off, delta};
    }
    // The part of 32 keys from j on in sum p (dout . v), which is delta too.
    __device__ __forceinline__ float product(const AttentionArgs &a, const RowTile &r, const char *kt, const char *vt, int j) const {
        const f16_t s = q.products(kt, 0, a.width, r.lane);
        const f16_t dp = dout.products(vt, 0, a.width, r.lane);
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float x = __builtin_amdgcn_exp2f(fmaf(s[i], a.dot_scale, -off)) * dp[i];
            sum += sees(j + 4 * (r.lane / 32) - r.lo, 8 * (i / 4) + i % 4, r.lo, r.hi) ? x : 0.0f;
        }
        return sum;
    }

    // 32 keys from j on.
    template <bool APART>
    __device__ __forceinline__ void step(const AttentionArgs &a, const RowTile &r, const char *kt, const char *vt, int j,
                                         char *room) {
        const bool whole = r.sight.whole(j, 32);
        const f16_t s = q.products(kt, 0, a.width, r.lane);
        const f16_t dp = dout.products(vt, 0, a.width, r.lane);
        float ds[16];
#pragma unroll
        for (int i = 0; i < 16; ++i)
            ds[i] = __builtin_amdgcn_exp2f(fmaf(s[i], a.dot_scale, -off)) * (dp[i] - delta);
        if (!whole) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                // A row's only key has weight 1 whatever its score is: ds is 0.
                ds[i] = sees(j + 4 * (r.lane / 32) - r.lo, 8 * (i / 4) + i % 4, r.lo, r.hi - r.lo == 1 ? r.lo : r.hi) ? ds[i] : 0.0f;
            }
        }
        held.hold(ds, acc);
        if (APART && !whole)
            add_rows_apart<T, DP>(acc, kt, 0, ds, room, r.lane, [&](int x) { return j + x >= r.lo && j + x < r.hi; });
        else
            add_rows<T, DP>(acc, kt, 0, Weights<T>(ds), r.lane);
    }
    __device__ __forceinline__ void store(const AttentionArgs &a, const RowTile &r) const {
        if (r.valid) store_column<T>(head_at<T>(a.dq, r.worker, r.t, r.head), a.width, acc, held.down(a.scale), r.lane);
    }
};

template <typename T, int DP, bool DIRECT, bool APART>
__device__ __forceinline__ void dq_over_keys(const AttentionArgs &a, const RowTile &r, QueryGradient<T, DP> &g,
                                             char (&lds)[2][2 * kKeyTile<T, DP> * Tile<T, DP>::kRowBytes], char *room) {
    constexpr int BN = kKeyTile<T, DP>, kRowBytes = Tile<T, DP>::kRowBytes;
    over_keys<T, DP, BN, DIRECT>(a, r, lds, [&](const char *tile, int j) __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < BN; b += 32)
            if (r.sight.any(j + b, 32))
                g.template step<APART>(a, r, tile + b * kRowBytes, tile + (BN + b) * kRowBytes, j + b, room);
    });
}

// Where a workgroup walks through this many keys at most, delta comes from a walk
// of its own: with out rounded to 16 bits it is off by 2^-9 of |dout| |out|, which
// of few keys is as much as the rounding of ds (gradients of sequences of 8, 64
// and 250: 1.8, 1.55 and 1.6 times the rounding of the result, without it 1.4).
constexpr int kExactKeys = 256;

template <typename T, int DP, bool DIRECT>
__device__ __forceinline__ void exact_delta(const AttentionArgs &a, const RowTile &r, QueryGradient<T, DP> &g,
                                            char (&lds)[2][2 * kKeyTile<T, DP> * Tile<T, DP>::kRowBytes]) {
    if (sizeof(T) == 4 || r.end - r.first > kExactKeys) return;
    constexpr int BN = kKeyTile<T, DP>, kRowBytes = Tile<T, DP>::kRowBytes;
    float sum = 0.0f;
    over_keys<T, DP, BN, DIRECT>(a, r, lds, [&](const char *tile, int j) __attribute__((always_inline)) {
#pragma unroll 1
        for (int b = 0; b < BN; b += 32)
            if (r.sight.any(j + b, 32)) sum += g.product(a, r, tile + b * kRowBytes, tile + (BN + b) * kRowBytes, j + b);
    });
    g.delta = sum + other_half(sum);
    __syncthreads();
}

template <typename T, int DP, bool DIRECT>
__global__ __launch_bounds__(256, (kQueryWaves<T, DP>)) void attention_dq_kernel(AttentionArgs a) {
    __shared__ __align__(16) char lds[2][2 * kKeyTile<T, DP> * Tile<T, DP>::kRowBytes];
    __shared__ int most[4][2];
    const RowTile r(a, blockIdx.x, most);
    QueryGradient<T, DP> g;
    g.start(a, r);
    exact_delta<T, DP, DIRECT>(a, r, g, lds);
    g.keep(a, r);
    dq_over_keys<T, DP, DIRECT, false>(a, r, g, lds, nullptr);
    const bool again = __syncthreads_or(r.valid && not_finite(g.acc));
    const AttentionArgs &later = later_arguments();
    if (threadIdx.x == 0) later.marks[blockIdx.x] = again;
    if (!again) g.store(later, r);
}

// The gradients of k and v: columns are keys, 128 of a workgroup, and rows the
// queries that see them, in tiles of 32 or 64.  Four products of the seven of both
// kernels: 231 us where dq takes 128, and 1130 (970 TFLOP/s) where it takes 800.
// Two waves a SIMD, which wait half of the time for LDS and each other; three do
// not fit the registers.  Loads are used a tile later, in put(): used where they
// are issued they would wait for all copies on their way (9.2 ms for 3.0).
template <typename T, int DP>
constexpr int kRowTile = Tile<T, DP>::kRowBytes > 128 ? 32 : 64;

// Whether the keys' own rows of v lie in LDS: at 128 entries of 16 bits the rows
// and sums of two arrays pass the 256 registers of two waves a SIMD.
template <typename T, int DP>
constexpr bool kValuesInLds = sizeof(T) == 2 && DP == 128;

// Which gradients a kernel of keys gives: of more than 128 entries dk and dv one
// after the other, since sums of both leave no registers for the keys' rows.
enum { kBoth = 0, kOnlyValues = 1, kOnlyKeys = 2 };
template <typename T, int DP>
constexpr bool kOneByOne = DP > 128;

template <typename T, int DP>
struct RowsInLds {
    char rows[2][kRowTile<T, DP> * Tile<T, DP>::kRowBytes];   // q, dout
    float stats[2][kRowTile<T, DP>];                          // lse in powers of two, delta
    int2 sees[kRowTile<T, DP>];
};

// The tiles of rows that a workgroup walks through.  Of 64 blocks of 32 rows at a
// time each lane looks at one: whether any of the workgroup's keys is seen from
// it, any of this wave's, and all of them from all of its rows.
struct Walk {
    int64_t worker;
    int j0, mine, base, part;
    unsigned long long open, any, whole;

    template <int BLOCKS>
    __device__ __forceinline__ void look(const AttentionArgs &a, int lane) {
        const int block = base + lane;
        Sight s{0, 0, 0, 0};
        if (block * 32 < a.rows) s = block_sight(a, worker, block);
        open = __ballot(s.any(j0, 128));
        any = __ballot(s.any(mine, 32));
        whole = __ballot(s.whole(mine, 32));
        if (BLOCKS == 2) open = (open | open >> 1) & 0x5555555555555555ull;
        // Tiles go round the parts.
        const int tile = (base + lane) / BLOCKS;
        open &= __ballot(tile % a.parts == part);
    }
    // The first block of the next tile from `block` on, or one behind the last.
    template <int BLOCKS>
    __device__ __forceinline__ int next(const AttentionArgs &a, int block, int blocks, int lane) {
        while (block < blocks) {
            if (block >= base + 64) {
                base = block & ~63;
                look<BLOCKS>(a, lane);
            }
            const unsigned long long left = open >> (block - base);
            if (left) return block + __builtin_ctzll(left);
            block = base + 64;
        }
        return blocks;
    }
};

template <typename T, int DP, int WHICH>
struct KeyGradient {
    typedef Tile<T, DP> L;
    static constexpr bool kInLds = kValuesInLds<T, DP>, kDk = WHICH != kOnlyValues, kDv = WHICH != kOnlyKeys;
    OwnRow<T, DP> k, v;
    const char *values;   // 32 rows of v
    f16_t dk[kDk ? L::kBlocks : 1], dv[kDv ? L::kBlocks : 1];
    int64_t worker;
    int kvh, j0, mine, key, lane, part;
    unsigned pair;
    bool valid;
    Held<T> held;   // with p in it, of ds times 2^kBackwardShift

    __device__ __forceinline__ void start(const AttentionArgs &a, unsigned at, int tile, int turn, char *own) {
        lane = threadIdx.x % kWave;
        pair = at, part = turn;
        worker = pair / a.kv;
        kvh = (int)(pair % a.kv);
        j0 = tile * 128, mine = j0 + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) * 32;
        key = mine + lane % 32;
        valid = key < a.keys;
        held.clear();
        k.load(head_at<const T>(a.k, worker, valid ? key : 0, kvh), a.width, valid, lane);
        const T *vrow = head_at<const T>(a.v, worker, valid ? key : 0, kvh);
        if constexpr (!kDk) {
        } else if constexpr (kInLds) {
            char *to = own + threadIdx.x / kWave * 32 * L::kRowBytes;
            values = to;
            for (int i = 0; i < L::kOwn; ++i)
                *reinterpret_cast<u4_t *>(to + L::at(lane % 32, 2 * i + lane / 32)) =
                    load_chunk<T>(vrow, (2 * i + lane / 32) * L::E, a.width, valid);
        } else {
            v.load(vrow, a.width, valid, lane);
        }
#pragma unroll
        for (f16_t &x : dk) x = f16_t{0};
#pragma unroll
        for (f16_t &x : dv) x = f16_t{0};
    }

    // 32 rows of a tile from row0 on.
    template <bool APART>
    __device__ __forceinline__ void step(const AttentionArgs &a, const RowsInLds<T, DP> &lds, int row0, bool whole, char *room) {
        const f16_t s = k.products(lds.rows[0], row0, a.width, lane);
        float p[16], ds[16];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f4_t off = *reinterpret_cast<const f4_t *>(&lds.stats[0][row0 + 8 * g + 4 * (lane / 32)]);
#pragma unroll
            for (int r = 0; r < 4; ++r) p[4 * g + r] = __builtin_amdgcn_exp2f(fmaf(s[4 * g + r], a.dot_scale, -off[r]));
        }
        f16_t dp;
        if constexpr (!kDk) dp = f16_t{0};
        else if constexpr (kInLds) dp = dots_in_lds<T, DP>(lds.rows[1], row0, values, 0, lane);
        else dp = v.products(lds.rows[1], row0, a.width, lane);
        unsigned there = 0xffff;
        if (!whole) {
            there = 0;
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                const i4_t x = *reinterpret_cast<const i4_t *>(&lds.sees[row0 + 8 * (i / 4) + 4 * (lane / 32) + i % 4]);
                const bool one = sees(key - x[0], 0, x[0], x[1]), two = sees(key - x[2], 0, x[2], x[3]);
                p[i] = one ? p[i] : 0.0f, p[i + 1] = two ? p[i + 1] : 0.0f;
                // Not the gradient of a row's only key: its weight is 1 whatever its score is.
                there |= (one && x[1] - x[0] != 1) << i | (two && x[3] - x[2] != 1) << (i + 1);
            }
        }
        const auto there_apart = [&](int r) {
            const int2 x = lds.sees[row0 + r];
            return sees(key - x.x, 0, x.x, x.y);
        };
        if constexpr (kDv) {
            if (APART && !whole) add_rows_apart<T, DP>(dv, lds.rows[1], row0, p, room, lane, there_apart);
            else add_rows<T, DP>(dv, lds.rows[1], row0, Weights<T>(p), lane);
        }
        if constexpr (kDk) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f4_t delta = *reinterpret_cast<const f4_t *>(&lds.stats[1][row0 + 8 * g + 4 * (lane / 32)]);
#pragma unroll
                for (int r = 0; r < 4; ++r) ds[4 * g + r] = p[4 * g + r] * (dp[4 * g + r] - delta[r]);
            }
            // A weight of 0 times an infinity is none.
            if (!whole) {
#pragma unroll
                for (int i = 0; i < 16; ++i) ds[i] = there >> i & 1 ? ds[i] : 0.0f;
            }
            held.hold(ds, dk);
            if (APART && !whole) add_rows_apart<T, DP>(dk, lds.rows[0], row0, ds, room, lane, there_apart);
            else add_rows<T, DP>(dk, lds.rows[0], row0, Weights<T>(ds), lane);
        }
    }

    template <bool DIRECT, bool APART>
    __device__ __forceinline__ void over_rows(const AttentionArgs &a, RowsInLds<T, DP> (&lds)[2], char *room) {
        constexpr int BR = kRowTile<T, DP>, kTileBlocks = BR / 32;
        const int blocks = (a.rows + 31) / 32;
        const char *qbase = reinterpret_cast<const char *>(head_at<const T>(a.q, worker, 0, kvh * a.group));
        const char *obase = reinterpret_cast<const char *>(head_at<const T>(a.dout, worker, 0, kvh * a.group));
        Stage<T, DP, BR, 256, DIRECT> qs, os;
        // A group that divides a tile has its rows at the same places of every one.
        const bool steady = BR % a.group == 0;
        float2 stat = {0.0f, 0.0f};
        int2 range = {0, 0};
        const auto fetch = [&](int block, RowsInLds<T, DP> &to) __attribute__((always_inline)) {
            const int row0 = block * 32, t0 = token_of(a, row0), rows = min(BR, a.rows - row0);
            const auto at = [&](const Heads &x) {
                return [&, rs = x.rs, hs = x.hs](int r) {
                    const int row = row0 + r, t = token_of(a, row);
                    return ((t - t0) * rs + (row - t * a.group) * hs) * (int64_t)sizeof(T);
                };
            };
            // What comes into registers is used only in put().
            if (threadIdx.x < BR) {
                const int row = row0 + threadIdx.x;
                stat = float2{0.0f, 0.0f}, range = int2{0, 0};
                if (row < a.rows) {
                    stat = a.stats[(int64_t)pair * a.rows + row];
                    const int t = token_of(a, row);
                    range = a.ranges ? a.ranges[worker * a.range_stride + t] : seen(a, worker, t);
                }
            }
            if (!steady) {
                qs.places(threadIdx.x, at(a.q));
                os.places(threadIdx.x, at(a.dout));
            }
            qs.load(qbase + t0 * a.q.rs * (int64_t)sizeof(T), to.rows[0], a.width, rows, threadIdx.x, at(a.q));
            os.load(obase + t0 * a.dout.rs * (int64_t)sizeof(T), to.rows[1], a.width, rows, threadIdx.x, at(a.dout));
        };
        const auto put = [&](RowsInLds<T, DP> &to) {
            qs.put(to.rows[0], threadIdx.x);
            os.put(to.rows[1], threadIdx.x);
            if (threadIdx.x < BR) {
                to.stats[0][threadIdx.x] = stat.x - kBackwardShift<T>;
                to.stats[1][threadIdx.x] = stat.y;
                to.sees[threadIdx.x] = int2{max(range.x, 0), max(0, min(range.y, a.keys))};
            }
        };
        if (DIRECT && a.width < DP) {
#pragma unroll
            for (int i = 0; i < 4; ++i) qs.clear(lds[i / 2].rows[i % 2], threadIdx.x);
            __syncthreads();
        }
        // Without ranges the rows that see a key are all from one on.
        int block = 0;
        if (!a.ranges && a.causal)
            block = (int)(max((int64_t)0, (int64_t)j0 + a.tokens - a.keys) * a.group / BR) * kTileBlocks;
        Walk walk{worker, j0, mine, -64, part, 0, 0, 0};
        block = walk.next<kTileBlocks>(a, block, blocks, lane);
        if (block >= blocks) return;
        unsigned any = (unsigned)(walk.any >> (block - walk.base)), whole = (unsigned)(walk.whole >> (block - walk.base));
        if (steady) {
            const auto at = [&](const Heads &x) {
                return [&, rs = x.rs, hs = x.hs](int r) {
                    const int t = token_of(a, r);
                    return (t * rs + (r - t * a.group) * hs) * (int64_t)sizeof(T);
                };
            };
            qs.places(threadIdx.x, at(a.q));
            os.places(threadIdx.x, at(a.dout));
        }
        fetch(block, lds[0]);
        put(lds[0]);
        for (int half = 0; block < blocks; half ^= 1) {
            __syncthreads();
            block = walk.next<kTileBlocks>(a, block + kTileBlocks, blocks, lane);
            if (block < blocks) fetch(block, lds[half ^ 1]);
#pragma unroll
            for (int b = 0; b < kTileBlocks; ++b)
                if (any >> b & 1) step<APART>(a, lds[half], 32 * b, whole >> b & 1, room);
            if (block < blocks) {
                put(lds[half ^ 1]);
                any = (unsigned)(walk.any >> (block - walk.base)), whole = (unsigned)(walk.whole >> (block - walk.base));
            }
        }
    }

    __device__ __forceinline__ void store(const AttentionArgs &a) const {
        if (!valid) return;
        const float fv = ldexpf(1.0f, -(int)kBackwardShift<T>), fk = held.down(a.scale * fv);
        if (a.parts > 1) {
            float *to = a.part_out + (((int64_t)pair * a.keys + key) * a.parts + part) * 2 * a.width;
            if constexpr (kDk) store_column<float>(to, a.width, dk, fk, lane);
            if constexpr (kDv) store_column<float>(to + a.width, a.width, dv, fv, lane);
        } else {
            if constexpr (kDk) store_column<T>(head_at<T>(a.dk, worker, key, kvh), a.width, dk, fk, lane);
            if constexpr (kDv) store_column<T>(head_at<T>(a.dv, worker, key, kvh), a.width, dv, fv, lane);
        }
    }
};

// The key head, tile of keys and part of a workgroup.
struct KeyTile {
    unsigned pair;
    int tile, part;
    __device__ __forceinline__ KeyTile(const AttentionArgs &a, unsigned block) {
        const unsigned at = block / a.parts;
        part = (int)(block % a.parts);
        // The first keys are seen by the most rows, without ranges.
        pair = at % a.pairs;
        tile = (int)(at / a.pairs);
        if (a.order && a.bound_stride) {
            tile = a.order[at / a.kv];
            pair = tile / a.tiles * a.kv + at % a.kv;
            tile %= a.tiles;
        } else if (a.order) {
            tile = a.order[tile];
        }
    }
};

template <typename T, int DP, bool DIRECT, int WHICH>
__global__ __launch_bounds__(256, (kKeyWaves<T, DP>)) void attention_dkv_kernel(AttentionArgs a) {
    __shared__ __align__(16) RowsInLds<T, DP> lds[2];
    __shared__ __align__(16) char own[kValuesInLds<T, DP> ? 128 * Tile<T, DP>::kRowBytes : 16];
    const KeyTile at(a, blockIdx.x);
    KeyGradient<T, DP, WHICH> g;
    g.start(a, at.pair, at.tile, at.part, own);
    g.template over_rows<DIRECT, false>(a, lds, nullptr);
    const bool again = __syncthreads_or(g.valid && ((g.kDk && not_finite(g.dk)) || (g.kDv && not_finite(g.dv))));
    const AttentionArgs &later = later_arguments();
    // What the values' kernel has marked stays so.
    if (threadIdx.x == 0 && (again || WHICH != kOnlyKeys)) later.key_marks[blockIdx.x] = again;
    if (!again) g.store(later);
}

// What the two kernels above have marked.
template <typename T, int DP>
__global__ __launch_bounds__(256) void attention_grad_apart_kernel(AttentionArgs a, int64_t row_blocks, int64_t key_blocks) {
    constexpr int kRowBytes = Tile<T, DP>::kRowBytes;
    __shared__ __align__(16) union {
        char keys[2][2 * kKeyTile<T, DP> * kRowBytes];
        RowsInLds<T, DP> rows[2];
    } lds;
    __shared__ __align__(16) char own[kValuesInLds<T, DP> ? 128 * kRowBytes : 16];
    __shared__ __align__(16) char room[4][kApartBytes<T>];
    __shared__ int most[4][2];
    const int tiles = a.tiles;
    a.tiles = (a.rows + 127) / 128;
    over_marks(a.marks, row_blocks, [&](unsigned block) {
        const RowTile r(a, block, most);
        QueryGradient<T, DP> g;
        g.start(a, r);
        exact_delta<T, DP, false>(a, r, g, lds.keys);
        dq_over_keys<T, DP, false, true>(a, r, g, lds.keys, room[r.wave]);
        g.store(a, r);
    });
    a.tiles = tiles;
    over_marks(a.key_marks, key_blocks, [&](unsigned block) {
        const KeyTile at(a, block);
        const auto one = [&](auto which) {
            KeyGradient<T, DP, decltype(which)::value> g;
            g.start(a, at.pair, at.tile, at.part, own);
            g.template over_rows<false, true>(a, lds.rows, room[threadIdx.x / kWave]);
            g.store(a);
        };
        if constexpr (kOneByOne<T, DP>) {
            one(Int<kOnlyValues>());
            __syncthreads();
            one(Int<kOnlyKeys>());
        } else {
            one(Int<kBoth>());
        }
    });
}

// Adds up the parts of dk and dv, in their order: four entries a thread.
template <typename T>
__global__ __launch_bounds__(256) void attention_dkv_join_kernel(AttentionArgs a, int64_t total) {
    const int per = (2 * a.width + 3) / 4;
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= total * per) return;
    const int64_t row = at / per, pair = row / a.keys, worker = pair / a.kv;
    const int key = (int)(row % a.keys), kvh = (int)(pair % a.kv), k0 = (int)(at % per) * 4;
    const float *from = a.part_out + row * a.parts * 2 * a.width + k0;
    const int left = 2 * a.width - k0;
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int p = 0; p < a.parts; ++p, from += 2 * a.width)
        if (left >= 4) {
            f4_t v;
            __builtin_memcpy(&v, from, sizeof v);
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] += v[i];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] += i < left ? from[i] : 0.0f;
        }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int k = k0 + i;
        if (k < a.width) head_at<T>(a.dk, worker, key, kvh)[k] = (T)sum[i];
        else if (k < 2 * a.width) head_at<T>(a.dv, worker, key, kvh)[k - a.width] = (T)sum[i];
    }
}

// ---- launches ---------------------------------------------------------------------------

template <typename F>
void with_width(int64_t width, F f) {
    if (width <= 64) f(Int<64>());
    else if (width <= 128) f(Int<128>());
    else f(Int<256>());
}

// Whether rows start on 16 bytes and have whole chunks of them, and the places
// of a tile fit 32 bits: of up to 64 rows (2^30 bytes), `heads` heads of each.
bool direct(const Heads &h, int64_t bytes, int64_t width, int64_t heads) {
    const auto whole = [&](int64_t entries) { return entries * bytes % 16 == 0; };
    return (uintptr_t)h.data % 16 == 0 && whole(width) && whole(h.ws) && whole(h.rs) && whole(h.hs) &&
           h.rs * bytes < 1 << 24 && heads * h.hs * bytes < (int64_t)1 << 31;
}

}  // namespace

template <typename T>
void attention::launch_attention(const AttentionArgs &a, const ForwardPlan &p, hipStream_t st) {
    with_width(a.width, [&](auto dp) {
        constexpr int DP = decltype(dp)::value;
        if (p.split) {
            hipLaunchKernelGGL(HIP_KERNEL_NAME(attention_split_kernel<T, DP>), dim3((unsigned)p.blocks),
                               dim3(64 * split_waves(sizeof(T), DP)), 0, st, a);
            return;
        }
        if (direct(a.k, sizeof(T), a.width, 1) && direct(a.v, sizeof(T), a.width, 1))
            hipLaunchKernelGGL(HIP_KERNEL_NAME(attention_kernel<T, DP, true>), dim3((unsigned)p.blocks), dim3(256), 0, st, a);
        else
            hipLaunchKernelGGL(HIP_KERNEL_NAME(attention_kernel<T, DP, false>), dim3((unsigned)p.blocks), dim3(256), 0, st, a);
        hipLaunchKernelGGL(HIP_KERNEL_NAME(attention_apart_kernel<T, DP>), dim3((unsigned)std::min<int64_t>(p.blocks, kApartBlocks)),
                           dim3(256), 0, st, a, p.blocks);
    });
    if (p.parts > 1)
        hipLaunchKernelGGL(attention_join_kernel<T>, dim3((unsigned)((int64_t)a.pairs * a.rows)),
                           dim3(64 * kJoinWaves), 0, st, a);
}

template <typename T>
void attention::launch_attention_backward(AttentionArgs a, int32_t n, hipStream_t st) {
    a.tiles = (int32_t)tiles(a.keys, 128);
    if (a.ranges && a.tokens) {
        const int workers = a.range_stride ? n : 1;
        const int64_t total = workers * tiles(a.rows, 32);
        hipLaunchKernelGGL(HIP_KERNEL_NAME(attention_bounds_kernel<T>), dim3((unsigned)tiles(total, 8)), dim3(256), 0, st, a, total);
        // Not where all run at once.
        if ((int64_t)workers * a.tiles <= kMostOrdered && (int64_t)a.pairs * a.tiles * a.parts > 2 * kCus)
            hipLaunchKernelGGL(attention_order_kernel<T>, dim3(1), dim3(1024), 0, st, a, workers);
        else
            a.order = nullptr;
    } else {
        a.order = nullptr;
    }
    with_width(a.width, [&](auto dp) {
        constexpr int DP = decltype(dp)::value;
        const dim3 keys_grid((unsigned)(a.pairs * tiles(a.keys, 128) * a.parts)), rows_grid((unsigned)(a.pairs * tiles(a.rows, 128)));
        a.tiles = (int32_t)tiles(a.rows, 128);
        if (a.tokens && direct(a.k, sizeof(T), a.width, 1) && direct(a.v, sizeof(T), a.width, 1))
            hipLaunchKernelGGL(HIP_KERNEL_NAME(attention_dq_kernel<T, DP, true>), rows_grid, dim3(256), 0, st, a);
        else if (a.tokens)
            hipLaunchKernelGGL(HIP_KERNEL_NAME(attention_dq_kernel<T, DP, false>), rows_grid, dim3(256), 0, st, a);
        a.tiles = (int32_t)tiles(a.keys, 128);
        const bool whole = direct(a.q, sizeof(T), a.width, a.group) && direct(a.dout, sizeof(T), a.width, a.group);
        const auto keys = [&](auto which) {
            constexpr int kWhich = decltype(which)::value;
            if (whole)
                hipLaunchKernelGGL(HIP_KERNEL_NAME(attention_dkv_kernel<T, DP, true, kWhich>), keys_grid, dim3(256), 0, st, a);
            else
                hipLaunchKernelGGL(HIP_KERNEL_NAME(attention_dkv_kernel<T, DP, false, kWhich>), keys_grid, dim3(256), 0, st, a);
        };
        if constexpr (kOneByOne<T, DP>) {
            if (a.keys) keys(Int<kOnlyValues>()), keys(Int<kOnlyKeys>());
        } else if (a.keys) {
            keys(Int<kBoth>());
        }
        // Without rows or keys everything is 0.
        if (a.tokens && a.keys)
            hipLaunchKernelGGL(HIP_KERNEL_NAME(attention_grad_apart_kernel<T, DP>),
                               dim3(std::min(std::max(rows_grid.x, keys_grid.x), (unsigned)kApartBlocks)), dim3(256), 0, st, a,
                               (int64_t)rows_grid.x, (int64_t)keys_grid.x);
    });
    if (a.parts > 1) {
        const int64_t total = (int64_t)a.pairs * a.keys;
        hipLaunchKernelGGL(attention_dkv_join_kernel<T>, dim3((unsigned)tiles(total * tiles(2 * a.width, 4), 256)), dim3(256), 0,
                           st, a, total);
    }
}
