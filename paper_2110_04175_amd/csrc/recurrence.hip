// A gated linear recurrence over n workers' packed sequences, and its
// gradients, on CDNA4 (gfx950); the C ABI is in relaysum.h.
//
//   h_t = a_t h_(t-1) + c_t x_t,   a = sigmoid(gate), c = 1 - a = sigmoid(-gate)
//   dh_t = dy_t + a_(t+1) dh_(t+1)
//   dgate_t = dh_t (h_(t-1) - x_t) a_t c_t,   dx_t = c_t dh_t
//
// channel by channel.  A run of tokens takes a state s to A s + B; runs compose,
// so a sequence is cut into chunks of 64 tokens and those into a wave's 8.  A
// workgroup has 256 channels of a chunk in registers.
//
// Where a sequence starts (in the gradients: ends) nothing is carried, whatever
// it is: such a run is marked by a negative A (a is not), and no product with
// what came before is formed, which may be an infinity or a NaN.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "layer_call.hpp"

namespace {

constexpr int kChunk = 64;      // tokens of a workgroup
constexpr int kSteps = 8;       // of a wave
constexpr int kChannels = 4;    // of a lane
constexpr int kBlock = kWave * kChannels;
constexpr int kThreads = kChunk / kSteps * kWave;

struct RecurrenceArgs {
    Rows gate, x, h;                   // h: out, or dy
    Rows dgate, dx;
    Rows initial, last;                // [n][count]: initial, dinitial; last, dlast
    Rows dinitial;
    float *saved;                      // [n][chunks][width]: the state before each chunk
    float2 *runs;                      // [n][chunks][width]: A and B of each chunk
    const int32_t *starts;
    int64_t starts_stride;
    int32_t tokens, width, count, chunks, blocks;   // blocks: of channels
};

// Where a wave's tokens lie: lane i has token i's.
struct Places {
    int seq;
    unsigned inside, starts, ends;   // a bit for each token

    __device__ __forceinline__ Places(const RecurrenceArgs &a, int64_t worker, int t0, int lane) {
        const int t = t0 + lane % kSteps;
        bool in = t < a.tokens, first, final;
        if (a.starts) {
            const int32_t *s = a.starts + worker * a.starts_stride;
            int low = 0, high = a.count + 1;
            while (low < high) {
                const int mid = (low + high) / 2;
                if (s[mid] <= t) low = mid + 1;
                else high = mid;
            }
            in = in && low > 0 && low <= a.count;
            seq = in ? low - 1 : 0;
            first = in && s[seq] == t;
            final = in && (s[seq + 1] - 1 == t || t == a.tokens - 1);
        } else {
            seq = 0;
            first = in && t == 0;
            final = in && t == a.tokens - 1;
        }
        constexpr unsigned kMask = (1u << kSteps) - 1;
        inside = (unsigned)__ballot(in) & kMask;
        starts = (unsigned)__ballot(first) & kMask;
        ends = (unsigned)__ballot(final) & kMask;
    }
    __device__ __forceinline__ int sequence(int i) const { return __builtin_amdgcn_readlane(seq, i); }
};

__device__ __forceinline__ bool empty_sequence(const RecurrenceArgs &a, int64_t worker, int s) {
    if (!a.starts) return a.tokens == 0;
    const int32_t *st = a.starts + worker * a.starts_stride;
    return st[s] >= st[s + 1];
}

struct Run {
    float A, B;
    __device__ __forceinline__ float from(float s) const { return A < 0.0f ? B : fmaf(A, s, B); }
};
// First p, then r.
__device__ __forceinline__ Run then(const Run &p, const Run &r) {
    return Run{r.A < 0.0f ? r.A : p.A < 0.0f ? -1.0f : p.A * r.A, r.from(p.B)};
}

template <typename T>
__device__ __forceinline__ void load4(const T *p, int left, float (&v)[4]) {
    typedef T t4 __attribute__((ext_vector_type(4)));
    if (left >= 4) {
        t4 t;
        __builtin_memcpy(&t, p, sizeof t);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (float)t[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < left ? (float)p[i] : 0.0f;
    }
}

template <typename T>
__device__ __forceinline__ void store4(T *p, int left, const float (&v)[4]) {
    typedef T t4 __attribute__((ext_vector_type(4)));
    if (left >= 4) {
        t4 t;
#pragma unroll
        for (int i = 0; i < 4; ++i) t[i] = (T)v[i];
        __builtin_memcpy(p, &t, sizeof t);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) p[i] = (T)v[i];
    }
}

// The waves' runs of a chunk, in LDS: what leads from the chunk's edge to this
// wave, and over the whole chunk.
struct Chunk {
    Run runs[kChunk / kSteps][kBlock];

    template <bool REVERSE>
    __device__ __forceinline__ void join(int wave, int lane, const Run (&own)[4], Run (&before)[4], Run (&all)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            runs[wave][lane * 4 + i] = own[i];
            before[i] = all[i] = Run{1.0f, 0.0f};
        }
        __syncthreads();
        for (int k = 0; k < kChunk / kSteps; ++k) {
            const int w = REVERSE ? kChunk / kSteps - 1 - k : k;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (w == wave) before[i] = all[i];
                all[i] = then(all[i], runs[w][lane * 4 + i]);
            }
        }
    }
};

struct Where {
    int64_t worker;
    int chunk, channel, left, wave, lane, t0;
    __device__ __forceinline__ explicit Where(const RecurrenceArgs &a) {
        const unsigned block = blockIdx.x % a.blocks, at = blockIdx.x / a.blocks;
        worker = at / a.chunks;
        chunk = (int)(at % a.chunks);
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        lane = threadIdx.x % kWave;
        channel = (int)block * kBlock + lane * 4;
        left = a.width - channel;
        t0 = chunk * kChunk + wave * kSteps;
    }
    __device__ __forceinline__ int64_t slot(const RecurrenceArgs &a) const {
        return (worker * a.chunks + chunk) * a.width + channel;
    }
};

// The forward pass.  APART: only the chunk's run is wanted, for the kernel that
// carries states over chunks.
template <typename T, bool APART>
__global__ __launch_bounds__(kThreads) void recurrence_kernel(RecurrenceArgs a) {
    __shared__ Chunk chunk;
    const Where w(a);
    const Places at(a, w.worker, w.t0, w.lane);
    float av[kSteps][4], bv[kSteps][4];
    Run own[4];
    if (w.t0 < a.tokens) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int64_t t = min(w.t0 + s, a.tokens - 1);
            load4(row_at<const T>(a.gate, w.worker, t) + w.channel, w.left, av[s]);
            load4(row_at<const T>(a.x, w.worker, t) + w.channel, w.left, bv[s]);
        }
    } else {
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) av[s][i] = bv[s][i] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) own[i] = Run{1.0f, 0.0f};
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        const bool in = at.inside >> s & 1, first = at.starts >> s & 1;
        float init[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (first && a.initial.data)
            load4(row_at<const float>(a.initial, w.worker, at.sequence(s)) + w.channel, w.left, init);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float c;
            const float x = bv[s][i];
            gates<T>(av[s][i], av[s][i], c);
            bv[s][i] = c * x;
            if (first) bv[s][i] = fmaf(av[s][i], init[i], bv[s][i]);
            // Rows of no sequence leave no state.
            if (!in) bv[s][i] = 0.0f;
            if (first || !in) av[s][i] = -1.0f;
            own[i] = then(own[i], Run{av[s][i], bv[s][i]});
        }
    }
    Run before[4], all[4];
    chunk.join<false>(w.wave, w.lane, own, before, all);
    if (APART) {
        if (w.wave == 0)
            for (int i = 0; i < 4 && i < w.left; ++i) a.runs[w.slot(a) + i] = float2{all[i].A, all[i].B};
        return;
    }
    float h[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (a.chunks > 1) load4(a.saved + w.slot(a), w.left, h);
    else if (a.saved && w.wave == 0) store4(a.saved + w.slot(a), w.left, h);
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = before[i].from(h[i]);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        if (w.t0 + s >= a.tokens) break;
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = Run{av[s][i], bv[s][i]}.from(h[i]);
        store4(row_at<T>(a.h, w.worker, w.t0 + s) + w.channel, w.left, h);
        if (a.last.data && at.ends >> s & 1)
            store4(row_at<float>(a.last, w.worker, at.sequence(s)) + w.channel, w.left, h);
    }
    // Sequences of no token keep their state.
    if (a.last.data)
        for (int s = w.chunk * (kChunk / kSteps) + w.wave; s < a.count; s += a.chunks * (kChunk / kSteps)) {
            if (!empty_sequence(a, w.worker, s)) continue;
            float init[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            if (a.initial.data) load4(row_at<const float>(a.initial, w.worker, s) + w.channel, w.left, init);
            store4(row_at<float>(a.last, w.worker, s) + w.channel, w.left, init);
        }
}

// The backward pass.  Runs go back in time: what a token's state gets from the
// one after it.
template <typename T, bool APART>
__global__ __launch_bounds__(kThreads) void recurrence_grad_kernel(RecurrenceArgs a) {
    __shared__ Chunk chunk;
    const Where w(a);
    const Places at(a, w.worker, w.t0, w.lane);
    float av[kSteps][4], cv[kSteps][4], kv[kSteps][4], dv[kSteps][4];
    Run own[4], before[4], all[4];
    if (w.t0 < a.tokens) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int64_t t = min(w.t0 + s, a.tokens - 1);
            load4(row_at<const T>(a.gate, w.worker, t) + w.channel, w.left, av[s]);
            if (!APART) load4(row_at<const T>(a.x, w.worker, t) + w.channel, w.left, kv[s]);
            load4(row_at<const T>(a.h, w.worker, t) + w.channel, w.left, dv[s]);
        }
    } else {
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) av[s][i] = kv[s][i] = dv[s][i] = 0.0f;
    }
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) gates<T>(av[s][i], av[s][i], cv[s][i]);
    if (!APART) {
        // The states before each token, from the chunk's: kv = (h_(t-1) - x) a c.
#pragma unroll
        for (int i = 0; i < 4; ++i) own[i] = Run{1.0f, 0.0f};
        const auto initial = [&](int s, float (&init)[4]) {
#pragma unroll
            for (int i = 0; i < 4; ++i) init[i] = 0.0f;
            if (at.starts >> s & 1 && a.initial.data)
                load4(row_at<const float>(a.initial, w.worker, at.sequence(s)) + w.channel, w.left, init);
        };
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const bool in = at.inside >> s & 1, first = at.starts >> s & 1;
            float init[4];
            initial(s, init);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float b = cv[s][i] * kv[s][i];
                own[i] = then(own[i], !in     ? Run{-1.0f, 0.0f}
                                      : first ? Run{-1.0f, fmaf(av[s][i], init[i], b)}
                                              : Run{av[s][i], b});
            }
        }
        chunk.join<false>(w.wave, w.lane, own, before, all);
        __syncthreads();
        float h[4];
        load4(a.saved + w.slot(a), w.left, h);
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = before[i].from(h[i]);
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const bool in = at.inside >> s & 1, first = at.starts >> s & 1;
            float init[4];
            initial(s, init);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float prior = first ? init[i] : h[i], x = kv[s][i];
                h[i] = in ? fmaf(av[s][i], prior, cv[s][i] * x) : 0.0f;
                kv[s][i] = (prior - x) * (av[s][i] * cv[s][i]);
            }
        }
    }
    // From the last token to the first: g is what comes from behind.
#pragma unroll
    for (int i = 0; i < 4; ++i) own[i] = Run{1.0f, 0.0f};
#pragma unroll
    for (int s = kSteps - 1; s >= 0; --s) {
        const bool in = at.inside >> s & 1, first = at.starts >> s & 1, final = at.ends >> s & 1;
        float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (final && a.last.data)
            load4(row_at<const float>(a.last, w.worker, at.sequence(s)) + w.channel, w.left, d);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            // g -> a (dy + g), from a sequence's last token on from dlast alone; what
            // passes its first one is its initial state's.
            if (final) own[i] = Run{-1.0f, d[i]};
            own[i] = !in ? Run{-1.0f, 0.0f} : then(own[i], Run{av[s][i], av[s][i] * dv[s][i]});
            if (first) own[i] = Run{-1.0f, 0.0f};
        }
    }
    chunk.join<true>(w.wave, w.lane, own, before, all);
    if (APART) {
        if (w.wave == 0)
            for (int i = 0; i < 4 && i < w.left; ++i) a.runs[w.slot(a) + i] = float2{all[i].A, all[i].B};
        return;
    }
    float g[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    // The carrying kernel left in A what comes into the chunk.
    if (a.chunks > 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < w.left) g[i] = a.runs[w.slot(a) + i].x;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) g[i] = before[i].from(g[i]);
#pragma unroll
    for (int s = kSteps - 1; s >= 0; --s) {
        if (w.t0 + s >= a.tokens) continue;
        const bool in = at.inside >> s & 1, first = at.starts >> s & 1, final = at.ends >> s & 1;
        if (final) {
#pragma unroll
            for (int i = 0; i < 4; ++i) g[i] = 0.0f;
            if (a.last.data) load4(row_at<const float>(a.last, w.worker, at.sequence(s)) + w.channel, w.left, g);
        }
        float dgate[4], dx[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float dh = dv[s][i] + g[i];
            dgate[i] = in ? dh * kv[s][i] : 0.0f;
            dx[i] = in ? dh * cv[s][i] : 0.0f;
            g[i] = in ? dh * av[s][i] : 0.0f;
        }
        store4(row_at<T>(a.dgate, w.worker, w.t0 + s) + w.channel, w.left, dgate);
        store4(row_at<T>(a.dx, w.worker, w.t0 + s) + w.channel, w.left, dx);
        if (first) {
            if (a.dinitial.data) store4(row_at<float>(a.dinitial, w.worker, at.sequence(s)) + w.channel, w.left, g);
#pragma unroll
            for (int i = 0; i < 4; ++i) g[i] = 0.0f;
        }
    }
    if (a.dinitial.data)
        for (int s = w.chunk * (kChunk / kSteps) + w.wave; s < a.count; s += a.chunks * (kChunk / kSteps)) {
            if (!empty_sequence(a, w.worker, s)) continue;
            float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            if (a.last.data) load4(row_at<const float>(a.last, w.worker, s) + w.channel, w.left, d);
            store4(row_at<float>(a.dinitial, w.worker, s) + w.channel, w.left, d);
        }
}

// Carries states over the chunks of a channel.  A workgroup has 16 channels and
// 16 stretches of chunks: each stretch's run, then the states.
template <bool REVERSE>
__global__ __launch_bounds__(256) void carry_kernel(RecurrenceArgs a) {
    __shared__ Run runs[16][16];
    const unsigned blocks = (a.width + 15) / 16;
    const int64_t worker = blockIdx.x / blocks;
    const int c = (int)(blockIdx.x % blocks) * 16 + threadIdx.x % 16, part = threadIdx.x / 16;
    const int per = (a.chunks + 15) / 16, from = min(part * per, a.chunks), to = min(from + per, a.chunks);
    const auto at = [&](int k) {
        return (worker * a.chunks + (REVERSE ? a.chunks - 1 - k : k)) * a.width + c;
    };
    Run r{1.0f, 0.0f};
    if (c < a.width)
#pragma unroll 8
        for (int k = from; k < to; ++k) {
            const float2 v = a.runs[at(k)];
            r = then(r, Run{v.x, v.y});
        }
    runs[part][threadIdx.x % 16] = r;
    __syncthreads();
    if (c >= a.width) return;
    float s = 0.0f;
    for (int k = 0; k < part; ++k) s = runs[k][threadIdx.x % 16].from(s);
#pragma unroll 8
    for (int k = from; k < to; ++k) {
        const float2 v = a.runs[at(k)];
        if (REVERSE) a.runs[at(k)].x = s;
        else a.saved[at(k)] = s;
        s = Run{v.x, v.y}.from(s);
    }
}

// ---- host side -------------------------------------------------------------------------

constexpr int64_t kMaxTokens = 1 << 30;

int64_t chunks_of(int64_t tokens) { return tiles(tokens, kChunk); }

struct RecurrenceCall : Call {
    bool shape(int32_t n, int64_t tokens, int64_t width, int32_t count) {
        if (!sizes(n, tokens, width, "tokens")) return false;
        if (tokens > kMaxTokens) fail(refuse("tokens must be in 0..2^30"));
        else if (count < 1 || count > 1 << 30) fail(refuse("count must be in 1..2^30"));
        else if ((__int128)n * count * width > ((__int128)1 << 50)) fail(refuse("n * count * width is more than 2^50"));
        else if (n * chunks_of(tokens) * tiles(width, kBlock) > kMaxBlocks || n * tiles(width, 16) > kMaxBlocks)
            fail(refuse("n * tokens * width is too large for a launch"));
        return code == RELAYSUM_OK;
    }

    void sequences(const int32_t *starts, int64_t stride, int32_t n, int32_t count) {
        if (code != RELAYSUM_OK) return;
        if (!starts) {
            if (count != 1) fail(refuse("without starts there is one sequence"));
            return;
        }
        if (n == 1) stride = 0;
        if (stride < 0 || stride > ((int64_t)1 << 40) / n)
            return fail(refuse("starts_stride is negative or reaches past 2^40 entries"));
        span("starts", starts, (size_t)((n - 1) * stride + count + 1) * 4, 4, false);
    }

    void states(const char *name, const relaysum_rows *r, int32_t n, int32_t count, int64_t width, bool out) {
        if (code != RELAYSUM_OK || !r) return;
        rows(name, r, n, count, width, out);
        if (code == RELAYSUM_OK && r->type != RELAYSUM_FLOAT) fail(refuse("%s must be of type float", name));
    }
};

template <typename F>
void with_grid(const RecurrenceArgs &a, int32_t n, F f) {
    f(dim3((unsigned)(n * (int64_t)a.chunks * a.blocks)), dim3(kThreads), dim3((unsigned)(n * ((a.width + 15) / 16))));
}

}  // namespace

extern "C" {

int64_t relaysum_recurrence_chunks(int64_t tokens) {
    return tokens < 0 || tokens > kMaxTokens ? -1 : std::max<int64_t>(1, chunks_of(tokens));
}

int64_t relaysum_recurrence_workspace(int32_t n, int64_t tokens, int64_t width) {
    RecurrenceCall c;
    if (!c.shape(n, tokens, width, 1)) return -1;
    g_error[0] = '\0';
    const int64_t chunks = chunks_of(tokens);
    return chunks > 1 ? n * chunks * width * 12 : 0;
}

int relaysum_recurrence(int32_t n, int64_t tokens, int64_t width, int32_t count, const int32_t *starts,
                        int64_t starts_stride, const relaysum_rows *gate, const relaysum_rows *x,
                        const relaysum_rows *initial, const relaysum_rows *h, const relaysum_rows *last,
                        float *saved, void *workspace, size_t workspace_bytes, void *hip_stream) {
    RecurrenceCall c;
    const int64_t chunks = std::max<int64_t>(1, chunks_of(tokens));
    if (c.shape(n, tokens, width, count)) {
        c.rows("gate", gate, n, tokens, width, false);
        c.rows("x", x, n, tokens, width, false);
        c.rows("h", h, n, tokens, width, true);
        if (c.code == RELAYSUM_OK && (gate->type != x->type || gate->type != h->type))
            c.fail(refuse("gate, x and h must have one type"));
        c.sequences(starts, starts_stride, n, count);
        c.states("initial", initial, n, count, width, false);
        c.states("last", last, n, count, width, true);
        if (saved) c.span("saved", saved, (size_t)n * chunks * width * 4, 4, true);
        const size_t need = chunks > 1 ? (size_t)n * chunks * width * 12 : 0;
        if (need > workspace_bytes)
            c.fail(refuse("the workspace has %zu bytes, %zu are needed", workspace_bytes, need));
        c.span("workspace", workspace, need, 8, true);
    }
    if (!c.ready()) return c.code;
    RecurrenceArgs a{};
    a.gate = rows_of(gate, n, tokens), a.x = rows_of(x, n, tokens), a.h = rows_of(h, n, tokens);
    a.initial = rows_of(initial, n, count), a.last = rows_of(last, n, count);
    a.runs = static_cast<float2 *>(workspace);
    a.saved = saved || chunks == 1 ? saved : reinterpret_cast<float *>(a.runs + n * chunks * width);
    a.starts = starts, a.starts_stride = n > 1 ? starts_stride : 0;
    a.tokens = (int32_t)tokens, a.width = (int32_t)width, a.count = count;
    a.chunks = (int32_t)chunks, a.blocks = (int32_t)tiles(width, kBlock);
    const hipStream_t st = (hipStream_t)hip_stream;
    with_type(gate->type, [&](auto zero) {
        using T = decltype(zero);
        with_grid(a, n, [&](dim3 grid, dim3 block, dim3 carry) {
            if (chunks > 1) {
                hipLaunchKernelGGL(HIP_KERNEL_NAME(recurrence_kernel<T, true>), grid, block, 0, st, a);
                hipLaunchKernelGGL(HIP_KERNEL_NAME(carry_kernel<false>), carry, dim3(256), 0, st, a);
            }
            hipLaunchKernelGGL(HIP_KERNEL_NAME(recurrence_kernel<T, false>), grid, block, 0, st, a);
        });
    });
    return done("relaysum_recurrence");
}

int relaysum_recurrence_backward(int32_t n, int64_t tokens, int64_t width, int32_t count, const int32_t *starts,
                                 int64_t starts_stride, const relaysum_rows *dh, const relaysum_rows *dlast,
                                 const relaysum_rows *gate, const relaysum_rows *x, const relaysum_rows *initial,
                                 const float *saved, const relaysum_rows *dgate, const relaysum_rows *dx,
                                 const relaysum_rows *dinitial, void *workspace, size_t workspace_bytes,
                                 void *hip_stream) {
    RecurrenceCall c;
    const int64_t chunks = std::max<int64_t>(1, chunks_of(tokens));
    if (c.shape(n, tokens, width, count)) {
        c.rows("dh", dh, n, tokens, width, false);
        c.rows("gate", gate, n, tokens, width, false);
        c.rows("x", x, n, tokens, width, false);
        c.rows("dgate", dgate, n, tokens, width, true);
        c.rows("dx", dx, n, tokens, width, true);
        if (c.code == RELAYSUM_OK && (gate->type != x->type || gate->type != dh->type || gate->type != dgate->type ||
                                      gate->type != dx->type))
            c.fail(refuse("dh, gate, x, dgate and dx must have one type"));
        c.sequences(starts, starts_stride, n, count);
        c.states("initial", initial, n, count, width, false);
        c.states("dlast", dlast, n, count, width, false);
        c.states("dinitial", dinitial, n, count, width, true);
        c.span("saved", saved, (size_t)n * chunks * width * 4, 4, false);
        const size_t need = chunks > 1 ? (size_t)n * chunks * width * 8 : 0;
        if (need > workspace_bytes)
            c.fail(refuse("the workspace has %zu bytes, %zu are needed", workspace_bytes, need));
        c.span("workspace", workspace, need, 8, true);
    }
    if (!c.ready()) return c.code;
    RecurrenceArgs a{};
    a.gate = rows_of(gate, n, tokens), a.x = rows_of(x, n, tokens), a.h = rows_of(dh, n, tokens);
    a.dgate = rows_of(dgate, n, tokens), a.dx = rows_of(dx, n, tokens);
    a.initial = rows_of(initial, n, count), a.last = rows_of(dlast, n, count), a.dinitial = rows_of(dinitial, n, count);
    a.runs = static_cast<float2 *>(workspace);
    a.saved = const_cast<float *>(saved);
    a.starts = starts, a.starts_stride = n > 1 ? starts_stride : 0;
    a.tokens = (int32_t)tokens, a.width = (int32_t)width, a.count = count;
    a.chunks = (int32_t)chunks, a.blocks = (int32_t)tiles(width, kBlock);
    const hipStream_t st = (hipStream_t)hip_stream;
    with_type(gate->type, [&](auto zero) {
        using T = decltype(zero);
        with_grid(a, n, [&](dim3 grid, dim3 block, dim3 carry) {
            if (chunks > 1) {
                hipLaunchKernelGGL(HIP_KERNEL_NAME(recurrence_grad_kernel<T, true>), grid, block, 0, st, a);
                hipLaunchKernelGGL(HIP_KERNEL_NAME(carry_kernel<true>), carry, dim3(256), 0, st, a);
            }
            hipLaunchKernelGGL(HIP_KERNEL_NAME(recurrence_grad_kernel<T, false>), grid, block, 0, st, a);
        });
    });
    return done("relaysum_recurrence_backward");
}

}  // extern "C"
