// A gated linear recurrence over n workers' packed sequences, and its
// gradients, on CDNA4 (gfx950); the C ABI is in relaysum.h.
//
//   h_t = a_t h_(t-1) + c_t x_t,   a = sigmoid(gate), c = 1 - a = sigmoid(-gate)
//   dh_t = dy_t + a_(t+1) dh_(t+1)
//   dgate_t = dh_t (h_(t-1) - x_t) a_t c_t,   dx_t = c_t dh_t
//
// channel by channel.  A run of tokens takes a state s to A s + B, and runs
// compose.  A workgroup has 64 channels, one for each lane, and walks through its
// tokens in tiles of 128: each of its 16 waves has 8 of them in registers, the
// waves' runs go through LDS, and the next tile is on its way meanwhile.  So gate
// and x are read once.  Where there are too few channels for the device, tokens
// are split into parts: a first kernel finds the run of each part, and every
// workgroup begins with those that lead to its own.
//
// Where a sequence starts (in the gradients: ends) nothing is carried, whatever
// it is: such a run is marked by a negative A (a is not), and no product with
// what came before is formed, which may be an infinity or a NaN.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cstdint>
#include <type_traits>

#include "layer_call.hpp"

namespace {

constexpr int kChunk = 64;      // tokens between the states that are kept
constexpr int kSteps = 8;      // tokens of a wave in a tile
constexpr int kWaves = 16;
constexpr int kTile = kSteps * kWaves;
constexpr int kThreads = kWaves * kWave;

struct RecurrenceArgs {
    Rows gate, x, h;                   // h: out, or dy
    Rows dgate, dx;
    Rows initial, last;                // [n][count]: initial, dinitial; last, dlast
    Rows dinitial;
    float *saved;                      // [n][chunks][width]: the state before each chunk
    float2 *runs;                      // [n][parts][width]: A and B of each part
    const int32_t *starts;
    int64_t starts_stride;
    int32_t tokens, width, count, chunks, blocks;   // blocks: of channels
    int32_t tiles, parts, per;                      // of tokens; tiles of a part
};

// Where a wave's tokens lie.  `plain`: all within one sequence that neither
// starts nor ends at them.
struct Places {
    bool plain;
    int seq;                         // lane i: the sequence of token i
    unsigned inside, starts, ends;   // a bit for each token
    __device__ __forceinline__ int sequence(int i) const { return __builtin_amdgcn_readlane(seq, i); }
};

// A worker's starts, one for each lane where they are no more than that.
struct Starts {
    const int32_t *at;
    int count, tokens, lane, own;
    bool few;

    __device__ __forceinline__ Starts(const RecurrenceArgs &a, int64_t worker, int l) {
        at = a.starts ? a.starts + worker * a.starts_stride : nullptr;
        count = a.count, tokens = a.tokens, lane = l;
        few = count < kWave;
        own = INT_MAX;
        if (!at) own = lane == 0 ? 0 : lane == 1 ? tokens : INT_MAX;
        else if (few && lane <= count) own = at[lane];
    }
    // How many start at or before token t.
    __device__ __forceinline__ int upto(int t) const { return __popcll(__ballot(own <= t)); }

    __device__ __forceinline__ Places places(int t0) const {
        Places p{false, 0, 0, 0, 0};
        if (few) {
            int c = upto(t0 - 1), next = upto(t0);
            if (next > 0 && next <= count && t0 + kSteps < tokens && !__ballot(own >= t0 && own <= t0 + kSteps)) {
                p.plain = true;
                return p;
            }
#pragma unroll 1
            for (int i = 0; i < kSteps; ++i) {
                const int t = t0 + i, before = c;
                c = next;
                next = upto(t + 1);
                if (t >= tokens || c == 0 || c > count) continue;
                p.inside |= 1u << i;
                p.starts |= (unsigned)(c > before) << i;
                p.ends |= (unsigned)(next > c || t == tokens - 1) << i;
                p.seq = lane == i ? c - 1 : p.seq;
            }
            return p;
        }
        const int t = t0 + lane % kSteps;
        int low = 0, high = count + 1;
        while (low < high) {
            const int mid = (low + high) / 2;
            if (at[mid] <= t) low = mid + 1;
            else high = mid;
        }
        const bool in = t < tokens && low > 0 && low <= count;
        p.seq = in ? low - 1 : 0;
        const bool first = in && at[p.seq] == t;
        const bool final = in && (at[p.seq + 1] - 1 == t || t == tokens - 1);
        constexpr unsigned kMask = (1u << kSteps) - 1;
        p.inside = (unsigned)__ballot(in) & kMask;
        p.starts = (unsigned)__ballot(first) & kMask;
        p.ends = (unsigned)__ballot(final) & kMask;
        p.plain = p.inside == kMask && !p.starts && !p.ends;
        return p;
    }
    __device__ __forceinline__ bool empty(int s) const {
        return at ? at[s] >= at[s + 1] : tokens == 0;
    }
};

struct Run {
    float A, B;
    __device__ __forceinline__ float from(float s) const { return A < 0.0f ? B : fmaf(A, s, B); }
};
// First p, then r.
__device__ __forceinline__ Run then(const Run &p, const Run &r) {
    return Run{r.A < 0.0f ? r.A : p.A < 0.0f ? -1.0f : p.A * r.A, r.from(p.B)};
}

// A workgroup's channels and tokens; `channel` is in range for every lane, and
// `live` says whether it is the lane's own.
struct Where {
    int64_t worker;
    int part, wave, lane, channel;
    bool live;
    __device__ __forceinline__ explicit Where(const RecurrenceArgs &a) {
        const unsigned block = blockIdx.x % a.blocks, at = blockIdx.x / a.blocks;
        worker = at / a.parts;
        part = (int)(at % a.parts);
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        lane = threadIdx.x % kWave;
        channel = (int)block * kWave + lane;
        live = channel < a.width;
        channel = min(channel, a.width - 1);
    }
    template <typename T>
    __device__ __forceinline__ float get(const Rows &r, int64_t row) const { return (float)row_at<const T>(r, worker, row)[channel]; }
    __device__ __forceinline__ float state(const Rows &r, int64_t s) const { return r.data ? get<float>(r, s) : 0.0f; }
    template <typename T>
    __device__ __forceinline__ void put(const Rows &r, int64_t row, float v) const {
        if (live) row_at<T>(r, worker, row)[channel] = (T)v;
    }
};

// A lane's entries of the tokens from t0 on; those behind the last repeat it.
template <typename T>
__device__ __forceinline__ void load_steps(const RecurrenceArgs &a, const Where &w, const Rows &r, int t0, T (&v)[kSteps]) {
    const T *p = row_at<const T>(r, w.worker, min(t0, a.tokens - 1));
    if (t0 + kSteps <= a.tokens) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i, p += r.rs) v[i] = p[w.channel];
        return;
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        v[i] = p[w.channel];
        if (t0 + i + 1 < a.tokens) p += r.rs;
    }
}

// The run of a wave's tokens.  av and bv are its a and c x; states of zero where
// the tokens are in no sequence.
__device__ __forceinline__ Run run_of(const RecurrenceArgs &a, const Where &w, const Places &at, float (&av)[kSteps],
                                      float (&bv)[kSteps]) {
    Run own{1.0f, 0.0f};
    if (!at.plain) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const bool in = at.inside >> i & 1, first = at.starts >> i & 1;
            if (first) bv[i] = fmaf(av[i], w.state(a.initial, at.sequence(i)), bv[i]);
            if (!in) bv[i] = 0.0f;
            if (first || !in) av[i] = -1.0f;
            own = then(own, Run{av[i], bv[i]});
        }
        return own;
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        own.A *= av[i];
        own.B = fmaf(av[i], own.B, bv[i]);
    }
    return own;
}

// The state before a part, from the runs of those that lead to it.
template <bool REVERSE>
__device__ __forceinline__ float state_before(const RecurrenceArgs &a, const Where &w) {
    float s = 0.0f;
    const int many = REVERSE ? a.parts - 1 - w.part : w.part;
#pragma unroll 8
    for (int k = 0; k < many; ++k) {
        const float2 v = a.runs[(w.worker * a.parts + (REVERSE ? a.parts - 1 - k : k)) * a.width + w.channel];
        s = Run{v.x, v.y}.from(s);
    }
    return s;
}

// The run of a part: each wave's of its own stretch, then all of them.
template <typename T, bool REVERSE>
__global__ __launch_bounds__(kThreads) void recurrence_part_kernel(RecurrenceArgs a) {
    __shared__ Run runs[kWaves][kWave];
    const Where w(a);
    // Nothing follows the last part.
    if (w.part == (REVERSE ? 0 : a.parts - 1)) return;
    const Starts starts(a, w.worker, w.lane);
    Run all{1.0f, 0.0f};
    const int turn = REVERSE ? kWaves - 1 - w.wave : w.wave;
#pragma unroll 1
    for (int k = 0; k < a.per; ++k) {
        const int t0 = (w.part * a.per * kWaves + w.wave * a.per + (REVERSE ? a.per - 1 - k : k)) * kSteps;
        if (t0 >= a.tokens) continue;
        T graw[kSteps], xraw[kSteps];
        load_steps(a, w, a.gate, t0, graw);
        load_steps(a, w, REVERSE ? a.h : a.x, t0, xraw);
        const Places at = starts.places(t0);
        float av[kSteps], bv[kSteps];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            float c;
            gates((float)graw[i], av[i], c);
            bv[i] = REVERSE ? (float)xraw[i] : c * (float)xraw[i];
        }
        if (!REVERSE) {
            all = then(all, run_of(a, w, at, av, bv));
        } else if (at.plain) {
            float product = 1.0f;
#pragma unroll
            for (int i = kSteps - 1; i >= 0; --i) {
                all.B = av[i] * (all.B + bv[i]);
                product *= av[i];
            }
            all.A = all.A < 0.0f ? all.A : all.A * product;
        } else {
#pragma unroll
            for (int i = kSteps - 1; i >= 0; --i) {
                const bool in = at.inside >> i & 1, first = at.starts >> i & 1, final = at.ends >> i & 1;
                if (final) all = Run{-1.0f, w.state(a.last, at.sequence(i))};
                all = !in ? Run{-1.0f, 0.0f} : then(all, Run{av[i], av[i] * bv[i]});
                if (first) all = Run{-1.0f, 0.0f};
            }
        }
    }
    runs[turn][w.lane] = all;
    __syncthreads();
    if (w.wave) return;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) all = k ? then(all, runs[k][w.lane]) : runs[0][w.lane];
    if (w.live) a.runs[(w.worker * a.parts + w.part) * a.width + w.channel] = float2{all.A, all.B};
}

// The forward pass.
template <typename T>
__global__ __launch_bounds__(kThreads, 4) void recurrence_kernel(RecurrenceArgs a) {
    __shared__ Run runs[2][kWaves][kWave];
    const Where w(a);
    const Starts starts(a, w.worker, w.lane);
    const int first = w.part * a.per, end = min(first + a.per, a.tiles);
    T graw[kSteps], xraw[kSteps];
    if (first < end) {
        load_steps(a, w, a.gate, first * kTile + w.wave * kSteps, graw);
        load_steps(a, w, a.x, first * kTile + w.wave * kSteps, xraw);
    }
    float carry = state_before<false>(a, w);
#pragma unroll 1
    for (int tile = first; tile < end; ++tile) {
        const int t0 = tile * kTile + w.wave * kSteps;
        const Places at = starts.places(t0);
        float av[kSteps], bv[kSteps];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            float c;
            gates((float)graw[i], av[i], c);
            bv[i] = c * (float)xraw[i];
        }
        if (tile + 1 < end) {
            load_steps(a, w, a.gate, t0 + kTile, graw);
            load_steps(a, w, a.x, t0 + kTile, xraw);
        }
        runs[tile & 1][w.wave][w.lane] = run_of(a, w, at, av, bv);
        __syncthreads();
        float h = 0.0f;
#pragma unroll
        for (int k = 0; k < kWaves; ++k) {
            if (k == w.wave) h = carry;
            carry = runs[tile & 1][k][w.lane].from(carry);
        }
        if (t0 >= a.tokens) continue;
        if (a.saved && t0 % kChunk == 0 && w.live) a.saved[(w.worker * a.chunks + t0 / kChunk) * a.width + w.channel] = h;
        if (at.plain) {
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                h = fmaf(av[i], h, bv[i]);
                w.put<T>(a.h, t0 + i, h);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                if (t0 + i >= a.tokens) break;
                h = Run{av[i], bv[i]}.from(h);
                w.put<T>(a.h, t0 + i, h);
                if (a.last.data && at.ends >> i & 1) w.put<float>(a.last, at.sequence(i), h);
            }
        }
    }
    if (a.tiles == 0 && a.saved && w.wave == 0 && w.live) a.saved[w.worker * a.chunks * a.width + w.channel] = 0.0f;
    // Sequences of no token keep their state.
    if (a.last.data)
        for (int s = w.part * kWaves + w.wave; s < a.count; s += a.parts * kWaves)
            if (starts.empty(s)) w.put<float>(a.last, s, w.state(a.initial, s));
}

// The backward pass, tile by tile from the last one on.
template <typename T>
__global__ __launch_bounds__(kThreads, 4) void recurrence_grad_kernel(RecurrenceArgs a) {
    __shared__ Run runs_ahead[2][kWaves][kWave], runs_back[2][kWaves][kWave];
    const Where w(a);
    const Starts starts(a, w.worker, w.lane);
    const int first = w.part * a.per, end = min(first + a.per, a.tiles);
    T graw[kSteps], xraw[kSteps], draw[kSteps];
    float sraw = 0.0f;
    const auto load = [&](int t0) {
        load_steps(a, w, a.gate, t0, graw);
        load_steps(a, w, a.x, t0, xraw);
        load_steps(a, w, a.h, t0, draw);
        sraw = a.saved[(w.worker * a.chunks + min(t0 / kChunk, a.chunks - 1)) * a.width + w.channel];
    };
    if (first < end) load((end - 1) * kTile + w.wave * kSteps);
    float carry = state_before<true>(a, w);
#pragma unroll 1
    for (int tile = end - 1; tile >= first; --tile) {
        const int t0 = tile * kTile + w.wave * kSteps;
        const Places at = starts.places(t0);
        float av[kSteps], cv[kSteps], xv[kSteps], dv[kSteps], h = sraw;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            gates((float)graw[i], av[i], cv[i]);
            xv[i] = (float)xraw[i], dv[i] = (float)draw[i];
        }
        if (tile > first) load(t0 - kTile);
        Run ahead{1.0f, 0.0f}, back{1.0f, 0.0f};
        if (at.plain) {
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                ahead.A *= av[i];
                ahead.B = fmaf(av[i], ahead.B, cv[i] * xv[i]);
            }
#pragma unroll
            for (int i = kSteps - 1; i >= 0; --i) back.B = av[i] * (back.B + dv[i]);
            back.A = ahead.A;
        } else {
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const bool in = at.inside >> i & 1, start = at.starts >> i & 1;
                float b = cv[i] * xv[i];
                if (start) b = fmaf(av[i], w.state(a.initial, at.sequence(i)), b);
                ahead = then(ahead, !in ? Run{-1.0f, 0.0f} : Run{start ? -1.0f : av[i], b});
            }
#pragma unroll
            for (int i = kSteps - 1; i >= 0; --i) {
                const bool in = at.inside >> i & 1, start = at.starts >> i & 1, final = at.ends >> i & 1;
                // g -> a (dy + g), from a sequence's last token on from dlast alone; what
                // passes its first one is its initial state's.
                if (final) back = Run{-1.0f, w.state(a.last, at.sequence(i))};
                back = !in ? Run{-1.0f, 0.0f} : then(back, Run{av[i], av[i] * dv[i]});
                if (start) back = Run{-1.0f, 0.0f};
            }
        }
        runs_ahead[tile & 1][w.wave][w.lane] = ahead;
        runs_back[tile & 1][w.wave][w.lane] = back;
        __syncthreads();
        for (int k = w.wave & ~(kChunk / kSteps - 1); k < w.wave; ++k) h = runs_ahead[tile & 1][k][w.lane].from(h);
        float g = 0.0f;
#pragma unroll
        for (int k = kWaves - 1; k >= 0; --k) {
            if (k == w.wave) g = carry;
            carry = runs_back[tile & 1][k][w.lane].from(carry);
        }
        if (t0 >= a.tokens) continue;
        if (at.plain) {
            // xv: what dh is times in dgate.
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const float x = xv[i];
                xv[i] = (h - x) * (av[i] * cv[i]);
                h = fmaf(av[i], h, cv[i] * x);
            }
#pragma unroll
            for (int i = kSteps - 1; i >= 0; --i) {
                const float dh = dv[i] + g;
                w.put<T>(a.dgate, t0 + i, dh * xv[i]);
                w.put<T>(a.dx, t0 + i, dh * cv[i]);
                g = dh * av[i];
            }
            continue;
        }
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const bool in = at.inside >> i & 1, start = at.starts >> i & 1;
            const float prior = start ? w.state(a.initial, at.sequence(i)) : h, x = xv[i];
            h = in ? fmaf(av[i], prior, cv[i] * x) : 0.0f;
            xv[i] = (prior - x) * (av[i] * cv[i]);
        }
#pragma unroll
        for (int i = kSteps - 1; i >= 0; --i) {
            if (t0 + i >= a.tokens) continue;
            const bool in = at.inside >> i & 1, start = at.starts >> i & 1, final = at.ends >> i & 1;
            if (final) g = w.state(a.last, at.sequence(i));
            const float dh = dv[i] + g;
            w.put<T>(a.dgate, t0 + i, in ? dh * xv[i] : 0.0f);
            w.put<T>(a.dx, t0 + i, in ? dh * cv[i] : 0.0f);
            g = in ? dh * av[i] : 0.0f;
            if (start) {
                if (a.dinitial.data) w.put<float>(a.dinitial, at.sequence(i), g);
                g = 0.0f;
            }
        }
    }
    if (a.dinitial.data)
        for (int s = w.part * kWaves + w.wave; s < a.count; s += a.parts * kWaves)
            if (starts.empty(s)) w.put<float>(a.dinitial, s, w.state(a.last, s));
}

// ---- host side -------------------------------------------------------------------------

constexpr int64_t kMaxTokens = 1 << 30;

int64_t chunks_of(int64_t tokens) { return tiles(tokens, kChunk); }

// Parts of the tokens, and tiles of each.  Two workgroups for a CU; three
// quarters of them will do where that needs no parts, which read gate and x twice.
struct RecurrencePlan {
    int32_t tiles, parts, per;
    size_t workspace;
    RecurrencePlan(int32_t n, int64_t tokens, int64_t width) {
        const int64_t blocks = n * layer_plan::tiles(width, kWave);
        tiles = (int32_t)layer_plan::tiles(tokens, kTile);
        const int64_t want = blocks >= kCus * 3 / 4 ? 1 : std::min<int64_t>(layer_plan::tiles(2 * kCus, blocks), tiles / 2);
        per = (int32_t)layer_plan::tiles(std::max(tiles, 1), std::max<int64_t>(want, 1));
        parts = (int32_t)layer_plan::tiles(std::max(tiles, 1), per);
        workspace = parts > 1 ? (size_t)n * parts * width * 8 : 0;
    }
};

struct RecurrenceCall : Call {
    bool shape(int32_t n, int64_t tokens, int64_t width, int32_t count) {
        if (!sizes(n, tokens, width, "tokens")) return false;
        if (tokens > kMaxTokens) fail(refuse("tokens must be in 0..2^30"));
        else if (count < 1 || count > 1 << 30) fail(refuse("count must be in 1..2^30"));
        else if ((__int128)n * count * width > ((__int128)1 << 50)) fail(refuse("n * count * width is more than 2^50"));
        else if (n * tiles(width, kWave) > kMaxBlocks)
            fail(refuse("n * width is too large for a launch"));
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

}  // namespace

extern "C" {

int64_t relaysum_recurrence_chunks(int64_t tokens) {
    return tokens < 0 || tokens > kMaxTokens ? -1 : std::max<int64_t>(1, chunks_of(tokens));
}

int64_t relaysum_recurrence_workspace(int32_t n, int64_t tokens, int64_t width) {
    RecurrenceCall c;
    if (!c.shape(n, tokens, width, 1)) return -1;
    g_error[0] = '\0';
    return (int64_t)RecurrencePlan(n, tokens, width).workspace;
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
        const size_t need = RecurrencePlan(n, tokens, width).workspace;
        if (need > workspace_bytes)
            c.fail(refuse("the workspace has %zu bytes, %zu are needed", workspace_bytes, need));
        c.span("workspace", workspace, need, 8, true);
    }
    if (!c.ready()) return c.code;
    RecurrenceArgs a{};
    a.gate = rows_of(gate, n, tokens), a.x = rows_of(x, n, tokens), a.h = rows_of(h, n, tokens);
    a.initial = rows_of(initial, n, count), a.last = rows_of(last, n, count);
    a.runs = static_cast<float2 *>(workspace);
    a.saved = saved;
    a.starts = starts, a.starts_stride = n > 1 ? starts_stride : 0;
    a.tokens = (int32_t)tokens, a.width = (int32_t)width, a.count = count;
    a.chunks = (int32_t)chunks, a.blocks = (int32_t)tiles(width, kWave);
    const RecurrencePlan p(n, tokens, width);
    a.tiles = p.tiles, a.parts = p.parts, a.per = p.per;
    const dim3 grid((unsigned)((int64_t)n * a.blocks * a.parts)), block(kThreads);
    const hipStream_t st = (hipStream_t)hip_stream;
    with_type(gate->type, [&](auto zero) {
        using T = decltype(zero);
        if (a.parts > 1)
            hipLaunchKernelGGL(HIP_KERNEL_NAME(recurrence_part_kernel<T, false>), grid, block, 0, st, a);
        hipLaunchKernelGGL(recurrence_kernel<T>, grid, block, 0, st, a);
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
        const size_t need = RecurrencePlan(n, tokens, width).workspace;
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
    a.chunks = (int32_t)chunks, a.blocks = (int32_t)tiles(width, kWave);
    const RecurrencePlan p(n, tokens, width);
    a.tiles = p.tiles, a.parts = p.parts, a.per = p.per;
    const dim3 grid((unsigned)((int64_t)n * a.blocks * a.parts)), block(kThreads);
    const hipStream_t st = (hipStream_t)hip_stream;
    with_type(gate->type, [&](auto zero) {
        using T = decltype(zero);
        if (a.parts > 1)
            hipLaunchKernelGGL(HIP_KERNEL_NAME(recurrence_part_kernel<T, true>), grid, block, 0, st, a);
        hipLaunchKernelGGL(recurrence_grad_kernel<T>, grid, block, 0, st, a);
    });
    return done("relaysum_recurrence_backward");
}

}  // extern "C"
