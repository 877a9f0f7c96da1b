// The norms around a block of n workers' models on CDNA4 (gfx950), the one
// behind it with its gate and residual scale and the one in front of the next
// block, in one pass, and their gradients; the C ABI is in relaysum.h.
//
//   u = z * post_rstd * post_weight          post_rstd = 1 / sqrt(mean(z^2) + eps)
//   s = residual + scale * sigmoid(gate) * u
//   y = s * rstd * weight                    rstd = 1 / sqrt(mean(s^2) + eps)
//
// With zh = z * post_rstd, sh = s * rstd, g = sigmoid(gate):
//   ds = dsum + rstd * (dy * weight - sh * mean(dy * weight * sh))
//   dgate = ds * scale * u * g (1 - g),   v = ds * scale * g * post_weight
//   dz = post_rstd * (v - zh * mean(v * zh))
//   dweight = sum dy * sh,  dpost_weight = sum ds * scale * g * zh,  dscale = sum ds * g * u
//
// Bound by memory: a row stays in registers from its first load to its last store.
// 16 x 2048 x 1024 bfloat16 with what the backward pass needs 82 us (4.9 TB/s).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "layer_call.hpp"

namespace {

struct BlockNormArgs {
    Rows z, gate, r, sum;
    Packed y, saved;
    const float *post_weight, *weight, *scale;
    int64_t post_stride, weight_stride, scale_stride;
    float *post_rstd, *rstd;
    int64_t rows, total;
    int32_t width, stride;
    float eps;
};

// 1 / sqrt(mean(v^2) + eps) of a row that TPR threads hold, and in `rstd` that of
// the row as it was: rows outside binary32's range are scaled in place.
template <int TPR, int J>
__device__ __forceinline__ float row_rstd(float (&v)[J][8], float width, float eps, float &rstd, float *redf,
                                          unsigned *redu) {
    float sq = 0.0f;
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) sq = fmaf(v[j][i], v[j][i], sq);
    sq = row_reduce<TPR, float, pick_sum>(sq, redf);
    const float mean = sq / width + eps;
    rstd = 1.0f / sqrtf(mean);
    if (mean >= 0x1p-100f && mean < INFINITY) return rstd;
    return scaled_rstd<TPR, J>(v, width, eps, rstd, redf, redu);
}

// A sum of floats rounded to T: to a float first, as in the other types.  The fused
// instruction of binary16 would round but once, and 6 sums of 100,000 that lie next to
// the middle of two neighbours the other way than the same rows as floats.
template <typename T>
__device__ __forceinline__ float rounded(float v) {
    if constexpr (std::is_same<T, _Float16>::value) asm("" : "+v"(v));
    return (float)(T)v;
}

template <typename T, int TPR, int J, bool GATE, bool KEEP>
__global__ __launch_bounds__(block_of(TPR)) void blocknorm_kernel(BlockNormArgs a) {
    __shared__ float redf[16];
    __shared__ unsigned redu[16];
    constexpr int kRows = block_of(TPR) / TPR;
    const int lane = threadIdx.x % TPR;
    for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR; row < a.total;
         row += (int64_t)gridDim.x * kRows) {
        const int64_t worker = row / a.rows, t = row - worker * a.rows;
        const float scale = a.scale[worker * a.scale_stride];
        float s[J][8];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int at = (lane + j * TPR) * 8;
            load8(row_at<const T>(a.z, worker, t) + at, a.width - at, s[j]);
        }
        float rstd;
        float inv = row_rstd<TPR, J>(s, (float)a.width, a.eps, rstd, redf, redu);
        if (lane == 0) a.post_rstd[row] = rstd;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int at = (lane + j * TPR) * 8;
            float w[8], r[8], f[8];
            load8(a.post_weight + worker * a.post_stride + at, a.width - at, w);
            load8(row_at<const T>(a.r, worker, t) + at, a.width - at, r);
            if (GATE) load8(row_at<const T>(a.gate, worker, t) + at, a.width - at, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // As exact as a float's, whatever the type: rstd and y follow from s in
                // 32 bits.
                float g = 1.0f, rest;
                if (GATE) gates(f[i], g, rest);
                s[j][i] = rounded<T>(fmaf(scale * g, s[j][i] * inv * w[i], r[i]));
            }
            // Behind the width everything stays 0 (gates and all).
            if (a.width - at < 8) {
#pragma unroll
                for (int i = 0; i < 8; ++i) s[j][i] = at + i < a.width ? s[j][i] : 0.0f;
            }
            store8(row_at<T>(a.sum, worker, t) + at, a.width - at, s[j]);
        }
        if (KEEP) write_grouped<TPR, J>(a.saved, row, a.stride, lane, s);
        inv = row_rstd<TPR, J>(s, (float)a.width, a.eps, rstd, redf, redu);
        if (lane == 0) a.rstd[row] = rstd;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int at = (lane + j * TPR) * 8;
            float w[8];
            load8(a.weight + worker * a.weight_stride + at, a.width - at, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[j][i] = s[j][i] * inv * w[i];
        }
        write_whole<TPR, J>(a.y, row, a.stride, lane, s, redu);
    }
}

struct BlockNormGradArgs {
    Rows dy, dsum, z, gate, dz, dgate, ds;
    Packed saved;
    const float *post_weight, *weight, *scale, *post_rstd, *rstd;
    int64_t post_stride, weight_stride, scale_stride;
    float *partial;      // [n][parts][2 * width + 1]: of weight, post_weight and scale
    float *dpost, *dweight, *dscale;
    int64_t dpost_stride, dweight_stride, dscale_stride;
    int64_t rows;
    int32_t width, stride, parts;
};

// What a thread reads of a row, as it lies in memory.
template <typename T, int TPR, int J, bool GATE>
struct GradRow {
    v8_t<T> dy[J], z[J], dsum[J], gate[GATE ? J : 1];
    u2_t codes[J];
    int8_t exps[J];
    float rstd, post_rstd;

    static __device__ __forceinline__ v8_t<T> chunk(const Rows &r, int64_t worker, int64_t t, int at, int left) {
        v8_t<T> v = {};
        if (!r.data || left <= 0) return v;
        const T *p = row_at<const T>(r, worker, t) + at;
        if (left >= 8) {
            __builtin_memcpy(&v, p, sizeof v);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : (T)0.0f;
        }
        return v;
    }
    __device__ __forceinline__ void load(const BlockNormGradArgs &a, int64_t worker, int64_t t, int lane) {
        const int64_t row = worker * a.rows + t;
        rstd = a.rstd[row], post_rstd = a.post_rstd[row];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int at = (lane + j * TPR) * 8, left = a.width - at;
            dy[j] = chunk(a.dy, worker, t, at, left);
            z[j] = chunk(a.z, worker, t, at, left);
            dsum[j] = chunk(a.dsum, worker, t, at, left);
            if (GATE) gate[j] = chunk(a.gate, worker, t, at, left);
            codes[j] = u2_t{0, 0};
            exps[j] = 0;
            if (left > 0) {
                codes[j] = *reinterpret_cast<const u2_t *>(a.saved.codes + row * a.stride + at);
                exps[j] = a.saved.exps[row * a.saved.groups + (a.saved.groups > 1 ? at / kGroup : 0)];
            }
        }
    }
};

// A workgroup owns every parts-th block of rows of one worker; threads keep
// their columns' sums in registers over all of them and, but in workgroups of
// 1024 (which have 128 registers), the worker's weights and the next row: at
// 16 x 2048 x 1024 bfloat16 118 us (4.3 TB/s) for 268 us without them.
template <typename T, int TPR, int J, bool GATE>
__global__ __launch_bounds__(block_of(TPR), (TPR > 256 ? 4 : J == 1 ? 3 : 2)) void blocknorm_grad_kernel(BlockNormGradArgs a) {
    constexpr int kRows = block_of(TPR) / TPR;
    constexpr bool kAhead = TPR <= 256;
    __shared__ float red[16];
    __shared__ float sums[kRows > 1 ? kRows * TPR * J * 8 : 1];
    const int lane = threadIdx.x % TPR;
    // The same for a whole wave, where that is one row's or part of it.
    const int slot = TPR < kWave ? threadIdx.x / TPR : __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
    const int64_t worker = blockIdx.x / a.parts;
    const int part = blockIdx.x % a.parts;
    const float scale = a.scale[worker * a.scale_stride];
    const int64_t step = (int64_t)a.parts * kRows;
    float dw[J][8], dp[J][8], dscale = 0.0f;
    float weight[kAhead ? J : 1][8], post[kAhead ? J : 1][8];
#pragma unroll
    for (int j = 0; j < J; ++j) {
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[j][i] = dp[j][i] = 0.0f;
        if constexpr (kAhead) {
            const int at = (lane + j * TPR) * 8;
            load8(a.weight + worker * a.weight_stride + at, a.width - at, weight[j]);
            load8(a.post_weight + worker * a.post_stride + at, a.width - at, post[j]);
        }
    }
    GradRow<T, TPR, J, GATE> in;
    int64_t t = (int64_t)part * kRows + slot;
    if (kAhead && t < a.rows) in.load(a, worker, t, lane);
    for (; t < a.rows; t += step) {
        if (!kAhead) in.load(a, worker, t, lane);
        const float rstd = in.rstd, post_rstd = in.post_rstd;
        float ds[J][8], zh[J][8], sh[J][8], dot = 0.0f, dot2 = 0.0f;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int at = (lane + j * TPR) * 8;
            const float sc = at < a.width ? rstd * scale_of(in.exps[j]) : 0.0f;
            float w[8];
            if constexpr (!kAhead) load8(a.weight + worker * a.weight_stride + at, a.width - at, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if constexpr (kAhead) w[i] = weight[j][i];
                ds[j][i] = (float)in.dy[j][i];
                sh[j][i] = code_at(i < 4 ? in.codes[j].x : in.codes[j].y, i % 4) * sc;
                dw[j][i] = fmaf(ds[j][i], sh[j][i], dw[j][i]);
                ds[j][i] *= w[i];
                dot = fmaf(ds[j][i], sh[j][i], dot);
            }
        }
        dot = row_reduce<TPR, float, pick_sum>(dot, red) / (float)a.width;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int at = (lane + j * TPR) * 8;
            float w[8], dgate[8];
            if constexpr (!kAhead) load8(a.post_weight + worker * a.post_stride + at, a.width - at, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if constexpr (kAhead) w[i] = post[j][i];
                const float own = rstd * fmaf(-sh[j][i], dot, ds[j][i]);
                ds[j][i] = a.dsum.data ? (float)in.dsum[j][i] + own : own;
                zh[j][i] = (float)in.z[j][i] * post_rstd;
                float gate = 1.0f, rest = 0.0f;
                if (GATE) gates((float)in.gate[GATE ? j : 0][i], gate, rest);
                const float dg = ds[j][i] * gate;            // of scale * u
                const float u = zh[j][i] * w[i];
                if (at + i < a.width) dscale = fmaf(dg, u, dscale);
                dgate[i] = dg * scale * u * rest;
                dp[j][i] = fmaf(dg * scale, zh[j][i], dp[j][i]);
                sh[j][i] = dg * scale * w[i];                // of zh
                if (at + i < a.width) dot2 = fmaf(sh[j][i], zh[j][i], dot2);
            }
            if (GATE) store8(row_at<T>(a.dgate, worker, t) + at, a.width - at, dgate);
        }
        if (kAhead && t + step < a.rows) in.load(a, worker, t + step, lane);
        dot2 = row_reduce<TPR, float, pick_sum>(dot2, red) / (float)a.width;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int at = (lane + j * TPR) * 8;
            store8(row_at<T>(a.ds, worker, t) + at, a.width - at, ds[j]);
#pragma unroll
            for (int i = 0; i < 8; ++i) sh[j][i] = post_rstd * fmaf(-zh[j][i], dot2, sh[j][i]);
            store8(row_at<T>(a.dz, worker, t) + at, a.width - at, sh[j]);
        }
    }
    // Columns' sums: of the rows' slots of the workgroup, then to the parts.
    float *out[2] = {a.dweight + worker * a.dweight_stride, a.dpost + worker * a.dpost_stride};
    float *one = a.dscale + worker * a.dscale_stride;
    if (a.parts > 1) {
        float *p = a.partial + (worker * a.parts + part) * (2 * (int64_t)a.width + 1);
        out[0] = p, out[1] = p + a.width, one = p + 2 * a.width;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const auto &d = k ? dp : dw;
        if (kRows == 1) {
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const int at = (lane + j * TPR) * 8;
                store8(out[k] + at, a.width - at, d[j]);
            }
            continue;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) sums[(slot * J * TPR + j * TPR + lane) * 8 + i] = d[j][i];
        __syncthreads();
        for (int c = threadIdx.x; c < a.width; c += block_of(TPR)) {
            float v = sums[c];
#pragma unroll
            for (int s = 1; s < kRows; ++s) v += sums[s * J * TPR * 8 + c];
            out[k][c] = v;
        }
    }
    dscale = row_reduce<block_of(TPR), float, pick_sum>(dscale, red);
    if (threadIdx.x == 0) *one = dscale;
}

// The parts' sums into the three gradients: as many columns as they have, 32 of
// them and 8 sums of every eighth part in a workgroup, added in a fixed order.
__global__ __launch_bounds__(256) void blocknorm_sum_kernel(BlockNormGradArgs a) {
    __shared__ float sums[8][32];
    const int64_t columns = 2 * (int64_t)a.width + 1;
    const unsigned per = (unsigned)((columns + 31) / 32);
    const int64_t worker = blockIdx.x / per;
    const int lane = threadIdx.x % 32, group = threadIdx.x / 32;
    const int64_t c = (int64_t)(blockIdx.x % per) * 32 + lane;
    float v = 0.0f;
    if (c < columns) {
        const float *p = a.partial + worker * a.parts * columns + c;
#pragma unroll 8
        for (int k = group; k < a.parts; k += 8) v += p[k * columns];
    }
    sums[group][lane] = v;
    __syncthreads();
    if (group || c >= columns) return;
#pragma unroll
    for (int k = 1; k < 8; ++k) v += sums[k][lane];
    if (c < a.width) a.dweight[worker * a.dweight_stride + c] = v;
    else if (c < 2 * (int64_t)a.width) a.dpost[worker * a.dpost_stride + c - a.width] = v;
    else a.dscale[worker * a.dscale_stride] = v;
}

// ---- host side -------------------------------------------------------------------------

// The gradient holds five rows and four sums of them at once: fewer chunks a thread.
template <typename F>
void with_grad_layout(int64_t stride, F f) {
    const int64_t chunks = stride / 8;
    if (chunks <= 16) f(Int<16>(), Int<1>());
    else if (chunks <= 64) f(Int<64>(), Int<1>());
    else if (chunks <= 128) f(Int<64>(), Int<2>());
    else if (chunks <= 256) f(Int<256>(), Int<1>());
    else if (chunks <= 512) f(Int<256>(), Int<2>());
    else if (chunks <= 1024) f(Int<1024>(), Int<1>());
    else if (chunks <= 2048) f(Int<1024>(), Int<2>());
    else f(Int<1024>(), Int<4>());
}

size_t grad_workspace(int32_t n, int64_t rows, int64_t width) {
    const int parts = norm_parts(n, rows);
    return parts > 1 ? (size_t)n * parts * (2 * width + 1) * 4 : 0;
}

struct BlockNormCall : Call {
    void vector(const char *name, const float *w, int32_t n, int64_t stride, int64_t width) {
        if (code != RELAYSUM_OK) return;
        if (n == 1) stride = 0;
        if (stride < 0 || stride > ((int64_t)1 << 44) / n)
            return fail(refuse("%s's stride is negative or reaches past 2^44 entries", name));
        add(Span{name, reinterpret_cast<const char *>(w), (size_t)((n - 1) * stride + width) * 4, false, false, width * 4,
                 stride * 4, 0, n, 1}, 4);
    }
    void gradient(const char *name, const relaysum_rows *r, int32_t n, int64_t width) {
        rows(name, r, n, 1, width, true);
        if (code == RELAYSUM_OK && r->type != RELAYSUM_FLOAT) fail(refuse("%s must be of type float", name));
    }
    void same(const char *name, const relaysum_rows *r, int32_t type) {
        if (code == RELAYSUM_OK && r && r->type != type) fail(refuse("%s is not of z's type", name));
    }
};

}  // namespace

extern "C" {

int relaysum_blocknorm(int32_t n, int64_t tokens, int64_t width, const relaysum_rows *z, const relaysum_rows *gate,
                       const relaysum_rows *residual, const float *post_weight, int64_t post_weight_stride,
                       const float *scale, int64_t scale_stride, const float *weight, int64_t weight_stride, float eps,
                       const relaysum_rows *sum, const relaysum_packed *y, float *post_rstd, float *rstd,
                       const relaysum_packed *saved, void *hip_stream) {
    BlockNormCall c;
    c.in_place = true;
    if (c.sizes(n, tokens, width, "tokens")) {
        c.rows("z", z, n, tokens, width, false);
        if (gate) c.rows("gate", gate, n, tokens, width, false);
        c.rows("residual", residual, n, tokens, width, false);
        c.rows("sum", sum, n, tokens, width, true);
        if (c.code == RELAYSUM_OK) {
            c.same("gate", gate, z->type);
            c.same("residual", residual, z->type);
            c.same("sum", sum, z->type);
        }
        c.vector("post_weight", post_weight, n, post_weight_stride, width);
        c.vector("scale", scale, n, scale_stride, 1);
        c.vector("weight", weight, n, weight_stride, width);
        if (y && !whole_rows(y, width)) c.fail(refuse("y is packed by whole rows (group 0)"));
        c.packed("y", y, n, tokens, width, true);
        c.span("post_rstd", post_rstd, (size_t)n * tokens * 4, 4, true);
        c.span("rstd", rstd, (size_t)n * tokens * 4, 4, true);
        if (saved) c.packed("saved", saved, n, tokens, width, true);
        if (saved && whole_rows(saved, width) && width > kGroup) c.fail(refuse("saved is packed in groups of %d", kGroup));
        if (!(eps >= 0.0f)) c.fail(refuse("eps must not be negative"));
    }
    if (!c.ready()) return c.code;
    if (tokens == 0) return done("relaysum_blocknorm");
    BlockNormArgs a{rows_of(z, n, tokens), rows_of(gate, n, tokens), rows_of(residual, n, tokens), rows_of(sum, n, tokens),
                    packed_of(y, width), packed_of(saved, width), post_weight, weight, scale,
                    n > 1 ? post_weight_stride : 0, n > 1 ? weight_stride : 0, n > 1 ? scale_stride : 0,
                    post_rstd, rstd, tokens, n * tokens, (int32_t)width, (int32_t)code_stride(width), eps};
    with_type(z->type, [&](auto zero) {
        using T = decltype(zero);
        with_layout(a.stride, [&](auto tpr, auto chunks) {
            constexpr int TPR = decltype(tpr)::value, J = decltype(chunks)::value;
            const dim3 grid(row_grid(a.total, block_of(TPR) / TPR)), block(block_of(TPR));
            const hipStream_t st = (hipStream_t)hip_stream;
            if (gate && saved)
                hipLaunchKernelGGL(HIP_KERNEL_NAME(blocknorm_kernel<T, TPR, J, true, true>), grid, block, 0, st, a);
            else if (gate)
                hipLaunchKernelGGL(HIP_KERNEL_NAME(blocknorm_kernel<T, TPR, J, true, false>), grid, block, 0, st, a);
            else if (saved)
                hipLaunchKernelGGL(HIP_KERNEL_NAME(blocknorm_kernel<T, TPR, J, false, true>), grid, block, 0, st, a);
            else
                hipLaunchKernelGGL(HIP_KERNEL_NAME(blocknorm_kernel<T, TPR, J, false, false>), grid, block, 0, st, a);
        });
    });
    return done("relaysum_blocknorm");
}

int64_t relaysum_blocknorm_workspace(int32_t n, int64_t tokens, int64_t width) {
    Call c;
    if (!c.sizes(n, tokens, width, "tokens")) return -1;
    g_error[0] = '\0';
    return (int64_t)grad_workspace(n, tokens, width);
}

int relaysum_blocknorm_backward(int32_t n, int64_t tokens, int64_t width, const relaysum_rows *dy,
                                const relaysum_rows *dsum, const relaysum_rows *z, const relaysum_rows *gate,
                                const relaysum_packed *saved, const float *post_rstd, const float *rstd,
                                const float *post_weight, int64_t post_weight_stride, const float *scale,
                                int64_t scale_stride, const float *weight, int64_t weight_stride,
                                const relaysum_rows *dz, const relaysum_rows *dgate, const relaysum_rows *ds,
                                const relaysum_rows *post_weight_grad, const relaysum_rows *scale_grad,
                                const relaysum_rows *weight_grad, void *workspace, size_t workspace_bytes,
                                void *hip_stream) {
    BlockNormCall c;
    c.in_place = true;
    int parts = 1;
    if (c.sizes(n, tokens, width, "tokens")) {
        parts = norm_parts(n, tokens);
        c.rows("z", z, n, tokens, width, false);
        c.rows("dy", dy, n, tokens, width, false);
        if (dsum) c.rows("dsum", dsum, n, tokens, width, false);
        if (!gate != !dgate) c.fail(refuse("gate and dgate come together"));
        if (gate) c.rows("gate", gate, n, tokens, width, false);
        if (dgate) c.rows("dgate", dgate, n, tokens, width, true);
        c.rows("dz", dz, n, tokens, width, true);
        c.rows("ds", ds, n, tokens, width, true);
        if (c.code == RELAYSUM_OK) {
            c.same("dy", dy, z->type);
            c.same("dsum", dsum, z->type);
            c.same("gate", gate, z->type);
            c.same("dgate", dgate, z->type);
            c.same("dz", dz, z->type);
            c.same("ds", ds, z->type);
        }
        c.packed("saved", saved, n, tokens, width, false);
        c.span("post_rstd", post_rstd, (size_t)n * tokens * 4, 4, false);
        c.span("rstd", rstd, (size_t)n * tokens * 4, 4, false);
        c.vector("post_weight", post_weight, n, post_weight_stride, width);
        c.vector("scale", scale, n, scale_stride, 1);
        c.vector("weight", weight, n, weight_stride, width);
        c.gradient("post_weight_grad", post_weight_grad, n, width);
        c.gradient("scale_grad", scale_grad, n, 1);
        c.gradient("weight_grad", weight_grad, n, width);
        const size_t need = grad_workspace(n, tokens, width);
        if (need > workspace_bytes)
            c.fail(refuse("the workspace has %zu bytes, %zu are needed", workspace_bytes, need));
        c.span("workspace", workspace, need, 4, true);
        if ((int64_t)n * std::max<int64_t>(parts, (2 * width + 32) / 32) > kMaxBlocks) c.fail(refuse("n is too large"));
    }
    if (!c.ready()) return c.code;
    const Rows dp = rows_of(post_weight_grad, n, 1), dsc = rows_of(scale_grad, n, 1), dw = rows_of(weight_grad, n, 1);
    BlockNormGradArgs a{rows_of(dy, n, tokens), rows_of(dsum, n, tokens), rows_of(z, n, tokens), rows_of(gate, n, tokens),
                        rows_of(dz, n, tokens), rows_of(dgate, n, tokens), rows_of(ds, n, tokens), packed_of(saved, width),
                        post_weight, weight, scale, post_rstd, rstd, n > 1 ? post_weight_stride : 0,
                        n > 1 ? weight_stride : 0, n > 1 ? scale_stride : 0, static_cast<float *>(workspace),
                        reinterpret_cast<float *>(dp.data), reinterpret_cast<float *>(dw.data),
                        reinterpret_cast<float *>(dsc.data), dp.ws, dw.ws, dsc.ws, tokens, (int32_t)width,
                        (int32_t)code_stride(width), parts};
    const hipStream_t st = (hipStream_t)hip_stream;
    with_type(z->type, [&](auto zero) {
        using T = decltype(zero);
        with_grad_layout(a.stride, [&](auto tpr, auto chunks) {
            constexpr int TPR = decltype(tpr)::value, J = decltype(chunks)::value;
            const dim3 grid((unsigned)(n * parts)), block(block_of(TPR));
            if (gate)
                hipLaunchKernelGGL(HIP_KERNEL_NAME(blocknorm_grad_kernel<T, TPR, J, true>), grid, block, 0, st, a);
            else
                hipLaunchKernelGGL(HIP_KERNEL_NAME(blocknorm_grad_kernel<T, TPR, J, false>), grid, block, 0, st, a);
        });
    });
    if (parts > 1)
        hipLaunchKernelGGL(blocknorm_sum_kernel, dim3((unsigned)(n * ((2 * width + 32) / 32))), dim3(256), 0, st, a);
    return done("relaysum_blocknorm_backward");
}

}  // extern "C"
