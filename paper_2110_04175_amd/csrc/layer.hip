// Layer operators on CDNA4 (gfx950): what n workers, each with weights of its
// own, compute between two RelaySum rounds.  RMS norm with the residual's
// addition into 8-bit rows, its gradient, products of 8-bit rows and their
// gradients, and packing; the C ABI is in relaysum.h.
//
// 8-bit rows.  A group of entries v (a whole row, or 128 entries of it) is
// held as q = rint(v * 2^-e), the smallest e >= -126 with max|v| <= 127 * 2^e.
// The scale is a power of two because of the backward pass: there the scaled
// rows lie on the contracted axis (dX = dY W sums over channels, dW = dY^T X
// over tokens), so the scale has to enter an operand of the matrix
// instructions.  q * 2^e has 7 significant bits and is exact in bfloat16; a
// 24-bit scale would cost a rounding of the operand (2^-9) or several
// products.  The price is a quantum up to twice that of max|v| / 127.
// A row's codes take its width rounded up to 128 bytes, zeros behind the
// width: rows start on 128-byte lines, and a contraction over the width has
// no tail.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <type_traits>

#include "relaysum.h"

namespace {

constexpr int kWave = 64;
constexpr int kCus = 256;
constexpr int64_t kMaxWidth = 32768;   // 127^2 * 32768 < 2^31: integer sums cannot overflow
constexpr int64_t kMaxChannels = 1 << 24;
constexpr int kGroup = 128;            // entries that share a scale in grouped rows, and the
                                       // bytes a row of codes is rounded up to
constexpr int kNotANumber = -128;      // exponent of a group that held a NaN or an infinity

typedef int i4_t __attribute__((ext_vector_type(4)));
typedef float f4_t __attribute__((ext_vector_type(4)));
typedef __bf16 b8_t __attribute__((ext_vector_type(8)));
typedef unsigned u2_t __attribute__((ext_vector_type(2)));
typedef unsigned u4_t __attribute__((ext_vector_type(4)));

// ---- elements ------------------------------------------------------------------

template <typename T>
using v8_t = T __attribute__((ext_vector_type(8)));

// Eight entries of a row as floats, those from `left` on as zeros.  Whole
// chunks are one or two 16-byte loads at any alignment of the type.
template <typename T>
__device__ __forceinline__ void load8(const T *p, int64_t left, float (&v)[8]) {
    if (left >= 8) {
        v8_t<T> t;
        __builtin_memcpy(&t, p, sizeof t);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)t[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? (float)p[i] : 0.0f;
    }
}

template <typename T>
__device__ __forceinline__ void store8(T *p, int64_t left, const float (&v)[8]) {
    if (left >= 8) {
        v8_t<T> t;
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = (T)v[i];
        __builtin_memcpy(p, &t, sizeof t);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = (T)v[i];
    }
}

__device__ __forceinline__ unsigned bits_of(float f) { return __builtin_bit_cast(unsigned, f); }
__device__ __forceinline__ float float_of(unsigned u) { return __builtin_bit_cast(float, u); }

// Exponent of a group whose largest |v| has these bits.  127 = 1.984375 * 2^6:
// |v| = m * 2^p fits 2^(p-6) if m <= 1.984375 (mantissa field 0x7e0000), else
// 2^(p-5).  As integers, the bits of NaN are above infinity's, above every
// number's, so one integer maximum finds the largest entry and what is none.
__device__ __forceinline__ int exponent_of(unsigned maxbits) {
    if (maxbits >= 0x7f800000u) return kNotANumber;
    return max((int)((maxbits + 0x1ffffu) >> 23) - 133, -126);
}

// 2^-e, or 0 for a group that is not a number (every code is then 0: NaN and
// infinity times 0 is NaN, which converts to 0).
__device__ __forceinline__ float inverse_scale(int e) {
    return e == kNotANumber ? 0.0f : float_of((unsigned)(127 - e) << 23);
}

__device__ __forceinline__ float scale_of(int e) {
    return e == kNotANumber ? float_of(0x7fc00000u) : float_of((unsigned)(127 + e) << 23);
}

__device__ __forceinline__ u2_t codes8(const float (&v)[8], float inv) {
    unsigned w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        w[i / 4] |= ((unsigned)__float2int_rn(v[i] * inv) & 0xffu) << (8 * (i % 4));
    return u2_t{w[0], w[1]};
}

__device__ __forceinline__ float code_at(unsigned w, int byte) {
    return (float)(int)(int8_t)(w >> (8 * byte));
}

template <int J>
__device__ __forceinline__ unsigned max_bits(const float (&v)[J][8]) {
    unsigned m = 0;
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, bits_of(v[j][i]) & 0x7fffffffu);
    return m;
}

// ---- reductions over the TPR threads that share a row ----------------------------
//
// 16 or 64 threads: lanes of one wave.  256 or 1024: a whole workgroup, through
// LDS; `red` holds one value per wave.

__device__ __forceinline__ float pick_sum(float a, float b) { return a + b; }
__device__ __forceinline__ unsigned pick_max(unsigned a, unsigned b) { return max(a, b); }

template <int TPR, typename V, V (*F)(V, V)>
__device__ __forceinline__ V row_reduce(V v, V *red) {
#pragma unroll
    for (int m = 1; m < (TPR < kWave ? TPR : kWave); m *= 2) v = F(v, __shfl_xor(v, m));
    if (TPR > kWave) {
        const int wave = threadIdx.x / kWave;
        __syncthreads();
        if (threadIdx.x % kWave == 0) red[wave] = v;
        __syncthreads();
        v = red[0];
#pragma unroll
        for (int w = 1; w < TPR / kWave; ++w) v = F(v, red[w]);
    }
    return v;
}

constexpr int block_of(int tpr) { return tpr > 256 ? tpr : 256; }

// ---- rows of n workers -----------------------------------------------------------

struct Rows {
    char *data;
    int64_t ws, rs;   // strides in entries
};

template <typename T>
__device__ __forceinline__ T *row_at(const Rows &r, int64_t worker, int64_t row) {
    return reinterpret_cast<T *>(r.data) + worker * r.ws + row * r.rs;
}

struct Packed {
    int8_t *codes, *exps;
    int32_t groups;   // exponents of a row
};

struct PackArgs {
    Rows v;
    Packed out;
    int64_t rows, total;   // rows of a worker, of all workers
    int32_t width, stride;
};

// Codes of a row that TPR threads hold in v (chunk j of thread `lane`: entries
// 8 * (lane + j * TPR)), as whole rows or in groups of 128 entries, which 16
// neighbouring lanes hold.
template <int TPR, int J>
__device__ __forceinline__ void write_grouped(const Packed &out, int64_t row, int32_t stride,
                                              int lane, const float (&v)[J][8]) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int chunk = lane + j * TPR;
        unsigned m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, bits_of(v[j][i]) & 0x7fffffffu);
#pragma unroll
        for (int s = 1; s < 16; s *= 2) m = max(m, (unsigned)__shfl_xor((int)m, s));
        if (chunk * 8 >= stride) continue;
        const int e = exponent_of(m);
        if (lane % 16 == 0) out.exps[row * out.groups + chunk / 16] = (int8_t)e;
        *reinterpret_cast<u2_t *>(out.codes + row * stride + chunk * 8) =
            codes8(v[j], inverse_scale(e));
    }
}

template <int TPR, int J>
__device__ __forceinline__ void write_whole(const Packed &out, int64_t row, int32_t stride,
                                            int lane, const float (&v)[J][8], unsigned *red) {
    const int e = exponent_of(row_reduce<TPR, unsigned, pick_max>(max_bits(v), red));
    const float inv = inverse_scale(e);
    if (lane == 0) out.exps[row] = (int8_t)e;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int chunk = lane + j * TPR;
        if (chunk * 8 < stride)
            *reinterpret_cast<u2_t *>(out.codes + row * stride + chunk * 8) = codes8(v[j], inv);
    }
}

template <typename T, int TPR, int J, bool GROUPED>
__global__ __launch_bounds__(block_of(TPR)) void pack_kernel(PackArgs a) {
    __shared__ unsigned red[16];
    constexpr int kRows = block_of(TPR) / TPR;
    const int lane = threadIdx.x % TPR;
    for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR; row < a.total;
         row += (int64_t)gridDim.x * kRows) {
        const int64_t worker = row / a.rows;
        const T *p = row_at<const T>(a.v, worker, row - worker * a.rows);
        float v[J][8];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int at = (lane + j * TPR) * 8;
            load8(p + at, a.width - at, v[j]);
        }
        if (GROUPED)
            write_grouped<TPR, J>(a.out, row, a.stride, lane, v);
        else
            write_whole<TPR, J>(a.out, row, a.stride, lane, v, red);
    }
}

template <typename T, int TPR>
__global__ __launch_bounds__(256) void unpack_kernel(PackArgs a) {
    constexpr int kRows = 256 / TPR;
    const int lane = threadIdx.x % TPR;
    for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR; row < a.total;
         row += (int64_t)gridDim.x * kRows) {
        const int64_t worker = row / a.rows;
        T *p = row_at<T>(a.v, worker, row - worker * a.rows);
        for (int at = lane * 8; at < a.width; at += TPR * 8) {
            const u2_t q = *reinterpret_cast<const u2_t *>(a.out.codes + row * a.stride + at);
            const float s =
                scale_of(a.out.exps[row * a.out.groups + (a.out.groups > 1 ? at / kGroup : 0)]);
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = code_at(i < 4 ? q.x : q.y, i % 4) * s;
            store8(p + at, a.width - at, v);
        }
    }
}

// ---- RMS norm ----------------------------------------------------------------------

struct NormArgs {
    Rows h, r, sum;
    Packed y, saved;
    const float *weight;
    float *rstd;
    int64_t weight_stride;
    int64_t rows, total;
    int32_t width, stride;
    float eps;
};

// s = h + r, rounded to the rows' type because that is what the stream goes on
// with; y = s * rstd * w is not rounded before it is packed.  One pass: the row
// stays in registers between the sum of squares and the codes.
template <typename T, int TPR, int J, bool RESIDUAL, bool KEEP>
__global__ __launch_bounds__(block_of(TPR)) void norm_kernel(NormArgs a) {
    __shared__ float redf[16];
    __shared__ unsigned redu[16];
    constexpr int kRows = block_of(TPR) / TPR;
    const int lane = threadIdx.x % TPR;
    for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR; row < a.total;
         row += (int64_t)gridDim.x * kRows) {
        const int64_t worker = row / a.rows, t = row - worker * a.rows;
        const T *h = row_at<const T>(a.h, worker, t);
        const float *w = a.weight + worker * a.weight_stride;
        float s[J][8], sq = 0.0f;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int at = (lane + j * TPR) * 8;
            load8(h + at, a.width - at, s[j]);
            if (RESIDUAL) {
                float r[8];
                load8(row_at<const T>(a.r, worker, t) + at, a.width - at, r);
#pragma unroll
                for (int i = 0; i < 8; ++i) s[j][i] = (float)(T)(s[j][i] + r[i]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) sq = fmaf(s[j][i], s[j][i], sq);
        }
        if (RESIDUAL) {
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const int at = (lane + j * TPR) * 8;
                store8(row_at<T>(a.sum, worker, t) + at, a.width - at, s[j]);
            }
        }
        sq = row_reduce<TPR, float, pick_sum>(sq, redf);
        const float rstd = 1.0f / sqrtf(sq / (float)a.width + a.eps);
        if (lane == 0) a.rstd[row] = rstd;
        if (KEEP) write_grouped<TPR, J>(a.saved, row, a.stride, lane, s);
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int at = (lane + j * TPR) * 8;
            float wv[8];
            load8(w + at, a.width - at, wv);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[j][i] = s[j][i] * rstd * wv[i];
        }
        write_whole<TPR, J>(a.y, row, a.stride, lane, s, redu);
    }
}

struct NormGradArgs {
    Rows dy, dsum, ds;
    Packed saved;
    const float *weight, *rstd;
    float *partial;    // [n][parts][width], or the gradient's rows if parts == 1
    int64_t weight_stride, partial_stride;   // partial_stride: between workers
    int64_t rows;
    int32_t width, stride, parts;
};

// A workgroup owns every parts-th block of rows of one worker: threads keep
// their columns' weights and sums of dy * xh in registers over all of them.
template <typename T, int TPR, int J, bool DSUM>
__global__ __launch_bounds__(block_of(TPR)) void norm_grad_kernel(NormGradArgs a) {
    constexpr int kRows = block_of(TPR) / TPR;
    __shared__ float red[16];
    __shared__ float sums[kRows > 1 ? kRows * TPR * J * 8 : 1];
    const int lane = threadIdx.x % TPR, slot = threadIdx.x / TPR;
    const int64_t worker = blockIdx.x / a.parts;
    const int part = blockIdx.x % a.parts;
    float w[J][8], dw[J][8];
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int at = (lane + j * TPR) * 8;
        load8(a.weight + worker * a.weight_stride + at, a.width - at, w[j]);
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[j][i] = 0.0f;
    }
    for (int64_t t = (int64_t)part * kRows + slot; t < a.rows; t += (int64_t)a.parts * kRows) {
        const int64_t row = worker * a.rows + t;
        const float rstd = a.rstd[row];
        float u[J][8], xh[J][8], dot = 0.0f;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int at = (lane + j * TPR) * 8;
            load8(row_at<const T>(a.dy, worker, t) + at, a.width - at, u[j]);
            u2_t q = {0, 0};
            float sc = 0.0f;
            if (at < a.width) {
                q = *reinterpret_cast<const u2_t *>(a.saved.codes + row * a.stride + at);
                sc = rstd * scale_of(a.saved.exps[row * a.saved.groups +
                                                  (a.saved.groups > 1 ? at / kGroup : 0)]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                xh[j][i] = code_at(i < 4 ? q.x : q.y, i % 4) * sc;
                dw[j][i] = fmaf(u[j][i], xh[j][i], dw[j][i]);
                u[j][i] *= w[j][i];
                dot = fmaf(u[j][i], xh[j][i], dot);
            }
        }
        dot = row_reduce<TPR, float, pick_sum>(dot, red) / (float)a.width;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int at = (lane + j * TPR) * 8;
            float d[8];
            if (DSUM) load8(row_at<const T>(a.dsum, worker, t) + at, a.width - at, d);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float g = rstd * fmaf(-xh[j][i], dot, u[j][i]);
                d[i] = DSUM ? d[i] + g : g;
            }
            store8(row_at<T>(a.ds, worker, t) + at, a.width - at, d);
        }
    }
    float *out = a.partial + worker * a.partial_stride + (int64_t)part * a.width;
    if (kRows == 1) {
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int at = (lane + j * TPR) * 8;
            store8(out + at, a.width - at, dw[j]);
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) sums[(slot * J * TPR + j * TPR + lane) * 8 + i] = dw[j][i];
    __syncthreads();
    for (int c = threadIdx.x; c < a.width; c += block_of(TPR)) {
        float v = sums[c];
#pragma unroll
        for (int k = 1; k < kRows; ++k) v += sums[k * J * TPR * 8 + c];
        out[c] = v;
    }
}

// out[i][c] = sum over parts of partial[i][p][c], p ascending: the order is
// fixed, so equal inputs give equal bits.
__global__ __launch_bounds__(256) void sum_parts_kernel(const float *partial, float *out,
                                                        int64_t out_stride, int32_t parts,
                                                        int32_t width) {
    const int per = (width + 255) / 256;
    const int64_t worker = blockIdx.x / per;
    const int c = (int)(blockIdx.x % per) * 256 + threadIdx.x;
    if (c >= width) return;
    const float *p = partial + worker * parts * (int64_t)width + c;
    float v = 0.0f;
    for (int k = 0; k < parts; ++k) v += p[(int64_t)k * width];
    out[worker * out_stride + c] = v;
}

// ---- products ------------------------------------------------------------------------
//
// LDS tiles of both products: rows of 128 bytes (128 codes, or 64 bfloat16 of
// the contracted axis) as 8 chunks of 16 bytes; chunk c of row r lies at
// position c ^ swizzle(r).  16 lanes that read the same chunk of 16 neighbouring
// rows then touch 16 different 16-byte bank groups, and so do the lanes that
// write one chunk of rows 4 apart.
__device__ __forceinline__ int swizzle(int row) { return ((row >> 1) & 7) ^ ((row >> 4) & 1); }
__device__ __forceinline__ int tile_at(int row, int chunk) {
    return row * 128 + ((chunk ^ swizzle(row)) << 4);
}

// Blocks go round the 8 XCDs; each takes a run of neighbouring tiles, which
// share rows in its L2.
__device__ __forceinline__ int64_t xcd_tile(int64_t block, int64_t blocks) {
    const int64_t run = blocks / 8, rest = blocks % 8, x = block % 8;
    return x * run + (x < rest ? x : rest) + block / 8;
}

struct LinearArgs {
    Packed x, w;
    Rows y;
    int64_t tokens;
    int32_t width, stride, channels;
    int64_t tiles_m;
    int32_t tiles_n;
};

// Y[t][c] = 2^(ex[t] + ew[c]) * sum_k qx[t][k] qw[c][k]: whole numbers until
// the one conversion (rounded to 24 bits from 2^24 on, then to the type).
template <typename T, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void linear_kernel(LinearArgs a) {
    constexpr int kThreads = 64 * WM * WN;
    constexpr int TM = BM / WM / 16, TN = BN / WN / 16;
    __shared__ __align__(16) char lds[(BM + BN) * 128];
    const int64_t tile = xcd_tile(blockIdx.x, gridDim.x);
    const int64_t per = a.tiles_m * a.tiles_n;
    const int64_t worker = tile / per, in = tile - worker * per;
    const int64_t m0 = (in / a.tiles_n) * BM;
    const int n0 = (int)(in % a.tiles_n) * BN;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);
    const int8_t *xq = a.x.codes + worker * a.tokens * a.stride;
    const int8_t *wq = a.w.codes + worker * (int64_t)a.channels * a.stride;
    i4_t acc[TM][TN] = {};
    for (int k0 = 0; k0 < a.stride; k0 += 128) {
        u4_t st[(BM + BN) * 8 / kThreads];
#pragma unroll
        for (int i = 0; i < (BM + BN) * 8 / kThreads; ++i) {
            const int u = i * kThreads + threadIdx.x, r = u / 8, ch = u % 8;
            // Rows past the end repeat the last one; what they give is not stored.
            const int8_t *p = r < BM ? xq + min(m0 + r, a.tokens - 1) * a.stride
                                     : wq + (int64_t)min(n0 + r - BM, a.channels - 1) * a.stride;
            st[i] = *reinterpret_cast<const u4_t *>(p + k0 + ch * 16);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < (BM + BN) * 8 / kThreads; ++i) {
            const int u = i * kThreads + threadIdx.x;
            *reinterpret_cast<u4_t *>(lds + tile_at(u / 8, u % 8)) = st[i];
        }
        __syncthreads();
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            i4_t xf[TM], wf[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i)
                xf[i] = *reinterpret_cast<const i4_t *>(
                    lds + tile_at(wm + i * 16 + lane % 16, ks * 4 + lane / 16));
#pragma unroll
            for (int j = 0; j < TN; ++j)
                wf[j] = *reinterpret_cast<const i4_t *>(
                    lds + tile_at(BM + wn + j * 16 + lane % 16, ks * 4 + lane / 16));
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[j], xf[i], acc[i][j], 0, 0, 0);
        }
    }
    // A lane has four neighbouring channels of one token in each accumulator.
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t t = m0 + wm + i * 16 + lane % 16;
        if (t >= a.tokens) continue;
        const int ex = a.x.exps[worker * a.tokens + t];
        T *y = row_at<T>(a.y, worker, t);
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int c0 = n0 + wn + j * 16 + lane / 16 * 4;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (c0 + k >= a.channels) continue;
                const int ew = a.w.exps[worker * a.channels + c0 + k];
                const float v = ldexpf((float)acc[i][j][k], ex + ew);
                y[c0 + k] = (T)(ex == kNotANumber || ew == kNotANumber ? float_of(0x7fc00000u) : v);
            }
        }
    }
}

struct GradArgs {
    Rows a;            // dY
    Packed b;          // [n][r][stride]
    Rows out;
    float *partial;    // split > 1: [split][n][m][cols]
    int64_t m, r;      // rows of the result, the contracted axis
    int32_t cols, stride, split;
    int64_t tiles_m;
    int32_t tiles_n;
    int32_t workers;
};

// A float as a sum of P bfloat16: exactly, for the 8, 11 and 24 significant
// bits of the three types and P = 1, 2, 3.
template <int P>
__device__ __forceinline__ void split(float v, __bf16 (&part)[P]) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
        part[p] = (__bf16)v;
        // An infinity has no rest.
        if (p + 1 < P) v = (bits_of((float)part[p]) & 0x7f800000u) == 0x7f800000u ? 0.0f : v - (float)part[p];
    }
}

template <typename T> struct Parts { static constexpr int n = 1; };
template <> struct Parts<_Float16> { static constexpr int n = 2; };
template <> struct Parts<float> { static constexpr int n = 3; };

// out[m][k] = sum_r A(m, r) * q[r][k] 2^e[r][k / group], with A(m, r) = dY[m][r]
// (dX: m tokens, r channels) or dY[r][m] (ALONG_R, dW: m channels, r tokens).
// Both operands are brought into LDS as bfloat16 rows along r: 8 x 4 blocks of
// codes, and of dY for dW, are turned in registers on the way.
template <typename T, typename O, bool ALONG_R, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void grad_kernel(GradArgs a) {
    constexpr int kThreads = 64 * WM * WN, P = Parts<T>::n, BR = 64;
    constexpr int TM = BM / WM / 16, TN = BN / WN / 16;
    __shared__ __align__(16) char lds[(P * BM + BN) * 128];
    char *ldb = lds + P * BM * 128;
    const int64_t per = a.tiles_m * a.tiles_n;
    const int64_t tile = xcd_tile(blockIdx.x, gridDim.x);
    const int64_t job = tile / per, in = tile - job * per;
    const int64_t worker = job / a.split;
    const int part = (int)(job - worker * a.split);
    const int64_t m0 = (in / a.tiles_n) * BM;
    const int n0 = (int)(in % a.tiles_n) * BN;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);
    // This part's share of the contracted axis, in whole tiles.
    const int64_t steps = (a.r + BR - 1) / BR;
    const int64_t s0 = steps * part / a.split, s1 = steps * (part + 1) / a.split;
    f4_t acc[TM][TN] = {};
    for (int64_t s = s0; s < s1; ++s) {
        const int64_t r0 = s * BR;
        __syncthreads();
        if (ALONG_R) {
#pragma unroll
            for (int i = 0; i < BM * BR / 32 / kThreads; ++i) {
                const int u = i * kThreads + threadIdx.x;
                const int mm = u % (BM / 4) * 4, rr = u / (BM / 4) * 8;
                __bf16 p[4][8][P];
#pragma unroll
                for (int y = 0; y < 8; ++y) {
                    const int64_t r = r0 + rr + y;
                    const T *src = row_at<const T>(a.a, worker, r) + m0 + mm;
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        split<P>(r < a.r && m0 + mm + x < a.m ? (float)src[x] : 0.0f, p[x][y]);
                }
#pragma unroll
                for (int x = 0; x < 4; ++x)
#pragma unroll
                    for (int k = 0; k < P; ++k) {
                        b8_t v;
#pragma unroll
                        for (int y = 0; y < 8; ++y) v[y] = p[x][y][k];
                        *reinterpret_cast<b8_t *>(lds + tile_at(k * BM + mm + x, rr / 8)) = v;
                    }
            }
        } else {
#pragma unroll
            for (int i = 0; i < BM * 8 / kThreads; ++i) {
                const int u = i * kThreads + threadIdx.x, mm = u / 8, ch = u % 8;
                const int64_t m = min(m0 + mm, a.m - 1), r = r0 + ch * 8;
                float v[8];
                load8(row_at<const T>(a.a, worker, m) + r, a.r - r, v);
                b8_t q[P];
#pragma unroll
                for (int y = 0; y < 8; ++y) {
                    __bf16 p[P];
                    split<P>(v[y], p);
#pragma unroll
                    for (int k = 0; k < P; ++k) q[k][y] = p[k];
                }
#pragma unroll
                for (int k = 0; k < P; ++k)
                    *reinterpret_cast<b8_t *>(lds + tile_at(k * BM + mm, ch)) = q[k];
            }
        }
#pragma unroll
        for (int i = 0; i < BN * BR / 32 / kThreads; ++i) {
            const int u = i * kThreads + threadIdx.x;
            const int nn = u % (BN / 4) * 4, rr = u / (BN / 4) * 8;
            const int col = min(n0 + nn, a.stride - 4);
            unsigned q[8];
            float sc[8];
#pragma unroll
            for (int y = 0; y < 8; ++y) {
                const int64_t r = r0 + rr + y, rc = worker * a.r + min(r, a.r - 1);
                q[y] = *reinterpret_cast<const unsigned *>(a.b.codes + rc * a.stride + col);
                const float e = scale_of(a.b.exps[rc * a.b.groups + (a.b.groups > 1 ? col / kGroup : 0)]);
                sc[y] = r < a.r ? e : 0.0f;
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                b8_t v;
#pragma unroll
                for (int y = 0; y < 8; ++y) v[y] = (__bf16)(code_at(q[y], x) * sc[y]);
                *reinterpret_cast<b8_t *>(ldb + tile_at(nn + x, rr / 8)) = v;
            }
        }
        __syncthreads();
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            b8_t bf[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j)
                bf[j] = *reinterpret_cast<const b8_t *>(
                    ldb + tile_at(wn + j * 16 + lane % 16, ks * 4 + lane / 16));
#pragma unroll
            for (int k = P - 1; k >= 0; --k)   // the smallest part first
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    const b8_t af = *reinterpret_cast<const b8_t *>(
                        lds + tile_at(k * BM + wm + i * 16 + lane % 16, ks * 4 + lane / 16));
#pragma unroll
                    for (int j = 0; j < TN; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf[j], af, acc[i][j], 0, 0, 0);
                }
        }
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t m = m0 + wm + i * 16 + lane % 16;
        if (m >= a.m) continue;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int c0 = n0 + wn + j * 16 + lane / 16 * 4;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (c0 + k >= a.cols) continue;
                if (a.split > 1)
                    a.partial[(((int64_t)part * a.workers + worker) * a.m + m) * a.cols + c0 + k] = acc[i][j][k];
                else
                    row_at<O>(a.out, worker, m)[c0 + k] = (O)acc[i][j][k];
            }
        }
    }
}

// The sum of the parts of a split product, in ascending order.
__global__ __launch_bounds__(256) void join_kernel(GradArgs a) {
    const int64_t per = a.m * a.cols, all = per * a.workers;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        float v = 0.0f;
        for (int s = 0; s < a.split; ++s) v += a.partial[s * all + i];
        const int64_t worker = i / per, at = i - worker * per, m = at / a.cols;
        row_at<float>(a.out, worker, m)[at - m * a.cols] = v;
    }
}

// ---- host side -------------------------------------------------------------------------

thread_local char g_error[256];

int refuse(const char *format, ...) __attribute__((format(printf, 1, 2)));
int refuse(const char *format, ...) {
    va_list ap;
    va_start(ap, format);
    std::vsnprintf(g_error, sizeof g_error, format, ap);
    va_end(ap);
    return RELAYSUM_ERR_INVALID_ARG;
}

int device_error(const char *what, hipError_t e) {
    std::snprintf(g_error, sizeof g_error, "%s: %s", what, hipGetErrorString(e));
    return RELAYSUM_ERR_DEVICE;
}

int done(const char *what) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return device_error(what, e);
    g_error[0] = '\0';
    return RELAYSUM_OK;
}

int64_t code_stride(int64_t width) { return (width + kGroup - 1) / kGroup * kGroup; }

size_t type_bytes(int32_t type) { return type == RELAYSUM_FLOAT ? 4 : 2; }

// One array of a call: where it lies, for the checks that follow.
struct Span {
    const char *name;
    const char *p;
    size_t bytes;
    bool out;
    int64_t ws, rs;   // strides of typed rows; -1 for other arrays
};

// Collects a call's arrays and says what is wrong with them.
struct Call {
    Span spans[12];
    int count = 0;
    int code = RELAYSUM_OK;
    int device = 0;
    // Whether rows may be written over rows read with the same strides: the
    // threads of a row read all of it before they write.
    bool in_place = false;

    void fail(int c) { code = code == RELAYSUM_OK ? c : code; }

    bool sizes(int32_t n, int64_t rows, int64_t width, const char *what) {
        if (n < 1 || n > RELAYSUM_MAX_WORKERS)
            fail(refuse("n must be in 1..%d", RELAYSUM_MAX_WORKERS));
        else if (rows < 0 || rows > (int64_t)1 << 40)
            fail(refuse("%s must be in 0..2^40", what));
        else if (width < 1 || width > kMaxWidth)
            fail(refuse("the width must be in 1..%d", (int)kMaxWidth));
        else if ((__int128)n * (rows + 1) * width > ((__int128)1 << 50))
            fail(refuse("n * %s * width is more than 2^50", what));
        return code == RELAYSUM_OK;
    }

    // The product's result has a row of `channels` entries for each token.
    bool product(int32_t n, int64_t tokens, int64_t width, int64_t channels) {
        if (!sizes(n, tokens, width, "tokens")) return false;
        if (channels < 1 || channels > kMaxChannels)
            fail(refuse("channels must be in 1..%d", (int)kMaxChannels));
        else if ((__int128)n * (tokens + width) * channels > ((__int128)1 << 50))
            fail(refuse("n * (tokens + width) * channels is more than 2^50"));
        return code == RELAYSUM_OK;
    }

    void span(const char *name, const void *p, size_t bytes, size_t align, bool out,
              int64_t ws = -1, int64_t rs = -1) {
        if (code != RELAYSUM_OK || !bytes) return;
        if (!p)
            fail(refuse("%s must not be NULL", name));
        else if ((uintptr_t)p % align)
            fail(refuse("%s must be %d-byte aligned", name, (int)align));
        else
            spans[count++] = Span{name, static_cast<const char *>(p), bytes, out, ws, rs};
    }

    void rows(const char *name, const relaysum_rows *r, int32_t n, int64_t rows, int64_t width,
              bool out) {
        if (code != RELAYSUM_OK) return;
        if (!r) return fail(refuse("%s must not be NULL", name));
        if (r->type < RELAYSUM_FLOAT || r->type > RELAYSUM_HALF)
            return fail(refuse("%s: unknown type %d", name, r->type));
        const int64_t ws = n > 1 ? r->worker_stride : 0, rs = rows > 1 ? r->row_stride : 0;
        const int64_t most = (int64_t)1 << 44;
        if (ws < 0 || rs < 0 || (n > 1 && ws > most / n) || (rows > 1 && rs > most / rows))
            return fail(refuse("%s: a stride is negative or reaches past 2^44 entries", name));
        if (!rows) return;
        // Rows that are written must not share entries: they follow one
        // another within a worker, or the workers follow one another in a row.
        const bool within = (rows == 1 || rs >= width) && (n == 1 || ws >= (rows - 1) * rs + width);
        const bool across = (n == 1 || ws >= width) && (rows == 1 || rs >= (n - 1) * ws + width);
        if (out && !within && !across) return fail(refuse("%s: its rows overlap", name));
        const size_t entries = (size_t)((n - 1) * ws + (rows - 1) * rs + width);
        span(name, r->data, entries * type_bytes(r->type), type_bytes(r->type), out, ws, rs);
    }

    void packed(const char *name, const relaysum_packed *p, int32_t n, int64_t rows, int64_t width,
                bool out) {
        if (code != RELAYSUM_OK) return;
        if (!p) return fail(refuse("%s must not be NULL", name));
        if (p->group != 0 && p->group != kGroup)
            return fail(refuse("%s: the group must be 0 (whole rows) or %d", name, kGroup));
        const int64_t stride = code_stride(width);
        span(name, p->codes, (size_t)n * rows * stride, 16, out);
        span(name, p->exps, (size_t)n * rows * (p->group ? stride / kGroup : 1), 1, out);
    }

    // Overlaps, then each array against the allocation that holds it.
    bool ready() {
        if (code != RELAYSUM_OK) return false;
        for (int i = 0; i < count; ++i)
            for (int j = 0; j < i; ++j) {
                const Span &a = spans[i], &b = spans[j];
                if (!(a.out || b.out) || a.p >= b.p + b.bytes || b.p >= a.p + a.bytes) continue;
                if (in_place && a.out != b.out && a.p == b.p && a.bytes == b.bytes && a.ws >= 0 &&
                    a.ws == b.ws && a.rs == b.rs)
                    continue;
                fail(refuse("%s and %s share memory", b.name, a.name));
                return false;
            }
        hipError_t e = hipGetDevice(&device);
        if (e != hipSuccess) {
            fail(device_error("hipGetDevice", e));
            return false;
        }
        for (int i = 0; i < count; ++i)
            if (!on_device(spans[i].p, spans[i].bytes)) {
                fail(refuse("%s does not lie within one allocation of device memory on the current GPU",
                            spans[i].name));
                return false;
            }
        return true;
    }

    // hipPointerGetAttributes gives the memory's kind and GPU,
    // hipMemGetAddressRange the allocation (memory it cannot place, such as
    // mappings made with the virtual-memory calls, passes on its kind and GPU).
    bool on_device(const void *p, size_t bytes) const {
        hipPointerAttribute_t at;
        if (hipPointerGetAttributes(&at, p) != hipSuccess) {
            (void)hipGetLastError();
            return false;
        }
        if (at.type != hipMemoryTypeDevice && at.type != hipMemoryTypeManaged) return false;
        if (at.type == hipMemoryTypeDevice && at.device != device) return false;
        hipDeviceptr_t base = nullptr;
        size_t size = 0;
        if (hipMemGetAddressRange(&base, &size, const_cast<void *>(p)) != hipSuccess || !base) {
            (void)hipGetLastError();
            return true;
        }
        const uintptr_t b = (uintptr_t)base, q = (uintptr_t)p;
        return q >= b && q - b <= size && bytes <= size - (q - b);
    }
};

Rows rows_of(const relaysum_rows *r, int32_t n, int64_t rows) {
    if (!r) return Rows{nullptr, 0, 0};
    return Rows{static_cast<char *>(r->data), n > 1 ? r->worker_stride : 0, rows > 1 ? r->row_stride : 0};
}

Packed packed_of(const relaysum_packed *p, int64_t width) {
    if (!p) return Packed{nullptr, nullptr, 0};
    return Packed{p->codes, p->exps, (int32_t)(p->group ? code_stride(width) / kGroup : 1)};
}

// Whether a row has one exponent; up to 128 entries both groups have.
bool whole_rows(const relaysum_packed *p, int64_t width) { return p->group == 0 || width <= kGroup; }

template <int V>
using Int = std::integral_constant<int, V>;

// Calls f with the row layout for a row of `stride` codes: the threads that
// share a row and the 8-entry chunks each of them holds.
template <typename F>
void with_layout(int64_t stride, F f) {
    const int64_t chunks = stride / 8;
    if (chunks <= 16) f(Int<16>(), Int<1>());
    else if (chunks <= 64) f(Int<64>(), Int<1>());
    else if (chunks <= 128) f(Int<64>(), Int<2>());
    else if (chunks <= 256) f(Int<64>(), Int<4>());
    else if (chunks <= 512) f(Int<256>(), Int<2>());
    else if (chunks <= 1024) f(Int<256>(), Int<4>());
    else if (chunks <= 2048) f(Int<1024>(), Int<2>());
    else f(Int<1024>(), Int<4>());
}

template <typename F>
void with_type(int32_t type, F f) {
    if (type == RELAYSUM_FLOAT) f((float)0);
    else if (type == RELAYSUM_BFLOAT) f((__bf16)0);
    else f((_Float16)0);
}

constexpr int64_t kMaxBlocks = 0x3fffff;   // a launch has fewer than 2^32 threads
constexpr int64_t kMaxGrid = 1 << 20;   // workgroups; kernels over rows loop beyond

unsigned row_grid(int64_t rows, int per) {
    return (unsigned)std::min<int64_t>((rows + per - 1) / per, kMaxGrid);
}

int chunks_layout(int64_t stride) { return stride <= 128 ? 16 : stride <= 2048 ? 64 : 256; }

// Workgroups per worker of the norm's gradient: enough for four on each CU, no
// more than one for 16 rows.
int norm_parts(int32_t n, int64_t rows) {
    const int64_t want = (4 * kCus + n - 1) / n;
    return (int)std::max<int64_t>(1, std::min<int64_t>(want, (rows + 15) / 16));
}

constexpr int kTile = 128;

int64_t tiles(int64_t size, int64_t tile) { return (size + tile - 1) / tile; }

// Parts of the contracted axis of dW: where the result has fewer tiles than
// there are CUs, so many that every CU has one, each at least 8 steps of 64 tokens.
int weight_split(int32_t n, int64_t tokens, int64_t width, int64_t channels) {
    const int64_t have = n * tiles(width, kTile) * tiles(channels, kTile);
    const int64_t want = (kCus + have - 1) / have;
    return (int)std::max<int64_t>(1, std::min<int64_t>(want, tokens / 512));
}

}  // namespace

extern "C" {

const char *relaysum_layer_error(void) { return g_error; }

int64_t relaysum_packed_stride(int64_t width) {
    return width < 1 || width > kMaxWidth ? -1 : code_stride(width);
}

int relaysum_pack(int32_t n, int64_t rows, int64_t width, const relaysum_rows *v,
                  const relaysum_packed *out, void *hip_stream) {
    Call c;
    if (c.sizes(n, rows, width, "rows")) {
        c.rows("v", v, n, rows, width, false);
        c.packed("out", out, n, rows, width, true);
    }
    if (!c.ready()) return c.code;
    if (rows == 0) return done("relaysum_pack");
    PackArgs a{rows_of(v, n, rows), packed_of(out, width), rows, n * rows, (int32_t)width,
               (int32_t)code_stride(width)};
    const bool grouped = out->group != 0;
    with_type(v->type, [&](auto zero) {
        using T = decltype(zero);
        with_layout(a.stride, [&](auto tpr, auto chunks) {
            constexpr int TPR = decltype(tpr)::value, J = decltype(chunks)::value;
            const unsigned grid = row_grid(a.total, block_of(TPR) / TPR);
            hipLaunchKernelGGL(HIP_KERNEL_NAME(grouped ? pack_kernel<T, TPR, J, true> : pack_kernel<T, TPR, J, false>),
                               dim3(grid), dim3(block_of(TPR)), 0, (hipStream_t)hip_stream, a);
        });
    });
    return done("relaysum_pack");
}

int relaysum_unpack(int32_t n, int64_t rows, int64_t width, const relaysum_packed *p,
                    const relaysum_rows *out, void *hip_stream) {
    Call c;
    if (c.sizes(n, rows, width, "rows")) {
        c.packed("p", p, n, rows, width, false);
        c.rows("out", out, n, rows, width, true);
    }
    if (!c.ready()) return c.code;
    if (rows == 0) return done("relaysum_unpack");
    PackArgs a{rows_of(out, n, rows), packed_of(p, width), rows, n * rows, (int32_t)width,
               (int32_t)code_stride(width)};
    with_type(out->type, [&](auto zero) {
        using T = decltype(zero);
        const int tpr = chunks_layout(a.stride);
        const dim3 grid(row_grid(a.total, 256 / tpr));
        const hipStream_t st = (hipStream_t)hip_stream;
        if (tpr == 16) hipLaunchKernelGGL(HIP_KERNEL_NAME(unpack_kernel<T, 16>), grid, dim3(256), 0, st, a);
        else if (tpr == 64) hipLaunchKernelGGL(HIP_KERNEL_NAME(unpack_kernel<T, 64>), grid, dim3(256), 0, st, a);
        else hipLaunchKernelGGL(HIP_KERNEL_NAME(unpack_kernel<T, 256>), grid, dim3(256), 0, st, a);
    });
    return done("relaysum_unpack");
}

int relaysum_rmsnorm(int32_t n, int64_t tokens, int64_t width, const relaysum_rows *h,
                     const relaysum_rows *residual, const float *weight, int64_t weight_stride,
                     float eps, const relaysum_rows *sum, const relaysum_packed *y, float *rstd,
                     const relaysum_packed *saved, void *hip_stream) {
    Call c;
    c.in_place = true;
    if (c.sizes(n, tokens, width, "tokens")) {
        c.rows("h", h, n, tokens, width, false);
        if (!residual != !sum)
            c.fail(refuse("residual and sum come together"));
        else if (residual && h && (residual->type != h->type || sum->type != h->type))
            c.fail(refuse("h, residual and sum must have one type"));
        if (residual) {
            c.rows("residual", residual, n, tokens, width, false);
            c.rows("sum", sum, n, tokens, width, true);
        }
        if (c.code == RELAYSUM_OK && n > 1 && (weight_stride < 0 || weight_stride > ((int64_t)1 << 44) / n))
            c.fail(refuse("weight_stride is negative or reaches past 2^44 entries"));
        const int64_t wspan = (n > 1 ? (n - 1) * weight_stride : 0) + width;
        c.span("weight", weight, c.code == RELAYSUM_OK ? (size_t)wspan * 4 : 0, 4, false);
        if (y && !whole_rows(y, width)) c.fail(refuse("y is packed by whole rows (group 0)"));
        c.packed("y", y, n, tokens, width, true);
        c.span("rstd", rstd, (size_t)n * tokens * 4, 4, true);
        if (saved) c.packed("saved", saved, n, tokens, width, true);
        if (saved && whole_rows(saved, width) && width > kGroup) c.fail(refuse("saved is packed in groups of %d", kGroup));
        if (!(eps >= 0.0f)) c.fail(refuse("eps must not be negative"));
    }
    if (!c.ready()) return c.code;
    if (tokens == 0) return done("relaysum_rmsnorm");
    NormArgs a{rows_of(h, n, tokens), rows_of(residual, n, tokens), rows_of(sum, n, tokens),
               packed_of(y, width), packed_of(saved, width), weight, rstd,
               n > 1 ? weight_stride : 0, tokens, n * tokens, (int32_t)width,
               (int32_t)code_stride(width), eps};
    with_type(h->type, [&](auto zero) {
        using T = decltype(zero);
        with_layout(a.stride, [&](auto tpr, auto chunks) {
            constexpr int TPR = decltype(tpr)::value, J = decltype(chunks)::value;
            const dim3 grid(row_grid(a.total, block_of(TPR) / TPR)), block(block_of(TPR));
            const hipStream_t st = (hipStream_t)hip_stream;
            if (residual && saved)
                hipLaunchKernelGGL(HIP_KERNEL_NAME(norm_kernel<T, TPR, J, true, true>), grid, block, 0, st, a);
            else if (residual)
                hipLaunchKernelGGL(HIP_KERNEL_NAME(norm_kernel<T, TPR, J, true, false>), grid, block, 0, st, a);
            else if (saved)
                hipLaunchKernelGGL(HIP_KERNEL_NAME(norm_kernel<T, TPR, J, false, true>), grid, block, 0, st, a);
            else
                hipLaunchKernelGGL(HIP_KERNEL_NAME(norm_kernel<T, TPR, J, false, false>), grid, block, 0, st, a);
        });
    });
    return done("relaysum_rmsnorm");
}

int64_t relaysum_rmsnorm_workspace(int32_t n, int64_t tokens, int64_t width) {
    Call c;
    if (!c.sizes(n, tokens, width, "tokens")) return -1;
    const int parts = norm_parts(n, tokens);
    return parts > 1 ? (int64_t)n * parts * width * 4 : 0;
}

int relaysum_rmsnorm_backward(int32_t n, int64_t tokens, int64_t width, const relaysum_rows *dy,
                              const relaysum_rows *dsum, const relaysum_packed *saved,
                              const float *rstd, const float *weight, int64_t weight_stride,
                              const relaysum_rows *ds, const relaysum_rows *weight_grad,
                              void *workspace, size_t workspace_bytes, void *hip_stream) {
    Call c;
    c.in_place = true;
    int parts = 1;
    if (c.sizes(n, tokens, width, "tokens")) {
        parts = norm_parts(n, tokens);
        c.rows("dy", dy, n, tokens, width, false);
        if (dy && ds && (dy->type != ds->type || (dsum && dsum->type != dy->type)))
            c.fail(refuse("dy, dsum and ds must have one type"));
        if (dsum) c.rows("dsum", dsum, n, tokens, width, false);
        c.packed("saved", saved, n, tokens, width, false);
        c.span("rstd", rstd, (size_t)n * tokens * 4, 4, false);
        if (c.code == RELAYSUM_OK && n > 1 && (weight_stride < 0 || weight_stride > ((int64_t)1 << 44) / n))
            c.fail(refuse("weight_stride is negative or reaches past 2^44 entries"));
        const int64_t wspan = (n > 1 ? (n - 1) * weight_stride : 0) + width;
        c.span("weight", weight, c.code == RELAYSUM_OK ? (size_t)wspan * 4 : 0, 4, false);
        c.rows("ds", ds, n, tokens, width, true);
        c.rows("weight_grad", weight_grad, n, 1, width, true);
        if (weight_grad && weight_grad->type != RELAYSUM_FLOAT)
            c.fail(refuse("weight_grad must be of type float"));
        const size_t need = parts > 1 ? (size_t)n * parts * width * 4 : 0;
        if (need > workspace_bytes)
            c.fail(refuse("the workspace has %zu bytes, %zu are needed", workspace_bytes, need));
        c.span("workspace", workspace, need, 4, true);
    }
    if (!c.ready()) return c.code;
    const Rows grad = rows_of(weight_grad, n, 1);
    NormGradArgs a{rows_of(dy, n, tokens), rows_of(dsum, n, tokens), rows_of(ds, n, tokens),
                   packed_of(saved, width), weight, rstd,
                   parts > 1 ? static_cast<float *>(workspace) : reinterpret_cast<float *>(grad.data),
                   n > 1 ? weight_stride : 0, parts > 1 ? parts * width : grad.ws, tokens,
                   (int32_t)width, (int32_t)code_stride(width), parts};
    if ((int64_t)n * parts > kMaxBlocks) return refuse("n is too large");
    const hipStream_t st = (hipStream_t)hip_stream;
    with_type(dy->type, [&](auto zero) {
        using T = decltype(zero);
        with_layout(a.stride, [&](auto tpr, auto chunks) {
            constexpr int TPR = decltype(tpr)::value, J = decltype(chunks)::value;
            const dim3 grid((unsigned)(n * parts)), block(block_of(TPR));
            if (dsum)
                hipLaunchKernelGGL(HIP_KERNEL_NAME(norm_grad_kernel<T, TPR, J, true>), grid, block, 0, st, a);
            else
                hipLaunchKernelGGL(HIP_KERNEL_NAME(norm_grad_kernel<T, TPR, J, false>), grid, block, 0, st, a);
        });
    });
    if (parts > 1)
        hipLaunchKernelGGL(sum_parts_kernel, dim3((unsigned)(n * ((width + 255) / 256))), dim3(256), 0, st,
                           a.partial, reinterpret_cast<float *>(grad.data), grad.ws, parts, (int32_t)width);
    return done("relaysum_rmsnorm_backward");
}

int relaysum_linear(int32_t n, int64_t tokens, int64_t width, int64_t channels,
                    const relaysum_packed *x, const relaysum_packed *w, const relaysum_rows *y,
                    void *hip_stream) {
    Call c;
    if (c.product(n, tokens, width, channels)) {
        c.packed("x", x, n, tokens, width, false);
        c.packed("w", w, n, channels, width, false);
        if (c.code == RELAYSUM_OK && !(whole_rows(x, width) && whole_rows(w, width)))
            c.fail(refuse("the product takes rows packed whole (group 0)"));
        c.rows("y", y, n, tokens, channels, true);
    }
    if (!c.ready()) return c.code;
    if (tokens == 0) return done("relaysum_linear");
    LinearArgs a{packed_of(x, width), packed_of(w, width), rows_of(y, n, tokens), tokens,
                 (int32_t)width, (int32_t)code_stride(width), (int32_t)channels,
                 tiles(tokens, kTile), (int32_t)tiles(channels, kTile)};
    const int64_t grid = n * a.tiles_m * a.tiles_n;
    if (grid > kMaxBlocks) return refuse("the result has more than %d tiles", (int)kMaxBlocks);
    with_type(y->type, [&](auto zero) {
        using T = decltype(zero);
        hipLaunchKernelGGL(HIP_KERNEL_NAME(linear_kernel<T, kTile, kTile, 2, 2>), dim3((unsigned)grid), dim3(256),
                           0, (hipStream_t)hip_stream, a);
    });
    return done("relaysum_linear");
}

int relaysum_linear_backward_input(int32_t n, int64_t tokens, int64_t width, int64_t channels,
                                   const relaysum_rows *dy, const relaysum_packed *w,
                                   const relaysum_rows *dx, void *hip_stream) {
    Call c;
    if (c.product(n, tokens, width, channels)) {
        c.rows("dy", dy, n, tokens, channels, false);
        c.packed("w", w, n, channels, width, false);
        c.rows("dx", dx, n, tokens, width, true);
        if (c.code == RELAYSUM_OK && dy->type != dx->type)
            c.fail(refuse("dy and dx must have one type"));
    }
    if (!c.ready()) return c.code;
    if (tokens == 0) return done("relaysum_linear_backward_input");
    GradArgs a{rows_of(dy, n, tokens), packed_of(w, width), rows_of(dx, n, tokens), nullptr,
               tokens, channels, (int32_t)width, (int32_t)code_stride(width), 1,
               tiles(tokens, kTile), (int32_t)tiles(width, kTile), n};
    const int64_t grid = n * a.tiles_m * a.tiles_n;
    if (grid > kMaxBlocks) return refuse("the result has more than %d tiles", (int)kMaxBlocks);
    with_type(dy->type, [&](auto zero) {
        using T = decltype(zero);
        hipLaunchKernelGGL(HIP_KERNEL_NAME(grad_kernel<T, T, false, kTile, kTile, 2, 2>), dim3((unsigned)grid),
                           dim3(256), 0, (hipStream_t)hip_stream, a);
    });
    return done("relaysum_linear_backward_input");
}

int64_t relaysum_linear_workspace(int32_t n, int64_t tokens, int64_t width, int64_t channels) {
    Call c;
    if (!c.product(n, tokens, width, channels)) return -1;
    const int split = weight_split(n, tokens, width, channels);
    return split > 1 ? (int64_t)split * n * width * channels * 4 : 0;
}

int relaysum_linear_backward_weight(int32_t n, int64_t tokens, int64_t width, int64_t channels,
                                    const relaysum_rows *dy, const relaysum_packed *x,
                                    const relaysum_rows *weight_grad, void *workspace,
                                    size_t workspace_bytes, void *hip_stream) {
    Call c;
    int split = 1;
    if (c.product(n, tokens, width, channels)) {
        c.rows("dy", dy, n, tokens, channels, false);
        c.packed("x", x, n, tokens, width, false);
        c.rows("weight_grad", weight_grad, n, channels, width, true);
        if (c.code == RELAYSUM_OK && weight_grad->type != RELAYSUM_FLOAT)
            c.fail(refuse("weight_grad must be of type float"));
        split = weight_split(n, tokens, width, channels);
        const size_t need = split > 1 ? (size_t)split * n * width * channels * 4 : 0;
        if (need > workspace_bytes)
            c.fail(refuse("the workspace has %zu bytes, %zu are needed", workspace_bytes, need));
        c.span("workspace", workspace, need, 16, true);
    }
    if (!c.ready()) return c.code;
    GradArgs a{rows_of(dy, n, tokens), packed_of(x, width), rows_of(weight_grad, n, channels),
               static_cast<float *>(workspace), channels, tokens, (int32_t)width,
               (int32_t)code_stride(width), split, tiles(channels, kTile), (int32_t)tiles(width, kTile), n};
    const int64_t grid = n * split * a.tiles_m * a.tiles_n;
    if (grid > kMaxBlocks) return refuse("the result has more than %d tiles", (int)kMaxBlocks);
    const hipStream_t st = (hipStream_t)hip_stream;
    with_type(dy->type, [&](auto zero) {
        using T = decltype(zero);
        hipLaunchKernelGGL(HIP_KERNEL_NAME(grad_kernel<T, float, true, kTile, kTile, 2, 2>), dim3((unsigned)grid),
                           dim3(256), 0, st, a);
    });
    if (split > 1) {
        const int64_t all = (int64_t)n * channels * width;
        hipLaunchKernelGGL(join_kernel, dim3((unsigned)std::min<int64_t>((all + 255) / 256, 16 * kCus)), dim3(256),
                           0, st, a);
    }
    return done("relaysum_linear_backward_weight");
}

}  // extern "C"
