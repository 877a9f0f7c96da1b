// Layer operators on CDNA4 (gfx950): what n workers, each with weights of its
// own, compute between two RelaySum rounds.  RMS norm with the residual's
// addition into 8-bit rows, its gradient, products of 8-bit rows and their
// gradients, and packing; the C ABI is in relaysum.h.  (With them a feed-forward
// sub-layer is complete but for its activation; there is no attention.)
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

#include "layer_plan.hpp"
#include "relaysum.h"

using namespace layer_plan;

namespace {

constexpr int kWave = 64;
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
    return float_of(e == kNotANumber ? 0u : (unsigned)(127 - e) << 23);
}

__device__ __forceinline__ float scale_of(int e) {
    return float_of(e == kNotANumber ? 0x7fc00000u : (unsigned)(127 + e) << 23);
}

__device__ __forceinline__ u2_t codes8(const float (&v)[8], float inv) {
    unsigned w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        w[i / 4] |= ((unsigned)__float2int_rn(v[i] * inv) & 0xffu) << (8 * (i % 4));
    return u2_t{w[0], w[1]};
}

// Two floats as two bfloat16, the first in the lower half.
__device__ __forceinline__ unsigned bf16_pair(float a, float b) {
    typedef float f2_t __attribute__((ext_vector_type(2)));
    typedef __bf16 b2_t __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(unsigned, __builtin_convertvector((f2_t{a, b}), b2_t));
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

// Packing: one pass, the row in registers between its maximum and its codes.
// Bound by memory: an entry's bytes in, one byte out.  16 x 4096 x 2048
// bfloat16 by 128: 403 MB in 73 us, 5.5 TB/s (a flat copy: 6.5); a weight of
// 16 workers, 2048 x 1024 out of model rows of odd length: 168 MB in 25 us.
// Rows of up to 128 entries take 16 lanes, up to 2048 a wave, wider ones a
// workgroup: the fewer threads share a row, the fewer steps its maximum takes,
// but 4 chunks of 8 entries a thread are what the registers hold well.
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

// Unpacking: a byte in, an entry out; 403 MB in 70 us, 5.8 TB/s.
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

// 1 / sqrt(mean(s^2) + eps) of a row whose squares, or their sum, may lie
// outside binary32's range: s is scaled by the power of two that brings the
// row's largest entry, or the root of eps if that is larger, to 1 or 2.  Leaves
// the scaled row in s and returns what it is to be multiplied by; rstd is that
// of the row as it was, an infinity where it passes the range (rows of numbers
// below 2^-128).  Rows of zeros, and those with a NaN or an infinity, stay.
// Every thread of the row takes part.
template <int TPR, int J>
__device__ __forceinline__ float scaled_rstd(float (&s)[J][8], float width, float eps, float &rstd,
                                             float *redf, unsigned *redu) {
    const unsigned most = row_reduce<TPR, unsigned, pick_max>(max_bits(s), redu);
    if (most == 0 || most >= 0x7f800000u) return rstd;
    const int p = max(ilogbf(float_of(most)), ilogbf(eps) >> 1);
    float sq = 0.0f;
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            s[j][i] = ldexpf(s[j][i], -p);
            sq = fmaf(s[j][i], s[j][i], sq);
        }
    sq = row_reduce<TPR, float, pick_sum>(sq, redf);
    const float inv = 1.0f / sqrtf(sq / width + ldexpf(eps, -2 * p));
    rstd = ldexpf(inv, -p);
    return inv;
}

// s = h + r, rounded to the rows' type because that is what the stream goes on
// with; y = s * rstd * w is not rounded before it is packed.  One pass: the row
// stays in registers between the sum of squares and the codes.  Bound by
// memory: 16 x 2048 x 1024 bfloat16 with s kept reads 4 bytes of an entry and
// writes 4: 268 MB in 45 us, 6.0 TB/s (37 us without s, 6.3; a flat copy: 6.5).
// The weights, a row for each worker, come from the caches.
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
        const float mean = sq / (float)a.width + a.eps;
        float rstd = 1.0f / sqrtf(mean), inv = rstd;
        if (KEEP) write_grouped<TPR, J>(a.saved, row, a.stride, lane, s);
        // Squares that were lost below 2^-149 are less than 2^-50 of 2^-100.
        if (!(mean >= 0x1p-100f && mean < INFINITY))
            inv = scaled_rstd<TPR, J>(s, (float)a.width, a.eps, rstd, redf, redu);
        if (lane == 0) a.rstd[row] = rstd;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int at = (lane + j * TPR) * 8;
            float wv[8];
            load8(w + at, a.width - at, wv);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[j][i] = s[j][i] * inv * wv[i];
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

// ds = dsum + rstd * (u - xh * mean(u * xh)), u = dy * w, xh = rstd * s, and this
// part's share of dw = sum of dy * xh.  A workgroup owns every parts-th block of
// rows of one worker: threads keep their columns' weights and sums of dy * xh
// in registers over all of them, so dw costs no memory traffic but one row for
// each workgroup.  Bound by memory: 16 x 2048 x 1024 bfloat16, 7 bytes of an
// entry, 235 MB in 40 us with the sum of the parts (5 us of it), 5.9 TB/s.
// From 16385 entries on a row does not fit the 128 registers that 1024 threads
// have each, and part of it goes to scratch: 4 x 512 x 32768 453 us, 1.0 TB/s
// (x 16384: 46 us, 5.1).
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

// out[i][c] = sum over parts of partial[i][p][c].  A workgroup has 32 columns
// of one worker and 8 sums of every eighth part each, added in a fixed order,
// so equal inputs give equal bits.
__global__ __launch_bounds__(256) void sum_parts_kernel(const float *partial, float *out,
                                                        int64_t out_stride, int32_t parts,
                                                        int32_t width) {
    __shared__ float sums[8][32];
    const unsigned per = (width + 31) / 32;
    const int64_t worker = blockIdx.x / per;
    const int lane = threadIdx.x % 32, group = threadIdx.x / 32;
    const int c = (int)(blockIdx.x % per) * 32 + lane;
    float v = 0.0f;
    if (c < width) {
        const float *p = partial + worker * parts * (int64_t)width + c;
#pragma unroll 4
        for (int k = group; k < parts; k += 8) v += p[(int64_t)k * width];
    }
    sums[group][lane] = v;
    __syncthreads();
    if (group == 0 && c < width) {
#pragma unroll
        for (int k = 1; k < 8; ++k) v += sums[k][lane];
        out[worker * out_stride + c] = v;
    }
}

// ---- products ------------------------------------------------------------------------
//
// LDS tiles of both products: rows of 128 bytes (128 codes, or 64 bfloat16 of
// the contracted axis) as 8 chunks of 16 bytes; chunk c of row r lies at
// position c ^ swizzle(r).  The swizzle takes row bits 1..5 to 3 bits so that
// bits {1,2,3}, {1,4,5}, {1,3,4} and {2,3,4} each reach all 8 positions (bit 0
// moves a row by half of the 64 banks): lanes that read one chunk of 16
// neighbouring rows, or of 4 times 4 rows 16 or 8 apart, touch different banks,
// and so do lanes that write one chunk of rows 4 apart.
__device__ __forceinline__ int swizzle(int row) {
    return ((row >> 1) & 7) ^ (((row >> 4) & 1) * 3) ^ (((row >> 5) & 1) << 2);
}
__device__ __forceinline__ int tile_at(int row, int chunk) {
    return row * 128 + ((chunk ^ swizzle(row)) << 4);
}

// Which result a matrix instruction's row r of tile j is: tiles go by Q, and a
// lane's 4 rows of each of them are neighbours, so that a lane ends up with
// 4 * Q entries in a row of the result, 32 bytes of it (dW of 16 x 2048 x 4096
// -> 1024 takes 7% more with 64 bytes, the product in bfloat16 6% more with 16).
template <typename O>
constexpr int kFours = 8 / (int)sizeof(O);
template <int Q>
__device__ __forceinline__ int tile_row(int j, int r) {
    return j / Q * 16 * Q + r / 4 * 4 * Q + j % Q * 4 + r % 4;
}

// A lane's place in a tile for reading 16 of its rows (tile_row<Q> of tile 0,
// chunk lane / 16), and from there the place for tile j and chunk 4 * ks +
// lane / 16: the swizzle is linear in the row's bits, so the two differ by a
// constant number of rows and a constant change of the chunk's bits.  `fresh`
// keeps the compiler from holding all of these sums in registers for the
// whole loop, which it has not got.
template <int Q>
__device__ __forceinline__ int read_at(int row0, int lane) {
    return tile_at(row0 + tile_row<Q>(0, lane % 16), lane / 16);
}
template <int Q>
__device__ __forceinline__ int moved(int at, int j, int ks) {
    const int row = tile_row<Q>(j, 0);
    return (at ^ ((ks * 4 ^ swizzle(row)) << 4)) + row * 128;
}
// From a chunk's place in a row that 4 divides to the same chunk x < 4 rows on.
__device__ __forceinline__ int column_at(int at, int x) { return (at ^ (swizzle(x) << 4)) + x * 128; }
__device__ __forceinline__ int fresh(int v) {
    asm volatile("" : "+v"(v));
    return v;
}

// 16 bytes for each lane from memory into LDS at `to` + 16 * lane, without
// registers in between; `to` is the same for the whole wave.
__device__ __forceinline__ void copy_to_lds(const void *from, char *to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                     (__attribute__((address_space(3))) void *)to, 16, 0, 0);
}

__device__ __forceinline__ void wait_for_copies() { __builtin_amdgcn_s_waitcnt(0x0f70); }   // vmcnt(0)

// Blocks go round the 8 XCDs; each takes a run of neighbouring tiles, which
// share rows in its L2.
__device__ __forceinline__ unsigned xcd_tile(unsigned block, unsigned blocks) {
    const unsigned run = blocks / 8, rest = blocks % 8, x = block % 8;
    return x * run + (x < rest ? x : rest) + block / 8;
}

// 4 * Q entries of a row of `cols`, from column c0 on.
template <int Q, typename O, typename V>
__device__ __forceinline__ void write_entries(O *row, int c0, int cols, const V *v) {
    O out[4 * Q];
#pragma unroll
    for (int k = 0; k < 4 * Q; ++k) out[k] = (O)v[k / 4][k % 4];
    if (c0 + 4 * Q <= cols) {
        __builtin_memcpy(row + c0, out, sizeof out);
    } else {
#pragma unroll
        for (int k = 0; k < 4 * Q; ++k)
            if (c0 + k < cols) row[c0 + k] = out[k];
    }
}

// Kinds of instructions for the scheduler's groups.
constexpr int kMfma = 0x8, kDsRead = 0x100;

struct LinearArgs {
    Packed x, w;
    Rows y;
    int32_t *partial;   // split > 1: [split][n][tokens][channels]
    int64_t tokens;
    int32_t stride, channels, split;
    int32_t tiles_m, tiles_n;
    int32_t workers;
};

// Y[t][c] = 2^(ex[t] + ew[c]) * sum_k qx[t][k] qw[c][k]: whole numbers until
// the one conversion (rounded to 24 bits from 2^24 on, then to the type).
//
// A step multiplies 128 codes of every row of the tile while the next 128 are
// copied into the other half of LDS.  With 256 x 256 results and 8 waves of
// 128 x 64 a step reads 192 KB of LDS, 768 cycles of it by the counters, and
// copies 64 KB in, for 2048 cycles of matrix instructions; reads of the second
// half of a step are placed among the products of the first.  Measured: 16 x 2048 x 1024 ->
// 4096 bfloat16 in 178 us, 1550 TOP/s; 4 x 8192 x 4096 -> 1024 in 115 us, 2400
// (the library's 8192^3 product of int8: 2030-2080).  The shorter one's matrix
// units are busy for 31% of the cycles: it writes 268 MB of results, at the end
// of every tile with nothing to compute beside; it reads 303 MB where X and W
// have 101, W once for every two rows of tiles, since tiles go along the
// channels first; and each step waits for its own copies, one step in flight.
// Two workgroups of 4 waves of 64 x 128 on a CU, one buffer each, took 3% more,
// 128 x 128 tiles 30%, 4 waves of 128 x 128 33%.
//
// Few tokens: tiles of 16 x 128 (4 to a CU), so that 16 workers' weights for
// one token are spread over all CUs: 25 MB in 5.1 us, 4.9 TB/s.  In between:
// 64 x 128 (3 to a CU).  plan_product has the rule.
template <int BM, int BN, int WM, int WN, int QMAX>
struct LinearTile {
    static constexpr int kThreads = 64 * WM * WN, kBytes = (BM + BN) * 128;
    static constexpr int TM = BM / WM / 16, TN = BN / WN / 16, Q = TN < QMAX ? TN : QMAX;
    static constexpr int kCopies = ((BM + BN) * 8 + kThreads - 1) / kThreads;
    static_assert(BM % 8 == 0 && BN % 8 == 0, "a wave's copy, 8 rows, is of one operand");

    // Starts the copies of 128 codes of every row of the tile.
    static __device__ __forceinline__ void fetch(const int8_t *x, const int8_t *w,
                                                 const unsigned (&at)[kCopies], char *lds) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            const int u = i * kThreads + wave * kWave;
            if ((BM + BN) * 8 % kThreads && u >= (BM + BN) * 8) break;
            copy_to_lds((u / 8 < BM ? x : w) + at[i], lds + u * 16);
        }
    }

    // xat, wat: read_at of the wave's first token and channel.
    static __device__ __forceinline__ void multiply(const char *lds, int xat, int wat, i4_t (&acc)[TM][TN]) {
        xat = fresh(xat);
        wat = fresh(wat);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            i4_t xf[TM], wf[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j) wf[j] = *reinterpret_cast<const i4_t *>(lds + moved<Q>(wat, j, ks));
#pragma unroll
            for (int i = 0; i < TM; ++i) xf[i] = *reinterpret_cast<const i4_t *>(lds + moved<1>(xat, i, ks));
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[j], xf[i], acc[i][j], 0, 0, 0);
        }
        // All of the first half's reads, then one more for every two products.
        __builtin_amdgcn_sched_group_barrier(kDsRead, TN + TM, 0);
#pragma unroll
        for (int q = 0; q < TM * TN / 2; ++q) {
            __builtin_amdgcn_sched_group_barrier(kMfma, 2, 0);
            __builtin_amdgcn_sched_group_barrier(kDsRead, 1, 0);
        }
    }
};

template <typename T, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN, 2) void linear_kernel(LinearArgs a) {
    using L = LinearTile<BM, BN, WM, WN, kFours<T>>;
    constexpr int TM = L::TM, TN = L::TN, Q = L::Q;
    __shared__ __align__(16) char lds[2 * L::kBytes];
    const unsigned tile = xcd_tile(blockIdx.x, gridDim.x);
    const unsigned per = (unsigned)a.tiles_m * a.tiles_n;
    const unsigned job = tile / per, in = tile % per;
    const int64_t worker = job / a.split;
    const int part = (int)(job % a.split);
    const int64_t m0 = (int64_t)(in / a.tiles_n) * BM;
    const int n0 = (int)(in % a.tiles_n) * BN;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);
    // Rows past the end repeat the last one; what they give is not stored.
    const int8_t *x = a.x.codes + (worker * a.tokens + m0) * a.stride;
    const int8_t *w = a.w.codes + (worker * a.channels + n0) * (int64_t)a.stride;
    const int last_m = (int)min(a.tokens - m0, (int64_t)BM) - 1, last_n = min(a.channels - n0, BN) - 1;
    unsigned at[L::kCopies];
#pragma unroll
    for (int i = 0; i < L::kCopies; ++i) {
        const int u = i * L::kThreads + threadIdx.x, r = u / 8 < BM ? u / 8 : u / 8 - BM;
        at[i] = (unsigned)min(r, u / 8 < BM ? last_m : last_n) * a.stride + (((u % 8) ^ swizzle(r)) << 4);
    }
    const int xat = read_at<1>(wm, lane), wat = BM * 128 + read_at<Q>(wn, lane);
    // This part's share of the width, in whole steps of 128 codes.
    const int steps = a.stride / 128;
    const int k1 = (int)((int64_t)steps * (part + 1) / a.split) * 128;
    int k0 = (int)((int64_t)steps * part / a.split) * 128, cur = 0;
    i4_t acc[TM][TN] = {};
    L::fetch(x + k0, w + k0, at, lds);
    for (k0 += 128; k0 <= k1; k0 += 128) {
        wait_for_copies();
        __syncthreads();
        if (k0 < k1) L::fetch(x + k0, w + k0, at, lds + (cur ^ L::kBytes));
        L::multiply(lds + cur, xat, wat, acc);
        cur ^= L::kBytes;
    }
    if (a.split > 1) {
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int64_t t = m0 + wm + i * 16 + lane % 16;
            if (t >= a.tokens) continue;
            int32_t *row = a.partial + (((int64_t)part * a.workers + worker) * a.tokens + t) * a.channels;
#pragma unroll
            for (int j0 = 0; j0 < TN; j0 += Q)
                write_entries<Q>(row, n0 + wn + tile_row<Q>(j0, lane / 16 * 4), a.channels, &acc[i][j0]);
        }
        return;
    }
    // A lane has 4 * Q neighbouring channels of one token in Q accumulators.
    const int64_t t0 = m0 + wm + lane % 16;
    int ex[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) ex[i] = a.x.exps[worker * a.tokens + min(t0 + i * 16, a.tokens - 1)];
#pragma unroll
    for (int j0 = 0; j0 < TN; j0 += Q) {
        const int c0 = n0 + wn + tile_row<Q>(j0, lane / 16 * 4);
        int ew[4 * Q];
#pragma unroll
        for (int k = 0; k < 4 * Q; ++k) ew[k] = a.w.exps[worker * a.channels + min(c0 + k, a.channels - 1)];
        // A whole number of at most 2^29 times 2^ex is a normal number, or 0,
        // up to ex = 98; the second factor then makes the one rounding that
        // can be left.
        int most = ex[0];
#pragma unroll
        for (int i = 1; i < TM; ++i) most = max(most, ex[i]);
        const bool wide = __any(most > 98);
        float sw[4 * Q];
#pragma unroll
        for (int k = 0; k < 4 * Q; ++k) sw[k] = scale_of(ew[k]);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            T v[4 * Q];
            if (wide) {
#pragma unroll
                for (int k = 0; k < 4 * Q; ++k) {
                    const float f = ldexpf((float)acc[i][j0 + k / 4][k % 4], ex[i] + ew[k]);
                    v[k] = (T)(ex[i] == kNotANumber || ew[k] == kNotANumber ? float_of(0x7fc00000u) : f);
                }
            } else {
                const float sx = scale_of(ex[i]);
#pragma unroll
                for (int k = 0; k < 4 * Q; ++k) v[k] = (T)((float)acc[i][j0 + k / 4][k % 4] * sx * sw[k]);
            }
            const int64_t t = t0 + i * 16;
            if (t >= a.tokens) continue;
            T *y = row_at<T>(a.y, worker, t);
            if (c0 + 4 * Q <= a.channels) {
                __builtin_memcpy(y + c0, v, sizeof v);
            } else {
#pragma unroll
                for (int k = 0; k < 4 * Q; ++k)
                    if (c0 + k < a.channels) y[c0 + k] = v[k];
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
    int32_t tiles_m, tiles_n;
    int32_t workers;
};

// Two floats as sums of P bfloat16 each: exactly, for the 8, 11 and 24
// significant bits of the three types and P = 1, 2, 3, as long as the last part
// is not below the smallest bfloat16, 2^-133, to whose multiples floats are
// rounded (a float of 1e-34 keeps 22 bits).  All parts but the last are cut and
// not rounded: a rounded one would pass the largest bfloat16 for floats in the
// last 2^-9 of their range.  8 bits a part are enough that way too.
template <int P>
__device__ __forceinline__ void split_pair(float a, float b, unsigned (&part)[P]) {
#pragma unroll
    for (int p = 0; p + 1 < P; ++p) {
        const unsigned x = bits_of(a) & 0xffff0000u, y = bits_of(b) & 0xffff0000u;
        part[p] = x >> 16 | y;
        // An infinity has no rest; a NaN that was cut to an infinity has a NaN.
        a = (bits_of(a) & 0x7fffffffu) == 0x7f800000u ? 0.0f : a - float_of(x);
        b = (bits_of(b) & 0x7fffffffu) == 0x7f800000u ? 0.0f : b - float_of(y);
    }
    part[P - 1] = bf16_pair(a, b);
}

template <typename T> struct Parts { static constexpr int n = 1; };
template <> struct Parts<_Float16> { static constexpr int n = 2; };
template <> struct Parts<float> { static constexpr int n = 3; };

// out[m][k] = sum_r A(m, r) * q[r][k] 2^e[r][k / group], with A(m, r) = dY[m][r]
// (dX: m tokens, r channels) or dY[r][m] (ALONG_R, dW: m channels, r tokens).
// Both operands are brought into LDS as bfloat16 rows along r, 64 of r a step:
// 8 x 4 blocks of codes, and of dY for dW, are turned in registers on the way,
// codes converted once for the workgroup and not by each wave that reads them.
// The products are exact in 32 bits; sums are bfloat16 matrix instructions'
// 32-bit ones.  dY of 16 or 32 bits goes in as 2 or 3 bfloat16 that add up to it.
//
// Bound by the matrix unit together with what feeds it: a step of 256 x 256 has
// 2048 cycles of matrix instructions on each SIMD, conversions and addresses
// about 900 of the vector unit, and LDS is busy for 1280.  dX takes some 4300
// cycles a step (matrix units busy 48%), so a quarter is waiting; dW, which
// also writes four times the bytes at the end of its tiles, 5500 (37%).
// 16 x 2048 bfloat16 tokens, 4096 channels, width 1024: dX in 250 us,
// 1100 TFLOP/s; dW 295-305 us, 900-930 (the library's bfloat16 product of
// 8192^3: 1130-1150), 312 with X packed by 128.  Float gradients (three products
// each): 909 and 1139 us; binary16 (two): 491 and 654.  The tile is as large as
// two steps of all parts fit in LDS; floats, with a quarter of bfloat16's tile,
// have twice the LDS reads for a matrix instruction that they would have there.
template <typename T, int QMAX, bool ALONG_R, bool GROUPED, int BM, int BN, int WM, int WN>
struct GradTile {
    static constexpr int kThreads = 64 * WM * WN, P = Parts<T>::n, BR = 64;
    static constexpr int kA = P * BM * 128, kBytes = kA + BN * 128;
    static constexpr int TM = BM / WM / 16, TN = BN / WN / 16, Q = TN < QMAX ? TN : QMAX;
    // Units of one thread: 8 r of one m (dX), or 8 r of 4 m (dW); 8 r of 4 columns.
    static constexpr int kUnitsA = BM * BR / (ALONG_R ? 32 : 8), kUnitsB = BN * BR / 32;
    static constexpr int UA = (kUnitsA + kThreads - 1) / kThreads, UB = (kUnitsB + kThreads - 1) / kThreads;
    typedef T t4_t __attribute__((ext_vector_type(4)));

    // What a thread holds of a step on its way to LDS: dY and codes as they
    // are, and the exponents of its 8 rows of codes.
    struct Held {
        v8_t<T> a[ALONG_R ? 1 : UA];
        t4_t at[ALONG_R ? UA : 1][8];
        unsigned q[UB][8];
        u2_t e[GROUPED ? 1 : UB];
        int8_t eg[GROUPED ? UB : 1][8];
    };

    // Thread's unit i of a tile `span` wide in units of 4: its place along r.
    // The same for a whole wave where 64 units fit the width, which leaves
    // addresses to the scalar unit.
    static __device__ __forceinline__ int unit_r(int i, int span) {
        const int r = (i * kThreads + threadIdx.x) / (span / 4) * 8;
        return span / 4 % kWave == 0 ? __builtin_amdgcn_readfirstlane(r) : r;
    }

    // Loads the step at r0.  FULL: all of it is inside; else entries past the
    // contracted axis' end count as zeros, and only entries inside are touched.
    // Rows (dX) or columns (both) past the result's end repeat others: what
    // they give is not stored.
    template <bool FULL>
    static __device__ __forceinline__ void load(const GradArgs &g, int64_t worker, int64_t m0, int n0,
                                                int64_t r0, Held &h) {
#pragma unroll
        for (int i = 0; i < UA; ++i) {
            const int u = i * kThreads + threadIdx.x;
            if (kUnitsA % kThreads && u >= kUnitsA) break;
            if (ALONG_R) {
                const int rr = unit_r(i, BM);
                const T *p = row_at<const T>(g.a, worker, r0 + rr);
                int64_t m = m0 + u % (BM / 4) * 4;
                if (FULL) m = min(m, g.m - 4);
#pragma unroll
                for (int y = 0; y < 8; ++y) {
                    if (FULL) {
                        __builtin_memcpy(&h.at[i][y], p + y * g.a.rs + m, sizeof h.at[i][y]);
                    } else {
#pragma unroll
                        for (int x = 0; x < 4; ++x)
                            h.at[i][y][x] = r0 + rr + y < g.r && m + x < g.m ? p[y * g.a.rs + m + x] : (T)0.0f;
                    }
                }
            } else {
                const T *p = row_at<const T>(g.a, worker, min(m0 + u / 8, g.m - 1)) + r0 + u % 8 * 8;
                if (FULL) {
                    __builtin_memcpy(&h.a[i], p, sizeof h.a[i]);
                } else {
#pragma unroll
                    for (int y = 0; y < 8; ++y) h.a[i][y] = r0 + u % 8 * 8 + y < g.r ? p[y] : (T)0.0f;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < UB; ++i) {
            const int u = i * kThreads + threadIdx.x;
            if (kUnitsB % kThreads && u >= kUnitsB) break;
            const int rr = unit_r(i, BN), col = min(n0 + u % (BN / 4) * 4, g.stride - 4);
            const int64_t row = worker * g.r + r0 + rr;
            const int8_t *q = g.b.codes + row * g.stride;
            const int8_t *e = g.b.exps + row * g.b.groups + (GROUPED ? col / kGroup : 0);
            const int left = (int)min(g.r - r0 - rr, (int64_t)8);
#pragma unroll
            for (int y = 0; y < 8; ++y)
                h.q[i][y] = FULL || y < left ? *reinterpret_cast<const unsigned *>(q + y * (int64_t)g.stride + col) : 0u;
            if (GROUPED) {
#pragma unroll
                for (int y = 0; y < 8; ++y) h.eg[i][y] = FULL || y < left ? e[y * (int64_t)g.b.groups] : (int8_t)0;
            } else if (FULL) {
                __builtin_memcpy(&h.e[i], e, sizeof h.e[i]);
            } else {
                h.e[i] = u2_t{0, 0};
#pragma unroll
                for (int y = 0; y < 8; ++y)
                    if (y < left) h.e[i][y / 4] |= (unsigned)(uint8_t)e[y] << (8 * (y % 4));
            }
        }
    }

    // Chunks of dY that the result's edge would cut were loaded from up to 3
    // columns before (load<true>): moves their entries to their places.
    static __device__ __forceinline__ void align_edge(const GradArgs &g, int64_t m0, Held &h) {
#pragma unroll
        for (int i = 0; i < (ALONG_R ? UA : 0); ++i) {
            const int64_t before = m0 + (i * kThreads + threadIdx.x) % (BM / 4) * 4 - (g.m - 4);
            const int by = (int)max((int64_t)0, min(before, (int64_t)3));
#pragma unroll
            for (int y = 0; y < 8; ++y) {
                const t4_t v = h.at[i][y];
#pragma unroll
                for (int x = 0; x < 3; ++x)
                    h.at[i][y][x] = by == 0 ? v[x] : by == 1 ? v[x + 1] : by == 2 && x < 2 ? v[x + 2 & 3] : v[3];
            }
        }
    }

    static __device__ __forceinline__ void store(const Held &h, char *lds) {
#pragma unroll
        for (int i = 0; i < UB; ++i) {
            const int u = i * kThreads + threadIdx.x;
            if (kUnitsB % kThreads && u >= kUnitsB) break;
            const int at = tile_at(u % (BN / 4) * 4, u / (BN / 4));
            // The exponents are the same for a wave where its rows are; taken from
            // the first lane here and not, with a wait for memory, where they
            // are loaded.
            u2_t e = GROUPED ? u2_t{0, 0} : h.e[i];
            if (!GROUPED) {
                asm volatile("" : "+v"(e));
                if (BN / 4 % kWave == 0)
                    e = u2_t{(unsigned)__builtin_amdgcn_readfirstlane(e.x), (unsigned)__builtin_amdgcn_readfirstlane(e.y)};
            }
            float scale[8];
#pragma unroll
            for (int y = 0; y < 8; ++y)
                scale[y] = scale_of(GROUPED ? h.eg[i][y] : (int)(int8_t)(e[y / 4] >> (8 * (y % 4))));
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                u4_t v;
#pragma unroll
                for (int y = 0; y < 8; y += 2)
                    v[y / 2] = bf16_pair(code_at(h.q[i][y], x) * scale[y], code_at(h.q[i][y + 1], x) * scale[y + 1]);
                *reinterpret_cast<u4_t *>(lds + kA + column_at(at, x)) = v;
            }
        }
#pragma unroll
        for (int i = 0; i < UA; ++i) {
            const int u = i * kThreads + threadIdx.x;
            if (kUnitsA % kThreads && u >= kUnitsA) break;
            const int at = ALONG_R ? tile_at(u % (BM / 4) * 4, u / (BM / 4)) : tile_at(u / 8, u % 8);
#pragma unroll
            for (int x = 0; x < (ALONG_R ? 4 : 1); ++x) {
                u4_t v[P];
#pragma unroll
                for (int y = 0; y < 8; y += 2) {
                    const T a = ALONG_R ? h.at[i][y][x] : h.a[i][y], b = ALONG_R ? h.at[i][y + 1][x] : h.a[i][y + 1];
                    unsigned p[P];
                    if constexpr (P == 1)
                        p[0] = __builtin_bit_cast(unsigned short, a) | (unsigned)__builtin_bit_cast(unsigned short, b) << 16;
                    else
                        split_pair<P>((float)a, (float)b, p);
#pragma unroll
                    for (int k = 0; k < P; ++k) v[k][y / 2] = p[k];
                }
#pragma unroll
                for (int k = 0; k < P; ++k)
                    *reinterpret_cast<u4_t *>(lds + k * BM * 128 + column_at(at, x)) = v[k];
            }
        }
    }

    static __device__ __forceinline__ void multiply(const char *lds, int aat, int bat, f4_t (&acc)[TM][TN]) {
        aat = fresh(aat);
        bat = fresh(bat);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            b8_t bf[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j) bf[j] = *reinterpret_cast<const b8_t *>(lds + moved<Q>(bat, j, ks));
#pragma unroll
            for (int k = P - 1; k >= 0; --k) {   // the smallest part first
                b8_t af[TM];
#pragma unroll
                for (int i = 0; i < TM; ++i)
                    af[i] = *reinterpret_cast<const b8_t *>(lds + k * BM * 128 + moved<1>(aat, i, ks));
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf[j], af[i], acc[i][j], 0, 0, 0);
            }
        }
        // All of the first half's reads, then the second half's among the products.
        constexpr int M = TM * TN * P;
        __builtin_amdgcn_sched_group_barrier(kDsRead, TN + P * TM, 0);
#pragma unroll
        for (int q = 0; q < M / 2; ++q) {
            __builtin_amdgcn_sched_group_barrier(kMfma, 2, 0);
            __builtin_amdgcn_sched_group_barrier(kDsRead, 1, 0);
        }
    }
};

template <typename T, typename O, bool ALONG_R, bool GROUPED, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN, 2) void grad_kernel(GradArgs a) {
    using G = GradTile<T, kFours<O>, ALONG_R, GROUPED, BM, BN, WM, WN>;
    constexpr int TM = G::TM, TN = G::TN, Q = G::Q;
    __shared__ __align__(16) char lds[2 * G::kBytes];
    const unsigned per = (unsigned)a.tiles_m * a.tiles_n;
    const unsigned tile = xcd_tile(blockIdx.x, gridDim.x);
    const unsigned job = tile / per, in = tile % per;
    const int64_t worker = job / a.split;
    const int part = (int)(job % a.split);
    const int64_t m0 = (int64_t)(in / a.tiles_n) * BM;
    const int n0 = (int)(in % a.tiles_n) * BN;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);
    const int aat = read_at<1>(wm, lane), bat = G::kA + read_at<Q>(wn, lane);
    // This part's share of the contracted axis, in whole steps.
    const int64_t steps = (a.r + G::BR - 1) / G::BR;
    const int64_t s0 = steps * part / a.split, s1 = steps * (part + 1) / a.split;
    f4_t acc[TM][TN] = {};
    if (s0 < s1) {
        typename G::Held h;
        // Steps that are loaded in whole chunks: not the one that the axis ends
        // in, and none of a result with fewer rows than a chunk.
        const int64_t whole = ALONG_R && a.m < 4 ? 0 : a.r / G::BR;
        const bool edge = ALONG_R && a.m % 4 && m0 + BM > a.m;
        auto load = [&](int64_t s) {
            if (s < whole) G::template load<true>(a, worker, m0, n0, s * G::BR, h);
            else G::template load<false>(a, worker, m0, n0, s * G::BR, h);
        };
        // Two waves share a SIMD: one multiplies step s first and then brings
        // s + 1 into LDS, the other the other way round, so that one's vector
        // instructions run beside the other's matrix instructions.
        const bool late = WM * WN == 8 && wave >= 4;
        auto store = [&](int64_t s, char *to) {
            if (edge && s < whole) G::align_edge(a, m0, h);
            G::store(h, to);
        };
        int cur = 0;
        load(s0);
        store(s0, lds);
        if (late && s0 + 1 < s1) load(s0 + 1);
        __syncthreads();
        int64_t s = s0;
        for (; s + 2 < min(s1, whole); ++s) {
            if (late) store(s + 1, lds + (cur ^ G::kBytes));
            G::template load<true>(a, worker, m0, n0, (s + 1 + late) * G::BR, h);
            G::multiply(lds + cur, aat, bat, acc);
            cur ^= G::kBytes;
            if (!late) store(s + 1, lds + cur);
            __syncthreads();
        }
        for (; s < s1; ++s) {
            if (late && s + 1 < s1) store(s + 1, lds + (cur ^ G::kBytes));
            if (s + 1 + late < s1) load(s + 1 + late);
            G::multiply(lds + cur, aat, bat, acc);
            cur ^= G::kBytes;
            if (!late && s + 1 < s1) store(s + 1, lds + cur);
            __syncthreads();
        }
    }
    // A lane has 4 * Q neighbouring columns of one row in Q accumulators.
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t m = m0 + wm + i * 16 + lane % 16;
        if (m >= a.m) continue;
#pragma unroll
        for (int j0 = 0; j0 < TN; j0 += Q) {
            const int c0 = n0 + wn + tile_row<Q>(j0, lane / 16 * 4);
            if (a.split > 1)
                write_entries<Q>(a.partial + (((int64_t)part * a.workers + worker) * a.m + m) * a.cols, c0, a.cols,
                                 &acc[i][j0]);
            else
                write_entries<Q>(row_at<O>(a.out, worker, m), c0, a.cols, &acc[i][j0]);
        }
    }
}

// The sum of the parts of a split product, in ascending order, so that equal
// inputs give equal bits: four
// neighbouring entries of [n][rows][cols] for each thread, given to
// f(worker, row, column, sum) one by one.
template <typename V, typename F>
__device__ __forceinline__ void join_parts(const V *partial, int split, int64_t workers, int64_t rows, int cols, F f) {
    const int64_t all = workers * rows * cols;
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < all; i += (int64_t)gridDim.x * 1024) {
        V v[4] = {0, 0, 0, 0};
        if (i + 4 <= all) {
            // Eight parts' loads at a time.
            for (int s0 = 0; s0 < split; s0 += 8) {
                V p[8][4];
#pragma unroll
                for (int s = 0; s < 8; ++s)
                    __builtin_memcpy(p[s], partial + min(s0 + s, split - 1) * all + i, sizeof p[s]);
#pragma unroll
                for (int s = 0; s < 8; ++s)
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] += s0 + s < split ? p[s][k] : 0;
            }
        } else {
            for (int s = 0; s < split; ++s)
                for (int k = 0; i + k < all; ++k) v[k] += partial[s * all + i + k];
        }
        int64_t row = i / cols;
        int col = (int)(i - row * cols);
        int64_t worker = row / rows;
        row -= worker * rows;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (i + k >= all) break;
            f(worker, row, col, v[k]);
            if (++col == cols) {
                col = 0;
                if (++row == rows) row = 0, ++worker;
            }
        }
    }
}

template <typename T>
__global__ __launch_bounds__(256) void join_linear_kernel(LinearArgs a) {
    join_parts(a.partial, a.split, a.workers, a.tokens, a.channels, [&](int64_t worker, int64_t t, int c, int v) {
        const int ex = a.x.exps[worker * a.tokens + t], ew = a.w.exps[worker * a.channels + c];
        const float f = ldexpf((float)v, ex + ew);
        row_at<T>(a.y, worker, t)[c] = (T)(ex == kNotANumber || ew == kNotANumber ? float_of(0x7fc00000u) : f);
    });
}

template <typename O>
__global__ __launch_bounds__(256) void join_grad_kernel(GradArgs a) {
    join_parts(a.partial, a.split, a.workers, a.m, a.cols,
               [&](int64_t worker, int64_t m, int c, float v) { row_at<O>(a.out, worker, m)[c] = (O)v; });
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

// One array of a call: where it lies, for the checks that follow.  Row t of
// worker i is the `row` bytes at p + i * ws + t * rs; a dense array is one row.
struct Span {
    const char *name;
    const char *p;
    size_t bytes;     // from the first row's start to the last one's end
    bool out;
    bool typed;       // rows of a type, which a call may allow to be written in place
    int64_t row, ws, rs, n, rows;

    // The bytes that rows reach over when all of them are moved by multiples of
    // m to where the first lies.
    int64_t reach(int64_t m) const {
        return row + (ws % m ? (n - 1) * ws : 0) + (rs % m ? (rows - 1) * rs : 0);
    }
};

// Whether no byte is in both: one array ends before the other starts, or both
// keep to their own part of every stretch of m bytes, m a stride of either
// (models and gradients as halves of one tensor, say).
bool apart(const Span &a, const Span &b) {
    if (a.p >= b.p + b.bytes || b.p >= a.p + a.bytes) return true;
    for (const int64_t m : {a.ws, a.rs, b.ws, b.rs}) {
        if (m <= 0) continue;
        const int64_t from = (int64_t)(b.p - a.p) % m, start = from < 0 ? from + m : from;
        if (start >= a.reach(m) && start + b.reach(m) <= m) return true;
    }
    return false;
}

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

    // A product's workgroups and workspace.
    template <typename P>
    void product_launch(const P &plan, const void *workspace, size_t bytes) {
        if (code != RELAYSUM_OK) return;
        // Not even the largest tile's fit a launch.
        if (plan.blocks > kMaxBlocks) return fail(refuse("the result has more than %d tiles", (int)kMaxBlocks));
        if (plan.workspace > bytes)
            return fail(refuse("the workspace has %zu bytes, %zu are needed", bytes, plan.workspace));
        span("workspace", workspace, plan.workspace, 16, true);
    }

    void span(const char *name, const void *p, size_t bytes, size_t align, bool out) {
        add(Span{name, static_cast<const char *>(p), bytes, out, false, (int64_t)bytes, 0, 0, 1, 1}, align);
    }

    void add(const Span &s, size_t align) {
        if (code != RELAYSUM_OK || !s.bytes) return;
        if (!s.p)
            fail(refuse("%s must not be NULL", s.name));
        else if ((uintptr_t)s.p % align)
            fail(refuse("%s must be %d-byte aligned", s.name, (int)align));
        else
            spans[count++] = s;
    }

    // The norm's weights: a row of floats for each worker.
    void weights(const float *w, int32_t n, int64_t stride, int64_t width) {
        if (code != RELAYSUM_OK) return;
        if (n == 1) stride = 0;
        if (stride < 0 || stride > ((int64_t)1 << 44) / n)
            return fail(refuse("weight_stride is negative or reaches past 2^44 entries"));
        const size_t entries = (size_t)((n - 1) * stride + width);
        add(Span{"weight", reinterpret_cast<const char *>(w), entries * 4, false, false, width * 4, stride * 4, 0, n, 1}, 4);
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
        const int64_t b = (int64_t)type_bytes(r->type);
        add(Span{name, static_cast<const char *>(r->data), entries * b, out, true, width * b, ws * b, rs * b, n, rows},
            type_bytes(r->type));
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
                if (!(a.out || b.out) || apart(a, b)) continue;
                if (in_place && a.out != b.out && a.p == b.p && a.bytes == b.bytes && a.typed && b.typed &&
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

// Workgroups of a kernel over rows.  Packing and the norm loop over rows from
// 16 a CU on (one workgroup for every 4 rows took 6% more on a norm of 16 x 2048
// x 1024 bfloat16, 11% more packing 16 x 4096 x 2048 by 128); unpacking has
// nothing to keep between rows and does better without (6%).
unsigned row_grid(int64_t rows, int per, int64_t most = 16 * kCus) {
    return (unsigned)std::min<int64_t>((rows + per - 1) / per, most);
}

int chunks_layout(int64_t stride) { return stride <= 128 ? 16 : stride <= 2048 ? 64 : 256; }

// Workgroups per worker of the norm's gradient: enough for four on each CU, no
// more than one for 8 rows (5 x 777 x 1001 floats, 15.2 us a call, took 13% more
// with one for 16 rows, 4% more for 4).
int norm_parts(int32_t n, int64_t rows) {
    const int64_t want = (4 * kCus + n - 1) / n;
    return (int)std::max<int64_t>(1, std::min<int64_t>(want, (rows + 7) / 8));
}

// Calls f with the large or the small tile of a type: BM, BN, WM, WN.
template <typename T, typename F>
void with_grad_tile(int tile, F f) {
    constexpr int P = Parts<T>::n;
    if (tile == 0) f(Int<P == 1 ? 256 : 128>(), Int<P == 3 ? 128 : 256>(), Int<2>(), Int<4>());
    else f(Int<64>(), Int<128>(), Int<2>(), Int<2>());
}

template <typename F>
void with_linear_tile(int tile, F f) {
    if (tile == 0) f(Int<256>(), Int<256>(), Int<2>(), Int<4>());
    else if (tile == 1) f(Int<64>(), Int<128>(), Int<2>(), Int<2>());
    else f(Int<16>(), Int<128>(), Int<1>(), Int<4>());
}

unsigned join_grid(int64_t entries) {
    return (unsigned)std::max<int64_t>(1, std::min<int64_t>((entries + 1023) / 1024, 8 * kCus));
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
        const dim3 grid(row_grid(a.total, 256 / tpr, 1 << 20));
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
        c.weights(weight, n, weight_stride, width);
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
        c.weights(weight, n, weight_stride, width);
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
        hipLaunchKernelGGL(sum_parts_kernel, dim3((unsigned)(n * ((width + 31) / 32))), dim3(256), 0, st,
                           a.partial, reinterpret_cast<float *>(grad.data), grad.ws, parts, (int32_t)width);
    return done("relaysum_rmsnorm_backward");
}

int64_t relaysum_linear_workspace_of(int32_t product, int32_t n, int64_t tokens, int64_t width,
                                     int64_t channels, int32_t type) {
    Call c;
    if (!c.product(n, tokens, width, channels)) return -1;
    if (type < RELAYSUM_FLOAT || type > RELAYSUM_HALF) {
        refuse("unknown type %d", type);
        return -1;
    }
    g_error[0] = '\0';
    switch (product) {
    case RELAYSUM_LINEAR: return (int64_t)plan_linear(n, tokens, width, channels).workspace;
    case RELAYSUM_LINEAR_BACKWARD_INPUT: return (int64_t)plan_grad(type, n, tokens, width, channels).workspace;
    case RELAYSUM_LINEAR_BACKWARD_WEIGHT: return (int64_t)plan_grad(type, n, channels, width, tokens).workspace;
    }
    refuse("unknown product %d", product);
    return -1;
}

int64_t relaysum_linear_workspace(int32_t n, int64_t tokens, int64_t width, int64_t channels, int32_t type) {
    int64_t most = -1;
    for (const int32_t product : {RELAYSUM_LINEAR, RELAYSUM_LINEAR_BACKWARD_INPUT, RELAYSUM_LINEAR_BACKWARD_WEIGHT})
        most = std::max(most, relaysum_linear_workspace_of(product, n, tokens, width, channels, type));
    return most;
}

int relaysum_linear(int32_t n, int64_t tokens, int64_t width, int64_t channels,
                    const relaysum_packed *x, const relaysum_packed *w, const relaysum_rows *y,
                    void *workspace, size_t workspace_bytes, void *hip_stream) {
    Call c;
    Plan p;
    if (c.product(n, tokens, width, channels)) {
        c.packed("x", x, n, tokens, width, false);
        c.packed("w", w, n, channels, width, false);
        if (c.code == RELAYSUM_OK && !(whole_rows(x, width) && whole_rows(w, width)))
            c.fail(refuse("the product takes rows packed whole (group 0)"));
        c.rows("y", y, n, tokens, channels, true);
        p = plan_linear(n, tokens, width, channels);
        c.product_launch(p, workspace, workspace_bytes);
    }
    if (!c.ready()) return c.code;
    if (tokens == 0) return done("relaysum_linear");
    const LinearArgs a{packed_of(x, width), packed_of(w, width), rows_of(y, n, tokens),
                       static_cast<int32_t *>(workspace), tokens, (int32_t)code_stride(width),
                       (int32_t)channels, p.split, (int32_t)p.tiles_m, (int32_t)p.tiles_n, n};
    const hipStream_t st = (hipStream_t)hip_stream;
    with_type(y->type, [&](auto zero) {
        using T = decltype(zero);
        with_linear_tile(p.tile, [&](auto bm, auto bn, auto wm, auto wn) {
            constexpr int BM = decltype(bm)::value, BN = decltype(bn)::value;
            constexpr int WM = decltype(wm)::value, WN = decltype(wn)::value;
            hipLaunchKernelGGL(HIP_KERNEL_NAME(linear_kernel<T, BM, BN, WM, WN>), dim3((unsigned)p.blocks),
                               dim3(64 * WM * WN), 0, st, a);
        });
        if (p.split > 1)
            hipLaunchKernelGGL(join_linear_kernel<T>, dim3(join_grid(n * tokens * channels)), dim3(256), 0, st, a);
    });
    return done("relaysum_linear");
}

int relaysum_linear_backward_input(int32_t n, int64_t tokens, int64_t width, int64_t channels,
                                   const relaysum_rows *dy, const relaysum_packed *w,
                                   const relaysum_rows *dx, void *workspace, size_t workspace_bytes,
                                   void *hip_stream) {
    Call c;
    Plan p;
    if (c.product(n, tokens, width, channels)) {
        c.rows("dy", dy, n, tokens, channels, false);
        c.packed("w", w, n, channels, width, false);
        c.rows("dx", dx, n, tokens, width, true);
        if (c.code == RELAYSUM_OK && dy->type != dx->type)
            c.fail(refuse("dy and dx must have one type"));
        if (c.code == RELAYSUM_OK && !whole_rows(w, width))
            c.fail(refuse("w must be packed by whole rows (group 0)"));
        if (c.code == RELAYSUM_OK) p = plan_grad(dy->type, n, tokens, width, channels);
        c.product_launch(p, workspace, workspace_bytes);
    }
    if (!c.ready()) return c.code;
    if (tokens == 0) return done("relaysum_linear_backward_input");
    const GradArgs a{rows_of(dy, n, tokens), packed_of(w, width), rows_of(dx, n, tokens),
                     static_cast<float *>(workspace), tokens, channels, (int32_t)width,
                     (int32_t)code_stride(width), p.split, (int32_t)p.tiles_m, (int32_t)p.tiles_n, n};
    const hipStream_t st = (hipStream_t)hip_stream;
    with_type(dy->type, [&](auto zero) {
        using T = decltype(zero);
        with_grad_tile<T>(p.tile, [&](auto bm, auto bn, auto wm, auto wn) {
            constexpr int BM = decltype(bm)::value, BN = decltype(bn)::value;
            constexpr int WM = decltype(wm)::value, WN = decltype(wn)::value;
            hipLaunchKernelGGL(HIP_KERNEL_NAME(grad_kernel<T, T, false, false, BM, BN, WM, WN>),
                               dim3((unsigned)p.blocks), dim3(64 * WM * WN), 0, st, a);
        });
        if (p.split > 1)
            hipLaunchKernelGGL(join_grad_kernel<T>, dim3(join_grid(n * tokens * width)), dim3(256), 0, st, a);
    });
    return done("relaysum_linear_backward_input");
}

int relaysum_linear_backward_weight(int32_t n, int64_t tokens, int64_t width, int64_t channels,
                                    const relaysum_rows *dy, const relaysum_packed *x,
                                    const relaysum_rows *weight_grad, void *workspace,
                                    size_t workspace_bytes, void *hip_stream) {
    Call c;
    Plan p;
    if (c.product(n, tokens, width, channels)) {
        c.rows("dy", dy, n, tokens, channels, false);
        c.packed("x", x, n, tokens, width, false);
        c.rows("weight_grad", weight_grad, n, channels, width, true);
        if (c.code == RELAYSUM_OK && weight_grad->type != RELAYSUM_FLOAT)
            c.fail(refuse("weight_grad must be of type float"));
        if (c.code == RELAYSUM_OK) p = plan_grad(dy->type, n, channels, width, tokens);
        c.product_launch(p, workspace, workspace_bytes);
    }
    if (!c.ready()) return c.code;
    const GradArgs a{rows_of(dy, n, tokens), packed_of(x, width), rows_of(weight_grad, n, channels),
                     static_cast<float *>(workspace), channels, tokens, (int32_t)width,
                     (int32_t)code_stride(width), p.split, (int32_t)p.tiles_m, (int32_t)p.tiles_n, n};
    const bool grouped = !whole_rows(x, width);
    const hipStream_t st = (hipStream_t)hip_stream;
    with_type(dy->type, [&](auto zero) {
        using T = decltype(zero);
        with_grad_tile<T>(p.tile, [&](auto bm, auto bn, auto wm, auto wn) {
            constexpr int BM = decltype(bm)::value, BN = decltype(bn)::value;
            constexpr int WM = decltype(wm)::value, WN = decltype(wn)::value;
            const dim3 grid((unsigned)p.blocks), block(64 * WM * WN);
            if (grouped)
                hipLaunchKernelGGL(HIP_KERNEL_NAME(grad_kernel<T, float, true, true, BM, BN, WM, WN>), grid, block, 0, st, a);
            else
                hipLaunchKernelGGL(HIP_KERNEL_NAME(grad_kernel<T, float, true, false, BM, BN, WM, WN>), grid, block, 0, st, a);
        });
    });
    if (p.split > 1)
        hipLaunchKernelGGL(join_grad_kernel<float>, dim3(join_grid(n * channels * width)), dim3(256), 0, st, a);
    return done("relaysum_linear_backward_weight");
}

}  // extern "C"
