// What the layer operators' kernels share: entries of a row as floats, 8-bit
// rows, reductions over a row, and copies into LDS.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

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

// ---- gates ------------------------------------------------------------------------

// a = 1 / (1 + e), c = e a with e = exp(-f): both to a few units of the last
// place, also where the other is near 1.  So in every type: a state is a product of
// hundreds of a's, and of 16-bit gates, which are often equal, their errors add up
// (the reciprocal as it comes and without log2(e)'s rest, gradients of states over
// 700 tokens were 9.6e-7 from 64 bits, where floats are 2.7e-7).
__device__ __forceinline__ void gates(float f, float &a, float &c) {
    constexpr double kLog2eWide = 1.44269504088896340736;
    constexpr float kLog2e = (float)kLog2eWide, kRest = (float)(kLog2eWide - (double)kLog2e);
    // Below -87 a is 2^-125 or less, above 200 it is 1; a NaN stays one.
    f = f < -87.0f ? -87.0f : f > 200.0f ? 200.0f : f;
    const float t = -f * kLog2e;
    float e = __builtin_amdgcn_exp2f(t);
    // What the product with log2(e) lost, and what its float lacks.
    const float lost = fmaf(-f, kLog2e, -t) - f * kRest;
    e = fmaf(e, lost * 0.69314718f, e);
    a = __builtin_amdgcn_rcpf(1.0f + e);
    a = fmaf(a, fmaf(-a, 1.0f + e, 1.0f), a);
    c = e * a;
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

// ---- copies and tiles -----------------------------------------------------------

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

}  // namespace
