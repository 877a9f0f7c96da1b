// Tiles of the attention kernels: rows of heads in LDS, and the two ways in
// which a wave multiplies by them.
//
// A wave works on 32 "columns" (queries, or keys in the gradients of K and V),
// one for each lane l % 32; the two lanes of a column share its other axis.
//   dots:     c[x][col] = sum over d of X[x][d] * B[d][col] for 32 rows x of a
//             tile, the columns' own rows B in registers
//   add_rows: acc[d][col] += sum over x of X[x][d] * w[x][col], with w as dots
//             leaves its results: register i of half h = l / 32 is row
//             8 * (i / 4) + 4 * h + i % 4
// So the weights that come out of one product go into the next as they are: no
// lane moves.  The order in which a matrix instruction adds up its rows is
// free, and X's rows are read in the order that w has them in.
#pragma once

#include "layer_rows.hpp"

namespace {

typedef float f16_t __attribute__((ext_vector_type(16)));
typedef _Float16 h8_t __attribute__((ext_vector_type(8)));
typedef short s4_t __attribute__((ext_vector_type(4)));

// Rows of DP entries (the heads' width rounded up) of 16-byte chunks.
template <typename T, int DP>
struct Tile {
    static constexpr int E = 16 / (int)sizeof(T);       // entries of a chunk
    static constexpr int kChunks = DP / E;              // of a row
    static constexpr int kRowBytes = DP * (int)sizeof(T);
    static constexpr int kOwn = DP / (2 * E);           // chunks of a column that one lane holds
    static constexpr int kBlocks = DP / 32;             // blocks of 32 entries

    // Chunk c of row r lies at position c ^ swizzle(r) of it.  Sixteen lanes
    // that read one chunk of neighbouring rows touch all banks once, and so do
    // those that read 64 bytes of each of 4 neighbouring rows.
    static __device__ __forceinline__ int swizzle(int row) {
        return kRowBytes == 128 ? ((row >> 1 & 1) << 2) | (row >> 2 & 3) : ((row & 3) << 2) | (row >> 2 & 3);
    }
    static __device__ __forceinline__ int at(int row, int chunk) {
        return row * kRowBytes + ((chunk ^ swizzle(row)) << 4);
    }
};

// A chunk of a row of `width` entries from entry `at` on, zeros behind.
template <typename T>
__device__ __forceinline__ u4_t load_chunk(const T *row, int at, int width, bool there) {
    constexpr int E = 16 / (int)sizeof(T);
    u4_t v = {0, 0, 0, 0};
    if (!there || at >= width) return v;
    if (at + E <= width) {
        __builtin_memcpy(&v, row + at, 16);
    } else {
        T t[E];
#pragma unroll
        for (int i = 0; i < E; ++i) t[i] = at + i < width ? row[at + i] : (T)0.0f;
        __builtin_memcpy(&v, t, 16);
    }
    return v;
}

// The sum of products of two chunks.
template <typename T>
__device__ __forceinline__ float chunk_dot(u4_t a, u4_t b, float sum) {
    constexpr int E = 16 / (int)sizeof(T);
    typedef T chunk_t __attribute__((ext_vector_type(E)));
    const chunk_t x = __builtin_bit_cast(chunk_t, a), y = __builtin_bit_cast(chunk_t, b);
#pragma unroll
    for (int i = 0; i < E; ++i) sum = fmaf((float)x[i], (float)y[i], sum);
    return sum;
}

__device__ __forceinline__ f16_t multiply(f16_t c, u4_t a, u4_t b, __bf16) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8_t, a), __builtin_bit_cast(b8_t, b), c, 0, 0, 0);
}
__device__ __forceinline__ f16_t multiply(f16_t c, u4_t a, u4_t b, _Float16) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8_t, a), __builtin_bit_cast(h8_t, b), c, 0, 0, 0);
}
__device__ __forceinline__ f16_t multiply(f16_t c, u4_t a, u4_t b, float) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(float_of(a[i]), float_of(b[i]), c, 0, 0, 0);
    return c;
}

// 32 rows of the tile from row0 (a multiple of 32) against the columns.
template <typename T, int DP>
__device__ __forceinline__ f16_t dots(const char *tile, int row0, const u4_t (&own)[Tile<T, DP>::kOwn], int lane) {
    typedef Tile<T, DP> L;
    f16_t c = {0};
    // Reads are on their way before the first product waits for one.
    u4_t x[L::kOwn];
#pragma unroll
    for (int i = 0; i < L::kOwn; ++i)
        x[i] = *reinterpret_cast<const u4_t *>(tile + row0 * L::kRowBytes + L::at(lane % 32, 2 * i + lane / 32));
    if (L::kOwn <= 4) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < L::kOwn; ++i) c = multiply(c, x[i], own[i], (T)0.0f);
    return c;
}

// The same with the columns' own rows in LDS, from row `col` of `own` on.
template <typename T, int DP>
__device__ __forceinline__ f16_t dots_in_lds(const char *tile, int row0, const char *own, int col, int lane) {
    typedef Tile<T, DP> L;
    f16_t c = {0};
#pragma unroll
    for (int i = 0; i < L::kOwn; ++i) {
        const int at = L::at(lane % 32, 2 * i + lane / 32);
        const u4_t a = *reinterpret_cast<const u4_t *>(tile + row0 * L::kRowBytes + at);
        const u4_t b = *reinterpret_cast<const u4_t *>(own + col * L::kRowBytes + at);
        c = multiply(c, a, b, (T)0.0f);
    }
    return c;
}

// The same with the columns' own rows in memory, where registers do not hold
// them: caches do.
template <typename T, int DP>
__device__ __forceinline__ f16_t dots_in_memory(const char *tile, int row0, const T *own, int width, bool valid, int lane) {
    typedef Tile<T, DP> L;
    f16_t c = {0};
#pragma unroll 8
    for (int i = 0; i < L::kOwn; ++i) {
        const u4_t a = *reinterpret_cast<const u4_t *>(tile + row0 * L::kRowBytes + L::at(lane % 32, 2 * i + lane / 32));
        c = multiply(c, a, load_chunk<T>(own, (2 * i + lane / 32) * L::E, width, valid), (T)0.0f);
    }
    return c;
}

// Weights of 32 rows as operands.
template <typename T>
struct Weights {
    u4_t part[2];
    __device__ __forceinline__ explicit Weights(const float (&w)[16]) {
        typedef T t8 __attribute__((ext_vector_type(8)));
        typedef float f8 __attribute__((ext_vector_type(8)));
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            f8 f;
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = w[8 * m + i];
            part[m] = __builtin_bit_cast(u4_t, __builtin_convertvector(f, t8));
        }
    }
};
template <>
struct Weights<float> {
    float part[16];
    __device__ __forceinline__ explicit Weights(const float (&w)[16]) {
#pragma unroll
        for (int i = 0; i < 16; ++i) part[i] = w[i];
    }
};

// 4 entries of each of 16 lanes' addresses, transposed: lane i of the 16 gets
// entry i % 4 of what lanes i / 4, 4 + i / 4, 8 + i / 4 and 12 + i / 4 point to.
__device__ __forceinline__ u2_t read_transposed(const char *p) {
    return __builtin_bit_cast(u2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) s4_t *)(p)));
}

template <typename T, int DP>
__device__ __forceinline__ void add_rows(f16_t (&acc)[DP / 32], const char *tile, int row0, const Weights<T> &w, int lane) {
    typedef Tile<T, DP> L;
    const int h = lane / 32, sub = lane / 16 % 2, i = lane % 16;
    if constexpr (sizeof(T) == 4) {
        // Two rows an instruction, one of each half.
#pragma unroll
        for (int x = 0; x < 16; ++x)
#pragma unroll
            for (int b = 0; b < DP / 32; ++b) {
                const float v = *reinterpret_cast<const float *>(
                    tile + row0 * L::kRowBytes + L::at(8 * (x / 4) + 4 * h + x % 4, 8 * b + lane % 32 / 4) + lane % 4 * 4);
                acc[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, w.part[x], acc[b], 0, 0, 0);
            }
    } else {
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int b = 0; b < DP / 32; ++b) {
                const int chunk = 4 * b + 2 * sub + i % 4 / 2, row = 4 * h + i / 4;
                const char *p = tile + (row0 + 16 * m) * L::kRowBytes + i % 2 * 8;
                const u2_t lo = read_transposed(p + L::at(row, chunk));
                const u2_t hi = read_transposed(p + L::at(row + 8, chunk));
                acc[b] = multiply(acc[b], u4_t{lo.x, lo.y, hi.x, hi.y}, w.part[m], (T)0.0f);
            }
    }
}

__device__ __forceinline__ void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Bytes of LDS for each wave that add_rows_apart needs.
template <typename T>
constexpr int kApartBytes = 16 * 32 * (int)sizeof(T);

// add_rows where a column must not touch rows that it does not see: in a matrix
// instruction an infinity or a NaN there would reach it even with weight 0.
// One row after the other, for tiles whose results came out not finite.
template <typename T, int DP, typename F>
__device__ __forceinline__ void add_rows_apart(f16_t (&acc)[DP / 32], const char *tile, int row0, const float (&w)[16],
                                            char *room, int lane, F sees) {
    typedef Tile<T, DP> L;
    typedef T t4 __attribute__((ext_vector_type(4)));
    T *weights = reinterpret_cast<T *>(room);
    const int h = lane / 32, col = lane % 32;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        wave_fence();
#pragma unroll
        for (int i = 0; i < 8; ++i) weights[(8 * (i / 4) + 4 * h + i % 4) * 32 + col] = (T)w[8 * m + i];
        wave_fence();
#pragma unroll 1
        for (int row = 0; row < 16; ++row) {
            const float f = (float)weights[row * 32 + col];
            if (!sees(16 * m + row)) continue;
#pragma unroll
            for (int b = 0; b < DP / 32; ++b)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int entry = 32 * b + 8 * g + 4 * h;
                    t4 x;
                    __builtin_memcpy(&x, tile + row0 * L::kRowBytes + L::at(16 * m + row, entry / L::E) +
                                             entry % L::E * (int)sizeof(T), sizeof x);
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[b][4 * g + r] = fmaf(f, (float)x[r], acc[b][4 * g + r]);
                }
        }
    }
    wave_fence();
}

// Whether any of a column's sums is an infinity or a NaN.
template <int B>
__device__ __forceinline__ bool not_finite(const f16_t (&acc)[B]) {
    float z = 0.0f;
#pragma unroll
    for (int b = 0; b < B; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) z = fmaf(acc[b][i], 0.0f, z);
    return !(z == 0.0f);
}

// Sums of a column as a row of `width` entries of type O, times f.
template <typename O, int B>
__device__ __forceinline__ void store_column(O *row, int width, const f16_t (&acc)[B], float f, int lane) {
    typedef O o4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int b = 0; b < B; ++b)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int at = 32 * b + 8 * g + 4 * (lane / 32);
            o4 v;
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] = (O)(acc[b][4 * g + r] * f);
            if (at + 4 <= width) {
                __builtin_memcpy(row + at, &v, sizeof v);
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (at + r < width) row[at + r] = v[r];
            }
        }
}

// One value of both lanes of a column.
__device__ __forceinline__ float other_half(float v) {
    const u2_t r = __builtin_bit_cast(u2_t, __builtin_amdgcn_permlane32_swap(bits_of(v), bits_of(v), false, false));
    return float_of(threadIdx.x % 64 < 32 ? r.y : r.x);
}

// 16 bytes for each lane from base + off into LDS at `to` + 16 * lane, on their
// way until wait_for_lds(); base and `to` are the same for the whole wave.  In
// assembly, because the compiler lets every later read of LDS wait for the
// builtin's copies, whatever tile it reads, so that none would overlap with work
// on another.  No register is written, and the address is read when it issues.
// The no-operations are what it takes from a scalar register's write to its use
// as an address.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"   // m0 is reserved: all the same it is overwritten
__device__ __forceinline__ void start_copy(const char *base, unsigned off, const char *to) {
    // The lower half of a pointer into LDS is the place there.
    const unsigned place = __builtin_amdgcn_readfirstlane((unsigned)reinterpret_cast<uint64_t>(to));
    const uint64_t at = reinterpret_cast<uint64_t>(base);
    const uint64_t from = (unsigned)__builtin_amdgcn_readfirstlane((unsigned)at) |
                          (uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((unsigned)(at >> 32)) << 32;
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2"
                 :: "s"(place), "v"(off), "s"(from) : "m0", "memory");
}
#pragma clang diagnostic pop
__device__ __forceinline__ void wait_for_lds() {
    asm volatile("" ::: "memory");
    wait_for_copies();
    asm volatile("" ::: "memory");
}

// R rows of a tile on their way from memory into LDS, by NT threads.  DIRECT:
// rows start on 16 bytes and have whole chunks, which are copied without
// registers in between; a lane's LDS place is fixed, so it takes the chunk that
// belongs there.  Rows that are not there then repeat the first one, and chunks
// behind the width stay as they are (zeros from clear()).  Otherwise through
// registers, at any alignment, zeros in both places.
template <typename T, int DP, int R, int NT, bool DIRECT>
struct Stage {
    typedef Tile<T, DP> L;
    static constexpr int kCount = R * L::kChunks / NT;
    static_assert(R * L::kChunks % NT == 0, "every thread has as many chunks");
    u4_t v[DIRECT ? 1 : kCount];
    unsigned off[DIRECT ? kCount : 1];

    static __device__ __forceinline__ void clear(char *tile, int thread) {
#pragma unroll
        for (int i = 0; i < kCount; ++i) *reinterpret_cast<u4_t *>(tile + (i * NT + thread) * 16) = u4_t{0, 0, 0, 0};
    }

    // Where a thread's chunks lie, from a tile's base on: at(r) is where row r
    // starts, in bytes.
    template <typename F>
    __device__ __forceinline__ void places(int thread, F at) {
        if (!DIRECT) return;
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            const int u = i * NT + thread, r = u / L::kChunks;
            off[i] = (unsigned)at(r) + (u % L::kChunks ^ L::swizzle(r)) * 16;
        }
    }

    // Starts the way of a tile whose places are known, of which `rows` are there.
    // DIRECT: in place of the others its first row.
    template <typename F>
    __device__ __forceinline__ void load(const char *base, char *tile, int width, int rows, int thread, F at) {
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            const int u = i * NT + thread, r = u / L::kChunks, place = u % L::kChunks;
            if (DIRECT) {
                const int chunk = place ^ L::swizzle(r);
                // A wave's first place in LDS.
                char *to = tile + (i * NT + __builtin_amdgcn_readfirstlane(thread & ~63)) * 16;
                if (chunk * L::E < width) start_copy(base, r < rows ? off[i] : chunk * 16u, to);
            } else {
                v[i] = load_chunk<T>(reinterpret_cast<const T *>(base + at(min(r, rows - 1))), place * L::E, width, r < rows);
            }
        }
    }
    // Ends it: with a barrier behind, all threads can read the tile.
    __device__ __forceinline__ void put(char *tile, int thread) const {
        if (DIRECT) {
            wait_for_lds();
            return;
        }
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            const int u = i * NT + thread;
            *reinterpret_cast<u4_t *>(tile + L::at(u / L::kChunks, u % L::kChunks)) = v[i];
        }
    }
};

}  // namespace
