// The layer calls' host side: checks of arguments, error texts, and the choice
// of a row kernel's shape.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <type_traits>

#include "layer_plan.hpp"
#include "layer_rows.hpp"
#include "relaysum.h"

// The calling thread's last failure, one for all of the library's layer calls.
inline thread_local __attribute__((visibility("hidden"))) char g_error[256];

namespace {

using namespace layer_plan;

inline int refuse(const char *format, ...) __attribute__((format(printf, 1, 2)));
inline int refuse(const char *format, ...) {
    va_list ap;
    va_start(ap, format);
    std::vsnprintf(g_error, sizeof g_error, format, ap);
    va_end(ap);
    return RELAYSUM_ERR_INVALID_ARG;
}

inline int device_error(const char *what, hipError_t e) {
    std::snprintf(g_error, sizeof g_error, "%s: %s", what, hipGetErrorString(e));
    return RELAYSUM_ERR_DEVICE;
}

inline int done(const char *what) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return device_error(what, e);
    g_error[0] = '\0';
    return RELAYSUM_OK;
}

inline int64_t code_stride(int64_t width) { return (width + kGroup - 1) / kGroup * kGroup; }

inline size_t type_bytes(int32_t type) { return type == RELAYSUM_FLOAT ? 4 : 2; }

// One array of a call: where it lies, for the checks that follow.  Row t of
// worker i is the `row` bytes at p + i * ws + t * rs, or, of an array with heads,
// those at + h * hs for every head h; a dense array is one row.
struct Span {
    const char *name;
    const char *p;
    size_t bytes;     // from the first row's start to the last one's end
    bool out;
    bool typed;       // rows of a type, which a call may allow to be written in place
    int64_t row, ws, rs, n, rows;
    int64_t hs = 0, heads = 1;

    // The bytes that rows reach over when all of them are moved by multiples of
    // m to where the first lies.
    int64_t reach(int64_t m) const {
        return row + (ws % m ? (n - 1) * ws : 0) + (rs % m ? (rows - 1) * rs : 0) + (hs % m ? (heads - 1) * hs : 0);
    }
};

// Whether no byte is in both: one array ends before the other starts, or both
// keep to their own part of every stretch of m bytes, m a stride of either
// (models and gradients as halves of one tensor, say).
inline bool apart(const Span &a, const Span &b) {
    if (a.p >= b.p + b.bytes || b.p >= a.p + a.bytes) return true;
    for (const int64_t m : {a.ws, a.rs, a.hs, b.ws, b.rs, b.hs}) {
        if (m <= 0) continue;
        const int64_t from = (int64_t)(b.p - a.p) % m, start = from < 0 ? from + m : from;
        if (start >= a.reach(m) && start + b.reach(m) <= m) return true;
    }
    return false;
}

// Collects a call's arrays and says what is wrong with them.
struct Call {
    Span spans[24];
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

inline Rows rows_of(const relaysum_rows *r, int32_t n, int64_t rows) {
    if (!r) return Rows{nullptr, 0, 0};
    return Rows{static_cast<char *>(r->data), n > 1 ? r->worker_stride : 0, rows > 1 ? r->row_stride : 0};
}

inline Packed packed_of(const relaysum_packed *p, int64_t width) {
    if (!p) return Packed{nullptr, nullptr, 0};
    return Packed{p->codes, p->exps, (int32_t)(p->group ? code_stride(width) / kGroup : 1)};
}

// Whether a row has one exponent; up to 128 entries both groups have.
inline bool whole_rows(const relaysum_packed *p, int64_t width) { return p->group == 0 || width <= kGroup; }

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
inline unsigned row_grid(int64_t rows, int per, int64_t most = 16 * kCus) {
    return (unsigned)std::min<int64_t>((rows + per - 1) / per, most);
}

inline int chunks_layout(int64_t stride) { return stride <= 128 ? 16 : stride <= 2048 ? 64 : 256; }

// Workgroups per worker of the norm's gradient: enough for four on each CU, no
// more than one for 8 rows (5 x 777 x 1001 floats, 15.2 us a call, took 13% more
// with one for 16 rows, 4% more for 4).
inline int norm_parts(int32_t n, int64_t rows) {
    const int64_t want = (4 * kCus + n - 1) / n;
    return (int)std::max<int64_t>(1, std::min<int64_t>(want, (rows + 7) / 8));
}

}  // namespace
