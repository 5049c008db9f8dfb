// Shared by the operators that go row by row (rms_norm.hip, checkpoint.hip,
// linear8.hip, weight_gradient.hip): rows of sequences, and sequences whose
// rows lie in one line.
#pragma once

#include "sequence.h"

namespace rocket {

// Columns of 8-bit rows come in multiples of this, the columns past the
// channels are zeros: a product needs no case for a rest, and every row starts
// on a 64-byte border.
constexpr int kPad8 = 64;
// Rows that share a channel's scale in a checkpoint.
constexpr int kKeepRows = 128;

inline int64_t padded8(int64_t channels) { return (channels + kPad8 - 1) / kPad8 * kPad8; }

struct View {
    char *data;
    int64_t series, step;  // strides, bytes
};

inline View view_of(const rocket_sequence *q, int32_t dtype) {
    const int64_t size = elem_size(dtype);
    return q ? View{(char *)q->data, q->series_stride * size, q->step_stride * size} : View{};
}

// The rows of sequences [n, steps]: row r is step r % steps of series r / steps.
struct Rows {
    int64_t count;
    int32_t n, steps;
    const int32_t *lengths;
};

// Where a row lies, and whether it holds data.
struct Place {
    int64_t i, t;
    bool live;
};

__device__ inline Place place_of(const Rows &rows, int64_t r) {
    Place p;
    if (rows.n == 1) {
        p.i = 0, p.t = r;
    } else if (rows.count < ((int64_t)1 << 32)) {
        const uint32_t i = (uint32_t)r / (uint32_t)rows.steps;
        p.i = i, p.t = (uint32_t)r - i * (uint32_t)rows.steps;
    } else {
        p.i = r / rows.steps, p.t = r - p.i * rows.steps;
    }
    p.live = !rows.lengths || p.t < rows.lengths[p.i];
    return p;
}

__device__ inline char *row_at(const View &v, const Place &p) { return v.data + p.i * v.series + p.t * v.step; }

// Rows of a shape.  Where no lengths are given and every view's rows lie at one
// distance, they are one series: no division for a row's place.
inline Rows rows_of(const rocket_sequence_shape *s, View **views, int count) {
    Rows r = {s->n * s->steps, (int32_t)s->n, (int32_t)s->steps, s->lengths};
    bool line = !s->lengths && r.count <= INT32_MAX;
    for (int k = 0; k < count; k++)
        if (views[k]->data && s->n > 1 && s->steps > 1 && views[k]->series != s->steps * views[k]->step) line = false;
    if (line) {
        if (s->steps == 1)
            for (int k = 0; k < count; k++) views[k]->step = views[k]->series;
        r.n = 1, r.steps = (int32_t)r.count;
    }
    return r;
}

// 8-bit rows, weights and checkpoints are the library's own layouts: 16-byte
// aligned, without gaps.
inline bool bytes_ok(const void *p) { return p && (uintptr_t)p % 16 == 0; }
inline bool floats_ok(const void *p) { return p && (uintptr_t)p % 4 == 0; }

// Kinds of values that stand for a row or a channel in 8 bits, by the largest
// magnitude's bits: a NaN or an infinity makes the whole NaN; below 2^-100 (its
// quotient could overflow) everything counts as 0.
constexpr uint32_t kNotFinite = 0x7f800000u, kTooSmall = 0x0d800000u;

// What values are multiplied by (0: all of them become 0).
__device__ inline float inverse8(uint32_t top) {
    return top >= kNotFinite || top < kTooSmall ? 0.0f : 127.0f / __builtin_bit_cast(float, top);
}

// The step between 8-bit values.
__device__ inline float step8(uint32_t top) {
    if (top >= kNotFinite) return __builtin_nanf("");
    return top < kTooSmall ? 0.0f : __builtin_bit_cast(float, top) / 127.0f;
}

__device__ inline uint32_t magnitude(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }
__device__ inline uint32_t larger(uint32_t a, uint32_t b) { return a > b ? a : b; }

// A value to the nearest whole number as a byte; inverse 0 gives 0 whatever the value.
// The inverse and the product are rounded, then ties go to even: off by less than
// 127 * 2 * 2^-24 before the last rounding, so that a value halfway between two whole
// numbers may go to either (777 x 129 x 331 fp16: 9,457 of 33 million are, and 1,101 of
// them go the other way than the quotient itself would).
__device__ inline uint32_t byte8(float x, float inverse) {
    return inverse == 0.0f ? 0u : (uint32_t)(int)__builtin_rintf(x * inverse) & 255u;
}

__device__ inline uint32_t four8(float a, float b, float c, float d, float inverse) {
    return byte8(a, inverse) | byte8(b, inverse) << 8 | byte8(c, inverse) << 16 | byte8(d, inverse) << 24;
}

}  // namespace rocket
