// Shared by the sequence operators (group_norm.hip, recurrence.hip,
// dropout.hip): element types, unaligned vector access, the logistic
// function, and the checks of their arguments.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "rocket.h"

namespace rocket {

// Elements are loaded and stored as raw 32-bit words: one fp32 element or two
// 16-bit elements, low half first.
template <int DT>
struct Elem;

template <>
struct Elem<ROCKET_FLOAT32> {
    using raw = float;
    using bits = uint32_t;
    static constexpr int kSize = 4, kPerWord = 1;
    static __device__ float get(uint32_t w, int) { return __builtin_bit_cast(float, w); }
    static __device__ uint32_t put(const float *x) { return __builtin_bit_cast(uint32_t, x[0]); }
    static __device__ float one(raw r) { return r; }
    static __device__ raw round(float x) { return x; }
};

template <>
struct Elem<ROCKET_BFLOAT16> {
    using raw = uint16_t;
    using bits = uint16_t;
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    static constexpr int kSize = 2, kPerWord = 2;
    static __device__ float get(uint32_t w, int j) {
        return __builtin_bit_cast(float, j ? w & 0xffff0000u : w << 16);
    }
    static __device__ uint32_t put(const float *x) {
        pair p;
        p[0] = (__bf16)x[0];
        p[1] = (__bf16)x[1];
        return __builtin_bit_cast(uint32_t, p);
    }
    static __device__ float one(raw r) { return __builtin_bit_cast(float, (uint32_t)r << 16); }
    static __device__ raw round(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
};

template <>
struct Elem<ROCKET_FLOAT16> {
    using raw = uint16_t;
    using bits = uint16_t;
    typedef _Float16 pair __attribute__((ext_vector_type(2)));
    static constexpr int kSize = 2, kPerWord = 2;
    static __device__ float get(uint32_t w, int j) { return (float)__builtin_bit_cast(pair, w)[j]; }
    static __device__ uint32_t put(const float *x) {
        pair p;
        p[0] = (_Float16)x[0];
        p[1] = (_Float16)x[1];
        return __builtin_bit_cast(uint32_t, p);
    }
    static __device__ float one(raw r) { return (float)__builtin_bit_cast(_Float16, r); }
    static __device__ raw round(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }
};

// V from an address of any alignment: one global_load of the full width (the
// hardware takes unaligned addresses; rows of an odd number of 16-bit
// channels start on 2-byte boundaries).
template <class V>
__device__ inline V load_at(const void *p) {
    V v;
    __builtin_memcpy(&v, p, sizeof(V));
    return v;
}

template <class V>
__device__ inline void store_at(void *p, const V &v) {
    __builtin_memcpy(p, &v, sizeof(V));
}

// exp(-|x|).  Of fp32 elements to about one unit in the last place: the
// product with log2(e) is taken in two parts, so that its rounding does not
// grow with |x|; below -120 the result is 0.  Of 16-bit elements the rounding
// of the product stays in: 2^-24 |x| relative, a ten-thousandth of a unit of
// the element's own rounding, and three instructions fewer.  NaN stays NaN.
template <int DT>
__device__ inline float exp_neg_abs(float x) {
    constexpr float kLog2e = 1.44269502162933349609375f, kLog2eLow = 1.925963033500011e-8f;
    if (DT != ROCKET_FLOAT32) return __builtin_amdgcn_exp2f(-__builtin_fabsf(x) * kLog2e);
    float y = -__builtin_fabsf(x);
    y = y < -120.0f ? -120.0f : y;
    float t = y * kLog2e;
    float low = __builtin_fmaf(y, kLog2eLow, __builtin_fmaf(y, kLog2e, -t));
    float e = __builtin_amdgcn_exp2f(t);
    return __builtin_fmaf(e, low * 0.693147180559945f, e);
}

// S(x) and 1 - S(x), S the logistic function, each to a few units in the last
// place at either end: the smaller one is never a difference of near-equals.
// FACTOR: s is one of many factors.  The reciprocal instruction is off by a tenth
// of 2^-24 on average, which adds up: after 2,000 steps of gates of 3 to 6 a state
// is off by 207 units of 2^-24 on average, by 1.4 with the step of Newton's method,
// which fp32 elements take (no time lost).  16-bit elements do without it: there
// 245 units are a thirtieth of an fp16 rounding, and the step costs 5 % (4 x 16384 x
// 256, bf16: 26.5 us against 25.3 us).
template <int DT, bool FACTOR = false>
__device__ inline void logistic(float x, float &s, float &rest) {
    float e = exp_neg_abs<DT>(x), d = 1.0f + e;
    float big = __builtin_amdgcn_rcpf(d);
    if (FACTOR && DT == ROCKET_FLOAT32) big = __builtin_fmaf(__builtin_fmaf(-d, big, 1.0f), big, big);
    float small = e * big;
    bool pos = x >= 0.0f;
    s = pos ? big : small;
    rest = pos ? small : big;
}

// Makes the compiler take the words as new, so that what it computed of them
// is computed again instead of being held in registers across a barrier.
template <int N>
__device__ inline void renew(uint32_t (&w)[N]) {
#pragma unroll
    for (int s = 0; s < N; s++) asm("" : "+v"(w[s]));
}

// The work item of a workgroup: workgroups go to the 8 XCDs in turn, and each
// XCD has an L2 of its own, so that items in a row (which share cache lines at
// their borders) are given to workgroups of one XCD.
__device__ inline uint32_t item_of_block() {
    const uint32_t b = blockIdx.x, x = b & 7, each = gridDim.x >> 3, more = gridDim.x & 7;
    return x * each + (x < more ? x : more) + (b >> 3);
}

// A value that is the same for the whole wavefront, into a scalar register.
__device__ inline int uniform(uint32_t x) { return __builtin_amdgcn_readfirstlane((int)x); }

// Steps of series i: its length, clamped into [0, L].
__device__ inline int32_t steps_of(const int32_t *lengths, int64_t i, int32_t L) {
    if (!lengths) return L;
    int32_t t = lengths[i];
    return t < 0 ? 0 : t > L ? L : t;
}

inline bool dtype_ok(int32_t dt) { return dt == ROCKET_FLOAT32 || dt == ROCKET_BFLOAT16 || dt == ROCKET_FLOAT16; }
inline int elem_size(int32_t dt) { return dt == ROCKET_FLOAT32 ? 4 : 2; }

// A shape the kernels' index arithmetic holds for.
inline bool shape_ok(const rocket_sequence_shape *s) {
    if (!s || s->n < 0 || s->steps < 0 || s->channels < 1 || !dtype_ok(s->dtype)) return false;
    if (s->n > INT32_MAX || s->steps > INT32_MAX || s->channels > (1 << 24)) return false;
    int64_t e;
    return !__builtin_mul_overflow(s->n, s->steps, &e) && !__builtin_mul_overflow(e, s->channels, &e) &&
           e <= ((int64_t)1 << 56);
}

inline bool empty(const rocket_sequence_shape *s) { return s->n == 0 || s->steps == 0; }

// A view of that shape: not null, aligned to its elements, strides whose
// largest offset fits (inputs may repeat rows: strides of 0).
inline bool view_ok(const rocket_sequence *q, const rocket_sequence_shape *s) {
    if (!q) return false;
    if (empty(s)) return true;
    if (!q->data || ((uintptr_t)q->data % elem_size(s->dtype)) != 0) return false;
    if (q->step_stride < 0 || q->series_stride < 0) return false;
    int64_t a, b;
    if (__builtin_mul_overflow(s->n, q->series_stride, &a) || __builtin_mul_overflow(s->steps, q->step_stride, &b) ||
        __builtin_add_overflow(a, b, &a))
        return false;
    return a <= ((int64_t)1 << 58);
}

// An output's rows must not overlap: along one of the two axes a step passes
// over everything the other axis spans.
inline bool out_ok(const rocket_sequence *q, const rocket_sequence_shape *s) {
    if (!view_ok(q, s)) return false;
    if (empty(s)) return true;
    int64_t C = s->channels;
    if ((s->n > 1 && q->series_stride < C) || (s->steps > 1 && q->step_stride < C)) return false;
    return s->n <= 1 || s->steps <= 1 || q->series_stride >= (s->steps - 1) * q->step_stride + C ||
           q->step_stride >= (s->n - 1) * q->series_stride + C;
}

// Workgroups that one launch takes: HIP refuses 2^32 threads and more.  Larger
// calls are cut into several launches.
inline int64_t most_groups(int64_t threads) { return (int64_t)UINT32_MAX / threads; }

inline rocket_status launched() { return hipGetLastError() == hipSuccess ? ROCKET_OK : ROCKET_ERR_HIP; }

}  // namespace rocket
