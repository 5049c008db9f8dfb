// RMS norm with the residual's addition, its output as a sequence or as 8-bit
// rows, its gradient, and 8-bit rows of any values.
//
//   s = x + residual rounded to the type,  k = 1 / sqrt(sum s^2 / C + eps),  y = s k w
//   8 bits: a = max |s w|,  q = rint(s w 127 / a),  scale = k a / 127
//   (k is a factor of the whole row, so q does not wait for it: one reduction
//   gives the sum of squares and the maximum)
//   gradient: g = dy w,  dx = k (g - s k mean(g s k)) + dtotal,  dw = sum over rows of dy s k
//
// Bound: HBM; a value takes some ten operations.  So a row is read once and
// stays in the registers of G threads (at least 16), 16 bytes a thread and load,
// up to 24,576 channels; wider rows are read twice.  The backward pass sums dw
// over a workgroup's rows in registers (of 1,024 threads in shared memory), a second
// kernel joins the workgroups' sums in a fixed order.
// Measured, bf16 where nothing else is said (a sum of two 256 MB tensors runs at
// 5.9 TB/s, a smaller set comes from the 256 MB cache):
//   s and y of x and a residual, 500 x 1000 x 256   178 us, 5.75 TB/s
//   y of x, 2048 x 20000 fp32                        65 us, 5.0 TB/s
//   dx and dw of dy, s and ds, 1000 x 1000 x 256    386 us, 5.3 TB/s
//   the same without ds, 100 x 1000 x 2000          240 to 245 us, 5.0 TB/s
#include <algorithm>

#include "rows.h"
#include "join.h"

namespace {

using rocket::Elem;
using rocket::Place;
using rocket::Rows;
using rocket::View;

typedef uint32_t Words __attribute__((ext_vector_type(4)));

// What a call makes of a row.
enum Kind { kSequence, kBytes, kBytesOfValues };

struct NormArgs {
    Rows rows;
    View x, r, total, y;  // r, total: null without a residual
    const float *weight;  // or null
    float *rstd;
    int8_t *q;
    float *scale;
    int64_t padded;  // bytes of a row of q
    int32_t channels;
    float eps;
};

struct BackArgs {
    Rows rows;
    View dy, s, dt, dx;  // dt or null
    const float *weight, *rstd;
    float *partial;  // [workgroups, channels]
    int32_t channels;
};

// By value: a cast of a vector's element as it stands takes its first one.
__device__ inline float float_of(uint32_t w) { return __builtin_bit_cast(float, w); }

template <int DT>
constexpr int kVec = 4 * Elem<DT>::kPerWord;  // elements of 16 bytes

// 16 bytes of a row from column c on; zeros past the row's end.  A row's last piece of
// 16-bit values is read as the row's last 16 bytes and moved down: by elements it would
// be up to seven loads that the whole wavefront waits for (300 x 1000 x 331 fp16 with a
// residual 215 us, else 281; its gradient 149, else 226).  Of fp32, up to three loads,
// it only costs registers (236 us, moved down 288), as in gradients of 1,024 threads.
template <int DT, bool MOVE = true>
__device__ inline Words load_chunk(const char *row, int c, int channels) {
    constexpr int V = kVec<DT>, kSize = Elem<DT>::kSize;
    if (MOVE && kSize == 2 && channels >= V) {
        const int over = c + V - channels;
        Words w = rocket::load_at<Words>(row + (int64_t)(over > 0 ? channels - V : c) * kSize);
        if (over > 0) {
            typedef uint64_t Two __attribute__((ext_vector_type(2)));
            Two t = __builtin_bit_cast(Two, w);
            const int bits = over * kSize * 8, less = bits & 63;
            const uint64_t carried = less ? t[1] << (64 - less) : 0;
            t[0] = bits < 64 ? t[0] >> less | carried : bits < 128 ? t[1] >> less : 0;
            t[1] = bits < 64 ? t[1] >> less : 0;
            w = __builtin_bit_cast(Words, t);
        }
        return w;
    }
    if (c + V <= channels) return rocket::load_at<Words>(row + (int64_t)c * kSize);
    Words w = {0, 0, 0, 0};
    using bits = typename Elem<DT>::bits;
#pragma unroll
    for (int e = 0; e < V; e++)
        if (c + e < channels) {
            const uint32_t v = ((const bits *)row)[c + e];
            w[e / Elem<DT>::kPerWord] |= Elem<DT>::kPerWord == 1 ? v : v << (16 * (e & 1));
        }
    return w;
}

template <int DT>
__device__ inline void store_chunk(char *row, int c, int channels, const Words &w) {
    constexpr int V = kVec<DT>;
    if (c + V <= channels) {
        rocket::store_at(row + (int64_t)c * Elem<DT>::kSize, w);
        return;
    }
    using bits = typename Elem<DT>::bits;
#pragma unroll
    for (int e = 0; e < V; e++)
        if (c + e < channels)
            ((bits *)row)[c + e] =
                (bits)(Elem<DT>::kPerWord == 1 ? w[e] : w[e / Elem<DT>::kPerWord] >> (16 * (e & 1)));
}

template <int DT>
__device__ inline void values_of(const Words &w, float (&f)[kVec<DT>]) {
#pragma unroll
    for (int e = 0; e < kVec<DT>; e++) f[e] = Elem<DT>::get(w[e / Elem<DT>::kPerWord], e % Elem<DT>::kPerWord);
}

template <int DT>
__device__ inline Words words_of(const float (&f)[kVec<DT>]) {
    Words w;
#pragma unroll
    for (int k = 0; k < 4; k++) w[k] = Elem<DT>::put(f + k * Elem<DT>::kPerWord);
    return w;
}

// Weights from column c on (1 where none are given), 0 past the row's end.
template <int V>
__device__ inline void load_weights(const float *weight, int c, int channels, float (&w)[V]) {
    if (weight && c + V <= channels) {
#pragma unroll
        for (int h = 0; h < V; h += 4) {
            const Words t = rocket::load_at<Words>(weight + c + h);
#pragma unroll
            for (int e = 0; e < 4; e++) w[h + e] = float_of(t[e]);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < V; e++) w[e] = c + e < channels ? (weight ? weight[c + e] : 1.0f) : 0.0f;
}

template <int CTRL>
__device__ inline float moved(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
}

template <int CTRL>
__device__ inline uint32_t moved(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xF, 0xF, true);
}

// The sum of s and the largest top over a row's G threads, to all of them.
// Lanes of a wavefront meet within rows of 16 (exchange of neighbours, of
// pairs, mirrored halves, mirrored rows), then by exchanges of rows and halves;
// wavefronts meet in shared memory.
template <int G, bool TOP>
__device__ inline void join_row(float &s, uint32_t &top, float *shared, int &turn) {
    s += moved<0xB1>(s);
    s += moved<0x4E>(s);
    s += moved<0x141>(s);
    s += moved<0x140>(s);
    if (TOP) {
        top = rocket::larger(top, moved<0xB1>(top));
        top = rocket::larger(top, moved<0x4E>(top));
        top = rocket::larger(top, moved<0x141>(top));
        top = rocket::larger(top, moved<0x140>(top));
    }
    if (G >= 32) {
        const uint32_t b = __builtin_bit_cast(uint32_t, s);
        const auto p = __builtin_amdgcn_permlane16_swap(b, b, false, false);
        s = float_of(p[0]) + float_of(p[1]);
        if (TOP) {
            const auto t = __builtin_amdgcn_permlane16_swap(top, top, false, false);
            top = rocket::larger(t[0], t[1]);
        }
    }
    if (G >= 64) {
        const uint32_t b = __builtin_bit_cast(uint32_t, s);
        const auto p = __builtin_amdgcn_permlane32_swap(b, b, false, false);
        s = float_of(p[0]) + float_of(p[1]);
        if (TOP) {
            const auto t = __builtin_amdgcn_permlane32_swap(top, top, false, false);
            top = rocket::larger(t[0], t[1]);
        }
    }
    if constexpr (G > 64) rocket::join_waves<G / 64, TOP>(s, top, shared, turn);
}

constexpr int threads_of(int G) { return G > 64 ? G : 256; }

__device__ inline float rstd_of(float squares, const NormArgs &a) {
    return 1.0f / __builtin_sqrtf(squares / (float)a.channels + a.eps);
}

// The chunk of s from column c on: x, or x + residual rounded, which is stored.
template <int DT>
__device__ inline Words sum_chunk(const NormArgs &a, const Words &x, const Words &r) {
    float f[kVec<DT>], g[kVec<DT>];
    values_of<DT>(x, f);
    values_of<DT>(r, g);
#pragma unroll
    for (int e = 0; e < kVec<DT>; e++) f[e] += g[e];
    return words_of<DT>(f);
}

template <int DT>
__device__ inline void store_bytes(const NormArgs &a, int64_t r, int c, const float (&f)[kVec<DT>],
                                   const float (&w)[kVec<DT>], float inverse) {
    if (c >= a.padded) return;
    float p[kVec<DT>];
#pragma unroll
    for (int e = 0; e < kVec<DT>; e++) p[e] = f[e] * w[e];
    int8_t *at = a.q + r * a.padded + c;
    const uint32_t lo = rocket::four8(p[0], p[1], p[2], p[3], inverse);
    if (kVec<DT> == 4) {
        *(uint32_t *)at = lo;
    } else {
        const uint32_t hi = rocket::four8(p[kVec<DT> - 4], p[kVec<DT> - 3], p[kVec<DT> - 2], p[kVec<DT> - 1], inverse);
        *(uint64_t *)at = (uint64_t)hi << 32 | lo;
    }
}

// G threads a row, CHUNKS loads of 16 bytes each.  CHUNKS 0: any width, the row
// is read twice (the second time from the cache that the first filled).
template <int DT, int G, int CHUNKS, int KIND>
__global__ __launch_bounds__(threads_of(G)) void norm_kernel(NormArgs a) {
    constexpr int V = kVec<DT>, kThreads = threads_of(G), kRows = kThreads / G, kHeld = CHUNKS ? CHUNKS : 1;
    __shared__ float shared[G > 64 ? 4 * (G / 64) : 1];
    const int j = threadIdx.x % G, C = a.channels;
    const int64_t stride = (int64_t)gridDim.x * kRows;
    const int end = KIND == kSequence ? C : (int)a.padded;
    float w[kHeld][V];
    if (CHUNKS && KIND != kBytesOfValues)
#pragma unroll
        for (int k = 0; k < kHeld; k++) load_weights<V>(a.weight, (k * G + j) * V, C, w[k]);
    int turn = 0;
    for (int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / G; r < a.rows.count; r += stride) {
        const Place p = rocket::place_of(a.rows, r);
        if (!p.live) {
            // nothing is read; a row's threads all come here, and none of them joins
            const Words zero = {0, 0, 0, 0};
            for (int c = j * V; c < end; c += G * V) {
                if (KIND == kSequence)
                    store_chunk<DT>(rocket::row_at(a.y, p), c, C, zero);
                else {
                    int8_t *at = a.q + r * a.padded + c;
                    if (V == 4)
                        *(uint32_t *)at = 0;
                    else
                        *(uint64_t *)at = 0;
                }
                if (a.r.data && c < C) store_chunk<DT>(rocket::row_at(a.total, p), c, C, zero);
            }
            if (j == 0) {
                if (KIND != kBytesOfValues) a.rstd[r] = 0.0f;
                if (KIND != kSequence) a.scale[r] = 0.0f;
            }
            continue;
        }
        const char *x = rocket::row_at(a.x, p);
        const char *res = a.r.data ? rocket::row_at(a.r, p) : nullptr;
        char *total = a.r.data ? rocket::row_at(a.total, p) : nullptr;
        Words s[kHeld];
        float squares = 0.0f;
        uint32_t top = 0;
        auto take = [&](const Words &t, const float (&u)[V]) {
            float f[V];
            values_of<DT>(t, f);
#pragma unroll
            for (int e = 0; e < V; e++) {
                if (KIND != kBytesOfValues) squares = __builtin_fmaf(f[e], f[e], squares);
                if (KIND != kSequence)
                    top = rocket::larger(top, rocket::magnitude(KIND == kBytes ? f[e] * u[e] : f[e]));
            }
        };
        if (CHUNKS) {
#pragma unroll
            for (int k = 0; k < kHeld; k++) s[k] = load_chunk<DT>(x, (k * G + j) * V, C);
            if (res) {
                Words t[kHeld];
#pragma unroll
                for (int k = 0; k < kHeld; k++) t[k] = load_chunk<DT>(res, (k * G + j) * V, C);
#pragma unroll
                for (int k = 0; k < kHeld; k++) {
                    s[k] = sum_chunk<DT>(a, s[k], t[k]);
                    store_chunk<DT>(total, (k * G + j) * V, C, s[k]);
                }
            }
#pragma unroll
            for (int k = 0; k < kHeld; k++) take(s[k], w[k]);
        } else {
            for (int c = j * V; c < C; c += G * V) {
                Words t = load_chunk<DT>(x, c, C);
                if (res) {
                    t = sum_chunk<DT>(a, t, load_chunk<DT>(res, c, C));
                    store_chunk<DT>(total, c, C, t);
                }
                if (KIND == kBytes) load_weights<V>(a.weight, c, C, w[0]);
                take(t, w[0]);
            }
        }
        join_row<G, KIND != kSequence>(squares, top, shared, turn);
        float k = 1.0f, inverse = 0.0f;
        if (KIND != kBytesOfValues) k = rstd_of(squares, a);
        if (KIND != kSequence) inverse = rocket::inverse8(top);
        if (j == 0) {
            if (KIND != kBytesOfValues) a.rstd[r] = k;
            if (KIND == kBytes) a.scale[r] = k * rocket::step8(top);
            if (KIND == kBytesOfValues) a.scale[r] = rocket::step8(top);
        }
        auto give = [&](const Words &t, int c, const float (&u)[V]) {
            float f[V];
            values_of<DT>(t, f);
            if (KIND == kSequence) {
#pragma unroll
                for (int e = 0; e < V; e++) f[e] = f[e] * k * u[e];
                store_chunk<DT>(rocket::row_at(a.y, p), c, C, words_of<DT>(f));
            } else if (KIND == kBytes) {
                store_bytes<DT>(a, r, c, f, u, inverse);
            } else {
                float one[V];
#pragma unroll
                for (int e = 0; e < V; e++) one[e] = 1.0f;
                store_bytes<DT>(a, r, c, f, one, inverse);
            }
        };
        if (CHUNKS) {
#pragma unroll
            for (int q = 0; q < kHeld; q++) give(s[q], (q * G + j) * V, w[q]);
        } else {
            for (int c = j * V; c < end; c += G * V) {
                const Words t = load_chunk<DT>(res ? total : x, c, C);
                if (KIND != kBytesOfValues) load_weights<V>(a.weight, c, C, w[0]);
                give(t, c, w[0]);
            }
        }
    }
}

// dw is summed too, in registers (CHUNKS 0: a kernel of its own sums it).  Rows of
// more than 16 elements a thread take the weights anew for every row: the registers
// hold s, dy and the sums.
template <int DT, int G, int CHUNKS>
__global__ __launch_bounds__(threads_of(G)) void back_kernel(BackArgs a) {
    constexpr int V = kVec<DT>, kThreads = threads_of(G), kRows = kThreads / G, kHeld = CHUNKS ? CHUNKS : 1;
    constexpr bool kHold = CHUNKS > 0 && kHeld * V <= 16, kMove = G < 1024;
    // 1,024 threads have 128 registers each: dw's sums lie in shared memory, four values of
    // a thread side by side (8 x 1000 x 20000: fp32 681 us in registers, of which 86 were
    // spilled, 414 so, bf16 446 and 257; x 12001 fp32 327 and 227)
    constexpr bool kAside = CHUNKS > 0 && G == 1024;
    typedef float Four __attribute__((ext_vector_type(4)));
    __shared__ float shared[G > 64 ? 4 * (G / 64) : CHUNKS ? kThreads * V : 1];
    __shared__ Four aside[kAside ? kThreads * kHeld * V / 4 : 1];
    const int j = threadIdx.x % G, C = a.channels;
    const int64_t stride = (int64_t)gridDim.x * kRows;
    const float inv_c = 1.0f / (float)C;
    float w[kHeld][V], dw[kHeld][V];
    if (kAside)
        for (int k = 0; k < kHeld * V / 4; k++) aside[k * kThreads + threadIdx.x] = Four{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < kHeld; k++) {
        if (kHold) load_weights<V>(a.weight, (k * G + j) * V, C, w[k]);
#pragma unroll
        for (int e = 0; e < V; e++) dw[k][e] = 0.0f;
    }
    int turn = 0;
    for (int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / G; r < a.rows.count; r += stride) {
        const Place p = rocket::place_of(a.rows, r);
        char *dx = rocket::row_at(a.dx, p);
        if (!p.live) {
            const Words zero = {0, 0, 0, 0};
            for (int c = j * V; c < C; c += G * V) store_chunk<DT>(dx, c, C, zero);
            continue;
        }
        const char *from_s = rocket::row_at(a.s, p), *from_dy = rocket::row_at(a.dy, p);
        const char *from_dt = a.dt.data ? rocket::row_at(a.dt, p) : nullptr;
        const float k = a.rstd[r];
        float inner = 0.0f;
        uint32_t none = 0;
        auto take = [&](const Words &ts, const Words &td, const float (&u)[V]) {
            float fs[V], fd[V];
            values_of<DT>(ts, fs);
            values_of<DT>(td, fd);
#pragma unroll
            for (int e = 0; e < V; e++) inner = __builtin_fmaf(fd[e] * u[e], fs[e] * k, inner);
        };
        auto give = [&](const Words &ts, const Words &td, const Words &tt, int c, const float (&u)[V], float mean) {
            float fs[V], fd[V], ft[V], out[V];
            values_of<DT>(ts, fs);
            values_of<DT>(td, fd);
            values_of<DT>(tt, ft);
#pragma unroll
            for (int e = 0; e < V; e++) {
                out[e] = k * __builtin_fmaf(-(fs[e] * k), mean, fd[e] * u[e]);
                if (a.dt.data) out[e] += ft[e];
            }
            store_chunk<DT>(dx, c, C, words_of<DT>(out));
        };
        const Words zero = {0, 0, 0, 0};
        if (CHUNKS) {
            Words s[kHeld], d[kHeld], t[kHeld];
#pragma unroll
            for (int q = 0; q < kHeld; q++) {
                s[q] = load_chunk<DT, kMove>(from_s, (q * G + j) * V, C);
                d[q] = load_chunk<DT, kMove>(from_dy, (q * G + j) * V, C);
                t[q] = kHold && from_dt ? load_chunk<DT, kMove>(from_dt, (q * G + j) * V, C) : zero;
            }
#pragma unroll
            for (int q = 0; q < kHeld; q++) {
                if (!kHold) load_weights<V>(a.weight, (q * G + j) * V, C, w[q]);
                take(s[q], d[q], w[q]);
                float fs[V], fd[V];
                values_of<DT>(s[q], fs);
                values_of<DT>(d[q], fd);
                if (kAside) {
#pragma unroll
                    for (int h = 0; h < V / 4; h++) {
                        Four &sum = aside[(q * (V / 4) + h) * kThreads + threadIdx.x];
                        Four v = sum;
#pragma unroll
                        for (int e = 0; e < 4; e++) v[e] = __builtin_fmaf(fd[4 * h + e], fs[4 * h + e] * k, v[e]);
                        sum = v;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < V; e++) dw[q][e] = __builtin_fmaf(fd[e], fs[e] * k, dw[q][e]);
                }
            }
            join_row<G, false>(inner, none, shared, turn);
            const float mean = inner * inv_c;
            // what was computed of the words is computed again, not held over the barrier
#pragma unroll
            for (int q = 0; q < kHeld; q++)
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    uint32_t ws = s[q][e], wd = d[q][e];
                    asm volatile("" : "+v"(ws), "+v"(wd));
                    s[q][e] = ws, d[q][e] = wd;
                }
#pragma unroll
            for (int q = 0; q < kHeld; q++) {
                const int c = (q * G + j) * V;
                if (!kHold) load_weights<V>(a.weight, c, C, w[q]);
                if (!kHold && from_dt) t[q] = load_chunk<DT, kMove>(from_dt, c, C);
                if (c < C) give(s[q], d[q], t[q], c, w[q], mean);
            }
        } else {
            for (int c = j * V; c < C; c += G * V) {
                load_weights<V>(a.weight, c, C, w[0]);
                take(load_chunk<DT, kMove>(from_s, c, C), load_chunk<DT, kMove>(from_dy, c, C), w[0]);
            }
            join_row<G, false>(inner, none, shared, turn);
            const float mean = inner * inv_c;
            for (int c = j * V; c < C; c += G * V) {
                load_weights<V>(a.weight, c, C, w[0]);
                give(load_chunk<DT, kMove>(from_s, c, C), load_chunk<DT, kMove>(from_dy, c, C),
                     from_dt ? load_chunk<DT, kMove>(from_dt, c, C) : zero, c, w[0], mean);
            }
        }
    }
    if (!CHUNKS || !a.partial) return;
    float *to = a.partial + (int64_t)blockIdx.x * C;
#pragma unroll
    for (int q = 0; q < kHeld; q++) {
        const int c = (q * G + j) * V;
        if (kRows > 1) {  // rows of a workgroup meet in shared memory, chunk by chunk
            __syncthreads();
#pragma unroll
            for (int e = 0; e < V; e++) shared[(threadIdx.x / G) * G * V + j * V + e] = dw[q][e];
            __syncthreads();
            for (int e = threadIdx.x; e < G * V; e += kThreads) {
                float sum = 0.0f;
#pragma unroll
                for (int g = 0; g < kRows; g++) sum += shared[g * G * V + e];
                if (q * G * V + e < C) to[q * G * V + e] = sum;
            }
        } else {
#pragma unroll
            for (int e = 0; e < V; e++) {
                const float sum = kAside ? aside[(q * (V / 4) + e / 4) * kThreads + threadIdx.x][e % 4] : dw[q][e];
                if (c + e < C) to[c + e] = sum;
            }
        }
    }
}

// dw of rows too wide for registers: a thread a column, the rows dealt to
// gridDim.y workgroups.
template <int DT>
__global__ __launch_bounds__(256) void weight_kernel(BackArgs a) {
    using raw = typename Elem<DT>::raw;
    const int c = blockIdx.x * 256 + threadIdx.x;
    float sum = 0.0f;
    for (int64_t r = blockIdx.y; r < a.rows.count; r += gridDim.y) {
        const Place p = rocket::place_of(a.rows, r);
        if (!p.live || c >= a.channels) continue;
        const float s = Elem<DT>::one(((const raw *)rocket::row_at(a.s, p))[c]);
        const float d = Elem<DT>::one(((const raw *)rocket::row_at(a.dy, p))[c]);
        sum = __builtin_fmaf(d, s * a.rstd[r], sum);
    }
    if (c < a.channels) a.partial[(int64_t)blockIdx.y * a.channels + c] = sum;
}

// Sums of `parts` rows of partial sums: 16 columns a workgroup, 64 rows at once,
// joined in a fixed order.
__global__ __launch_bounds__(1024) void join_kernel(const float *partial, float *sum, int64_t parts, int32_t channels) {
    __shared__ float shared[64][17];
    const int col = threadIdx.x % 16, row = threadIdx.x / 16;
    const int64_t c = (int64_t)blockIdx.x * 16 + col;
    float v = 0.0f;
    if (c < channels)
        for (int64_t p = row; p < parts; p += 64) v += partial[p * channels + c];
    shared[row][col] = v;
    __syncthreads();
    if (threadIdx.x < 16 && c < channels) {
        float t = 0.0f;
        for (int k = 0; k < 64; k++) t += shared[k][threadIdx.x];
        sum[c] = t;
    }
}

constexpr int kCus = 256;

// Workgroups of a call.  Of rows that a workgroup shares or holds in two loads each, as
// many as there are (500 x 1000 x 256 bf16 with a residual: 178 us; 211 us where only
// those that run at once go from row to row); of wider rows those that run at once,
// which keep the weights (20 x 1000 x 6000 bf16: 94 us against 114 us).
inline uint32_t grid_of(int64_t rows, int threads, int rows_each, int chunks) {
    const int64_t most = threads == 256 && chunks <= 2 ? 1 << 22 : (int64_t)kCus * (2048 / threads);
    return (uint32_t)std::min((rows + rows_each - 1) / rows_each, most);
}

template <int DT, int G, int CHUNKS, int KIND>
void norm_one(const NormArgs &a, hipStream_t s) {
    constexpr int kThreads = threads_of(G);
    norm_kernel<DT, G, CHUNKS, KIND><<<grid_of(a.rows.count, kThreads, kThreads / G, CHUNKS), kThreads, 0, s>>>(a);
}

// The threads and chunks that hold a row: as few threads as take at most 4
// chunks (2 of workgroups' rows), since a row's sum costs the same for few as
// for many chunks.
template <int DT, int KIND>
void norm_type(const NormArgs &a, hipStream_t s) {
    const int64_t chunks = ((KIND == kSequence ? a.channels : a.padded) + kVec<DT> - 1) / kVec<DT>;
    if (chunks <= 16) norm_one<DT, 16, 1, KIND>(a, s);
    else if (chunks <= 32) norm_one<DT, 32, 1, KIND>(a, s);
    else if (chunks <= 64) norm_one<DT, 64, 1, KIND>(a, s);
    else if (chunks <= 128) norm_one<DT, 64, 2, KIND>(a, s);
    else if (chunks <= 256) norm_one<DT, 64, 4, KIND>(a, s);
    else if (chunks <= 512) norm_one<DT, 256, 2, KIND>(a, s);
    else if (chunks <= 1024) norm_one<DT, 256, 4, KIND>(a, s);
    else if (chunks <= 2048) norm_one<DT, 1024, 2, KIND>(a, s);
    else if (chunks <= 24576 / kVec<DT>) norm_one<DT, 1024, 24 / kVec<DT>, KIND>(a, s);
    else norm_one<DT, 1024, 0, KIND>(a, s);
}

template <int KIND>
rocket_status norm_launch(const NormArgs &a, int32_t dtype, void *stream) {
    hipStream_t s = (hipStream_t)stream;
    if (dtype == ROCKET_FLOAT32)
        norm_type<ROCKET_FLOAT32, KIND>(a, s);
    else if (dtype == ROCKET_BFLOAT16)
        norm_type<ROCKET_BFLOAT16, KIND>(a, s);
    else
        norm_type<ROCKET_FLOAT16, KIND>(a, s);
    return rocket::launched();
}

// ------------------------------------------------------------ backward pass
constexpr int kWideParts = 64;     // the same of rows too wide for registers

int64_t chunks_of(const rocket_sequence_shape *s) {
    const int v = s->dtype == ROCKET_FLOAT32 ? 4 : 8;
    return (s->channels + v - 1) / v;
}

bool too_wide(const rocket_sequence_shape *s) { return s->channels > 24576; }

// Threads and loads of a row in the backward pass: at most 16 elements a thread, so
// that s, dy, the weights and their sums stay in registers (20 x 1000 x 6000 bf16: 210
// us, and 414 with 32 elements, where the weights are read for each row and a SIMD holds
// one wave; 2000 channels, 100 x 1000: 240 and 344).  The last kind, 24, reads them.
// The workgroups are at most those that run at once, each with a sum of dw in registers;
// more make waves of unlike length and more sums to join (100 x 1000 x 2000 bf16: 240 us, 274
// with two thirds of them, 308 with four thirds).
struct Row {
    int threads, chunks;
};

Row row_of(int64_t chunks, int vec) {
    const int most = 16 / vec;   // loads of a thread
    if (chunks <= 16) return {16, 1};
    if (chunks <= 32) return {32, 1};
    if (chunks <= 64) return {64, 1};
    if (chunks <= 128) return {64, 2};
    if (chunks <= 64 * most) return {64, most};
    for (int g = 128; g <= 1024; g *= 2)
        if (chunks <= g * most) return {g, most};
    return {1024, 24 / vec};
}

int64_t back_parts(const rocket_sequence_shape *s) {
    const int64_t rows = s->n * s->steps;
    if (too_wide(s)) return std::min<int64_t>(rows, kWideParts);
    const int vec = s->dtype == ROCKET_FLOAT32 ? 4 : 8;
    const Row row = row_of(chunks_of(s), vec);
    const int each = threads_of(row.threads) / row.threads;
    // waves of a SIMD: three, which is what rows of 16 elements a thread leave room for and
    // what feeds it where every thread's loads are whole; of narrower rows that leave
    // threads idle or end inside a load six (1,000,000 x 64 bf16 157 us with three, 103
    // with six; 1,000,000 x 256 386 and 423)
    const bool whole = s->channels % (row.threads * row.chunks * vec) == 0;
    const int waves = row.threads <= 64 && row.chunks * vec <= 8 && !whole ? 6 : 3;
    const int most = row.threads < 512 ? kCus * waves * 256 / threads_of(row.threads) : kCus;
    return std::min<int64_t>((rows + each - 1) / each, most);
}

template <int DT, int G, int CHUNKS>
void back_one(const BackArgs &a, int64_t parts, hipStream_t s) {
    constexpr int kThreads = threads_of(G);
    back_kernel<DT, G, CHUNKS><<<(uint32_t)parts, kThreads, 0, s>>>(a);
}

template <int DT>
void back_type(const BackArgs &a, int64_t parts, hipStream_t s) {
    constexpr int V = kVec<DT>, kMost = 16 / V;
    const int64_t chunks = (a.channels + V - 1) / V;
    if (a.channels > 24576) {
        if (a.partial)  // first: dx may be written over dy or s
            weight_kernel<DT><<<dim3((uint32_t)((a.channels + 255) / 256), (uint32_t)parts), 256, 0, s>>>(a);
        back_one<DT, 1024, 0>(a, std::min<int64_t>(a.rows.count, 2 * kCus), s);
        return;
    }
    const Row row = row_of(chunks, V);
    switch (row.threads) {
    case 16: back_one<DT, 16, 1>(a, parts, s); break;
    case 32: back_one<DT, 32, 1>(a, parts, s); break;
    case 64:
        if (row.chunks == 1)
            back_one<DT, 64, 1>(a, parts, s);
        else if (row.chunks == 2)
            back_one<DT, 64, 2>(a, parts, s);
        else
            back_one<DT, 64, kMost>(a, parts, s);
        break;
    case 128: back_one<DT, 128, kMost>(a, parts, s); break;
    case 256: back_one<DT, 256, kMost>(a, parts, s); break;
    case 512: back_one<DT, 512, kMost>(a, parts, s); break;
    default:
        if (row.chunks == kMost)
            back_one<DT, 1024, kMost>(a, parts, s);
        else
            back_one<DT, 1024, 24 / V>(a, parts, s);
    }
}

bool eps_ok(float eps) { return eps >= 0.0f && eps <= 3.4028234e38f; }

// The checks that the two forward passes share, and their arguments.
bool forward_args(const rocket_sequence_shape *shape, const rocket_sequence *x, const rocket_sequence *residual,
                  const float *weight, float eps, const rocket_sequence *total, const float *rstd, NormArgs &a) {
    if (!rocket::shape_ok(shape) || !eps_ok(eps) || !rocket::view_ok(x, shape)) return false;
    if ((residual != nullptr) != (total != nullptr)) return false;
    if (residual && (!rocket::view_ok(residual, shape) || !rocket::out_ok(total, shape))) return false;
    if (weight && !rocket::floats_ok(weight)) return false;
    if (!rocket::empty(shape) && !rocket::floats_ok(rstd)) return false;
    a.x = rocket::view_of(x, shape->dtype);
    a.r = rocket::view_of(residual, shape->dtype);
    a.total = rocket::view_of(total, shape->dtype);
    a.weight = weight, a.rstd = const_cast<float *>(rstd);
    a.channels = (int32_t)shape->channels, a.eps = eps;
    a.padded = rocket::padded8(shape->channels);
    return true;
}

}  // namespace

extern "C" rocket_status rocket_rms_norm_forward(const rocket_sequence_shape *shape, const rocket_sequence *x,
                                                 const rocket_sequence *residual, const float *weight, float eps,
                                                 const rocket_sequence *y, const rocket_sequence *total, float *rstd,
                                                 void *hip_stream) {
    NormArgs a = {};
    if (!forward_args(shape, x, residual, weight, eps, total, rstd, a) || !rocket::out_ok(y, shape))
        return ROCKET_ERR_INVALID_ARG;
    if (rocket::empty(shape)) return ROCKET_OK;
    if (total && total->data == y->data) return ROCKET_ERR_INVALID_ARG;   // one of the two would be lost
    a.y = rocket::view_of(y, shape->dtype);
    View *views[] = {&a.x, &a.r, &a.total, &a.y};
    a.rows = rocket::rows_of(shape, views, 4);
    return norm_launch<kSequence>(a, shape->dtype, hip_stream);
}

extern "C" rocket_status rocket_rms_norm_bytes_forward(const rocket_sequence_shape *shape, const rocket_sequence *x,
                                                  const rocket_sequence *residual, const float *weight, float eps,
                                                  int8_t *q, float *scale, const rocket_sequence *total, float *rstd,
                                                  void *hip_stream) {
    NormArgs a = {};
    if (!forward_args(shape, x, residual, weight, eps, total, rstd, a)) return ROCKET_ERR_INVALID_ARG;
    if (rocket::empty(shape)) return ROCKET_OK;
    if (!rocket::bytes_ok(q) || !rocket::floats_ok(scale)) return ROCKET_ERR_INVALID_ARG;
    a.q = q, a.scale = scale;
    View *views[] = {&a.x, &a.r, &a.total};
    a.rows = rocket::rows_of(shape, views, 3);
    return norm_launch<kBytes>(a, shape->dtype, hip_stream);
}

extern "C" rocket_status rocket_quantize_rows(const rocket_sequence_shape *shape, const rocket_sequence *x, int8_t *q,
                                              float *scale, void *hip_stream) {
    if (!rocket::shape_ok(shape) || !rocket::view_ok(x, shape)) return ROCKET_ERR_INVALID_ARG;
    if (rocket::empty(shape)) return ROCKET_OK;
    if (!rocket::bytes_ok(q) || !rocket::floats_ok(scale)) return ROCKET_ERR_INVALID_ARG;
    NormArgs a = {};
    a.x = rocket::view_of(x, shape->dtype);
    a.channels = (int32_t)shape->channels;
    a.padded = rocket::padded8(shape->channels);
    a.q = q, a.scale = scale;
    View *views[] = {&a.x};
    a.rows = rocket::rows_of(shape, views, 1);
    return norm_launch<kBytesOfValues>(a, shape->dtype, hip_stream);
}

extern "C" rocket_status rocket_rms_norm_workspace(const rocket_sequence_shape *shape, int64_t *bytes) {
    if (!bytes || !rocket::shape_ok(shape)) return ROCKET_ERR_INVALID_ARG;
    *bytes = 0;
    if (rocket::empty(shape)) return ROCKET_OK;
    const int64_t parts = back_parts(shape);
    if (parts > 1) *bytes = (parts * shape->channels * 4 + 7) / 8 * 8;
    return ROCKET_OK;
}

extern "C" rocket_status rocket_rms_norm_backward(const rocket_sequence_shape *shape, const rocket_sequence *dy,
                                                  const rocket_sequence *total, const float *weight, const float *rstd,
                                                  const rocket_sequence *dtotal, const rocket_sequence *dx,
                                                  float *dweight, void *workspace, int64_t workspace_bytes,
                                                  void *hip_stream) {
    if (!rocket::shape_ok(shape) || !rocket::view_ok(dy, shape) || !rocket::view_ok(total, shape) ||
        (dtotal && !rocket::view_ok(dtotal, shape)) || !rocket::out_ok(dx, shape))
        return ROCKET_ERR_INVALID_ARG;
    if ((weight && !rocket::floats_ok(weight)) || (dweight && !rocket::floats_ok(dweight)))
        return ROCKET_ERR_INVALID_ARG;
    hipStream_t s = (hipStream_t)hip_stream;
    const int32_t channels = (int32_t)shape->channels;
    if (rocket::empty(shape)) {  // a sum of no rows
        if (dweight) join_kernel<<<(uint32_t)((channels + 15) / 16), 1024, 0, s>>>(nullptr, dweight, 0, channels);
        return dweight ? rocket::launched() : ROCKET_OK;
    }
    int64_t need = 0;
    rocket_rms_norm_workspace(shape, &need);
    if (!rocket::floats_ok(rstd)) return ROCKET_ERR_INVALID_ARG;
    if (dweight && need && (!workspace || (uintptr_t)workspace % 8 != 0 || workspace_bytes < need))
        return ROCKET_ERR_INVALID_ARG;
    BackArgs a = {};
    a.dy = rocket::view_of(dy, shape->dtype), a.s = rocket::view_of(total, shape->dtype);
    a.dt = rocket::view_of(dtotal, shape->dtype), a.dx = rocket::view_of(dx, shape->dtype);
    a.weight = weight, a.rstd = rstd, a.channels = channels;
    const int64_t parts = back_parts(shape);
    a.partial = !dweight ? nullptr : parts > 1 ? (float *)workspace : dweight;
    View *views[] = {&a.dy, &a.s, &a.dt, &a.dx};
    a.rows = rocket::rows_of(shape, views, 4);
    if (shape->dtype == ROCKET_FLOAT32)
        back_type<ROCKET_FLOAT32>(a, parts, s);
    else if (shape->dtype == ROCKET_BFLOAT16)
        back_type<ROCKET_BFLOAT16>(a, parts, s);
    else
        back_type<ROCKET_FLOAT16>(a, parts, s);
    if (dweight && parts > 1)
        join_kernel<<<(uint32_t)((channels + 15) / 16), 1024, 0, s>>>(a.partial, dweight, parts, channels);
    return rocket::launched();
}
