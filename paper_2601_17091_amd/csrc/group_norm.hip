// Group norm with an activation over sequences [n, L, C], channels last.
//
// A series of T steps, a group of C / G channels, N = T C / G elements:
//   m = sum x / N,  s = sum (x - m)^2 / N,  r = 1 / sqrt(s + eps)
//   xh = (x - m) r,  z = xh w_c + b_c,  y = act(z)
// and backwards, with dz = dy act'(z) and g = dz w_c,
//   db_c = sum dz,  dw_c = sum dz xh  (over series and steps)
//   dx = r (g - mean(g) - xh mean(g xh))  (means over the group's N elements)
//
// A workgroup takes a slab: all steps of a few whole groups, mostly at least
// 128 bytes of channels wide.  Where the slab fits its registers it is read
// once: the sum, then the squares about the mean, then the output come from
// there (held).  Longer series are cut into chunks of steps: one launch leaves
// each chunk's mean and squares (or, backwards, its sums), a second one merges
// them in a fixed order and writes the output.  Groups wider than a workgroup's
// columns are cut along the channels in the same way.  There are no atomics:
// results do not change from call to call.
//
// A thread owns one column of 16 bytes of channels in every `rows`-th step.
// The last column of a slab is moved back so that it ends with the slab; the
// channels it shares with its neighbour are computed twice and counted once.
// Where every column lies in one group (groups of whole columns, or one group a
// slab) a thread's sums are one number a quantity, one barrier and a few
// shuffles join them, and a workgroup goes through several series whose columns
// load as the last series' are written.  Else the sums are joined channel by
// channel in shared memory.
//
// Bound: HBM, and the vector unit beside it.  Backward with SiLU, 1000 x 1000 x
// 256, bf16: 384 to 391 us, 4.0 TB/s of the 1,536 MB that have to move (a sum of
// two tensors of that size reaches 6.1 TB/s); the slope is computed twice, in the
// sums and again for dx, since dy times the slope in 32 bits would be half as much
// again to hold: 35 vector instructions an element, 66 % of the vector unit's time.
// Most kernels that hold 8 columns of x and of dy spill a few registers (this one
// 16 of 128, 52 bytes a thread).  Forward, 1000 x 1000 x 256 without an activation:
// 205 to 237 us in bf16, 378 us in fp32 (5.4 TB/s).  4 x 16384 x 512, bf16, GELU:
// 48 to 51 us, the slabs being read twice (15 us and 33 us).  777 x 129 x 924 in
// groups of 33, fp16, ReLU, ragged: 88 to 94 us.
#include <algorithm>
#include <iterator>
#include <type_traits>

#include "sequence.h"

namespace {

using rocket::Elem;

enum Mode { kHeld, kStats, kApply };

struct View {
    char *p;
    int64_t ss, ts;  // bytes
};

struct NormArgs {
    View x, dy, out;   // out: y, or dx
    int32_t n, L;
    int32_t C, G, width;       // width: channels of a group
    int32_t slabs, parts;      // slabs per series; parts > 1: slabs per group
    int32_t cols, rows;        // columns of a slab; steps a workgroup passes at once
    int32_t chunks;            // of steps
    int32_t most_groups;       // groups of a slab, at most
    int32_t in_place;          // the output is one of the inputs
    int32_t act;
    float eps;
    const float *w, *b;        // or null
    const int32_t *lengths;
    float *mean, *rstd;        // [n, G]: written forward, read backward
    float2 *stats;             // [n, G, chunks * parts]: (mean, squares), backward sums of dz w and of dz w xh
    float *sums;               // backward: [rows of sums, 2, C] sums of dz and dz xh
    int32_t series;            // backward, held: workgroups along the series
};

// A column's elements: 16 bytes, or one element where a row has fewer.
template <int DT, bool WIDE>
struct Pack {
    typedef uint32_t vec __attribute__((ext_vector_type(4)));
    static constexpr int kN = 4 * Elem<DT>::kPerWord;
    vec v;
    __device__ void load(const char *p) { v = rocket::load_at<vec>(p); }
    __device__ float get(int e) const { return Elem<DT>::get(v[e / Elem<DT>::kPerWord], e % Elem<DT>::kPerWord); }
    __device__ typename Elem<DT>::raw element(int e) const {
        using bits = typename Elem<DT>::bits;
        return __builtin_bit_cast(typename Elem<DT>::raw, (bits)(v[e / Elem<DT>::kPerWord] >> 16 * (e % Elem<DT>::kPerWord)));
    }
    __device__ void set(int e, float f) { v[e] = __builtin_bit_cast(uint32_t, f); }   // fp32 elements
    // Elements e to e + N, rounded.  Two neighbours write the channels that they
    // share, each at another e, so that all conversions are the same instruction.
    // Left to itself the compiler fuses some of those to fp16 with the operation
    // before them, which rounds that operation's exact result and may differ.
    template <int N>
    __device__ void put(int e, const float (&f)[N]) {
#pragma unroll
        for (int k = 0; k < N / Elem<DT>::kPerWord; k++) {
            uint32_t w;
            if constexpr (DT == ROCKET_FLOAT16)
                asm("v_cvt_pk_f16_f32 %0, %1, %2" : "=v"(w) : "v"(f[2 * k]), "v"(f[2 * k + 1]));
            else
                w = Elem<DT>::put(f + k * Elem<DT>::kPerWord);
            v[e / Elem<DT>::kPerWord + k] = w;
        }
    }
    __device__ void store(char *p) const { rocket::store_at(p, v); }
    __device__ void clear() { v = vec{0, 0, 0, 0}; }
    __device__ void renew() {
        uint32_t w[4] = {v[0], v[1], v[2], v[3]};
        rocket::renew(w);
        v = vec{w[0], w[1], w[2], w[3]};
    }
};

template <int DT>
struct Pack<DT, false> {
    using raw = typename Elem<DT>::raw;
    static constexpr int kN = 1;
    raw v;
    __device__ void load(const char *p) { v = *(const raw *)p; }
    __device__ float get(int) const { return Elem<DT>::one(v); }
    __device__ raw element(int) const { return v; }
    __device__ void set(int, float f) { v = f; }
    __device__ void put(int, const float (&f)[1]) { v = Elem<DT>::round(f[0]); }
    __device__ void store(char *p) const { *(raw *)p = v; }
    __device__ void clear() { v = 0; }
    __device__ void renew() {}
};

// The normal distribution function and e = exp(-z^2 / 2).  Its lower tail is
// e t P(t) with t = 1 / (1 + p |z|): exp(z^2 / 2) times the tail is smooth in t, and
// P is a polynomial fitted to it in the relative error (Lawson's weighted least
// squares), so that values far below 0 keep their digits.
//   fp32 elements: P of degree 8, 2e-8 relative; z^2 in two parts, so that the tail
//   is good to 12 units of 2^-24 down to z = -12.5; where |z| < 1, 1/2 + z Q(z^2)
//   with Q of degree 5, whose rounding is the result's own.
//   16-bit elements: P of degree 5, the lesser of 7.3e-8 and 1e-4 of the tail, a
//   fifth of an fp16 rounding.
template <int DT>
__device__ inline float normal_cdf(float z, float &e) {
    if (DT != ROCKET_FLOAT32) {
        e = rocket::exp_neg_abs<DT>(0.5f * z * z);
        const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_fabsf(z), 0.29f, 1.0f));
        float q = __builtin_fmaf(t, -0.08850604f, 0.28376429f);
        q = __builtin_fmaf(t, q, -0.09162589f);
        q = __builtin_fmaf(t, q, 0.17847331f);
        q = __builtin_fmaf(t, q, 0.10106501f);
        q = __builtin_fmaf(t, q, 0.11682939f);
        const float tail = q * t * e;
        return z < 0.0f ? tail : 1.0f - tail;
    }
    // at 15 e is 0; a NaN goes on through the callers' products with z
    const float u = __builtin_amdgcn_fmed3f(__builtin_fabsf(z), 0.0f, 15.0f);
    const float s = u * u, low = __builtin_fmaf(u, u, -s);
    e = rocket::exp_neg_abs<DT>(0.5f * s);
    e = __builtin_fmaf(e, -0.5f * low, e);
    float c = __builtin_fmaf(s, -7.654199180251453e-06f, 0.0001134863487095572f);
    c = __builtin_fmaf(s, c, -0.001186329871416092f);
    c = __builtin_fmaf(s, c, 0.009973322972655296f);
    c = __builtin_fmaf(s, c, -0.06649035960435867f);
    c = __builtin_fmaf(s, c, 0.3989422917366028f);
    c = __builtin_fmaf(z, c, 0.5f);
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(u, 0.21f, 1.0f));
    float q = __builtin_fmaf(t, -0.07122398912906647f, 0.28145527839660645f);
    q = __builtin_fmaf(t, q, -0.3257579207420349f);
    q = __builtin_fmaf(t, q, 0.34412485361099243f);
    q = __builtin_fmaf(t, q, -0.09015858173370361f);
    q = __builtin_fmaf(t, q, 0.12320016324520111f);
    q = __builtin_fmaf(t, q, 0.06964277476072311f);
    q = __builtin_fmaf(t, q, 0.08500158041715622f);
    q = __builtin_fmaf(t, q, 0.08371583372354507f);
    const float tail = q * t * e;
    return u < 1.0f ? c : z < 0.0f ? tail : 1.0f - tail;
}

template <int DT, int ACT>
__device__ inline float activate(float z) {
    if (ACT == ROCKET_ACT_RELU) return z < 0.0f ? 0.0f : z;
    if (ACT == ROCKET_ACT_SILU) {
        float s, rest;
        rocket::logistic<DT>(z, s, rest);
        return z * s;
    }
    if (ACT == ROCKET_ACT_GELU) {
        float e;
        return z * normal_cdf<DT>(z, e);
    }
    return z;
}

template <int DT, int ACT>
__device__ inline float slope(float z) {
    if (ACT == ROCKET_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
    if (ACT == ROCKET_ACT_SILU) {
        float s;
        if (DT == ROCKET_FLOAT32) {
            float rest;
            rocket::logistic<DT>(z, s, rest);
            return s * __builtin_fmaf(z, rest, 1.0f);
        }
        s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504f));
        return s * (1.0f + __builtin_fmaf(-s, z, z));
    }
    if (ACT == ROCKET_ACT_GELU) {
        float e;
        const float c = normal_cdf<DT>(z, e);
        return __builtin_fmaf(z * 0.39894228040143268f, e, c);
    }
    return 1.0f;
}

// Where a workgroup and a thread work.
struct Place {
    uint32_t i;           // series
    int slab, chunk;
    int c0, c1, g0, ng;   // the slab's channels and groups
    int row, col;         // the thread's first step in a pass, its column
    int c, skip;          // its first channel; leading channels that its neighbour counts
    bool active;
};

template <int NT, int VEC>
__device__ inline void place_thread(const NormArgs &a, Place &p) {
    if (a.parts == 1) {
        p.g0 = (int)((int64_t)a.G * p.slab / a.slabs);
        p.ng = (int)((int64_t)a.G * (p.slab + 1) / a.slabs) - p.g0;
        p.c0 = p.g0 * a.width;
        p.c1 = p.c0 + p.ng * a.width;
    } else {
        p.g0 = p.slab / a.parts;
        p.ng = 1;
        const int part = p.slab % a.parts, base = p.g0 * a.width;
        p.c0 = base + (int)((int64_t)a.width * part / a.parts);
        p.c1 = base + (int)((int64_t)a.width * (part + 1) / a.parts);
    }
    p.row = threadIdx.x / a.cols;
    p.col = threadIdx.x - p.row * a.cols;
    const int nominal = p.c0 + p.col * VEC;
    p.active = p.row < a.rows && nominal < p.c1;
    p.c = nominal + VEC <= p.c1 ? nominal : p.c1 - VEC;
    p.skip = nominal - p.c;
    // the threads left over load the slab's first column, which is in bounds
    if (!p.active) p.c = p.c0, p.skip = 0, p.row = 0;
}

// Shared memory of a slab, sized by the launch.  Arrays start on 16 bytes.
struct Scratch {
    float *group, *group2;   // [groups of a slab]
    float *rows;             // [rows][W]: the threads' sums, or [2][threads]
    float *chan;             // parts of the channels' sums
    float *of[4];            // [4][W]: what the elements of a channel are scaled by
    float *first;            // [W], backward
    float *total;            // [2][W], backward, held
};

// What a call's kernels keep there.  Where every column lies in one group, a
// thread's sums are one number a quantity, and the scales are read as needed.
// At most 57 KB, since 256 columns of 16 bytes, the widest slab, are chunks or
// kOne; but kOneBack of 1,024 threads takes 74 to 94 KB, and asks for it.
enum Keep { kSums, kSumsBack, kChunkBack, kOne, kOneBack };

__host__ __device__ inline int pad4(int n) { return (n + 3) / 4 * 4; }

__host__ __device__ inline int64_t scratch_floats(int threads, int vec, int cols, int rows, int groups, int keep) {
    const int W = cols * vec, head = 2 * pad4(groups);
    if (keep == kOne) return head + 2 * threads + 2 * W;
    if (keep == kOneBack) return head + 2 * threads + 2 * W + 2 * (int64_t)threads * vec;
    return head + (int64_t)rows * W + pad4(threads > W ? threads : W) + (keep == kSumsBack ? 7 : keep == kChunkBack ? 5 : 4) * W;
}

template <int NT, int VEC>
__device__ inline Scratch scratch_of(const NormArgs &a) {
    extern __shared__ __attribute__((aligned(16))) float shared[];
    const int W = a.cols * VEC;
    Scratch s;
    s.group = shared;
    s.group2 = s.group + pad4(a.most_groups);
    s.rows = s.group2 + pad4(a.most_groups);
    s.chan = s.rows + a.rows * W;
    s.of[0] = s.chan + pad4(NT > W ? NT : W);
    for (int k = 1; k < 4; k++) s.of[k] = s.of[k - 1] + W;
    s.first = s.of[3] + W;
    s.total = s.first + W;
    return s;
}

// The values of an array of channels for a thread's column, from its element
// `from` on.
template <int N>
__device__ inline void of_column(const float *of, const Place &p, float (&v)[N], int from = 0) {
    const float *at = of + (p.c - p.c0) + from;
#pragma unroll
    for (int e = 0; e < N; e++) v[e] = at[e];
}

// fn(channel of the slab, its group of the slab), a thread a channel.
template <int NT, class Fn>
__device__ inline void for_channels(const NormArgs &a, const Place &p, Fn fn) {
    for (int ch = threadIdx.x; ch < p.c1 - p.c0; ch += NT) fn(ch, a.parts == 1 ? ch / a.width : 0);
}

// Sums acc over the workgroup's rows: s.chan[part * W + channel], `parts`
// parts of every channel of the slab.
template <int NT, int VEC>
__device__ inline int sum_rows(const NormArgs &a, const Place &p, const float (&acc)[VEC], const Scratch &s) {
    const int W = p.c1 - p.c0;
    __syncthreads();   // rows and chan are free
    if (p.active) {
        float *at = s.rows + p.row * W + p.c - p.c0;
        if (p.skip == 0) {
#pragma unroll
            for (int e = 0; e < VEC; e++) at[e] = acc[e];
        } else {
#pragma unroll
            for (int e = 0; e < VEC; e++)
                if (e >= p.skip) at[e] = acc[e];
        }
    }
    __syncthreads();
    const int parts = W < NT ? min(NT / W, a.rows) : 1;
    const int per = W < NT ? W : NT;
    const int part = threadIdx.x / per;
    if (part < parts)
        for (int ch = threadIdx.x - part * per; ch < W; ch += NT) {
            float t = 0.0f;
            for (int r = part; r < a.rows; r += parts) t += s.rows[r * W + ch];
            s.chan[part * W + ch] = t;
        }
    __syncthreads();
    return parts;
}

// group[k] = the sum over the slab's channels of group k of scale_c times the
// channel's `parts` values in `of` (scale may be null).
template <int NT>
__device__ inline void sum_groups(const Place &p, const float *of, int parts, const float *scale, float *group) {
    const int W = p.c1 - p.c0, each = W / p.ng;
    auto channel = [&](int ch) {
        float u = 0.0f;
        for (int q = 0; q < parts; q++) u += of[q * W + ch];
        return scale ? scale[p.c0 + ch] * u : u;
    };
    if (each * parts <= 32) {
        for (int k = threadIdx.x; k < p.ng; k += NT) {
            float t = 0.0f;
            for (int ch = k * each; ch < (k + 1) * each; ch++) t += channel(ch);
            group[k] = t;
        }
    } else {
        for (int k = threadIdx.x >> 6; k < p.ng; k += NT >> 6) {
            float t = 0.0f;
            for (int ch = k * each + (threadIdx.x & 63); ch < (k + 1) * each; ch += 64) t += channel(ch);
#pragma unroll
            for (int off = 32; off; off /= 2) t += __shfl_xor(t, off);
            if ((threadIdx.x & 63) == 0) group[k] = t;
        }
    }
    __syncthreads();
}

// Where every column lies in one group: t1 and t2 become their sums over the
// threads of the thread's own group, in all of them.  `g`: its group of the slab.
template <int NT, int VEC>
__device__ inline void sum_two(const NormArgs &a, const Place &p, int g, float &t1, float &t2, float *rows,
                               float *group, float *group2) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (!p.active) t1 = 0.0f, t2 = 0.0f;
    if (p.ng == 1) {
#pragma unroll
        for (int off = 32; off; off /= 2) t1 += __shfl_xor(t1, off), t2 += __shfl_xor(t2, off);
        if (NT == 64) return;
        __syncthreads();   // rows is free
        if (lane == 0) rows[wave] = t1, rows[NT + wave] = t2;
        __syncthreads();
        t1 = 0.0f, t2 = 0.0f;
        for (int k = 0; k < NT / 64; k++) t1 += rows[k], t2 += rows[NT + k];
        return;
    }
    __syncthreads();   // rows and the groups are free
    rows[threadIdx.x] = t1, rows[NT + threadIdx.x] = t2;
    __syncthreads();
    const int each = a.width / VEC;   // columns of a group
    if (each * a.rows <= 16) {
        for (int k = threadIdx.x; k < 2 * p.ng; k += NT) {
            const float *at = rows + (k & 1) * NT + (k >> 1) * each;
            float u = 0.0f;
            for (int r = 0; r < a.rows; r++)
                for (int c = 0; c < each; c++) u += at[r * a.cols + c];
            (k & 1 ? group2 : group)[k >> 1] = u;
        }
    } else {
        const int side = each < 64 ? each : 64, down = 64 / side, r0 = lane / side, c0 = lane - r0 * side;
        for (int k = wave; k < 2 * p.ng; k += NT / 64) {
            const float *at = rows + (k & 1) * NT + (k >> 1) * each;
            float u = 0.0f;
            if (r0 < down)
                for (int r = r0; r < a.rows; r += down)
                    for (int c = c0; c < each; c += side) u += at[r * a.cols + c];
#pragma unroll
            for (int off = 32; off; off /= 2) u += __shfl_xor(u, off);
            if (lane == 0) (k & 1 ? group2 : group)[k >> 1] = u;
        }
    }
    __syncthreads();
    t1 = group[g], t2 = group2[g];
}

// The steps of chunk k, and how many of them are the series' own.
__device__ inline int chunk_rows(const NormArgs &a, int64_t T, int chunk, int64_t per, int64_t &first) {
    first = chunk * per;
    int64_t left = T - first;
    return (int)(left < 0 ? 0 : left < per ? left : per);
}

// The column of step `pass` + row of a workgroup's pass over `rows` steps, 0
// past the series' own steps.
template <class P>
__device__ inline void load_row(P &v, const char *at, int pass, int rows, int row, int own, int64_t stride) {
    if (pass + rows <= own) {   // the same for the whole workgroup
        v.load(at + pass * stride);
    } else {
        v.clear();
        if (pass + row < own) v.load(at + pass * stride);
    }
}

// Writes a column.  Where the output goes over an input that other threads
// have not read yet (a second launch over chunks, in place), a column that was
// moved back leaves the channels that its neighbour counts to the neighbour.
template <int DT, class P>
__device__ inline void store_column(char *at, const P &v, const Place &p, bool in_place) {
    if (!in_place || p.skip == 0) {
        v.store(at);
        return;
    }
    using raw = typename Elem<DT>::raw;
#pragma unroll
    for (int e = 0; e < P::kN; e++)
        if (e >= p.skip) ((raw *)at)[e] = v.element(e);
}

template <int DT>
__device__ inline char *column_at(const View &x, const Place &p, int64_t first) {
    return x.p + p.i * x.ss + (first + p.row) * x.ts + (int64_t)p.c * Elem<DT>::kSize;
}

// Forward.  R: passes over the rows that a thread holds.
template <int DT, bool WIDE, int NT, int R, int MODE, bool ONE>
__global__ __launch_bounds__(NT, NT == 512 ? 4 : 3) void norm_kernel(NormArgs a) {
    using P = Pack<DT, WIDE>;
    constexpr int VEC = P::kN;
    const Scratch s = scratch_of<NT, VEC>(a);
    Place p;
    const uint32_t b = rocket::item_of_block(), rest_of = rocket::uniform(b / a.slabs);
    p.slab = rocket::uniform(b - rest_of * a.slabs);
    p.i = rocket::uniform(rest_of / a.chunks);
    p.chunk = rocket::uniform(rest_of - p.i * a.chunks);
    place_thread<NT, VEC>(a, p);
    const int64_t T = rocket::steps_of(a.lengths, p.i, a.L), per = (int64_t)R * a.rows;
    int64_t first;
    const int own = chunk_rows(a, T, p.chunk, per, first);

    // Columns at a time: all that the thread holds, or four in a second launch.
    constexpr int H = MODE == kApply && R > 4 ? 4 : R;
    P held[H];
    const char *x = column_at<DT>(a.x, p, first);
    auto load = [&](int j0) {
#pragma unroll
        for (int j = 0; j < H; j++) load_row<P>(held[j], x, (j0 + j) * a.rows, a.rows, p.row, own, a.x.ts);
    };

    const int W = p.c1 - p.c0, each = W / p.ng;
    constexpr bool one = ONE;
    const int g = one && p.ng > 1 ? (p.c - p.c0) / a.width : 0;   // one: the column's group of the slab
    float m[VEC], sc[VEC], sh[VEC];
    if (MODE != kApply) {
        load(0);
        float acc[VEC];
#pragma unroll
        for (int e = 0; e < VEC; e++) acc[e] = 0.0f;
#pragma unroll
        for (int j = 0; j < R; j++)
            if (p.row + j * a.rows < own) {
#pragma unroll
                for (int e = 0; e < VEC; e++) acc[e] += held[j].get(e);
            }
        const float inv = own ? 1.0f / ((float)own * (float)each) : 0.0f;
        auto own_sum = [&]() {   // of the channels that this column counts
            float t = 0.0f;
#pragma unroll
            for (int e = 0; e < VEC; e++) t += e >= p.skip ? acc[e] : 0.0f;
            return t;
        };
        float mean = 0.0f, squares = 0.0f;   // one: of the column's group
        if (one) {
            float none = 0.0f;
            mean = own_sum();
            sum_two<NT, VEC>(a, p, g, mean, none, s.rows, s.group, s.group2);
            mean *= inv;
#pragma unroll
            for (int e = 0; e < VEC; e++) m[e] = mean;
        } else {
            const int parts = sum_rows<NT, VEC>(a, p, acc, s);
            sum_groups<NT>(p, s.chan, parts, nullptr, s.group);
            for_channels<NT>(a, p, [&](int ch, int k) { s.of[0][ch] = s.group[k] * inv; });
            __syncthreads();
            of_column<VEC>(s.of[0], p, m);
        }
#pragma unroll
        for (int e = 0; e < VEC; e++) acc[e] = 0.0f;
#pragma unroll
        for (int j = 0; j < H; j++) held[j].renew();
#pragma unroll
        for (int j = 0; j < R; j++)
            if (p.row + j * a.rows < own) {
#pragma unroll
                for (int e = 0; e < VEC; e++) {
                    float d = held[j].get(e) - m[e];
                    acc[e] = __builtin_fmaf(d, d, acc[e]);
                }
            }
        if (one) {
            float none = 0.0f;
            squares = own_sum();
            sum_two<NT, VEC>(a, p, g, squares, none, s.rows, s.group, s.group2);
        } else {
            const int parts = sum_rows<NT, VEC>(a, p, acc, s);
            sum_groups<NT>(p, s.chan, parts, nullptr, s.group2);
        }
        // one: the first thread of a group writes for it
        const bool leads = one && p.active && p.row == 0 && p.c == p.c0 + g * a.width;
        if (MODE == kStats) {
            const int K = a.chunks * a.parts, k = p.chunk * a.parts + (a.parts > 1 ? p.slab % a.parts : 0);
            float2 *at = a.stats + ((int64_t)p.i * a.G + p.g0) * K + k;
            if (leads) at[(int64_t)g * K] = make_float2(mean, squares);
            if (!one)
                for (int q = threadIdx.x; q < p.ng; q += NT)
                    at[(int64_t)q * K] = make_float2(s.group[q] * inv, s.group2[q]);
            return;
        }
        float *means = a.mean + (int64_t)p.i * a.G + p.g0, *rstds = a.rstd + (int64_t)p.i * a.G + p.g0;
        if (one) {
            const float rstd = own ? 1.0f / sqrtf(squares * inv + a.eps) : 0.0f;
            if (leads) means[g] = mean, rstds[g] = rstd;
#pragma unroll
            for (int e = 0; e < VEC; e++) sc[e] = rstd;
        } else {
            for (int q = threadIdx.x; q < p.ng; q += NT) {
                const float rstd = own ? 1.0f / sqrtf(s.group2[q] * inv + a.eps) : 0.0f;
                s.group[q] *= inv, s.group2[q] = rstd;
                means[q] = s.group[q], rstds[q] = rstd;
            }
        }
    } else {
        // merge the chunks' statistics: N = sum n_k, m = sum n_k m_k / N,
        // squares = sum (squares_k + n_k (m_k - m)^2)
        const int K = a.chunks * a.parts;
        const float inv = T ? 1.0f / ((float)T * (float)a.width) : 0.0f;
        for (int g = threadIdx.x >> 6; g < p.ng; g += NT >> 6) {
            const float2 *st = a.stats + ((int64_t)p.i * a.G + p.g0 + g) * K;
            float mean = 0.0f, sq = 0.0f;
            for (int pass = 0; pass < 2; pass++) {
                float t = 0.0f;
                for (int k = threadIdx.x & 63; k < K; k += 64) {
                    const int part = k % a.parts;
                    int64_t f0;
                    const float rows = (float)chunk_rows(a, T, k / a.parts, per, f0);
                    const int wide = (int)((int64_t)a.width * (part + 1) / a.parts) -
                                     (int)((int64_t)a.width * part / a.parts);
                    const float nk = rows * (float)wide, d = st[k].x - mean;
                    t += pass ? __builtin_fmaf(nk * d, d, st[k].y) : nk * inv * st[k].x;
                }
#pragma unroll
                for (int off = 32; off; off /= 2) t += __shfl_xor(t, off);
                if (pass)
                    sq = t;
                else
                    mean = t;
            }
            if ((threadIdx.x & 63) == 0) {
                const float rstd = T ? 1.0f / sqrtf(sq * inv + a.eps) : 0.0f;
                s.group[g] = mean, s.group2[g] = rstd;
                if (p.chunk == 0 && (a.parts == 1 || p.slab % a.parts == 0)) {
                    a.mean[(int64_t)p.i * a.G + p.g0 + g] = mean;
                    a.rstd[(int64_t)p.i * a.G + p.g0 + g] = rstd;
                }
            }
        }
    }
    if (one) {
        if (MODE == kApply) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < VEC; e++) m[e] = s.group[g], sc[e] = s.group2[g];
        }
        if (!p.active) return;
#pragma unroll
        for (int e = 0; e < VEC; e++) {
            if (a.w) sc[e] *= a.w[p.c + e];
            sh[e] = a.b ? a.b[p.c + e] : 0.0f;
        }
    } else {
        __syncthreads();
        for_channels<NT>(a, p, [&](int ch, int k) {
            s.of[0][ch] = s.group[k];
            s.of[1][ch] = s.group2[k] * (a.w ? a.w[p.c0 + ch] : 1.0f);
            s.of[2][ch] = a.b ? a.b[p.c0 + ch] : 0.0f;
        });
        __syncthreads();
        if (!p.active) return;
        of_column<VEC>(s.of[0], p, m);
        of_column<VEC>(s.of[1], p, sc);
        of_column<VEC>(s.of[2], p, sh);
    }
    char *out = column_at<DT>(a.out, p, first);
    const int64_t rest = a.L - first;
    auto write = [&](int j0, auto act) {
#pragma unroll
        for (int j = 0; j < H; j++) {
            const int pass = (j0 + j) * a.rows, r = p.row + pass;
            float y[VEC];
#pragma unroll
            for (int e = 0; e < VEC; e++) y[e] = 0.0f;
            if (r < own) {
#pragma unroll
                for (int e = 0; e < VEC; e++)
                    y[e] = activate<DT, act.value>(__builtin_fmaf(held[j].get(e) - m[e], sc[e], sh[e]));
            }
            if (r < rest) {
                P to;
                to.put(0, y);
                store_column<DT>(out + pass * a.out.ts, to, p, MODE == kApply && a.in_place);
            }
        }
    };
    for (int j0 = 0; j0 < R && j0 * a.rows < rest; j0 += H) {
        if (MODE == kApply) load(j0);
#pragma unroll
        for (int j = 0; j < H; j++) held[j].renew();
        switch (a.act) {
        case ROCKET_ACT_RELU: write(j0, std::integral_constant<int, ROCKET_ACT_RELU>()); break;
        case ROCKET_ACT_SILU: write(j0, std::integral_constant<int, ROCKET_ACT_SILU>()); break;
        case ROCKET_ACT_GELU: write(j0, std::integral_constant<int, ROCKET_ACT_GELU>()); break;
        default: write(j0, std::integral_constant<int, ROCKET_ACT_NONE>());
        }
    }
}

// Forward, held, every column in one group: a workgroup goes through the
// series b, b + a.series, ..., and the next series' columns load as this one's
// are written.
template <int DT, int NT, int R>
__global__ __launch_bounds__(NT, 5) void norm_one_kernel(NormArgs a) {
    using P = Pack<DT, true>;
    constexpr int VEC = P::kN;
    extern __shared__ __attribute__((aligned(16))) float shared[];
    const int W = a.cols * VEC;
    float *group = shared, *group2 = group + pad4(a.most_groups), *rows = group2 + pad4(a.most_groups);
    float *weight = rows + 2 * NT, *bias = weight + W;   // of the slab's channels
    Place p;
    const uint32_t b = rocket::item_of_block(), begin = rocket::uniform(b / a.slabs);
    p.slab = rocket::uniform(b - begin * a.slabs);
    p.chunk = 0;
    place_thread<NT, VEC>(a, p);
    for (int ch = threadIdx.x; ch < p.c1 - p.c0; ch += NT) {
        weight[ch] = a.w ? a.w[p.c0 + ch] : 1.0f;
        bias[ch] = a.b ? a.b[p.c0 + ch] : 0.0f;
    }
    const int g = p.ng > 1 ? (p.c - p.c0) / a.width : 0;
    const bool leads = p.active && p.row == 0 && p.c == p.c0 + g * a.width;   // writes for its group
    __syncthreads();

    P held[R];
    int own = rocket::steps_of(a.lengths, begin, a.L);   // all of them are held
    p.i = begin;
    const char *x = column_at<DT>(a.x, p, 0);
#pragma unroll
    for (int j = 0; j < R; j++) load_row<P>(held[j], x, j * a.rows, a.rows, p.row, own, a.x.ts);
    for (;;) {
        // as if new: what follows from them is not kept across series
        asm("" : "+v"(p.row), "+v"(p.c), "+s"(a.x.ts), "+s"(a.out.ts));
        float acc[VEC];
        auto own_sum = [&]() {   // of the channels that this column counts
            float t = 0.0f;
#pragma unroll
            for (int e = 0; e < VEC; e++) t += e >= p.skip ? acc[e] : 0.0f;
            return t;
        };
#pragma unroll
        for (int e = 0; e < VEC; e++) acc[e] = 0.0f;
#pragma unroll
        for (int j = 0; j < R; j++)
            if (j * a.rows < own) {   // columns past the own steps hold 0
#pragma unroll
                for (int e = 0; e < VEC; e++) acc[e] += held[j].get(e);
            }
        const float inv = own ? 1.0f / ((float)own * (float)a.width) : 0.0f;
        float mean = own_sum(), squares, none = 0.0f;
        sum_two<NT, VEC>(a, p, g, mean, none, rows, group, group2);
        mean *= inv;
#pragma unroll
        for (int e = 0; e < VEC; e++) acc[e] = 0.0f;
#pragma unroll
        for (int j = 0; j < R; j++) held[j].renew();
#pragma unroll
        for (int j = 0; j < R; j++)
            if (p.row + j * a.rows < own) {
#pragma unroll
                for (int e = 0; e < VEC; e++) {
                    const float d = held[j].get(e) - mean;
                    acc[e] = __builtin_fmaf(d, d, acc[e]);
                }
            }
        squares = own_sum(), none = 0.0f;
        sum_two<NT, VEC>(a, p, g, squares, none, rows, group, group2);
        const float rstd = own ? 1.0f / sqrtf(squares * inv + a.eps) : 0.0f;
        if (leads) {
            a.mean[(int64_t)p.i * a.G + p.g0 + g] = mean;
            a.rstd[(int64_t)p.i * a.G + p.g0 + g] = rstd;
        }
        float sc[VEC], sh[VEC];
        of_column<VEC>(weight, p, sc);
        of_column<VEC>(bias, p, sh);
#pragma unroll
        for (int e = 0; e < VEC; e++) sc[e] *= rstd;

        const uint32_t next = p.i + a.series;   // below 2^32
        char *out = column_at<DT>(a.out, p, 0);
        const int had = own;
        const bool more = next < (uint32_t)a.n;
        own = more ? rocket::steps_of(a.lengths, next, a.L) : 0;
        p.i = more ? next : p.i;
        x = column_at<DT>(a.x, p, 0);
        auto write = [&](auto act) {
#pragma unroll
            for (int j = 0; j < R; j++) {
                const int pass = j * a.rows, r = p.row + pass;
                if (pass >= a.L) break;
                float y[VEC];
#pragma unroll
                for (int e = 0; e < VEC; e++) y[e] = 0.0f;
                if (r < had) {
                    held[j].renew();
#pragma unroll
                    for (int e = 0; e < VEC; e++)
                        y[e] = activate<DT, act.value>(__builtin_fmaf(held[j].get(e) - mean, sc[e], sh[e]));
                }
                if (r < a.L && p.active) {
                    P to;
                    to.put(0, y);
                    to.store(out + pass * a.out.ts);
                }
                load_row<P>(held[j], x, pass, a.rows, p.row, own, a.x.ts);
            }
        };
        switch (a.act) {
        case ROCKET_ACT_RELU: write(std::integral_constant<int, ROCKET_ACT_RELU>()); break;
        case ROCKET_ACT_SILU: write(std::integral_constant<int, ROCKET_ACT_SILU>()); break;
        case ROCKET_ACT_GELU: write(std::integral_constant<int, ROCKET_ACT_GELU>()); break;
        default: write(std::integral_constant<int, ROCKET_ACT_NONE>());
        }
        if (!more) break;
    }
}

// What the backward pass keeps of an element's channel.  Everything is taken
// of d = x - m, whose rounding goes with the spread and not with the level.  z is
// the fused d A + B with A = r w and B = b, as in the forward pass, but for ReLU:
// there z is rounded step by step as the formula is written, since the slope
// jumps with z's sign.
template <int N, int ACT>
struct Channel {
    static constexpr bool kSteps = ACT == ROCKET_ACT_RELU;
    float A[N], B[N], m[N];   // d A + B; in steps: w and b
    float r[kSteps ? N : 1];
    __device__ float z(float d, int e) const {
        if (kSteps) return d * r[kSteps ? e : 0] * A[e] + B[e];
        return __builtin_fmaf(d, A[e], B[e]);
    }
    __device__ float scale(int e) const { return kSteps ? A[e] * r[kSteps ? e : 0] : A[e]; }
    __device__ void take(const Scratch &s, const Place &p, int from) {
        of_column(s.of[0], p, A, from);
        of_column(s.of[1], p, B, from);
        of_column(s.of[2], p, m, from);
        if constexpr (kSteps) of_column(s.of[3], p, r, from);
    }
};

// Elements of a column that norm_back_kernel takes at a time, through all the
// columns that the thread holds: what it keeps of eight channels at once does
// not fit beside 8 columns of x and of dy (777 x 129 x 924 in groups of 33, bf16,
// SiLU: 221 us, against 285 us with all eight).
template <int VEC>
constexpr int kAtOnce = VEC < 4 ? VEC : 4;

// Backward.  Held: a workgroup goes through the series b, b + a.series, ... and
// keeps the channel sums over them; kStats leaves the channel sums of a chunk.
// sum dz xh is gathered as sum dz (x - m), m the mean of the channel's own
// group, and multiplied by r once a channel: no group's values reach another's.
template <int DT, bool WIDE, int NT, int R, int MODE, int ACT>
__global__ __launch_bounds__(NT, 4) void norm_back_kernel(NormArgs a) {
    using P = Pack<DT, WIDE>;
    constexpr int VEC = P::kN, N = kAtOnce<VEC>;
    constexpr bool CENTRED = DT == ROCKET_FLOAT32 && MODE == kHeld;   // x - m goes over x's words
    const Scratch s = scratch_of<NT, VEC>(a);
    Place p;
    const uint32_t b = rocket::item_of_block(), rest_of = rocket::uniform(b / a.slabs);
    p.slab = rocket::uniform(b - rest_of * a.slabs);
    const uint32_t begin = MODE == kHeld ? rest_of : (uint32_t)rocket::uniform(rest_of / a.chunks);
    p.chunk = MODE == kHeld ? 0 : rocket::uniform(rest_of - begin * a.chunks);
    place_thread<NT, VEC>(a, p);
    const int W = p.c1 - p.c0;
    const int64_t per = (int64_t)R * a.rows;
    if (MODE == kHeld)
        for (int ch = threadIdx.x; ch < W; ch += NT) s.total[ch] = 0.0f, s.total[W + ch] = 0.0f;
    constexpr int H = MODE == kApply && R > 2 ? 2 : R;

    P hx[H], hg[H];
    int64_t first, T = rocket::steps_of(a.lengths, begin, a.L);
    int own = chunk_rows(a, T, p.chunk, per, first);
    p.i = begin;
    const char *x = column_at<DT>(a.x, p, first), *dy = column_at<DT>(a.dy, p, first);
    auto load = [&](int j, int j0) {
        load_row<P>(hx[j], x, (j0 + j) * a.rows, a.rows, p.row, own, a.x.ts);
        load_row<P>(hg[j], dy, (j0 + j) * a.rows, a.rows, p.row, own, a.dy.ts);
    };
    if (MODE != kApply) {
#pragma unroll
        for (int j = 0; j < H; j++) load(j, 0);
    }
    for (;;) {
        // as if new: what follows from them is not kept across series
        asm("" : "+v"(p.row), "+v"(p.c), "+s"(a.x.ts), "+s"(a.dy.ts), "+s"(a.out.ts));
        const float *mean = a.mean + (int64_t)p.i * a.G + p.g0, *rstd = a.rstd + (int64_t)p.i * a.G + p.g0;
        for_channels<NT>(a, p, [&](int ch, int g) {
            const float m = mean[g], r = rstd[g], w = a.w ? a.w[p.c0 + ch] : 1.0f, bias = a.b ? a.b[p.c0 + ch] : 0.0f;
            s.of[0][ch] = ACT == ROCKET_ACT_RELU ? w : r * w;
            s.of[1][ch] = bias, s.of[2][ch] = m;
            if (ACT == ROCKET_ACT_RELU) s.of[3][ch] = r;
        });
        __syncthreads();
        if (MODE != kApply) {
            float sd[VEC], sx[VEC];
#pragma unroll
            for (int e = 0; e < VEC; e++) sd[e] = 0.0f, sx[e] = 0.0f;
#pragma unroll
            for (int q = 0; q < VEC; q += N) {
                Channel<N, ACT> of;
                of.take(s, p, q);
#pragma unroll
                for (int j = 0; j < R; j++)
                    if (p.row + j * a.rows < own) {
#pragma unroll
                        for (int e = 0; e < N; e++) {
                            const float d = hx[j].get(q + e) - of.m[e];
                            const float dz = hg[j].get(q + e) * slope<DT, ACT>(of.z(d, e));
                            sd[q + e] += dz;
                            sx[q + e] = __builtin_fmaf(dz, d, sx[q + e]);
                            if (CENTRED) hx[j].set(q + e, d);
                        }
                    }
                __builtin_amdgcn_sched_barrier(0);
            }
            int parts = sum_rows<NT, VEC>(a, p, sd, s);
            for (int ch = threadIdx.x; ch < W; ch += NT) {
                float t = 0.0f;
                for (int q = 0; q < parts; q++) t += s.chan[q * W + ch];
                s.first[ch] = t;
            }
            sum_groups<NT>(p, s.chan, parts, a.w, s.group);
            parts = sum_rows<NT, VEC>(a, p, sx, s);
            for_channels<NT>(a, p, [&](int ch, int g) {
                const float d = s.first[ch];
                float t = 0.0f;
                for (int q = 0; q < parts; q++) t += s.chan[q * W + ch];
                t *= rstd[g];
                if (MODE == kHeld) {
                    s.total[ch] += d, s.total[W + ch] += t;
                } else {
                    float *sum = a.sums + ((int64_t)p.i * a.chunks + p.chunk) * 2 * a.C + p.c0 + ch;
                    sum[0] = d, sum[a.C] = t;
                }
                s.first[ch] = t;
            });
            __syncthreads();
            sum_groups<NT>(p, s.first, 1, a.w, s.group2);
            if (MODE == kStats) {
                const int K = a.chunks * a.parts, k = p.chunk * a.parts + (a.parts > 1 ? p.slab % a.parts : 0);
                for (int g = threadIdx.x; g < p.ng; g += NT)
                    a.stats[((int64_t)p.i * a.G + p.g0 + g) * K + k] = make_float2(s.group[g], s.group2[g]);
                return;
            }
        } else {
            // the groups' sums over the chunks
            const int K = a.chunks * a.parts;
            for (int g = threadIdx.x >> 6; g < p.ng; g += NT >> 6) {
                const float2 *st = a.stats + ((int64_t)p.i * a.G + p.g0 + g) * K;
                float t1 = 0.0f, t2 = 0.0f;
                for (int k = threadIdx.x & 63; k < K; k += 64) t1 += st[k].x, t2 += st[k].y;
#pragma unroll
                for (int off = 32; off; off /= 2) t1 += __shfl_xor(t1, off), t2 += __shfl_xor(t2, off);
                if ((threadIdx.x & 63) == 0) s.group[g] = t1, s.group2[g] = t2;
            }
            __syncthreads();
        }
        // dx = r (dz w - mean(g) - xh mean(g xh)) = dz r w - (d D + E)
        const float inv = T ? 1.0f / ((float)T * (float)a.width) : 0.0f;
        for_channels<NT>(a, p, [&](int ch, int g) {
            const float r = rstd[g];
            s.chan[ch] = r * r * (s.group2[g] * inv);
            s.first[ch] = r * (s.group[g] * inv);
        });
        __syncthreads();
        const int64_t rest = a.L - first, next = (int64_t)p.i + (MODE == kHeld ? a.series : a.n);
        char *out = column_at<DT>(a.out, p, first);
        const int had = own;
        if (MODE == kHeld) {   // the next series' columns are loaded as these are done with
            T = next < a.n ? rocket::steps_of(a.lengths, next, a.L) : 0;
            own = chunk_rows(a, T, 0, per, first);
            p.i = next < a.n ? (uint32_t)next : p.i;
            x = column_at<DT>(a.x, p, first), dy = column_at<DT>(a.dy, p, first);
        }
        for (int j0 = 0; j0 < R && j0 * a.rows < rest; j0 += H) {
            if (MODE == kApply) {
#pragma unroll
                for (int j = 0; j < H; j++) load(j, j0);
            }
#pragma unroll
            for (int q = 0; q < VEC; q += N) {   // dx goes over dy's words
                Channel<N, ACT> of;
                of.take(s, p, q);
                float D[N], E[N];
                of_column(s.chan, p, D, q);
                of_column(s.first, p, E, q);
#pragma unroll
                for (int j = 0; j < H; j++) {
                    const int pass = (j0 + j) * a.rows, r = p.row + pass;
                    float dx[N];
#pragma unroll
                    for (int e = 0; e < N; e++) dx[e] = 0.0f;
                    if (r < had) {
                        if (q == 0) hx[j].renew(), hg[j].renew();
#pragma unroll
                        for (int e = 0; e < N; e++) {
                            const float d = CENTRED ? hx[j].get(q + e) : hx[j].get(q + e) - of.m[e];
                            const float dz = hg[j].get(q + e) * slope<DT, ACT>(of.z(d, e));
                            dx[e] = __builtin_fmaf(dz, of.scale(e), -__builtin_fmaf(d, D[e], E[e]));
                        }
                    }
                    hg[j].put(q, dx);
                    if (q + N < VEC) continue;
                    if (r < rest && p.active)
                        store_column<DT>(out + pass * a.out.ts, hg[j], p, MODE == kApply && a.in_place);
                    if (MODE == kHeld) load(j, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (next >= a.n) break;
        if (MODE == kHeld) __syncthreads();   // the shared arrays are free again
    }
    if (MODE == kHeld)
        for (int q = 0; q < 2; q++)
            for (int ch = threadIdx.x; ch < W; ch += NT)
                a.sums[((int64_t)begin * 2 + q) * a.C + p.c0 + ch] = s.total[q * W + ch];
}

// Backward, held, every column in one group: a thread's sums for its group are
// one number each, and the channel sums stay in its own slots of shared memory
// until the workgroup's last series, so that a series takes three barriers.
// The next series' columns load as this one's are written.
template <int DT, int NT, int R, int ACT>
__global__ __launch_bounds__(NT, 4) void norm_back_one_kernel(NormArgs a) {
    using P = Pack<DT, true>;
    constexpr int VEC = P::kN, Q = VEC / 4;
    constexpr bool CENTRED = DT == ROCKET_FLOAT32;   // x - m goes over x's words, which saves
    // the second pass a subtraction (500 x 1000 x 256, fp32, SiLU: 370 us against 381 us)
    extern __shared__ __attribute__((aligned(16))) float shared[];
    const int W = a.cols * VEC;
    float *group = shared, *group2 = group + pad4(a.most_groups), *rows = group2 + pad4(a.most_groups);
    float *weight = rows + 2 * NT, *bias = weight + W;                       // of the slab's channels
    typedef float vec4 __attribute__((ext_vector_type(4)));
    vec4 *total = (vec4 *)(bias + W);                                        // [2 Q][NT]
    Place p;
    const uint32_t b = rocket::item_of_block(), begin = rocket::uniform(b / a.slabs);
    p.slab = rocket::uniform(b - begin * a.slabs);
    p.chunk = 0;
    place_thread<NT, VEC>(a, p);
    for (int ch = threadIdx.x; ch < p.c1 - p.c0; ch += NT) {
        weight[ch] = a.w ? a.w[p.c0 + ch] : 1.0f;
        bias[ch] = a.b ? a.b[p.c0 + ch] : 0.0f;
    }
#pragma unroll
    for (int k = 0; k < 2 * Q; k++) total[k * NT + threadIdx.x] = vec4{0, 0, 0, 0};
    const int g = p.ng > 1 ? (p.c - p.c0) / a.width : 0;
    __syncthreads();

    P hx[R], hg[R];
    int own = rocket::steps_of(a.lengths, begin, a.L);   // all of them are held
    p.i = begin;
    const char *x = column_at<DT>(a.x, p, 0), *dy = column_at<DT>(a.dy, p, 0);
    auto load = [&](int j) {
        load_row<P>(hx[j], x, j * a.rows, a.rows, p.row, own, a.x.ts);
        load_row<P>(hg[j], dy, j * a.rows, a.rows, p.row, own, a.dy.ts);
    };
#pragma unroll
    for (int j = 0; j < R; j++) load(j);
    for (;;) {
        // as if new: what follows from them is not kept across series
        asm("" : "+v"(p.row), "+v"(p.c), "+s"(a.x.ts), "+s"(a.dy.ts), "+s"(a.out.ts));
        const float mean = a.mean[(int64_t)p.i * a.G + p.g0 + g], rstd = a.rstd[(int64_t)p.i * a.G + p.g0 + g];
        Channel<VEC, ACT> of;
        auto scales = [&]() {
            of_column(weight, p, of.A);
            of_column(bias, p, of.B);
#pragma unroll
            for (int e = 0; e < VEC; e++) {
                if constexpr (ACT == ROCKET_ACT_RELU)
                    of.r[e] = rstd;
                else
                    of.A[e] *= rstd;
            }
        };
        scales();
        float sd[VEC], sx[VEC];
#pragma unroll
        for (int e = 0; e < VEC; e++) sd[e] = 0.0f, sx[e] = 0.0f;
#pragma unroll
        for (int j = 0; j < R; j++)
            if (p.row + j * a.rows < own) {
#pragma unroll
                for (int e = 0; e < VEC; e++) {
                    const float d = hx[j].get(e) - mean;
                    const float dz = hg[j].get(e) * slope<DT, ACT>(of.z(d, e));
                    sd[e] += dz;
                    sx[e] = __builtin_fmaf(dz, d, sx[e]);
                    if (CENTRED) hx[j].set(e, d);
                    if (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);   // four at a time: registers are short
                }
            }
        // r mean(g) N and mean(g xh) N of the thread's elements, and the channel sums
        float t1 = 0.0f, t2 = 0.0f;
#pragma unroll
        for (int e = 0; e < VEC; e++) {
            t1 = __builtin_fmaf(e >= p.skip ? of.scale(e) : 0.0f, sd[e], t1);
            t2 = __builtin_fmaf(e >= p.skip ? of.scale(e) : 0.0f, sx[e], t2);
        }
#pragma unroll
        for (int k = 0; k < Q; k++) {
            vec4 d = total[k * NT + threadIdx.x], q = total[(Q + k) * NT + threadIdx.x];
#pragma unroll
            for (int e = 0; e < 4; e++) {
                d[e] += sd[4 * k + e];
                q[e] = __builtin_fmaf(rstd, sx[4 * k + e], q[e]);
            }
            total[k * NT + threadIdx.x] = d, total[(Q + k) * NT + threadIdx.x] = q;
        }
        sum_two<NT, VEC>(a, p, g, t1, t2, rows, group, group2);
        // dx = r (dz w - mean(g) - xh mean(g xh)) = dz r w - (d D + E)
        const float inv = own ? 1.0f / ((float)own * (float)a.width) : 0.0f;
        const float D = rstd * rstd * (t2 * inv), E = t1 * inv;
        scales();

        const uint32_t next = p.i + a.series;   // below 2^32
        char *out = column_at<DT>(a.out, p, 0);
        const int had = own;
        const bool more = next < (uint32_t)a.n;
        own = more ? rocket::steps_of(a.lengths, next, a.L) : 0;
        p.i = more ? next : p.i;
        x = column_at<DT>(a.x, p, 0), dy = column_at<DT>(a.dy, p, 0);
#pragma unroll
        for (int j = 0; j < R; j++) {
            const int pass = j * a.rows, r = p.row + pass;
            float dx[VEC];
#pragma unroll
            for (int e = 0; e < VEC; e++) dx[e] = 0.0f;
            if (r < had) {
                hx[j].renew(), hg[j].renew();
#pragma unroll
                for (int e = 0; e < VEC; e++) {
                    const float d = CENTRED ? hx[j].get(e) : hx[j].get(e) - mean;
                    const float dz = hg[j].get(e) * slope<DT, ACT>(of.z(d, e));
                    dx[e] = __builtin_fmaf(dz, of.scale(e), -__builtin_fmaf(d, D, E));
                    if (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);
                }
            }
            if (r < a.L && p.active) {
                P to;
                to.put(0, dx);
                to.store(out + pass * a.out.ts);
            }
            load(j);
        }
        if (!more) break;
    }
    __syncthreads();
    // over the rows: channel ch is element ch % VEC of column ch / VEC; the last
    // column starts early
    const int wide = p.c1 - p.c0;
    for (int q = 0; q < 2; q++)
        for (int ch = threadIdx.x; ch < wide; ch += NT) {
            const int col = ch / VEC, at = col * VEC;
            const int e = ch - at + (at + VEC > wide ? at + VEC - wide : 0);
            float t = 0.0f;
            for (int r = 0; r < a.rows; r++) t += ((const float *)&total[(q * Q + e / 4) * NT + r * a.cols + col])[e % 4];
            a.sums[((int64_t)begin * 2 + q) * a.C + p.c0 + ch] = t;
        }
}

// Rows of channel sums to fewer rows: out[o, q, c] = the sum of in[r, q, c]
// over rows r of block o.  16 rows of 64 channels at a time.
__global__ __launch_bounds__(1024) void fold_kernel(const float *in, int64_t rows, int64_t per, int C, float *out0,
                                                    float *out1, int64_t out_stride) {
    __shared__ float part[16][64];
    const int blocks = (C + 63) / 64;
    const int cb = blockIdx.x % blocks, q = blockIdx.x / blocks & 1;
    const int64_t o = blockIdx.x / blocks / 2;
    const int c = cb * 64 + (threadIdx.x & 63), k = threadIdx.x >> 6;
    const int64_t end = (o + 1) * per < rows ? (o + 1) * per : rows;
    float t = 0.0f;
    if (c < C)
        for (int64_t r = o * per + k; r < end; r += 16) t += in[(r * 2 + q) * C + c];
    part[k][threadIdx.x & 63] = t;
    __syncthreads();
    if (k == 0 && c < C) {
        for (int j = 1; j < 16; j++) t += part[j][threadIdx.x & 63];
        float *out = q ? out1 : out0;
        if (out) out[o * out_stride + c] = t;
    }
}

// How a call is cut.
struct Cut {
    bool wide, held;
    bool one;           // every 16-byte column lies in one group
    int32_t width, slabs, parts, cols, rows, threads, run, chunks;
    int32_t series;     // backward, held
    int32_t groups;     // of a slab, at most
    int64_t each;       // workgroups of a series; 0: `series` times slabs go through all of them
    int64_t launch;     // series of a launch
    int64_t sum_rows;   // backward: rows of channel sums
    int64_t folded;     // rows after the first fold, 0: one fold is enough
};

// Rows of channel sums that one workgroup adds up before a second launch adds
// the rest; up to 4 times as many take one launch.
constexpr int kFold = 128;
// Forward, a workgroup goes through many series where a thread holds this many
// columns at most (10000 x 16 x 256, bf16: 63 us, against 86 us with a workgroup
// a series).  With 8 columns the next series' do not fit beside them (777 x 129 x
// 924 in groups of 33, fp32: 253 us against 187 us).
constexpr int kLoopRun = 4;
// Workgroups that hold a slab, the smallest that does is taken: threads, and
// 16-byte columns of a thread (of each operand).
struct Size {
    int threads, run;
};
constexpr Size kSizes[] = {{64, 4}, {256, 4}, {256, 8}, {512, 8}, {512, 16}};
// Backward, the largest size instead of slabs of 64 bytes (1000 x 1000 x 256, bf16,
// SiLU: 410 us against 474 us; 200 series: 119 us against 117 us).
constexpr int64_t kManySlabs = 1024;
constexpr Size kBackSizes[] = {{64, 4}, {256, 4}, {256, 8}, {512, 8}, {1024, 8}};
constexpr Size kChunk = {256, 16}, kBackChunk = {256, 8};   // of a chunk, and of rows of less than 16 bytes

// The slabs for `per` groups each, and the smallest workgroup that holds one.
bool hold(const rocket_sequence_shape *s, int32_t groups, int64_t per, int vec, bool back, Cut *cut) {
    const int64_t L = s->steps > 0 ? s->steps : 1;
    cut->slabs = (int32_t)((groups + per - 1) / per);
    const int64_t most = (groups + cut->slabs - 1) / cut->slabs;   // the most groups a slab gets
    cut->cols = (int32_t)((most * cut->width + vec - 1) / vec);
    cut->groups = (int32_t)most;
    auto holds = [&](const Size &z) {
        cut->threads = z.threads, cut->run = z.run, cut->rows = z.threads / cut->cols;
        return cut->rows >= 1 && (int64_t)cut->rows * z.run >= L &&
               (z.threads <= 512 || s->n * cut->slabs >= kManySlabs);
    };
    if (!cut->wide) return holds(back ? kBackChunk : kChunk);
    if (back) return std::any_of(std::begin(kBackSizes), std::end(kBackSizes), holds);
    return std::any_of(std::begin(kSizes), std::end(kSizes), holds);
}

bool cut_of(const rocket_sequence_shape *s, int32_t groups, bool back, Cut *cut) {
    const int size = rocket::elem_size(s->dtype), vec_wide = 16 / size;
    const int64_t C = s->channels, width = C / groups, L = s->steps > 0 ? s->steps : 1;
    cut->wide = C >= vec_wide;
    cut->width = (int32_t)width;
    const int vec = cut->wide ? vec_wide : 1;
    const int64_t most = 256 * (int64_t)vec;   // channels of a slab
    cut->parts = 1;
    cut->held = false;
    if (width > most) {
        cut->parts = (int32_t)((width + most - 1) / most);
        cut->slabs = (int32_t)(groups * cut->parts);
        cut->groups = 1;
        int64_t part = (width + cut->parts - 1) / cut->parts;
        cut->cols = (int32_t)((part + vec - 1) / vec);
    } else {
        // A slab is at least 128 bytes wide (a cache line), and wider while that
        // leaves workgroups for the whole chip and the slab is small: up to the
        // columns of a wavefront, or of 4 where a group is wider (8000 x 1 x 2000
        // in groups of 100, fp32, forward: 86 us with 2 groups a slab, 120 us with
        // 20), and not where columns would then lie in two groups (1000 x 16 x
        // 2000 in groups of 100, bf16: 25 us with a group a slab, 47 us with
        // more).  64 bytes where only that is held.
        int64_t per = 1, half = 1;
        while (half < groups && half * width * size < 64) half++;
        while (per < groups && per * width * size < 128) per++;
        const int64_t limit = width <= 64 * vec ? 64 * vec : most;
        const bool whole = width % vec == 0 || per > 1;
        while (whole && per * 2 <= groups && per * 2 * width <= limit && per * width * size * L < (16 << 10) &&
               s->n * ((groups + 2 * per - 1) / (2 * per)) >= 1024)
            per *= 2;
        cut->held = hold(s, groups, per, vec, back, cut) ||
                    (half < per && hold(s, groups, half, vec, back, cut));
        if (!cut->held) hold(s, groups, per, vec, back, cut);
    }
    // every column lies in one group: groups of whole columns, or one a slab
    cut->one = cut->wide && (width % vec == 0 || cut->groups == 1);
    cut->chunks = 1;
    cut->folded = 0;
    if (!cut->held) {
        cut->threads = kChunk.threads, cut->run = (back ? kBackChunk : kChunk).run;
        cut->rows = cut->threads / cut->cols;
        const int64_t step = (int64_t)cut->rows * cut->run, chunks = (L + step - 1) / step;
        cut->chunks = (int32_t)chunks;
        cut->each = chunks * cut->slabs;
        cut->sum_rows = s->n * chunks;
    } else if (back || (cut->one && cut->run <= kLoopRun)) {
        // as many workgroups as the registers take (20 wavefronts a CU), backward
        // more of them, whose loads and sums then overlap; all with as many series
        int64_t series = (256 * (back ? 32 : 20) * 64 / cut->threads + cut->slabs - 1) / cut->slabs;
        if (series > s->n) series = s->n;
        if (series < 1) series = 1;
        const int64_t each = (s->n + series - 1) / series;
        cut->series = (int32_t)(each > 0 ? (s->n + each - 1) / each : 1);
        cut->each = 0;
        cut->sum_rows = cut->series;
    } else {
        cut->each = cut->slabs;
    }
    cut->launch = s->n > 0 ? s->n : 1;
    if (cut->each) cut->launch = std::min(cut->launch, rocket::most_groups(cut->threads) / cut->each);
    if (back && cut->sum_rows > 4 * kFold) cut->folded = (cut->sum_rows + kFold - 1) / kFold;
    const int64_t fold_grid = (cut->folded ? cut->folded : 1) * 2 * ((C + 63) / 64);
    return cut->launch >= 1 && (!back || fold_grid <= rocket::most_groups(1024));
}

int64_t stats_of(const rocket_sequence_shape *s, int32_t groups, const Cut &c) {
    return c.held ? 0 : c.launch * groups * (int64_t)c.chunks * c.parts;
}

int64_t workspace_of(const rocket_sequence_shape *s, int32_t groups, bool back, const Cut &c) {
    const int64_t sums = back ? (c.sum_rows + c.folded) * 2 * s->channels * (int64_t)sizeof(float) : 0;
    return stats_of(s, groups, c) * (int64_t)sizeof(float2) + sums;
}

template <int DT, bool BACK, bool WIDE, int NT, int R, int MODE>
void go(const NormArgs &a, const Cut &c, hipStream_t s) {
    const uint32_t grid = (uint32_t)(c.each ? a.n * c.each : (int64_t)c.series * c.slabs);
    const bool one = WIDE && c.one && (!BACK || MODE == kHeld);
    const int keep = one ? (BACK ? kOneBack : kOne) : !BACK ? kSums : MODE == kHeld ? kSumsBack : kChunkBack;
    const int lds = (int)scratch_floats(NT, Pack<DT, WIDE>::kN, c.cols, c.rows, c.groups, keep) * 4;
    if constexpr (!BACK && WIDE && MODE == kHeld) {
        if (!one)
            norm_kernel<DT, true, NT, R, MODE, false><<<grid, NT, lds, s>>>(a);
        else if constexpr (R <= kLoopRun)
            norm_one_kernel<DT, NT, R><<<grid, NT, lds, s>>>(a);
        else
            norm_kernel<DT, true, NT, R, MODE, true><<<grid, NT, lds, s>>>(a);
    } else if constexpr (!BACK) {
        if (WIDE && one)
            norm_kernel<DT, WIDE, NT, R, MODE, WIDE><<<grid, NT, lds, s>>>(a);
        else
            norm_kernel<DT, WIDE, NT, R, MODE, false><<<grid, NT, lds, s>>>(a);
    } else {
        auto act = [&](auto k) {
            constexpr int ACT = decltype(k)::value;
            if constexpr (WIDE && MODE == kHeld) {
                if (one) {
                    if (lds > (64 << 10) &&
                        hipFuncSetAttribute((const void *)norm_back_one_kernel<DT, NT, R, ACT>,
                                            hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess)
                        return;   // the error is reported after the launch
                    norm_back_one_kernel<DT, NT, R, ACT><<<grid, NT, lds, s>>>(a);
                    return;
                }
            }
            norm_back_kernel<DT, WIDE, NT, R, MODE, ACT><<<grid, NT, lds, s>>>(a);
        };
        switch (a.act) {
        case ROCKET_ACT_RELU: act(std::integral_constant<int, ROCKET_ACT_RELU>()); break;
        case ROCKET_ACT_SILU: act(std::integral_constant<int, ROCKET_ACT_SILU>()); break;
        case ROCKET_ACT_GELU: act(std::integral_constant<int, ROCKET_ACT_GELU>()); break;
        default: act(std::integral_constant<int, ROCKET_ACT_NONE>());
        }
    }
}

// The held kernel of the size that the call was cut for.
template <int DT, bool BACK, int K = 0>
void run_held(const NormArgs &a, const Cut &c, hipStream_t s) {
    constexpr int kCount = BACK ? (int)std::size(kBackSizes) : (int)std::size(kSizes);
    if constexpr (K < kCount) {
        constexpr Size z = BACK ? kBackSizes[BACK ? K : 0] : kSizes[K];
        if (c.threads == z.threads && c.run == z.run)
            go<DT, BACK, true, z.threads, z.run, kHeld>(a, c, s);
        else
            run_held<DT, BACK, K + 1>(a, c, s);
    }
}

// The call's series from i on, as many as a launch takes.
template <bool BACK>
NormArgs part_of(NormArgs a, const Cut &c, int64_t i) {
    a.n = (int32_t)std::min<int64_t>(c.launch, a.n - i);
    for (View *x : {&a.x, &a.dy, &a.out})
        if (x->p) x->p += i * x->ss;
    if (a.lengths) a.lengths += i;
    a.mean += i * a.G, a.rstd += i * a.G;
    if (BACK) a.sums += i * c.chunks * 2 * a.C;   // several launches: a row of sums a chunk
    return a;
}

template <int DT, bool BACK>
void run(const NormArgs &a, const Cut &c, hipStream_t s) {
    constexpr Size z = BACK ? kBackChunk : kChunk;
    if (c.held && c.wide) {
        run_held<DT, BACK>(a, c, s);
    } else if (c.held) {
        go<DT, BACK, false, z.threads, z.run, kHeld>(a, c, s);
    } else if (c.wide) {
        go<DT, BACK, true, z.threads, z.run, kStats>(a, c, s);
        go<DT, BACK, true, z.threads, z.run, kApply>(a, c, s);
    } else {
        go<DT, BACK, false, z.threads, z.run, kStats>(a, c, s);
        go<DT, BACK, false, z.threads, z.run, kApply>(a, c, s);
    }
}

template <bool BACK>
void run_type(int32_t dtype, const NormArgs &call, const Cut &c, hipStream_t s) {
    for (int64_t i = 0; i < call.n; i += c.launch) {
        const NormArgs a = part_of<BACK>(call, c, i);
        if (dtype == ROCKET_FLOAT32)
            run<ROCKET_FLOAT32, BACK>(a, c, s);
        else if (dtype == ROCKET_BFLOAT16)
            run<ROCKET_BFLOAT16, BACK>(a, c, s);
        else
            run<ROCKET_FLOAT16, BACK>(a, c, s);
    }
}

View view(const rocket_sequence *q, int size) {
    return View{(char *)q->data, q->series_stride * size, q->step_stride * size};
}

bool aligned(const void *p, uintptr_t to) { return (uintptr_t)p % to == 0; }

bool args_ok(const rocket_sequence_shape *shape, int32_t groups, int32_t act, const float *w, const float *b) {
    return rocket::shape_ok(shape) && groups >= 1 && groups <= shape->channels && shape->channels % groups == 0 &&
           (int64_t)groups * shape->n <= ((int64_t)1 << 40) && act >= ROCKET_ACT_NONE && act <= ROCKET_ACT_GELU &&
           aligned(w, 4) && aligned(b, 4) && aligned(shape->lengths, 4);
}

NormArgs args_of(const rocket_sequence_shape *shape, int32_t groups, int32_t act, const float *w, const float *b,
                 const Cut &cut) {
    NormArgs a = {};
    a.n = (int32_t)shape->n, a.L = (int32_t)shape->steps, a.C = (int32_t)shape->channels, a.G = groups, a.width = cut.width;
    a.slabs = cut.slabs, a.parts = cut.parts, a.cols = cut.cols, a.rows = cut.rows, a.chunks = cut.chunks;
    a.most_groups = cut.groups, a.act = act, a.w = w, a.b = b, a.lengths = shape->lengths, a.series = cut.series;
    return a;
}

}  // namespace

extern "C" rocket_status rocket_group_norm_workspace(const rocket_sequence_shape *shape, int32_t groups,
                                                     int32_t backward, int64_t *bytes) {
    Cut cut = {};
    if (!bytes || !args_ok(shape, groups, ROCKET_ACT_NONE, nullptr, nullptr) ||
        !cut_of(shape, groups, backward != 0, &cut))
        return ROCKET_ERR_INVALID_ARG;
    *bytes = workspace_of(shape, groups, backward != 0, cut);
    return ROCKET_OK;
}

extern "C" rocket_status rocket_group_norm_forward(const rocket_sequence_shape *shape, int32_t groups,
                                                   const rocket_sequence *x, const float *weight, const float *bias,
                                                   float eps, int32_t activation, const rocket_sequence *y,
                                                   float *mean, float *rstd, void *workspace,
                                                   int64_t workspace_bytes, void *hip_stream) {
    Cut cut = {};
    if (!args_ok(shape, groups, activation, weight, bias) || !cut_of(shape, groups, false, &cut) ||
        !rocket::view_ok(x, shape) || !rocket::out_ok(y, shape) || !(eps >= 0.0f) || !(eps <= 3.0e38f) ||
        (shape->n > 0 && (!mean || !rstd)) || !aligned(mean, 4) || !aligned(rstd, 4))
        return ROCKET_ERR_INVALID_ARG;
    const int64_t need = workspace_of(shape, groups, false, cut);
    if (workspace_bytes < need || (need && (!workspace || !aligned(workspace, 8)))) return ROCKET_ERR_INVALID_ARG;
    if (shape->n == 0) return ROCKET_OK;
    const int size = rocket::elem_size(shape->dtype);
    NormArgs a = args_of(shape, groups, activation, weight, bias, cut);
    a.x = view(x, size), a.out = view(y, size);
    a.in_place = x->data == y->data;
    a.eps = eps, a.mean = mean, a.rstd = rstd, a.stats = (float2 *)workspace;
    run_type<false>(shape->dtype, a, cut, (hipStream_t)hip_stream);
    return rocket::launched();
}

extern "C" rocket_status rocket_group_norm_backward(const rocket_sequence_shape *shape, int32_t groups,
                                                    const rocket_sequence *dy, const rocket_sequence *x,
                                                    const float *weight, const float *bias, int32_t activation,
                                                    const float *mean, const float *rstd, const rocket_sequence *dx,
                                                    float *dweight, float *dbias, void *workspace,
                                                    int64_t workspace_bytes, void *hip_stream) {
    Cut cut = {};
    if (!args_ok(shape, groups, activation, weight, bias) || !cut_of(shape, groups, true, &cut) ||
        !rocket::view_ok(dy, shape) || !rocket::view_ok(x, shape) || !rocket::out_ok(dx, shape) ||
        (shape->n > 0 && (!mean || !rstd)) || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(dweight, 4) ||
        !aligned(dbias, 4))
        return ROCKET_ERR_INVALID_ARG;
    const int64_t need = workspace_of(shape, groups, true, cut);
    if (workspace_bytes < need || (need && (!workspace || !aligned(workspace, 8)))) return ROCKET_ERR_INVALID_ARG;
    hipStream_t s = (hipStream_t)hip_stream;
    const int size = rocket::elem_size(shape->dtype), C = (int)shape->channels;
    float *sums = (float *)((float2 *)workspace + stats_of(shape, groups, cut));
    int64_t rows = 0;
    if (!rocket::empty(shape)) {
        NormArgs a = args_of(shape, groups, activation, weight, bias, cut);
        a.x = view(x, size), a.dy = view(dy, size), a.out = view(dx, size);
        a.in_place = dx->data == dy->data || dx->data == x->data;
        a.mean = const_cast<float *>(mean), a.rstd = const_cast<float *>(rstd), a.sums = sums;
        a.stats = (float2 *)workspace;
        run_type<true>(shape->dtype, a, cut, s);
        rows = cut.sum_rows;
    }
    if (!dweight && !dbias) return rocket::launched();
    const uint32_t blocks = (uint32_t)((C + 63) / 64);
    if (rows && cut.folded) {
        float *next = sums + rows * 2 * C;
        fold_kernel<<<(uint32_t)cut.folded * 2 * blocks, 1024, 0, s>>>(sums, rows, kFold, C, next, next + C,
                                                                       2 * (int64_t)C);
        sums = next, rows = cut.folded;
    }
    fold_kernel<<<2 * blocks, 1024, 0, s>>>(sums, rows, rows ? rows : 1, C, dbias, dweight, 0);
    return rocket::launched();
}
