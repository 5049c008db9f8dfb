// Group norm with an activation over sequences [n, L, C], channels last.
//
// A series of T steps, a group of C / G channels, N = T C / G elements:
//   m = sum x / N,  s = sum (x - m)^2 / N,  r = 1 / sqrt(s + eps)
//   xh = (x - m) r,  z = xh w_c + b_c,  y = act(z)
// and backwards, with dz = dy act'(z) and g = dz w_c,
//   db_c = sum dz,  dw_c = sum dz xh  (over series and steps)
//   dx = r (g - mean(g) - xh mean(g xh))  (means over the group's N elements)
//
// A workgroup takes a slab: all steps of a few whole groups, at least 128
// bytes of channels wide.  Where the slab fits its registers it is read once:
// the sum, then the squares about the mean, then the output come from there
// (held).  Longer series are cut into chunks of steps: one launch leaves each
// chunk's mean and squares (or, backwards, its channel sums), a second one
// merges them in a fixed order and writes the output.  Groups wider than a
// workgroup's columns are cut along the channels in the same way.  There are
// no atomics: results do not change from call to call.
//
// A thread owns one column of 16 bytes of channels in every `rows`-th step.
// The last column of a slab is moved back so that it ends with the slab; the
// channels it shares with its neighbour are computed twice and counted once.
#include <algorithm>
#include <climits>
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
    int32_t act;
    float eps;
    const float *w, *b;        // or null
    const int32_t *lengths;
    float *mean, *rstd;        // [n, G]: written forward, read backward
    float2 *stats;             // forward: [n, G, chunks * parts] (mean, squares)
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
    __device__ static void store(char *p, const float *f) {
        vec o;
#pragma unroll
        for (int k = 0; k < 4; k++) o[k] = Elem<DT>::put(f + k * Elem<DT>::kPerWord);
        rocket::store_at(p, o);
    }
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
    __device__ static void store(char *p, const float *f) { *(raw *)p = Elem<DT>::round(f[0]); }
    __device__ void clear() { v = 0; }
    __device__ void renew() {}
};

// The normal distribution function and e = exp(-z^2 / 2).  fp32 elements: the
// library's erf.  16-bit elements: formula 7.1.26 of Abramowitz and Stegun
// (1964), erf to 1.5e-7, far below the elements' own rounding; its tail is a
// product, so that small values of z < 0 keep their digits.
template <int DT>
__device__ inline float normal_cdf(float z, float &e) {
    e = rocket::exp_neg_abs<DT>(0.5f * z * z);
    if (DT == ROCKET_FLOAT32) return 0.5f + 0.5f * erff(z * 0.70710678118654752f);
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_fabsf(z), 0.3275911f * 0.70710678f, 1.0f));
    float q = __builtin_fmaf(t, 0.5f * 1.061405429f, 0.5f * -1.453152027f);
    q = __builtin_fmaf(t, q, 0.5f * 1.421413741f);
    q = __builtin_fmaf(t, q, 0.5f * -0.284496736f);
    q = __builtin_fmaf(t, q, 0.5f * 0.254829592f);
    const float tail = q * t * e;
    return z < 0.0f ? tail : 1.0f - tail;
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
    if (!p.active) p.c = p.c0, p.skip = 0;
}

// Shared memory of a slab, sized by the launch.  Arrays of W start on 16 bytes.
struct Scratch {
    float *rows;             // [rows][W]: the threads' sums
    float *chan;             // parts of the channels' sums
    float *group, *group2;   // [groups of a slab]
    float *of[4];            // [4][W]: what the elements of a channel are scaled by
    float *first;            // [W], backward
    float *total;            // [2][W], backward, held
};

__host__ __device__ inline int64_t scratch_floats(int threads, int vec, int cols, int rows, int groups, bool back) {
    const int W = cols * vec;
    return (int64_t)rows * W + ((threads > W ? threads : W) + 3) / 4 * 4 + 2 * ((groups + 3) / 4 * 4) +
           (back ? 7 : 4) * W;
}

template <int NT, int VEC>
__device__ inline Scratch scratch_of(const NormArgs &a) {
    extern __shared__ __attribute__((aligned(16))) float shared[];
    const int W = a.cols * VEC, groups = (a.most_groups + 3) / 4 * 4;
    Scratch s;
    s.of[0] = shared;
    for (int k = 1; k < 4; k++) s.of[k] = s.of[k - 1] + W;
    s.rows = s.of[3] + W;
    s.chan = s.rows + a.rows * W;
    s.group = s.chan + ((NT > W ? NT : W) + 3) / 4 * 4;
    s.group2 = s.group + groups;
    s.first = s.group2 + groups;
    s.total = s.first + W;
    return s;
}

// The values of an array of channels for a thread's column.
template <int VEC>
__device__ inline void of_column(const float *of, const Place &p, float (&v)[VEC]) {
    const float *at = of + (p.c - p.c0);
#pragma unroll
    for (int e = 0; e < VEC; e++) v[e] = at[e];
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

template <int DT>
__device__ inline char *column_at(const View &x, const Place &p, int64_t first) {
    return x.p + p.i * x.ss + (first + p.row) * x.ts + (int64_t)p.c * Elem<DT>::kSize;
}

// Forward.  R: passes over the rows that a thread holds.
template <int DT, bool WIDE, int NT, int R, int MODE>
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
        int parts = sum_rows<NT, VEC>(a, p, acc, s);
        sum_groups<NT>(p, s.chan, parts, nullptr, s.group);
        const float inv = own ? 1.0f / ((float)own * (float)each) : 0.0f;
        for_channels<NT>(a, p, [&](int ch, int g) { s.of[0][ch] = s.group[g] * inv; });
        __syncthreads();
        float m[VEC];
        of_column<VEC>(s.of[0], p, m);
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
        parts = sum_rows<NT, VEC>(a, p, acc, s);
        sum_groups<NT>(p, s.chan, parts, nullptr, s.group2);
        if (MODE == kStats) {
            const int K = a.chunks * a.parts, k = p.chunk * a.parts + (a.parts > 1 ? p.slab % a.parts : 0);
            for (int g = threadIdx.x; g < p.ng; g += NT)
                a.stats[((int64_t)p.i * a.G + p.g0 + g) * K + k] = make_float2(s.group[g] * inv, s.group2[g]);
            return;
        }
        for (int g = threadIdx.x; g < p.ng; g += NT) {
            const float mean = s.group[g] * inv, rstd = own ? 1.0f / sqrtf(s.group2[g] * inv + a.eps) : 0.0f;
            s.group[g] = mean, s.group2[g] = rstd;
            a.mean[(int64_t)p.i * a.G + p.g0 + g] = mean;
            a.rstd[(int64_t)p.i * a.G + p.g0 + g] = rstd;
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
    __syncthreads();
    for_channels<NT>(a, p, [&](int ch, int g) {
        s.of[0][ch] = s.group[g];
        s.of[1][ch] = s.group2[g] * (a.w ? a.w[p.c0 + ch] : 1.0f);
        s.of[2][ch] = a.b ? a.b[p.c0 + ch] : 0.0f;
    });
    __syncthreads();

    if (!p.active) return;
    float m[VEC], sc[VEC], sh[VEC];
    of_column<VEC>(s.of[0], p, m);
    of_column<VEC>(s.of[1], p, sc);
    of_column<VEC>(s.of[2], p, sh);
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
            if (r < rest) P::store(out + pass * a.out.ts, y);
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

// What the backward pass keeps of an element's channel.  z is the fused
// x A + B with A = r w and B = b - m A, but for ReLU: there z is rounded step by
// step as the formula is written, since the slope jumps with z's sign.
template <int VEC, int ACT>
struct Channel {
    static constexpr bool kSteps = ACT == ROCKET_ACT_RELU;
    float A[VEC], B[VEC];                                // x A + B; in steps: w and b
    float m[kSteps ? VEC : 1], r[kSteps ? VEC : 1];
    __device__ float z(float x, int e) const {
        if (kSteps) return (x - m[kSteps ? e : 0]) * r[kSteps ? e : 0] * A[e] + B[e];
        return __builtin_fmaf(x, A[e], B[e]);
    }
    __device__ float scale(int e) const { return kSteps ? A[e] * r[kSteps ? e : 0] : A[e]; }
    __device__ void take(const Scratch &s, const Place &p) {
        of_column<VEC>(s.of[0], p, A);
        of_column<VEC>(s.of[1], p, B);
        if constexpr (kSteps) {
            of_column<VEC>(s.of[2], p, m);
            of_column<VEC>(s.of[3], p, r);
        }
    }
};

// Backward.  Held: a workgroup goes through the series b, b + a.series, ... and
// keeps the channel sums over them; kStats leaves the channel sums of a chunk.
// sum dz xh is gathered as sum dz (x - k), k the mean of the slab's first
// group, and completed once a channel: r (sum dz (x - k) - (m - k) sum dz).
template <int DT, bool WIDE, int NT, int R, int MODE, int ACT, bool ONE>
__global__ __launch_bounds__(NT, 4) void norm_back_kernel(NormArgs a) {
    using P = Pack<DT, WIDE>;
    constexpr int VEC = P::kN;
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
            if (ACT == ROCKET_ACT_RELU) {
                s.of[0][ch] = w, s.of[1][ch] = bias, s.of[2][ch] = m, s.of[3][ch] = r;
            } else {
                s.of[0][ch] = r * w, s.of[1][ch] = __builtin_fmaf(-m, r * w, bias);
            }
        });
        __syncthreads();
        if (MODE != kApply) {
            Channel<VEC, ACT> of;
            of.take(s, p);
            const float k = mean[0];
            float sd[VEC], sx[VEC];
#pragma unroll
            for (int e = 0; e < VEC; e++) sd[e] = 0.0f, sx[e] = 0.0f;
#pragma unroll
            for (int j = 0; j < R; j++)
                if (p.row + j * a.rows < own) {
#pragma unroll
                    for (int e = 0; e < VEC; e++) {
                        const float v = hx[j].get(e);
                        const float dz = hg[j].get(e) * slope<DT, ACT>(of.z(v, e));
                        sd[e] += dz;
                        sx[e] = __builtin_fmaf(dz, v - k, sx[e]);
                    }
                }
            int parts = sum_rows<NT, VEC>(a, p, sd, s);
            for (int ch = threadIdx.x; ch < W; ch += NT) {
                float t = 0.0f;
                for (int q = 0; q < parts; q++) t += s.chan[q * W + ch];
                s.first[ch] = t;
            }
            if (MODE == kHeld) sum_groups<NT>(p, s.chan, parts, a.w, s.group);
            parts = sum_rows<NT, VEC>(a, p, sx, s);
            for_channels<NT>(a, p, [&](int ch, int g) {
                const float d = s.first[ch];
                float t = 0.0f;
                for (int q = 0; q < parts; q++) t += s.chan[q * W + ch];
                t = rstd[g] * __builtin_fmaf(k - mean[g], d, t);
                if (MODE == kHeld) {
                    s.total[ch] += d, s.total[W + ch] += t;
                } else {
                    float *sum = a.sums + ((int64_t)p.i * a.chunks + p.chunk) * 2 * a.C + p.c0 + ch;
                    sum[0] = d, sum[a.C] = t;
                }
                s.first[ch] = t;
            });
            if (MODE == kStats) return;
            __syncthreads();
            sum_groups<NT>(p, s.first, 1, a.w, s.group2);
        } else {
            // the groups' sums from the chunks' channel sums
            for (int k = threadIdx.x >> 6; k < 2 * p.ng; k += NT >> 6) {
                const int q = k & 1, g = k >> 1;
                float t = 0.0f;
                for (int ch = threadIdx.x & 63; ch < a.width; ch += 64) {
                    const int c = (p.g0 + g) * a.width + ch;
                    const float *sum = a.sums + ((int64_t)p.i * a.chunks * 2 + q) * a.C + c;
                    float u = 0.0f;
                    for (int chunk = 0; chunk < a.chunks; chunk++) u += sum[(int64_t)chunk * 2 * a.C];
                    t += a.w ? a.w[c] * u : u;
                }
#pragma unroll
                for (int off = 32; off; off /= 2) t += __shfl_xor(t, off);
                if ((threadIdx.x & 63) == 0) (q ? s.group2 : s.group)[g] = t;
            }
            __syncthreads();
        }
        // dx = r (dz w - mean(g) - xh mean(g xh)) = dz r w - (x D + E)
        const float inv = T ? 1.0f / ((float)T * (float)a.width) : 0.0f;
        for_channels<NT>(a, p, [&](int ch, int g) {
            const float m = mean[g], r = rstd[g], D = r * r * (s.group2[g] * inv);
            s.chan[ch] = D;
            s.first[ch] = __builtin_fmaf(-m, D, r * (s.group[g] * inv));
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
        Channel<VEC, ACT> of;
        of.take(s, p);
        constexpr int kOwn = ONE ? 1 : VEC;
        float D[kOwn], E[kOwn];
        of_column<kOwn>(s.chan, p, D);
        of_column<kOwn>(s.first, p, E);
        for (int j0 = 0; j0 < R && j0 * a.rows < rest; j0 += H) {
            if (MODE == kApply) {
#pragma unroll
                for (int j = 0; j < H; j++) load(j, j0);
            }
#pragma unroll
            for (int j = 0; j < H; j++) {
                const int pass = (j0 + j) * a.rows, r = p.row + pass;
                float dx[VEC];
#pragma unroll
                for (int e = 0; e < VEC; e++) dx[e] = 0.0f;
                if (r < had) {
                    hx[j].renew(), hg[j].renew();
#pragma unroll
                    for (int e = 0; e < VEC; e++) {
                        const float v = hx[j].get(e), dz = hg[j].get(e) * slope<DT, ACT>(of.z(v, e));
                        dx[e] = __builtin_fmaf(dz, of.scale(e), -__builtin_fmaf(v, D[ONE ? 0 : e], E[ONE ? 0 : e]));
                    }
                }
                if (r < rest && p.active) P::store(out + pass * a.out.ts, dx);
                if (MODE == kHeld) load(j, 0);
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
    int64_t grid;
    int64_t sum_rows;   // backward: rows of channel sums
    int64_t folded;     // rows after the first fold, 0: one fold is enough
};

constexpr int kFold = 128;
// Workgroups that hold a slab: threads, and 16-byte columns of a thread (of
// each operand).
struct Size {
    int threads, run;
};
constexpr Size kSizes[] = {{64, 4}, {256, 4}, {256, 8}, {512, 8}, {512, 16}};
constexpr Size kBackSizes[] = {{64, 4}, {256, 4}, {256, 8}, {512, 8}};
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
        return cut->rows >= 1 && (int64_t)cut->rows * z.run >= L;
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
    cut->one = width % vec == 0;
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
        // A slab is at least 128 bytes wide (a cache line), and wider while
        // that leaves workgroups for the whole chip and the slab is small.
        // 64 bytes where only that is held.
        int64_t per = 1, half = 1;
        while (half < groups && half * width * size < 64) half++;
        while (per < groups && per * width * size < 128) per++;
        while (per * 2 <= groups && per * 2 * width <= most && per * width * size * L < (16 << 10) &&
               s->n * ((groups + 2 * per - 1) / (2 * per)) >= 1024)
            per *= 2;
        cut->held = hold(s, groups, per, vec, back, cut) ||
                    (half < per && hold(s, groups, half, vec, back, cut));
        if (!cut->held) hold(s, groups, per, vec, back, cut);
    }
    cut->chunks = 1;
    cut->folded = 0;
    if (!cut->held) {
        cut->threads = kChunk.threads, cut->run = (back ? kBackChunk : kChunk).run;
        cut->rows = cut->threads / cut->cols;
        const int64_t step = (int64_t)cut->rows * cut->run, chunks = (L + step - 1) / step;
        if (chunks > INT_MAX) return false;
        cut->chunks = (int32_t)chunks;
        if (__builtin_mul_overflow(s->n * chunks, (int64_t)cut->slabs, &cut->grid)) return false;
        cut->sum_rows = s->n * chunks;
    } else if (back) {
        int64_t series = (1024 + cut->slabs - 1) / cut->slabs;
        if (series > s->n) series = s->n;
        cut->series = (int32_t)(series > 0 ? series : 1);
        cut->grid = (int64_t)cut->series * cut->slabs;
        cut->sum_rows = cut->series;
    } else {
        cut->grid = s->n * cut->slabs;
    }
    if (back && cut->sum_rows > 4 * kFold) cut->folded = (cut->sum_rows + kFold - 1) / kFold;
    const int64_t fold_grid = (cut->folded ? cut->folded : 1) * 2 * ((C + 63) / 64);
    return cut->grid <= INT_MAX && (!back || fold_grid <= INT_MAX);
}

int64_t workspace_of(const rocket_sequence_shape *s, int32_t groups, bool back, const Cut &c) {
    if (back) return (c.sum_rows + c.folded) * 2 * s->channels * (int64_t)sizeof(float);
    return c.held ? 0 : s->n * groups * (int64_t)c.chunks * c.parts * (int64_t)sizeof(float2);
}

template <int DT, bool BACK, bool WIDE, int NT, int R, int MODE>
void go(const NormArgs &a, const Cut &c, hipStream_t s) {
    const uint32_t grid = (uint32_t)c.grid;
    const int lds = (int)scratch_floats(NT, Pack<DT, WIDE>::kN, c.cols, c.rows, c.groups, BACK) * 4;
    if constexpr (!BACK) {
        norm_kernel<DT, WIDE, NT, R, MODE><<<grid, NT, lds, s>>>(a);
    } else {
        // columns that lie in one group each, where registers are short
        const bool one = WIDE && MODE == kHeld && R > 4 && c.one;
        auto act = [&](auto k) {
            constexpr int ACT = decltype(k)::value;
            if constexpr (WIDE && MODE == kHeld && R > 4) {
                if (one) {
                    norm_back_kernel<DT, WIDE, NT, R, MODE, ACT, true><<<grid, NT, lds, s>>>(a);
                    return;
                }
            }
            norm_back_kernel<DT, WIDE, NT, R, MODE, ACT, false><<<grid, NT, lds, s>>>(a);
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
void run_type(int32_t dtype, const NormArgs &a, const Cut &c, hipStream_t s) {
    if (dtype == ROCKET_FLOAT32)
        run<ROCKET_FLOAT32, BACK>(a, c, s);
    else if (dtype == ROCKET_BFLOAT16)
        run<ROCKET_BFLOAT16, BACK>(a, c, s);
    else
        run<ROCKET_FLOAT16, BACK>(a, c, s);
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
    if (workspace_bytes < need || (need && (!workspace || !aligned(workspace, 4)))) return ROCKET_ERR_INVALID_ARG;
    hipStream_t s = (hipStream_t)hip_stream;
    const int size = rocket::elem_size(shape->dtype), C = (int)shape->channels;
    float *sums = (float *)workspace;
    int64_t rows = 0;
    if (!rocket::empty(shape)) {
        NormArgs a = args_of(shape, groups, activation, weight, bias, cut);
        a.x = view(x, size), a.dy = view(dy, size), a.out = view(dx, size);
        a.mean = const_cast<float *>(mean), a.rstd = const_cast<float *>(rstd), a.sums = sums;
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
