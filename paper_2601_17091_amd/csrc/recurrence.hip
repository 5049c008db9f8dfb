// Gated linear recurrence along the steps of sequences [n, L, C]:
//
//   h_t = S(f_t) h_{t-1} + (1 - S(f_t)) v_t,   y_t = S(o_t) h_t (or h_t)
//
// Any run of steps is an affine map of the state before it, h -> A h + B, and
// maps compose: (A2, B2) after (A1, B1) is (A2 A1, A2 B1 + B2).  So the time
// axis splits: a thread composes its own 16 steps, the lanes and wavefronts of
// a workgroup combine theirs into the map of a tile, and the tiles of a series
// combine over the grid.  Every combination runs in a fixed order, so results
// do not change from call to call.  The gradient is the same scan from the
// other end: with g_t = dy_t S(o_t), the gradient that reaches h_{t-1} is
//   e_t = S(f_t) (g_t + e_{t+1}),   e_L = the gradient of the last state,
// and with dh_t = g_t + e_{t+1}
//   dv = dh (1 - a),  df = dh (h_{t-1} - v) a (1 - a),  do = dy h S(o) (1 - S(o)).
// The states are held in fp32 throughout; y and the gradients are rounded once.
//
// Layout: a lane takes one 32-bit word of channels (one fp32, two 16-bit), so
// that a wavefront's load of one step is 256 contiguous bytes; where a series
// has fewer than 64 words of channels, the lanes left over take further runs
// of steps.  Steps past a series' length act as h -> h and are not read.
#include <climits>

#include "sequence.h"

namespace {

using rocket::Elem;

constexpr int kWaves = 8;
constexpr int kThreads = 64 * kWaves;
constexpr int kRun = 16;                       // steps of one thread
constexpr int kEvery = ROCKET_RECURRENCE_EVERY;  // steps between kept states
static_assert(kEvery % kRun == 0 && (kWaves * kRun) % kEvery == 0, "kept states fall on the starts of runs and tiles");

struct View {
    char *p;
    int64_t ss, ts;  // bytes
};

struct RecArgs {
    View v, f, o, y;        // y: forward
    View dy, dv, df, dO;    // backward
    int64_t n, L, C;
    const int32_t *lengths;
    const float *h0;        // forward, or null
    float *h_last;          // forward
    float *states;          // kept states [n, ceil(L / kEvery), C]: written (or null) forward, read backward
    const float *dh_last;   // backward, or null
    float *dh0;             // backward
    float2 *maps;           // [n, tiles, C], tiles > 1
    int32_t tiles, lanes;   // lanes over channels, a power of two
    int32_t blocks;         // channel blocks
};

// Where a thread works.
struct Place {
    int64_t i, len;   // series, its steps
    int64_t t0;       // first step of the thread's run
    int64_t c, c_ld;  // its first channel, and the channel it loads from
    int tile, wave, lane, lanes;
    int count;        // channels it owns: 0, 1 or 2
    bool high;        // its one channel is the high half of the word at c_ld
    bool single;      // C == 1 and 16-bit elements: no whole word to load
};

template <int DT>
__device__ inline Place place_of(const RecArgs &a) {
    constexpr int P = Elem<DT>::kPerWord;
    Place p;
    const int64_t b = blockIdx.x;
    const int64_t cb = b % a.blocks, rest = b / a.blocks;
    p.i = rest % a.n;
    p.tile = (int)(rest / a.n);
    p.wave = threadIdx.x >> 6;
    p.lane = threadIdx.x & 63;
    p.lanes = a.lanes;
    const int runs = 64 / a.lanes;
    const int cl = p.lane & (a.lanes - 1), q = p.lane / a.lanes;
    p.c = (cb * a.lanes + cl) * P;
    int64_t left = a.C - p.c;
    p.count = left <= 0 ? 0 : left < P ? 1 : P;
    p.high = P == 2 && p.count == 1 && a.C > 1;
    p.single = P == 2 && a.C == 1;
    p.c_ld = p.c + P <= a.C ? p.c : a.C > P ? a.C - P : 0;
    p.len = rocket::steps_of(a.lengths, p.i, a.L);
    p.t0 = (((int64_t)p.tile * kWaves + p.wave) * runs + q) * kRun;
    return p;
}

// The words of a run; steps past the series' length repeat its last one (they
// are masked later), and a series of no steps loads nothing.
template <int DT>
__device__ inline void load_run(const View &x, const Place &p, uint32_t (&w)[kRun]) {
    if (p.len == 0) {
#pragma unroll
        for (int s = 0; s < kRun; s++) w[s] = 0;
        return;
    }
    const char *base = x.p + p.i * x.ss + p.c_ld * Elem<DT>::kSize;
#pragma unroll
    for (int s = 0; s < kRun; s++) {
        int64_t t = p.t0 + s < p.len ? p.t0 + s : p.len - 1;
        if (p.single)
            w[s] = *(const typename Elem<DT>::raw *)(base + t * x.ts);
        else
            w[s] = rocket::load_at<uint32_t>(base + t * x.ts);
    }
    if (p.high) {
#pragma unroll
        for (int s = 0; s < kRun; s++) w[s] >>= 16;
    }
}

template <int DT>
__device__ inline void store_step(const View &x, const Place &p, int64_t t, const float *val) {
    char *q = x.p + p.i * x.ss + t * x.ts + p.c * Elem<DT>::kSize;
    if (p.count == Elem<DT>::kPerWord)
        rocket::store_at(q, Elem<DT>::put(val));
    else if (p.count == 1)
        *(typename Elem<DT>::raw *)q = Elem<DT>::round(val[0]);
}

// Composes the maps of the runs before a thread's own inside its tile:
// (eA, eB), applied to the state at the tile's start, gives the state at the
// run's start.  tA, tB: the whole tile's map.  REVERSE: from the last run to
// the first.
template <int P, bool REVERSE>
__device__ inline void compose_tile(const Place &p, const float *A, const float *B, float *eA, float *eB, float *tA,
                                    float *tB, float2 (*maps)[64 * 2]) {
    float sA[P], sB[P];
#pragma unroll
    for (int j = 0; j < P; j++) sA[j] = A[j], sB[j] = B[j];
    for (int off = p.lanes; off < 64; off *= 2) {
        bool on = REVERSE ? p.lane + off < 64 : p.lane >= off;
#pragma unroll
        for (int j = 0; j < P; j++) {
            float pa = REVERSE ? __shfl_down(sA[j], off) : __shfl_up(sA[j], off);
            float pb = REVERSE ? __shfl_down(sB[j], off) : __shfl_up(sB[j], off);
            if (on) {
                sB[j] = __builtin_fmaf(sA[j], pb, sB[j]);
                sA[j] *= pa;
            }
        }
    }
    const int cl = p.lane & (p.lanes - 1);
    const bool first = REVERSE ? p.lane + p.lanes >= 64 : p.lane < p.lanes;   // nothing before it in its wavefront
    const bool last = REVERSE ? p.lane < p.lanes : p.lane + p.lanes >= 64;
    if (last) {
#pragma unroll
        for (int j = 0; j < P; j++) maps[p.wave][cl * P + j] = make_float2(sA[j], sB[j]);
    }
#pragma unroll
    for (int j = 0; j < P; j++) {
        float xa = sA[j], xb = sB[j];
        if (p.lanes < 64) {
            xa = REVERSE ? __shfl_down(sA[j], p.lanes) : __shfl_up(sA[j], p.lanes);
            xb = REVERSE ? __shfl_down(sB[j], p.lanes) : __shfl_up(sB[j], p.lanes);
        }
        eA[j] = first ? 1.0f : xa;
        eB[j] = first ? 0.0f : xb;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < P; j++) {
        float wA = 1.0f, wB = 0.0f;   // the wavefronts before this one
        float aA = 1.0f, aB = 0.0f;   // all of them
#pragma unroll
        for (int k = 0; k < kWaves; k++) {
            const int w = REVERSE ? kWaves - 1 - k : k;
            if (w == p.wave) wA = aA, wB = aB;
            float2 m = maps[w][cl * P + j];
            aB = __builtin_fmaf(m.x, aB, m.y);
            aA *= m.x;
        }
        eB[j] = __builtin_fmaf(eA[j], wB, eB[j]);
        eA[j] *= wA;
        tA[j] = aA, tB[j] = aB;
    }
}

// The state at a tile's start: the maps of the tiles before it (REVERSE:
// after it) applied to `h` in order.  Each wavefront composes a range of them,
// then the ranges are applied in turn.
template <int P, bool REVERSE>
__device__ inline void apply_tiles(const RecArgs &a, const Place &p, float *h, float2 (*maps)[64 * 2]) {
    const int before = REVERSE ? a.tiles - 1 - p.tile : p.tile;
    if (before == 0) return;   // the same for the whole workgroup
    const int cl = p.lane & (p.lanes - 1);
    __syncthreads();           // maps is free again
    if (p.lane < p.lanes) {
        float A[P], B[P];
#pragma unroll
        for (int j = 0; j < P; j++) A[j] = 1.0f, B[j] = 0.0f;
        const int from = (int)((int64_t)before * p.wave / kWaves), to = (int)((int64_t)before * (p.wave + 1) / kWaves);
        for (int k = from; k < to; k++) {
            const int tile = REVERSE ? a.tiles - 1 - k : k;
            const float2 *m = a.maps + (p.i * a.tiles + tile) * a.C + p.c;
#pragma unroll
            for (int j = 0; j < P; j++)
                if (j < p.count) {
                    float2 x = m[j];
                    B[j] = __builtin_fmaf(x.x, B[j], x.y);
                    A[j] *= x.x;
                }
        }
#pragma unroll
        for (int j = 0; j < P; j++) maps[p.wave][cl * P + j] = make_float2(A[j], B[j]);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < P; j++)
#pragma unroll
        for (int w = 0; w < kWaves; w++) {
            float2 m = maps[w][cl * P + j];
            h[j] = __builtin_fmaf(m.x, h[j], m.y);
        }
}

// The forward pass over a tile.  MAPS: only the tile's map, for the tiles that
// follow; else everything.
template <int DT, bool MAPS, bool GATE>
__global__ __launch_bounds__(kThreads, 4) void forward_kernel(RecArgs a) {
    constexpr int P = Elem<DT>::kPerWord;
    __shared__ float2 maps[kWaves][64 * 2];
    const Place p = place_of<DT>(a);
    uint32_t wv[kRun], wf[kRun], wo[kRun];
    load_run<DT>(a.v, p, wv);
    load_run<DT>(a.f, p, wf);
    if (GATE && !MAPS) load_run<DT>(a.o, p, wo);

    float fa[kRun][P], fb[kRun][P], A[P], B[P];
#pragma unroll
    for (int j = 0; j < P; j++) A[j] = 1.0f, B[j] = 0.0f;
#pragma unroll
    for (int s = 0; s < kRun; s++)
#pragma unroll
        for (int j = 0; j < P; j++) {
            float keep, in;
            rocket::logistic(Elem<DT>::get(wf[s], j), keep, in);
            float b = in * Elem<DT>::get(wv[s], j);
            const bool live = p.t0 + s < p.len;
            fa[s][j] = live ? keep : 1.0f;
            fb[s][j] = live ? b : 0.0f;
            B[j] = __builtin_fmaf(fa[s][j], B[j], fb[s][j]);
            A[j] *= fa[s][j];
        }

    float eA[P], eB[P], tA[P], tB[P];
    compose_tile<P, false>(p, A, B, eA, eB, tA, tB, maps);
    if (MAPS) {
        if (p.wave == 0 && p.lane < p.lanes)
#pragma unroll
            for (int j = 0; j < P; j++)
                if (j < p.count) a.maps[(p.i * a.tiles + p.tile) * a.C + p.c + j] = make_float2(tA[j], tB[j]);
        return;
    }

    float h[P];
#pragma unroll
    for (int j = 0; j < P; j++) h[j] = a.h0 && j < p.count ? a.h0[p.i * a.C + p.c + j] : 0.0f;
    apply_tiles<P, false>(a, p, h, maps);
#pragma unroll
    for (int j = 0; j < P; j++) h[j] = __builtin_fmaf(eA[j], h[j], eB[j]);

    if (a.states && p.t0 % kEvery == 0 && p.t0 < a.L) {
        const int64_t per = (a.L + kEvery - 1) / kEvery;
#pragma unroll
        for (int j = 0; j < P; j++)
            if (j < p.count) a.states[(p.i * per + p.t0 / kEvery) * a.C + p.c + j] = h[j];
    }
#pragma unroll
    for (int s = 0; s < kRun; s++) {
        float y[P];
#pragma unroll
        for (int j = 0; j < P; j++) {
            h[j] = __builtin_fmaf(fa[s][j], h[j], fb[s][j]);
            y[j] = h[j];
            if (GATE) {
                float so, rest;
                rocket::logistic(Elem<DT>::get(wo[s], j), so, rest);
                y[j] *= so;
            }
            if (!(p.t0 + s < p.len)) y[j] = 0.0f;
        }
        if (p.t0 + s < a.L) store_step<DT>(a.y, p, p.t0 + s, y);
    }
    const int64_t end = a.L > 0 ? a.L - 1 : 0;
    if (p.t0 <= end && end < p.t0 + kRun)
#pragma unroll
        for (int j = 0; j < P; j++)
            if (j < p.count) a.h_last[p.i * a.C + p.c + j] = h[j];
}

// The backward pass over a tile.  MAPS: only the tile's map of the gradient
// that runs towards its start; else everything, from the kept state.
template <int DT, bool MAPS, bool GATE>
__global__ __launch_bounds__(kThreads, 4) void backward_kernel(RecArgs a) {
    constexpr int P = Elem<DT>::kPerWord;
    __shared__ float2 maps[kWaves][64 * 2];
    const Place p = place_of<DT>(a);
    uint32_t wv[kRun], wf[kRun], wo[kRun], wg[kRun];
    load_run<DT>(a.f, p, wf);
    load_run<DT>(a.dy, p, wg);
    if (GATE) load_run<DT>(a.o, p, wo);
    if (!MAPS) load_run<DT>(a.v, p, wv);

    float h[kRun][P];   // the state before each step
    float A[P], R[P], B[P];
#pragma unroll
    for (int j = 0; j < P; j++) A[j] = 1.0f, R[j] = 0.0f, B[j] = 0.0f;
#pragma unroll
    for (int s = kRun - 1; s >= 0; s--)
#pragma unroll
        for (int j = 0; j < P; j++) {
            float keep, in, so = 1.0f, rest;
            rocket::logistic(Elem<DT>::get(wf[s], j), keep, in);
            if (GATE) rocket::logistic(Elem<DT>::get(wo[s], j), so, rest);
            const float g = Elem<DT>::get(wg[s], j) * so;
            if (p.t0 + s < p.len) {
                R[j] = keep * (R[j] + g);
                if (!MAPS) B[j] = __builtin_fmaf(A[j], in * Elem<DT>::get(wv[s], j), B[j]);
                A[j] *= keep;
            }
        }

    float eA[P], eR[P], tA[P], tR[P];
    compose_tile<P, true>(p, A, R, eA, eR, tA, tR, maps);
    if (MAPS) {
        if (p.wave == 0 && p.lane < p.lanes)
#pragma unroll
            for (int j = 0; j < P; j++)
                if (j < p.count) a.maps[(p.i * a.tiles + p.tile) * a.C + p.c + j] = make_float2(tA[j], tR[j]);
        return;
    }
    float e[P];
#pragma unroll
    for (int j = 0; j < P; j++) e[j] = a.dh_last && j < p.count ? a.dh_last[p.i * a.C + p.c + j] : 0.0f;
    apply_tiles<P, true>(a, p, e, maps);
#pragma unroll
    for (int j = 0; j < P; j++) e[j] = __builtin_fmaf(eA[j], e[j], eR[j]);

    float fA[P], fB[P];
    __syncthreads();
    compose_tile<P, false>(p, A, B, fA, fB, tA, tR, maps);
    const int64_t start = p.tile * (int64_t)(kWaves * kRun) * (64 / p.lanes);   // the tile's first step
    const int64_t per = (a.L + kEvery - 1) / kEvery;
    float state[P];
#pragma unroll
    for (int j = 0; j < P; j++) {
        float s0 = start < a.L && j < p.count ? a.states[(p.i * per + start / kEvery) * a.C + p.c + j] : 0.0f;
        state[j] = __builtin_fmaf(fA[j], s0, fB[j]);
    }
#pragma unroll
    for (int s = 0; s < kRun; s++)
#pragma unroll
        for (int j = 0; j < P; j++) {
            float keep, in;
            rocket::logistic(Elem<DT>::get(wf[s], j), keep, in);
            h[s][j] = state[j];
            state[j] = __builtin_fmaf(keep, state[j], in * Elem<DT>::get(wv[s], j));
        }
#pragma unroll
    for (int s = kRun - 1; s >= 0; s--) {
        const bool live = p.t0 + s < p.len;
        float gv[P], gf[P], go[P];
#pragma unroll
        for (int j = 0; j < P; j++) {
            float keep, in, so = 1.0f, rest = 0.0f;
            rocket::logistic(Elem<DT>::get(wf[s], j), keep, in);
            if (GATE) rocket::logistic(Elem<DT>::get(wo[s], j), so, rest);
            const float v = Elem<DT>::get(wv[s], j), dy = Elem<DT>::get(wg[s], j);
            const float dh = __builtin_fmaf(dy, so, e[j]);
            gv[j] = live ? dh * in : 0.0f;
            gf[j] = live ? gv[j] * (h[s][j] - v) * keep : 0.0f;
            if (GATE) go[j] = live ? dy * __builtin_fmaf(keep, h[s][j], in * v) * so * rest : 0.0f;
            e[j] = live ? keep * dh : e[j];
        }
        if (p.t0 + s < a.L) {
            store_step<DT>(a.dv, p, p.t0 + s, gv);
            store_step<DT>(a.df, p, p.t0 + s, gf);
            if (GATE) store_step<DT>(a.dO, p, p.t0 + s, go);
        }
    }
    if (p.t0 == 0)
#pragma unroll
        for (int j = 0; j < P; j++)
            if (j < p.count) a.dh0[p.i * a.C + p.c + j] = e[j];
}

// One step of every series: a word of channels per thread.
struct StepArgs {
    const char *v, *f, *o;
    char *y;
    int64_t vs, fs, os, ys;  // row strides, bytes
    const float *h_in;
    float *h_out;
    int64_t n, C, words;     // words of channels per series
};

template <int DT, bool GATE>
__global__ __launch_bounds__(256) void step_kernel(StepArgs a) {
    using raw = typename Elem<DT>::raw;
    constexpr int P = Elem<DT>::kPerWord;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= a.n * a.words) return;
    const int64_t i = id / a.words, c = (id - i * a.words) * P;
    const int count = a.C - c < P ? 1 : P;
    const char *pv = a.v + i * a.vs + c * Elem<DT>::kSize, *pf = a.f + i * a.fs + c * Elem<DT>::kSize;
    const char *po = GATE ? a.o + i * a.os + c * Elem<DT>::kSize : nullptr;
    char *py = a.y + i * a.ys + c * Elem<DT>::kSize;
    uint32_t wv, wf, wo = 0;
    if (count == P) {
        wv = rocket::load_at<uint32_t>(pv), wf = rocket::load_at<uint32_t>(pf);
        if (GATE) wo = rocket::load_at<uint32_t>(po);
    } else {
        wv = *(const raw *)pv, wf = *(const raw *)pf;
        if (GATE) wo = *(const raw *)po;
    }
    float h[P], y[P];
#pragma unroll
    for (int j = 0; j < P; j++) h[j] = j < count ? a.h_in[i * a.C + c + j] : 0.0f;
#pragma unroll
    for (int j = 0; j < P; j++) {
        float keep, in;
        rocket::logistic(Elem<DT>::get(wf, j), keep, in);
        h[j] = __builtin_fmaf(keep, h[j], in * Elem<DT>::get(wv, j));
        y[j] = h[j];
        if (GATE) {
            float so, rest;
            rocket::logistic(Elem<DT>::get(wo, j), so, rest);
            y[j] *= so;
        }
    }
#pragma unroll
    for (int j = 0; j < P; j++)
        if (j < count) a.h_out[i * a.C + c + j] = h[j];
    if (count == P)
        rocket::store_at(py, Elem<DT>::put(y));
    else
        *(raw *)py = Elem<DT>::round(y[0]);
}

// How a call is cut.
struct Cut {
    int32_t lanes, blocks, tiles;
    int64_t grid;
};

// Lanes over channels: the power of two that covers the words of channels, 64
// at most; the wavefront's other lanes take further runs of steps, so that
// few channels do not leave lanes idle.
bool cut_of(const rocket_sequence_shape *s, Cut *cut) {
    const int64_t per_word = rocket::elem_size(s->dtype) == 4 ? 1 : 2;
    const int64_t words = (s->channels + per_word - 1) / per_word;
    cut->lanes = 1;
    while (cut->lanes < 64 && cut->lanes < words) cut->lanes *= 2;
    const int64_t steps = (int64_t)kWaves * kRun * (64 / cut->lanes);
    cut->blocks = (int32_t)((words + cut->lanes - 1) / cut->lanes);
    cut->tiles = (int32_t)(s->steps > steps ? (s->steps + steps - 1) / steps : 1);
    return !__builtin_mul_overflow(s->n * cut->blocks, (int64_t)cut->tiles, &cut->grid) && cut->grid <= INT_MAX;
}

int64_t workspace_of(const rocket_sequence_shape *s, const Cut &cut) {
    return cut.tiles > 1 ? s->n * cut.tiles * s->channels * (int64_t)sizeof(float2) : 0;
}

View view(const rocket_sequence *q, int size) {
    return q ? View{(char *)q->data, q->series_stride * size, q->step_stride * size} : View{nullptr, 0, 0};
}

bool aligned(const void *p, uintptr_t to) { return (uintptr_t)p % to == 0; }

template <int DT, bool GATE>
void run_forward(const RecArgs &a, const Cut &cut, hipStream_t s) {
    if (cut.tiles > 1) forward_kernel<DT, true, GATE><<<(uint32_t)cut.grid, kThreads, 0, s>>>(a);
    forward_kernel<DT, false, GATE><<<(uint32_t)cut.grid, kThreads, 0, s>>>(a);
}

template <int DT, bool GATE>
void run_backward(const RecArgs &a, const Cut &cut, hipStream_t s) {
    if (cut.tiles > 1) backward_kernel<DT, true, GATE><<<(uint32_t)cut.grid, kThreads, 0, s>>>(a);
    backward_kernel<DT, false, GATE><<<(uint32_t)cut.grid, kThreads, 0, s>>>(a);
}

template <int DT, bool GATE>
void run_step(const StepArgs &a, hipStream_t s) {
    const int64_t threads = a.n * a.words;
    step_kernel<DT, GATE><<<(uint32_t)((threads + 255) / 256), 256, 0, s>>>(a);
}

#define BY_TYPE(fn, dtype, gate, ...)                                                                       \
    do {                                                                                                    \
        if ((dtype) == ROCKET_FLOAT32)                                                                      \
            (gate) ? fn<ROCKET_FLOAT32, true>(__VA_ARGS__) : fn<ROCKET_FLOAT32, false>(__VA_ARGS__);        \
        else if ((dtype) == ROCKET_BFLOAT16)                                                                \
            (gate) ? fn<ROCKET_BFLOAT16, true>(__VA_ARGS__) : fn<ROCKET_BFLOAT16, false>(__VA_ARGS__);      \
        else                                                                                                \
            (gate) ? fn<ROCKET_FLOAT16, true>(__VA_ARGS__) : fn<ROCKET_FLOAT16, false>(__VA_ARGS__);        \
    } while (0)

}  // namespace

extern "C" rocket_status rocket_recurrence_workspace(const rocket_sequence_shape *shape, int64_t *bytes) {
    Cut cut;
    if (!bytes || !rocket::shape_ok(shape) || !cut_of(shape, &cut)) return ROCKET_ERR_INVALID_ARG;
    *bytes = workspace_of(shape, cut);
    return ROCKET_OK;
}

extern "C" rocket_status rocket_recurrence_forward(const rocket_sequence_shape *shape, const rocket_sequence *v,
                                                   const rocket_sequence *f, const rocket_sequence *o, const float *h0,
                                                   const rocket_sequence *y, float *h_last, float *states,
                                                   void *workspace, int64_t workspace_bytes, void *hip_stream) {
    Cut cut;
    if (!rocket::shape_ok(shape) || !cut_of(shape, &cut) || !rocket::view_ok(v, shape) || !rocket::view_ok(f, shape) ||
        (o && !rocket::view_ok(o, shape)) || !rocket::out_ok(y, shape) || (shape->n > 0 && !h_last))
        return ROCKET_ERR_INVALID_ARG;
    const int64_t need = workspace_of(shape, cut);
    if (workspace_bytes < need || (need && (!workspace || !aligned(workspace, 8)))) return ROCKET_ERR_INVALID_ARG;
    if (!aligned(h0, 4) || !aligned(h_last, 4) || !aligned(states, 4) || !aligned(shape->lengths, 4))
        return ROCKET_ERR_INVALID_ARG;
    if (shape->n == 0) return ROCKET_OK;
    const int size = rocket::elem_size(shape->dtype);
    RecArgs a = {};
    a.v = view(v, size), a.f = view(f, size), a.o = view(o, size), a.y = view(y, size);
    a.n = shape->n, a.L = shape->steps, a.C = shape->channels, a.lengths = shape->lengths;
    a.h0 = h0, a.h_last = h_last, a.states = states, a.maps = (float2 *)workspace;
    a.tiles = cut.tiles, a.lanes = cut.lanes, a.blocks = cut.blocks;
    BY_TYPE(run_forward, shape->dtype, o != nullptr, a, cut, (hipStream_t)hip_stream);
    return rocket::launched();
}

extern "C" rocket_status rocket_recurrence_backward(const rocket_sequence_shape *shape, const rocket_sequence *dy,
                                                    const rocket_sequence *v, const rocket_sequence *f,
                                                    const rocket_sequence *o, const float *states,
                                                    const float *dh_last, const rocket_sequence *dv,
                                                    const rocket_sequence *df, const rocket_sequence *dO, float *dh0,
                                                    void *workspace, int64_t workspace_bytes, void *hip_stream) {
    Cut cut;
    if (!rocket::shape_ok(shape) || !cut_of(shape, &cut) || !rocket::view_ok(dy, shape) ||
        !rocket::view_ok(v, shape) || !rocket::view_ok(f, shape) || (o && !rocket::view_ok(o, shape)) ||
        !rocket::out_ok(dv, shape) || !rocket::out_ok(df, shape) || (o != nullptr) != (dO != nullptr) ||
        (dO && !rocket::out_ok(dO, shape)) || (shape->n > 0 && !dh0) || (!rocket::empty(shape) && !states))
        return ROCKET_ERR_INVALID_ARG;
    const int64_t need = workspace_of(shape, cut);
    if (workspace_bytes < need || (need && (!workspace || !aligned(workspace, 8)))) return ROCKET_ERR_INVALID_ARG;
    if (!aligned(states, 4) || !aligned(dh_last, 4) || !aligned(dh0, 4) || !aligned(shape->lengths, 4))
        return ROCKET_ERR_INVALID_ARG;
    if (shape->n == 0) return ROCKET_OK;
    const int size = rocket::elem_size(shape->dtype);
    RecArgs a = {};
    a.v = view(v, size), a.f = view(f, size), a.o = view(o, size);
    a.dy = view(dy, size), a.dv = view(dv, size), a.df = view(df, size), a.dO = view(dO, size);
    a.n = shape->n, a.L = shape->steps, a.C = shape->channels, a.lengths = shape->lengths;
    a.states = const_cast<float *>(states), a.dh_last = dh_last, a.dh0 = dh0, a.maps = (float2 *)workspace;
    a.tiles = cut.tiles, a.lanes = cut.lanes, a.blocks = cut.blocks;
    BY_TYPE(run_backward, shape->dtype, o != nullptr, a, cut, (hipStream_t)hip_stream);
    return rocket::launched();
}

extern "C" rocket_status rocket_recurrence_step(int64_t n, int64_t channels, int32_t dtype, const void *v,
                                                int64_t v_stride, const void *f, int64_t f_stride, const void *o,
                                                int64_t o_stride, const float *h_in, float *h_out, void *y,
                                                int64_t y_stride, void *hip_stream) {
    rocket_sequence_shape shape = {n, 1, channels, dtype, nullptr};
    if (!rocket::shape_ok(&shape)) return ROCKET_ERR_INVALID_ARG;
    if (n == 0) return ROCKET_OK;
    rocket_sequence sv = {const_cast<void *>(v), v_stride, 0}, sf = {const_cast<void *>(f), f_stride, 0};
    rocket_sequence so = {const_cast<void *>(o), o_stride, 0}, sy = {y, y_stride, 0};
    if (!rocket::view_ok(&sv, &shape) || !rocket::view_ok(&sf, &shape) || (o && !rocket::view_ok(&so, &shape)) ||
        !rocket::out_ok(&sy, &shape) || !h_in || !h_out || !aligned(h_in, 4) || !aligned(h_out, 4))
        return ROCKET_ERR_INVALID_ARG;
    const int size = rocket::elem_size(dtype);
    StepArgs a;
    a.v = (const char *)v, a.f = (const char *)f, a.o = (const char *)o, a.y = (char *)y;
    a.vs = v_stride * size, a.fs = f_stride * size, a.os = o_stride * size, a.ys = y_stride * size;
    a.h_in = h_in, a.h_out = h_out, a.n = n, a.C = channels;
    const int64_t per_word = size == 4 ? 1 : 2;
    a.words = (channels + per_word - 1) / per_word;
    if ((n * a.words + 255) / 256 > INT_MAX) return ROCKET_ERR_INVALID_ARG;
    BY_TYPE(run_step, dtype, o != nullptr, a, (hipStream_t)hip_stream);
    return rocket::launched();
}
