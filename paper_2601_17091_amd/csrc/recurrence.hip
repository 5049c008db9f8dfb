// Gated linear recurrence along the steps of sequences [n, L, C]:
//
//   h_t = S(f_t) h_{t-1} + (1 - S(f_t)) v_t,   y_t = S(o_t) h_t (or h_t)
//
// Any run of steps is an affine map of the state before it, h -> A h + B, and
// maps compose: (A2, B2) after (A1, B1) is (A2 A1, A2 B1 + B2).  So the time
// axis splits: a thread composes its own run of steps, and the lanes and
// wavefronts of a workgroup combine theirs into the states at the runs' starts.
// The gradient is the same scan from the other end: with g_t = dy_t S(o_t), the
// gradient that reaches h_{t-1} is
//   e_t = S(f_t) (g_t + e_{t+1}),   e_L = the gradient of the last state,
// and with dh_t = g_t + e_{t+1}
//   dv = dh (1 - a),  df = dh (h_{t-1} - v) a (1 - a),  do = dy h S(o) (1 - S(o)).
// Every combination runs in a fixed order, so results do not change from call
// to call.  States, gates and gradients of states are held in fp32 throughout;
// y and the gradients are rounded once.
//
// Layout: a lane takes one 32-bit word of channels (one fp32, two 16-bit) of
// 16 elements' worth of steps; 32 lanes side by side take 128 contiguous bytes
// of a step, and the lanes left over take further runs.  A workgroup covers a
// tile of 128 steps (more where few channels leave lanes over) of one row, a
// row being a block of channels of one series.  Where the rows fill the chip, a
// workgroup goes through all tiles of its row, the state carried on, the next
// tile's loads in flight.  Where they do not, every tile has a workgroup of its
// own, and the tiles of a row meet through memory: a workgroup takes the row's
// next tile by a counter, publishes its tile's map, and waits for the maps of
// the tiles before it.  Tiles before it were taken before it and publish their
// maps without waiting for anything, so every wait ends.  To bound what a tile
// reads, every 32nd tile publishes the state behind it, and tiles start from
// that; it waits for earlier tiles only, so these waits end as well.  A map or
// state is one word written and read whole, and never equals the pattern that
// the workspace is filled with, so that it needs no flag and no fence.
// Everything is read once.  The backward pass goes through the tiles from the
// last to the first, each from the state that the forward pass kept there.
//
// Bound: HBM.  Measured: 64 x 1000 x 512, bf16, gated, backward 115 us, 4.0 TB/s
// of the 459 MB that have to move (a large copy reaches 5.0 to 5.3 TB/s); 8 x
// 10000 x 256, fp32, backward 89 us, 4.6 TB/s; 1000 x 1000 x 256, fp32, forward
// 550 us, 5.6 TB/s; 4 x 16384 x 256, bf16, forward 26 us, 3.9 TB/s: 16 rows,
// whose tiles wait for each other; 777 x 129 x 331, fp16, gated, ragged 65 to 71 us
// (full lengths 73 us, 336 channels 63 us: neither the bytes nor the odd rows, but
// workgroups that take as long when few of their wavefronts have steps).
// One counter a cache line: with the 16 rows' counters side by side the last
// but one took 40 us.
#include <algorithm>
#include <type_traits>

#include "sequence.h"

namespace {

using rocket::Elem;

constexpr int kEvery = ROCKET_RECURRENCE_EVERY;  // steps between kept states
constexpr int kElems = 16;                       // elements of a thread in a tile
constexpr int kMostLanes = 32;                   // lanes over channels
constexpr int kMostWaves = 16;                   // of a workgroup that takes a whole series at once
constexpr int kTileWaves = 8;                    // of one that takes a tile of 128 steps
constexpr int kMostChannels = 64;                // of a workgroup: 32 lanes x 2
constexpr int64_t kFill = 512;                   // rows that fill the chip
constexpr int kApart = 64;                       // words from counter to counter: each has its own cache line
// Tiles from one published state to the next: more are more maps to read for
// each tile, fewer are more states that wait for each other (4 x 16384 x 256,
// bf16, forward: 31 us at 64, 29 at 32, 28 at 16; 47, 46 and 46 us at 8 x 10000 x
// 256, fp32).  32 keeps the chain of states short in longer series.
constexpr int kGroup = 32;
// A workgroup's way through a row: all its tiles, one of many, the only one.
enum Way { kLoop, kSplit, kOne };
constexpr uint32_t kNone = 0xffffffffu;          // not published yet

struct View {
    char *p;
    int64_t ss, ts;  // bytes
};

struct RecArgs {
    View v, f, o, y;        // y: forward
    View dy, dv, df, dO;    // backward
    int32_t n, L;
    int64_t C;
    const int32_t *lengths;
    const float *h0;        // forward, or null
    float *h_last;          // forward
    float *states;          // kept states [n, ceil(L / kEvery), C]: written (or null) forward, read backward
    const float *dh_last;   // backward, or null
    float *dh0;             // backward
    uint64_t *maps;         // [rows, tiles, 64], split
    uint32_t *reached;      // [rows, ceil(tiles / kGroup), 64]: states, split
    uint32_t *taken;        // [rows][kApart]: tiles taken, less one, split
    int32_t blocks;         // channel blocks
    int32_t lanes;          // lanes over channels, a power of two
    int32_t waves;          // wavefronts of a workgroup
    int32_t tiles;          // tiles of a row
};

template <int DT>
constexpr int kRun = kElems / Elem<DT>::kPerWord;  // steps of one thread in a tile

// A gate that keeps the state: S = 1 and 1 - S = 0 to the bit.
template <int DT>
constexpr uint32_t kKeep = DT == ROCKET_FLOAT32 ? 0x7f800000u : DT == ROCKET_BFLOAT16 ? 0x7f807f80u : 0x7c007c00u;

// Where a thread works.
struct Place {
    uint32_t i, len;  // series, its steps
    uint32_t row, tile;   // row; steps of a tile
    int c, c_ld;      // first channel, and the channel it loads from
    int wave, lane, cl, run;
    int count;        // channels it owns: 0, 1 or 2
    bool high;        // its one channel is the high half of the word at c_ld
    bool single;      // C == 1 and 16-bit elements: no whole word to load
};

template <int DT>
__device__ inline Place place_of(const RecArgs &a) {
    constexpr int P = Elem<DT>::kPerWord;
    Place p;
    const uint32_t b = rocket::item_of_block();
    p.row = rocket::uniform(b % ((uint32_t)a.n * a.blocks));
    p.i = rocket::uniform(p.row / a.blocks);
    const int cb = (int)(p.row - p.i * a.blocks);
    p.wave = rocket::uniform(threadIdx.x >> 6);
    p.lane = threadIdx.x & 63;
    const int runs = 64 / a.lanes;
    p.cl = p.lane & (a.lanes - 1);
    p.run = p.wave * runs + p.lane / a.lanes;
    p.tile = (uint32_t)a.waves * runs * kRun<DT>;
    p.c = (cb * a.lanes + p.cl) * P;
    const int C = (int)a.C, left = C - p.c;
    p.count = left <= 0 ? 0 : left < P ? 1 : P;
    p.high = P == 2 && p.count == 1 && C > 1;
    p.single = P == 2 && C == 1;
    p.c_ld = p.c + P <= C ? p.c : C > P ? C - P : 0;
    p.len = rocket::steps_of(a.lengths, p.i, a.L);
    return p;
}

// The words of a run from step t0; steps past the series' length get `fill`.
template <int DT>
__device__ inline void load_run(const View &x, const Place &p, uint32_t t0, uint32_t fill, uint32_t (&w)[kRun<DT>]) {
    using raw = typename Elem<DT>::raw;
    const char *at = x.p + p.i * x.ss + t0 * x.ts + (int64_t)p.c_ld * Elem<DT>::kSize;
    if (p.single) {
#pragma unroll
        for (int s = 0; s < kRun<DT>; s++) w[s] = t0 + s < p.len ? (uint32_t)*(const raw *)(at + s * x.ts) : fill;
    } else if (t0 + kRun<DT> <= p.len) {
#pragma unroll
        for (int s = 0; s < kRun<DT>; s++) w[s] = rocket::load_at<uint32_t>(at + s * x.ts);
    } else {
#pragma unroll
        for (int s = 0; s < kRun<DT>; s++) w[s] = t0 + s < p.len ? rocket::load_at<uint32_t>(at + s * x.ts) : fill;
    }
    if (p.high) {
#pragma unroll
        for (int s = 0; s < kRun<DT>; s++) w[s] = t0 + s < p.len ? w[s] >> 16 : fill;
    }
}

// Whether a run's stores need no checks: whole words, all steps inside.
template <int DT>
__device__ inline bool whole_run(const Place &p, uint32_t t0, uint32_t L) {
    return p.count == Elem<DT>::kPerWord && t0 + kRun<DT> <= L;
}

// Writes the packed word of step t of a run that starts at `at`, checked
// unless the run is whole.
template <int DT, bool WHOLE>
__device__ inline void store_step(char *at, int64_t stride, const Place &p, int s, uint32_t left, uint32_t w) {
    using raw = typename Elem<DT>::raw;
    if (WHOLE)
        rocket::store_at(at + s * stride, w);
    else if ((uint32_t)s < left && p.count == Elem<DT>::kPerWord)
        rocket::store_at(at + s * stride, w);
    else if ((uint32_t)s < left && p.count == 1)
        *(raw *)(at + s * stride) = (raw)w;
}

template <int DT>
__device__ inline char *run_at(const View &x, const Place &p, uint32_t t0) {
    return x.p + p.i * x.ss + t0 * x.ts + (int64_t)p.c * Elem<DT>::kSize;
}

// Shared memory of one scan over the wavefronts of a workgroup.
template <int WAY>
struct Scan {
    static constexpr int kWaves = WAY == kOne ? kMostWaves : kTileWaves;
    float2 map[kWaves][kMostChannels];
    float start[kWaves][kMostChannels];
};

// Inclusive scan of the runs' maps over the lanes of a wavefront, then
// (A, B) becomes the map of the runs before the thread's own (REVERSE: after
// it), and the wavefront's whole map goes to shared memory.
template <int P, bool REVERSE, int WAY>
__device__ inline void scan_lanes(const RecArgs &a, const Place &p, float *A, float *B, Scan<WAY> &s) {
    for (int off = a.lanes; off < 64; off *= 2) {
        const bool on = REVERSE ? p.lane + off < 64 : p.lane >= off;
#pragma unroll
        for (int j = 0; j < P; j++) {
            const float pa = REVERSE ? __shfl_down(A[j], off) : __shfl_up(A[j], off);
            const float pb = REVERSE ? __shfl_down(B[j], off) : __shfl_up(B[j], off);
            B[j] = on ? __builtin_fmaf(A[j], pb, B[j]) : B[j];
            A[j] = on ? A[j] * pa : A[j];
        }
    }
    const bool first = REVERSE ? p.lane + a.lanes >= 64 : p.lane < a.lanes;   // nothing before it in its wavefront
    const bool last = REVERSE ? p.lane < a.lanes : p.lane + a.lanes >= 64;
    if (last) {
#pragma unroll
        for (int j = 0; j < P; j++) s.map[p.wave][p.cl * P + j] = make_float2(A[j], B[j]);
    }
#pragma unroll
    for (int j = 0; j < P; j++) {
        // always so (32 lanes at most); without the branch the compiler's order of
        // the loop costs 64 x 1000 x 512, fp32, gated, forward 6 % (108 us, not 102 us)
        float xa = A[j], xb = B[j];
        if (a.lanes < 64) {
            xa = REVERSE ? __shfl_down(A[j], a.lanes) : __shfl_up(A[j], a.lanes);
            xb = REVERSE ? __shfl_down(B[j], a.lanes) : __shfl_up(B[j], a.lanes);
        }
        A[j] = first ? 1.0f : xa;
        B[j] = first ? 0.0f : xb;
    }
}

// One thread per channel goes through the wavefronts' maps: the state at each
// wavefront's start, and in `carry` the state past the tile.
template <bool REVERSE, int WAY>
__device__ inline void scan_waves(int waves, int ch, float &carry, Scan<WAY> &s) {
    for (int k = 0; k < waves; k++) {
        const int w = REVERSE ? waves - 1 - k : k;
        const float2 m = s.map[w][ch];
        s.start[w][ch] = carry;
        carry = __builtin_fmaf(m.x, carry, m.y);
    }
}

// What a split row's tiles publish.
struct Meet {
    float2 map[kTileWaves][kMostChannels];
    int tile;
};

__device__ inline uint32_t published(float x) {
    const uint32_t w = __builtin_bit_cast(uint32_t, x);
    return w == kNone ? 0x7fc00000u : w;   // a NaN that is not the pattern
}

// The row's next tile.
__device__ inline int take_tile(const RecArgs &a, const Place &p, Meet &m) {
    if (threadIdx.x == 0)
        m.tile = (int)(__hip_atomic_fetch_add(a.taken + (int64_t)p.row * kApart, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1u);
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(m.tile);
}

// After the wavefronts' maps are in s.map: publishes the map of the row's
// order-th tile, waits for those before it back to the last published state,
// and returns, in the threads that scan, the state at the tile's start.  The
// whole workgroup calls it.
template <int P, bool REVERSE>
__device__ inline float meet(const RecArgs &a, const Place &p, int order, bool scans, float h, const Scan<kSplit> &s, Meet &m) {
    uint64_t *row = a.maps + (int64_t)p.row * a.tiles * kMostChannels;
    const int ch = threadIdx.x, channels = a.lanes * P;   // channels that are published
    if (scans) {
        float A = 1.0f, B = 0.0f;
        for (int k = 0; k < a.waves; k++) {
            const float2 x = s.map[REVERSE ? a.waves - 1 - k : k][ch];
            B = __builtin_fmaf(x.x, B, x.y);
            A *= x.x;
        }
        __hip_atomic_store(row + (int64_t)order * kMostChannels + ch,
                           (uint64_t)published(A) | (uint64_t)__builtin_bit_cast(uint32_t, B) << 32,
                           __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    asm volatile("" ::: "memory");   // published before anything is waited for
    const int from = order / kGroup * kGroup, before = order - from;
    {
        // each wavefront composes a range of the maps, four on their way at once
        float A = 1.0f, B = 0.0f;
        const int lo = from + before * p.wave / a.waves, hi = from + before * (p.wave + 1) / a.waves;
        if (p.lane < channels) {
            for (int k = lo; k < hi; k += 4) {
                uint64_t w[4];
#pragma unroll
                for (int j = 0; j < 4; j++)
                    if (k + j < hi)
                        w[j] = __hip_atomic_load(row + (int64_t)(k + j) * kMostChannels + p.lane, __ATOMIC_RELAXED,
                                                 __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
                for (int j = 0; j < 4; j++)
                    if (k + j < hi) {
                        while ((uint32_t)w[j] == kNone) {
                            __builtin_amdgcn_s_sleep(1);
                            w[j] = __hip_atomic_load(row + (int64_t)(k + j) * kMostChannels + p.lane,
                                                     __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                        }
                        const float x = __builtin_bit_cast(float, (uint32_t)w[j]);
                        B = __builtin_fmaf(x, B, __builtin_bit_cast(float, (uint32_t)(w[j] >> 32)));
                        A *= x;
                    }
            }
            m.map[p.wave][p.lane] = make_float2(A, B);
        }
    }
    __syncthreads();
    if (scans) {
        if (from > 0) {
            const uint32_t *at = a.reached + ((int64_t)p.row * ((a.tiles + kGroup - 1) / kGroup) + from / kGroup) *
                                                 kMostChannels + ch;
            uint32_t w;
            while ((w = __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) == kNone)
                __builtin_amdgcn_s_sleep(1);
            h = __builtin_bit_cast(float, w);
        }
        for (int w = 0; w < a.waves; w++) {
            const float2 x = m.map[w][ch];
            h = __builtin_fmaf(x.x, h, x.y);
        }
    }
    return h;
}

// Publishes the state behind the order-th tile where a later tile starts from it.
__device__ inline void reach(const RecArgs &a, const Place &p, int order, float h) {
    if ((order + 1) % kGroup == 0 && order + 1 < a.tiles)
        __hip_atomic_store(a.reached + ((int64_t)p.row * ((a.tiles + kGroup - 1) / kGroup) + (order + 1) / kGroup) *
                                           kMostChannels + threadIdx.x,
                           published(h), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The forward pass over a row, or over one tile of it.
template <int DT, int WAY, bool GATE>
__global__ __launch_bounds__(64 * (WAY == kOne ? kMostWaves : kTileWaves), WAY == kSplit && !GATE ? 8 : 4) void forward_kernel(RecArgs a) {
    constexpr int P = Elem<DT>::kPerWord, S = kRun<DT>;
    constexpr bool SPLIT = WAY == kSplit;
    __shared__ Scan<WAY> scan;
    __shared__ typename std::conditional<SPLIT, Meet, int>::type met;
    Place p = place_of<DT>(a);
    const bool scans = threadIdx.x < a.lanes * P;   // the threads that go through the wavefronts, one a channel
    const int64_t ch = (p.c - p.cl * P) + (int)threadIdx.x, per = ((int64_t)a.L + kEvery - 1) / kEvery;
    const uint32_t L = a.L;
    float carry = scans && ch < a.C && a.h0 ? a.h0[p.i * a.C + ch] : 0.0f;
    int k = 0;
    if constexpr (SPLIT) k = take_tile(a, p, met);
    uint32_t wv[S], wf[S], wo[S];
    auto load = [&](uint32_t t0) {
        load_run<DT>(a.v, p, t0, 0, wv);
        load_run<DT>(a.f, p, t0, kKeep<DT>, wf);
        if (GATE) load_run<DT>(a.o, p, t0, 0, wo);
    };
    load(k * p.tile + p.run * S);

    for (;; k++) {
        // as if new: what follows from them is not kept across tiles
        if (WAY == kLoop) {
            asm("" : "+v"(p.c), "+v"(p.c_ld), "+v"(p.run), "+v"(p.cl), "+v"(p.lane), "+s"(p.i));
            asm("" : "+s"(a.v.ts), "+s"(a.f.ts), "+s"(a.o.ts), "+s"(a.y.ts));
        }
        const uint32_t t0 = k * p.tile + p.run * S;
        const bool live = k * p.tile + p.wave * (64 / a.lanes) * S < p.len;   // of the wavefront
        float fa[S][P], fb[S][P], A[P], B[P];
#pragma unroll
        for (int j = 0; j < P; j++) A[j] = 1.0f, B[j] = 0.0f;
        if (live) {
#pragma unroll
            for (int s = 0; s < S; s++)
#pragma unroll
                for (int j = 0; j < P; j++) {
                    float in;
                    rocket::logistic<DT, true>(Elem<DT>::get(wf[s], j), fa[s][j], in);
                    fb[s][j] = in * Elem<DT>::get(wv[s], j);
                    B[j] = __builtin_fmaf(fa[s][j], B[j], fb[s][j]);
                    A[j] *= fa[s][j];
                }
        } else {
#pragma unroll
            for (int s = 0; s < S; s++)
#pragma unroll
                for (int j = 0; j < P; j++) fa[s][j] = 1.0f, fb[s][j] = 0.0f;
        }
        uint32_t go[S];   // the next tile's words go over these
        if (GATE) {
#pragma unroll
            for (int s = 0; s < S; s++) go[s] = wo[s];
        }
        if (WAY == kLoop && k + 1 < a.tiles) load(t0 + p.tile);   // on their way during the scan
        scan_lanes<P, false>(a, p, A, B, scan);
        __syncthreads();
        if constexpr (SPLIT) carry = meet<P, false>(a, p, k, scans, carry, scan, met);
        if (scans) scan_waves<false>(a.waves, threadIdx.x, carry, scan);
        if (SPLIT && scans) reach(a, p, k, carry);
        __syncthreads();
        float h[P];
#pragma unroll
        for (int j = 0; j < P; j++) h[j] = __builtin_fmaf(A[j], scan.start[p.wave][p.cl * P + j], B[j]);
        if (a.states && t0 % kEvery == 0 && t0 < L)
#pragma unroll
            for (int j = 0; j < P; j++)
                if (j < p.count) a.states[(p.i * per + t0 / kEvery) * a.C + p.c + j] = h[j];
        char *at = run_at<DT>(a.y, p, t0);
        const uint32_t left = t0 < L ? L - t0 : 0;
        auto steps = [&](auto whole) {
#pragma unroll
            for (int s = 0; s < S; s++) {
                float out[P];
#pragma unroll
                for (int j = 0; j < P; j++) {
                    h[j] = __builtin_fmaf(fa[s][j], h[j], fb[s][j]);
                    out[j] = h[j];
                    if (GATE) {
                        float so, rest;
                        rocket::logistic<DT>(Elem<DT>::get(go[s], j), so, rest);
                        out[j] *= so;
                    }
                }
                store_step<DT, whole.value>(at, a.y.ts, p, s, left, t0 + s < p.len ? Elem<DT>::put(out) : 0);
            }
        };
        if (!live) {
#pragma unroll
            for (int s = 0; s < S; s++) store_step<DT, false>(at, a.y.ts, p, s, left, 0);
        } else if (whole_run<DT>(p, t0, L)) {
            steps(std::true_type());
        } else {
            steps(std::false_type());
        }
        if (WAY != kLoop || k + 1 == a.tiles) break;
    }
    if (k == a.tiles - 1 && scans && ch < a.C) a.h_last[p.i * a.C + ch] = carry;
}

// The backward pass over a row from its last tile to its first, or over one
// tile of it.
template <int DT, int WAY, bool GATE>
__global__ __launch_bounds__(64 * (WAY == kOne ? kMostWaves : kTileWaves), 4) void backward_kernel(RecArgs a) {
    constexpr int P = Elem<DT>::kPerWord, S = kRun<DT>;
    constexpr bool SPLIT = WAY == kSplit;
    __shared__ Scan<WAY> scan, fscan;
    __shared__ typename std::conditional<SPLIT, Meet, int>::type met;
    Place p = place_of<DT>(a);
    const int channels = a.lanes * P;
    const bool scans = threadIdx.x < channels;                    // the threads that go through the gradients' maps
    const int other = a.waves > 1 ? 64 : 0;                       // and those that go through the states'
    const bool fscans = (int)threadIdx.x >= other && (int)threadIdx.x < other + channels;
    const int64_t c0 = p.c - p.cl * P, ch = c0 + threadIdx.x, fch = c0 + threadIdx.x - other;
    const int64_t per = ((int64_t)a.L + kEvery - 1) / kEvery;
    const uint32_t L = a.L;
    float carry = scans && ch < a.C && a.dh_last ? a.dh_last[p.i * a.C + ch] : 0.0f;
    int order = 0;
    if constexpr (SPLIT) order = take_tile(a, p, met);
    for (;; order++) {
        // as if new: what follows from them is not kept across tiles
        if (WAY == kLoop) {
            asm("" : "+v"(p.c), "+v"(p.c_ld), "+v"(p.run), "+v"(p.cl), "+v"(p.lane), "+s"(p.i));
            asm("" : "+s"(a.v.ts), "+s"(a.f.ts), "+s"(a.o.ts), "+s"(a.dy.ts));
            asm("" : "+s"(a.dv.ts), "+s"(a.df.ts), "+s"(a.dO.ts));
        }
        const uint32_t tile0 = (uint32_t)(a.tiles - 1 - order) * p.tile, t0 = tile0 + p.run * S;
        const bool live = tile0 + p.wave * (64 / a.lanes) * S < p.len;   // of the wavefront
        uint32_t wv[S], wf[S], wo[S], wg[S];
        load_run<DT>(a.f, p, t0, kKeep<DT>, wf);
        load_run<DT>(a.dy, p, t0, 0, wg);
        if (GATE) load_run<DT>(a.o, p, t0, 0, wo);
        load_run<DT>(a.v, p, t0, 0, wv);
        float state = 0.0f;
        if (fscans && tile0 < L && fch < a.C) state = a.states[(p.i * per + tile0 / kEvery) * a.C + fch];

        float fa[S][P], in[S][P], A[P], R[P], FA[P], B[P];
#pragma unroll
        for (int j = 0; j < P; j++) A[j] = 1.0f, R[j] = 0.0f, B[j] = 0.0f;
        if (live) {
#pragma unroll
            for (int s = S - 1; s >= 0; s--)
#pragma unroll
                for (int j = 0; j < P; j++) {
                    float so = 1.0f, rest;
                    rocket::logistic<DT, true>(Elem<DT>::get(wf[s], j), fa[s][j], in[s][j]);
                    if (GATE) rocket::logistic<DT>(Elem<DT>::get(wo[s], j), so, rest);
                    const float g = GATE ? Elem<DT>::get(wg[s], j) * so : Elem<DT>::get(wg[s], j);
                    R[j] = fa[s][j] * (R[j] + g);
                    B[j] = __builtin_fmaf(A[j], in[s][j] * Elem<DT>::get(wv[s], j), B[j]);
                    A[j] *= fa[s][j];
                }
        } else {
#pragma unroll
            for (int s = 0; s < S; s++)
#pragma unroll
                for (int j = 0; j < P; j++) fa[s][j] = 1.0f, in[s][j] = 0.0f;
        }
#pragma unroll
        for (int j = 0; j < P; j++) FA[j] = A[j];
        scan_lanes<P, true>(a, p, A, R, scan);
        scan_lanes<P, false>(a, p, FA, B, fscan);
        __syncthreads();
        if (fscans) scan_waves<false>(a.waves, (int)threadIdx.x - other, state, fscan);
        if constexpr (SPLIT) carry = meet<P, true>(a, p, order, scans, carry, scan, met);
        if (scans) scan_waves<true>(a.waves, threadIdx.x, carry, scan);
        if (SPLIT && scans) reach(a, p, order, carry);
        __syncthreads();

        rocket::renew(wv);
        rocket::renew(wg);
        if (GATE) rocket::renew(wo);
        char *at_v = run_at<DT>(a.dv, p, t0), *at_f = run_at<DT>(a.df, p, t0);
        const uint32_t left = t0 < L ? L - t0 : 0;
        char *at_o = GATE ? run_at<DT>(a.dO, p, t0) : nullptr;
        auto store = [&](auto whole, int s, uint32_t gv, uint32_t gf, uint32_t go) {
            store_step<DT, whole.value>(at_v, a.dv.ts, p, s, left, gv);
            store_step<DT, whole.value>(at_f, a.df.ts, p, s, left, gf);
            if (GATE) store_step<DT, whole.value>(at_o, a.dO.ts, p, s, left, go);
        };
        auto steps = [&](auto whole) {
            float h[S][P], e[P];   // the state before each step
#pragma unroll
            for (int j = 0; j < P; j++) {
                const int at = p.cl * P + j;
                e[j] = __builtin_fmaf(A[j], scan.start[p.wave][at], R[j]);
                h[0][j] = __builtin_fmaf(FA[j], fscan.start[p.wave][at], B[j]);
            }
#pragma unroll
            for (int s = 0; s + 1 < S; s++)
#pragma unroll
                for (int j = 0; j < P; j++)
                    h[s + 1][j] = __builtin_fmaf(fa[s][j], h[s][j], in[s][j] * Elem<DT>::get(wv[s], j));
#pragma unroll
            for (int s = S - 1; s >= 0; s--) {
                float xv[P], xf[P], xo[P];
#pragma unroll
                for (int j = 0; j < P; j++) {
                    float so = 1.0f, rest = 0.0f;
                    if (GATE) rocket::logistic<DT>(Elem<DT>::get(wo[s], j), so, rest);
                    const float v = Elem<DT>::get(wv[s], j), dy = Elem<DT>::get(wg[s], j);
                    const float dh = GATE ? __builtin_fmaf(dy, so, e[j]) : dy + e[j];
                    xv[j] = dh * in[s][j];
                    xf[j] = xv[j] * (h[s][j] - v) * fa[s][j];
                    if (GATE) xo[j] = dy * __builtin_fmaf(fa[s][j], h[s][j], in[s][j] * v) * so * rest;
                    e[j] = fa[s][j] * dh;
                }
                const bool own = t0 + s < p.len;
                store(whole, s, own ? Elem<DT>::put(xv) : 0, own ? Elem<DT>::put(xf) : 0,
                      GATE && own ? Elem<DT>::put(xo) : 0);
            }
        };
        if (!live) {
#pragma unroll
            for (int s = 0; s < S; s++) store(std::false_type(), s, 0, 0, 0);
        } else if (whole_run<DT>(p, t0, L)) {
            steps(std::true_type());
        } else {
            steps(std::false_type());
        }
        if (WAY != kLoop || order + 1 == a.tiles) break;
    }
    if (order == a.tiles - 1 && scans && ch < a.C) a.dh0[p.i * a.C + ch] = carry;
}

// Nothing is published yet, and no tile taken.
__global__ __launch_bounds__(256) void clear_kernel(uint64_t *p, int64_t words) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < words) p[i] = ~0ull;
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
        rocket::logistic<DT, true>(Elem<DT>::get(wf, j), keep, in);
        h[j] = __builtin_fmaf(keep, h[j], in * Elem<DT>::get(wv, j));
        y[j] = h[j];
        if (GATE) {
            float so, rest;
            rocket::logistic<DT>(Elem<DT>::get(wo, j), so, rest);
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
    int32_t lanes, waves, blocks, tiles;
    bool split;
    int64_t series, rows;   // of a launch
};

// 8-byte words of a split launch's maps, published states and counters.
int64_t map_words(const Cut &c) { return c.rows * c.tiles * kMostChannels; }
int64_t reached_words(const Cut &c) { return c.rows * ((c.tiles + kGroup - 1) / kGroup) * (kMostChannels / 2); }
int64_t workspace_words(const Cut &c) { return c.split ? map_words(c) + reached_words(c) + c.rows * (kApart / 2) : 0; }
int64_t workspace_of(const Cut &c) { return workspace_words(c) * 8; }

// Lanes over channels: the power of two that covers the words of channels, 32
// at most; the wavefront's other lanes take further runs of steps, so that
// few channels do not leave lanes idle.
//
// A series that is not much longer than a tile is one larger tile (777 x 129 x
// 331, fp16, gated, ragged: 67 us, against 92 us in two tiles): of up to 16
// wavefronts where rows are few (50 x 200 x 256: 10 us, split 16 us) and in the
// forward pass of 16-bit elements (1000 x 190 x 256: 72 against 89 us), 10 in
// its gated backward pass (1000 x 160 x 256: 154 against 182 us; of 12, 248
// against 243 us) and 8 else (fp32, 13 wavefronts, 1000 x 400 x 128, backward:
// 232 against 214 us).
//
// Split where rows alone do not fill the chip (8 x 10000 x 256, fp32, backward:
// 90 us, against 140 us with a first launch for the maps), and for three kinds
// of calls whose loop over tiles leaves more to be waited for than tiles that
// meet cost: long rows that fill it badly at last (600 rows of 4,000 steps,
// bf16: 187 us against 231 us; 1,000 rows: 83 against 86 us forward, 87 against
// 75 us backward); fp32 rows of 8 tiles and more (1000 x 1000 x 256, backward:
// 945 us against 1027 us; 256 x 300 x 512, 3 tiles: 188 against 167 us); and the
// gated backward pass of 16-bit elements, short of registers in its loop, where
// the tiles are mostly full (1000 x 1000 x 256: 788 us against 904 us; 1000 x
// 129 x 256, a last tile of one step: 197 against 173 us).
void cut_of(const rocket_sequence_shape *s, bool back, bool gate, Cut *cut) {
    const int64_t per_word = rocket::elem_size(s->dtype) == 4 ? 1 : 2;
    const int64_t words = (s->channels + per_word - 1) / per_word;
    cut->lanes = 1;
    while (cut->lanes < kMostLanes && cut->lanes < words) cut->lanes *= 2;
    const int64_t in_wave = (64 / cut->lanes) * (kElems / per_word);   // steps of a wavefront
    const int64_t L = s->steps > 0 ? s->steps : 1;
    cut->waves = (int32_t)(in_wave < kEvery ? kEvery / in_wave : 1);
    cut->blocks = (int32_t)((words + cut->lanes - 1) / cut->lanes);
    const int64_t rows = s->n * cut->blocks;
    // One tile holds the series.
    const int64_t one = (L + in_wave - 1) / in_wave;
    const int most = rows < kFill || (per_word == 2 && !back) ? kMostWaves : per_word == 2 && gate ? 10 : kTileWaves;
    if (one <= most) cut->waves = (int32_t)one;
    const int64_t tile = cut->waves * in_wave;
    cut->tiles = (int32_t)((L + tile - 1) / tile);
    const int64_t slots = (rows + kFill - 1) / kFill * kFill;   // of a loop, whole waves of workgroups
    cut->split = cut->tiles > 1 &&
                 (rows < kFill || (cut->tiles >= 8 && rows < 4 * kFill && 4 * rows < 3 * slots) ||
                  (per_word == 1 && cut->tiles >= 8) ||
                  (per_word == 2 && back && gate && 4 * L >= 3 * tile * cut->tiles));
    // Series of a launch: as many as its threads allow, and those of the launch
    // that clears the workspace (a word each).  A series whose tiles are too many
    // for one launch is not split.
    const int64_t limit = rocket::most_groups(256) * 256;
    cut->rows = cut->blocks;
    int64_t each = std::max<int64_t>((int64_t)cut->blocks * cut->tiles * 64 * cut->waves, workspace_words(*cut));
    cut->split = cut->split && each <= limit;
    if (!cut->split) each = (int64_t)cut->blocks * 64 * cut->waves;
    cut->series = std::min(std::max<int64_t>(s->n, 1), limit / each);
    cut->rows = cut->series * cut->blocks;
}

void set_cut(RecArgs &a, const Cut &c, void *workspace) {
    a.blocks = c.blocks, a.lanes = c.lanes, a.waves = c.waves, a.tiles = c.tiles;
    a.maps = (uint64_t *)workspace;
    if (c.split) {
        a.reached = (uint32_t *)(a.maps + map_words(c));
        a.taken = (uint32_t *)(a.maps + map_words(c) + reached_words(c));
    }
}

void clear(const RecArgs &a, const Cut &c, hipStream_t s) {
    const int64_t words = workspace_words(c);
    clear_kernel<<<(uint32_t)((words + 255) / 256), 256, 0, s>>>(a.maps, words);
}

View view(const rocket_sequence *q, int size) {
    return q ? View{(char *)q->data, q->series_stride * size, q->step_stride * size} : View{nullptr, 0, 0};
}

bool aligned(const void *p, uintptr_t to) { return (uintptr_t)p % to == 0; }

// The call's series from i on, as many as a launch takes.
RecArgs part_of(RecArgs a, const Cut &cut, int64_t i) {
    a.n = (int32_t)std::min<int64_t>(cut.series, a.n - i);
    for (View *x : {&a.v, &a.f, &a.o, &a.y, &a.dy, &a.dv, &a.df, &a.dO})
        if (x->p) x->p += i * x->ss;
    if (a.lengths) a.lengths += i;
    for (const float **x : {&a.h0, &a.dh_last})
        if (*x) *x += i * a.C;
    for (float **x : {&a.h_last, &a.dh0})
        if (*x) *x += i * a.C;
    if (a.states) a.states += i * (((int64_t)a.L + kEvery - 1) / kEvery) * a.C;
    return a;
}

template <int DT, bool GATE>
void run_forward(const RecArgs &call, const Cut &cut, hipStream_t s) {
    for (int64_t i = 0; i < call.n; i += cut.series) {
        const RecArgs a = part_of(call, cut, i);
        const uint32_t rows = (uint32_t)a.n * a.blocks, threads = 64 * cut.waves;
        if (cut.split) {
            clear(a, cut, s);
            forward_kernel<DT, kSplit, GATE><<<rows * cut.tiles, threads, 0, s>>>(a);
        } else if (cut.tiles > 1) {
            forward_kernel<DT, kLoop, GATE><<<rows, threads, 0, s>>>(a);
        } else {
            forward_kernel<DT, kOne, GATE><<<rows, threads, 0, s>>>(a);
        }
    }
}

template <int DT, bool GATE>
void run_backward(const RecArgs &call, const Cut &cut, hipStream_t s) {
    for (int64_t i = 0; i < call.n; i += cut.series) {
        const RecArgs a = part_of(call, cut, i);
        const uint32_t rows = (uint32_t)a.n * a.blocks, threads = 64 * cut.waves;
        if (cut.split) {
            clear(a, cut, s);
            backward_kernel<DT, kSplit, GATE><<<rows * cut.tiles, threads, 0, s>>>(a);
        } else if (cut.tiles > 1) {
            backward_kernel<DT, kLoop, GATE><<<rows, threads, 0, s>>>(a);
        } else {
            backward_kernel<DT, kOne, GATE><<<rows, threads, 0, s>>>(a);
        }
    }
}

template <int DT, bool GATE>
void run_step(StepArgs a, hipStream_t s) {
    const int64_t n = a.n, most = rocket::most_groups(256) * 256 / a.words;   // series of a launch
    for (int64_t i = 0; i < n; i += most) {
        a.n = std::min(most, n - i);
        step_kernel<DT, GATE><<<(uint32_t)((a.n * a.words + 255) / 256), 256, 0, s>>>(a);
        a.v += most * a.vs, a.f += most * a.fs, a.y += most * a.ys;
        if (GATE) a.o += most * a.os;
        a.h_in += most * a.C, a.h_out += most * a.C;
    }
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
    if (!bytes || !rocket::shape_ok(shape)) return ROCKET_ERR_INVALID_ARG;
    int64_t most = 0;
    for (int k = 0; k < 4; k++) {   // either pass, gated or not
        Cut cut;
        cut_of(shape, k & 1, k & 2, &cut);
        if (workspace_of(cut) > most) most = workspace_of(cut);
    }
    *bytes = most;
    return ROCKET_OK;
}

extern "C" rocket_status rocket_recurrence_forward(const rocket_sequence_shape *shape, const rocket_sequence *v,
                                                   const rocket_sequence *f, const rocket_sequence *o, const float *h0,
                                                   const rocket_sequence *y, float *h_last, float *states,
                                                   void *workspace, int64_t workspace_bytes, void *hip_stream) {
    if (!rocket::shape_ok(shape) || !rocket::view_ok(v, shape) || !rocket::view_ok(f, shape) ||
        (o && !rocket::view_ok(o, shape)) || !rocket::out_ok(y, shape) || (shape->n > 0 && !h_last))
        return ROCKET_ERR_INVALID_ARG;
    Cut cut;
    cut_of(shape, false, o != nullptr, &cut);
    const int64_t need = workspace_of(cut);
    if (workspace_bytes < need || (need && (!workspace || !aligned(workspace, 8)))) return ROCKET_ERR_INVALID_ARG;
    if (!aligned(h0, 4) || !aligned(h_last, 4) || !aligned(states, 4) || !aligned(shape->lengths, 4))
        return ROCKET_ERR_INVALID_ARG;
    if (shape->n == 0) return ROCKET_OK;
    const int size = rocket::elem_size(shape->dtype);
    RecArgs a = {};
    a.v = view(v, size), a.f = view(f, size), a.o = view(o, size), a.y = view(y, size);
    a.n = (int32_t)shape->n, a.L = (int32_t)shape->steps, a.C = shape->channels, a.lengths = shape->lengths;
    a.h0 = h0, a.h_last = h_last, a.states = states;
    set_cut(a, cut, workspace);
    BY_TYPE(run_forward, shape->dtype, o != nullptr, a, cut, (hipStream_t)hip_stream);
    return rocket::launched();
}

extern "C" rocket_status rocket_recurrence_backward(const rocket_sequence_shape *shape, const rocket_sequence *dy,
                                                    const rocket_sequence *v, const rocket_sequence *f,
                                                    const rocket_sequence *o, const float *states,
                                                    const float *dh_last, const rocket_sequence *dv,
                                                    const rocket_sequence *df, const rocket_sequence *dO, float *dh0,
                                                    void *workspace, int64_t workspace_bytes, void *hip_stream) {
    if (!rocket::shape_ok(shape) || !rocket::view_ok(dy, shape) ||
        !rocket::view_ok(v, shape) || !rocket::view_ok(f, shape) || (o && !rocket::view_ok(o, shape)) ||
        !rocket::out_ok(dv, shape) || !rocket::out_ok(df, shape) || (o != nullptr) != (dO != nullptr) ||
        (dO && !rocket::out_ok(dO, shape)) || (shape->n > 0 && !dh0) || (!rocket::empty(shape) && !states))
        return ROCKET_ERR_INVALID_ARG;
    Cut cut;
    cut_of(shape, true, o != nullptr, &cut);
    const int64_t need = workspace_of(cut);
    if (workspace_bytes < need || (need && (!workspace || !aligned(workspace, 8)))) return ROCKET_ERR_INVALID_ARG;
    if (!aligned(states, 4) || !aligned(dh_last, 4) || !aligned(dh0, 4) || !aligned(shape->lengths, 4))
        return ROCKET_ERR_INVALID_ARG;
    if (shape->n == 0) return ROCKET_OK;
    const int size = rocket::elem_size(shape->dtype);
    RecArgs a = {};
    a.v = view(v, size), a.f = view(f, size), a.o = view(o, size);
    a.dy = view(dy, size), a.dv = view(dv, size), a.df = view(df, size), a.dO = view(dO, size);
    a.n = (int32_t)shape->n, a.L = (int32_t)shape->steps, a.C = shape->channels, a.lengths = shape->lengths;
    a.states = const_cast<float *>(states), a.dh_last = dh_last, a.dh0 = dh0;
    set_cut(a, cut, workspace);
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
    BY_TYPE(run_step, dtype, o != nullptr, a, (hipStream_t)hip_stream);
    return rocket::launched();
}
