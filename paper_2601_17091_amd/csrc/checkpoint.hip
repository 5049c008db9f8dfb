// Checkpoints in 8 bits: rows of a sequence kept for the backward pass, and
// restored.
//
//   block b: rows 128 b .. 128 b + 127 of all series' steps in a row
//   a = max |x[t, c]| over the block,  scale[b, c] = a / 127
//   q[b, c, t - 128 b] = rint(x[t, c] 127 / a);  restored: q scale
//
// A scale for each channel and not for each row: features differ in level from
// channel to channel (a proportion beside a maximum), and a gradient of weights
// sums over rows, so that a channel's scale is a factor of the whole block's sum
// (weight_gradient.hip).  The rows of a channel lie side by side, as that sum
// reads them.
//
// Bound: HBM.  A workgroup takes 64 channels of a block: a thread 4 channels of
// 8 rows in registers (read once), the largest of each channel and the turn from
// rows to channels through shared memory.  64 x 1000 x 2000: fp32 kept in 137 us (640
// MB, 4.7 TB/s), restored to bf16 in 80 (384 MB, 4.8 TB/s); a copy runs at 5.3 TB/s.
#include <algorithm>

#include "rows.h"

namespace {

using rocket::Elem;
using rocket::kKeepRows;
using rocket::Place;
using rocket::Rows;
using rocket::View;

constexpr int kThreads = 256, kChannels = 64, kQuads = kChannels / 4, kBands = kThreads / kQuads;
constexpr int kRow = kKeepRows + 4;   // bytes of a channel in shared memory: words of neighbours in other banks

struct KeepArgs {
    Rows rows;
    View x;
    int8_t *q;
    float *scale;
    int32_t channels;
    int32_t tiles;   // of 64 channels
    int64_t first;   // the launch's first item
};

// Four channels of a row from column c on, as they are kept in memory.
template <int DT>
__device__ inline void load4(const char *row, int c, int channels, float (&f)[4]) {
    using raw = typename Elem<DT>::raw;
    typedef uint32_t vec __attribute__((ext_vector_type(4 / Elem<DT>::kPerWord)));
    if (c + 4 <= channels) {
        const vec w = rocket::load_at<vec>(row + (int64_t)c * Elem<DT>::kSize);
#pragma unroll
        for (int e = 0; e < 4; e++) f[e] = Elem<DT>::get(w[e / Elem<DT>::kPerWord], e % Elem<DT>::kPerWord);
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; e++) f[e] = c + e < channels ? Elem<DT>::one(((const raw *)row)[c + e]) : 0.0f;
}

template <int DT>
__device__ inline void store4(char *row, int c, int channels, const float (&f)[4]) {
    using raw = typename Elem<DT>::raw;
    typedef uint32_t vec __attribute__((ext_vector_type(4 / Elem<DT>::kPerWord)));
    if (c + 4 <= channels) {
        vec w;
#pragma unroll
        for (int k = 0; k < 4 / Elem<DT>::kPerWord; k++) w[k] = Elem<DT>::put(f + k * Elem<DT>::kPerWord);
        rocket::store_at(row + (int64_t)c * Elem<DT>::kSize, w);
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; e++)
        if (c + e < channels) ((raw *)row)[c + e] = Elem<DT>::round(f[e]);
}

// Where the rows of a block lie: 0 where there is none, the lowest bit set where it holds
// no data.  A row's place takes a division, so a thread finds one for all.
__device__ inline void look_up(const KeepArgs &a, int64_t block, uint64_t *rows) {
    if (threadIdx.x < kKeepRows) {
        const int64_t r = block * kKeepRows + threadIdx.x;
        uint64_t at = 0;
        if (r < a.rows.count) {
            const Place p = rocket::place_of(a.rows, r);
            at = (uint64_t)rocket::row_at(a.x, p) | (p.live ? 0 : 1);
        }
        rows[threadIdx.x] = at;
    }
    __syncthreads();
}

// Item: a tile of 64 channels of a block.  Thread: quad (4 channels) and band
// (rows 4 band .. 4 band + 3 of both halves of the block).
template <int DT>
__global__ __launch_bounds__(kThreads) void keep_kernel(KeepArgs a) {
    __shared__ uint32_t tops[kBands][kChannels];
    __shared__ uint64_t rows[kKeepRows];
    __shared__ __attribute__((aligned(16))) uint8_t turned[kChannels * kRow];
    const int64_t item = a.first + rocket::item_of_block();
    const int64_t block = item / a.tiles;
    const int c0 = (int)(item - block * a.tiles) * kChannels, quad = threadIdx.x % kQuads, band = threadIdx.x / kQuads;
    const int c = c0 + 4 * quad;
    float f[8][4];
    uint32_t top[4] = {0, 0, 0, 0};
    look_up(a, block, rows);
#pragma unroll
    for (int k = 0; k < 8; k++) {
        const uint64_t at = rows[(k / 4) * 64 + 4 * band + k % 4];
        if (at != 0 && !(at & 1) && c < a.channels) {
            load4<DT>((const char *)at, c, a.channels, f[k]);
        } else {
#pragma unroll
            for (int e = 0; e < 4; e++) f[k][e] = 0.0f;
        }
    }
#pragma unroll
    for (int k = 0; k < 8; k++)
#pragma unroll
        for (int e = 0; e < 4; e++) top[e] = rocket::larger(top[e], rocket::magnitude(f[k][e]));
#pragma unroll
    for (int e = 0; e < 4; e++) tops[band][4 * quad + e] = top[e];
    __syncthreads();
    if (threadIdx.x < kChannels) {
        uint32_t t = 0;
#pragma unroll
        for (int b = 0; b < kBands; b++) t = rocket::larger(t, tops[b][threadIdx.x]);
        tops[0][threadIdx.x] = t;
        if (c0 + (int)threadIdx.x < a.channels) a.scale[block * a.channels + c0 + threadIdx.x] = rocket::step8(t);
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 4; e++) {
        const float inverse = rocket::inverse8(tops[0][4 * quad + e]);
#pragma unroll
        for (int h = 0; h < 2; h++)
            *(uint32_t *)(turned + (4 * quad + e) * kRow + h * 64 + 4 * band) =
                rocket::four8(f[4 * h][e], f[4 * h + 1][e], f[4 * h + 2][e], f[4 * h + 3][e], inverse);
    }
    __syncthreads();
    // a channel's 128 bytes by 8 threads of 16
    typedef uint32_t vec __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int k = 0; k < kChannels * 8 / kThreads; k++) {
        const int at = k * kThreads + threadIdx.x, ch = at / 8;
        if (c0 + ch >= a.channels) continue;
        const uint32_t *from = (const uint32_t *)(turned + ch * kRow + at % 8 * 16);
        const vec v = {from[0], from[1], from[2], from[3]};
        *(vec *)(a.q + (block * a.channels + c0 + ch) * kKeepRows + at % 8 * 16) = v;
    }
}

template <int DT>
__global__ __launch_bounds__(kThreads) void restore_kernel(KeepArgs a) {
    __shared__ __attribute__((aligned(16))) uint8_t turned[kChannels * kRow];
    __shared__ uint64_t rows[kKeepRows];
    const int64_t item = a.first + rocket::item_of_block();
    const int64_t block = item / a.tiles;
    const int c0 = (int)(item - block * a.tiles) * kChannels, quad = threadIdx.x % kQuads, band = threadIdx.x / kQuads;
    const int c = c0 + 4 * quad;
    typedef uint32_t vec __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int k = 0; k < kChannels * 8 / kThreads; k++) {
        const int at = k * kThreads + threadIdx.x, ch = at / 8;
        if (c0 + ch >= a.channels) continue;
        const vec v = *(const vec *)(a.q + (block * a.channels + c0 + ch) * kKeepRows + at % 8 * 16);
        uint32_t *to = (uint32_t *)(turned + ch * kRow + at % 8 * 16);
#pragma unroll
        for (int e = 0; e < 4; e++) to[e] = v[e];
    }
    float scale[4];
#pragma unroll
    for (int e = 0; e < 4; e++) scale[e] = c + e < a.channels ? a.scale[block * a.channels + c + e] : 0.0f;
    look_up(a, block, rows);
    if (c >= a.channels) return;
#pragma unroll
    for (int h = 0; h < 2; h++) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; e++)
            w[e] = c + e < a.channels ? *(const uint32_t *)(turned + (4 * quad + e) * kRow + h * 64 + 4 * band) : 0u;
#pragma unroll
        for (int k = 0; k < 4; k++) {
            const uint64_t at = rows[h * 64 + 4 * band + k];
            if (at == 0) continue;
            float f[4];
#pragma unroll
            for (int e = 0; e < 4; e++) {
                f[e] = !(at & 1) ? (float)(int8_t)(w[e] >> 8 * k) * scale[e] : 0.0f;
                // the fp32 product is rounded before the type's rounding: fp16 is what
                // fp32's result rounds to (the compiler would make one instruction of both)
                if (DT == ROCKET_FLOAT16) asm("" : "+v"(f[e]));
            }
            store4<DT>((char *)(at & ~(uint64_t)1), c, a.channels, f);
        }
    }
}

template <int DT, bool RESTORE>
void launch(KeepArgs a, hipStream_t s) {
    const int64_t items = (a.rows.count + kKeepRows - 1) / kKeepRows * a.tiles, most = rocket::most_groups(kThreads);
    for (a.first = 0; a.first < items; a.first += most) {
        const uint32_t groups = (uint32_t)std::min(items - a.first, most);
        if (RESTORE)
            restore_kernel<DT><<<groups, kThreads, 0, s>>>(a);
        else
            keep_kernel<DT><<<groups, kThreads, 0, s>>>(a);
    }
}

template <bool RESTORE>
rocket_status call(const rocket_sequence_shape *shape, const rocket_sequence *x, const int8_t *q, const float *scale,
                   void *stream) {
    if (!rocket::shape_ok(shape) || !(RESTORE ? rocket::out_ok(x, shape) : rocket::view_ok(x, shape)))
        return ROCKET_ERR_INVALID_ARG;
    if (rocket::empty(shape)) return ROCKET_OK;
    if (!rocket::bytes_ok(q) || !rocket::floats_ok(scale)) return ROCKET_ERR_INVALID_ARG;
    KeepArgs a = {};
    a.x = rocket::view_of(x, shape->dtype);
    a.q = const_cast<int8_t *>(q), a.scale = const_cast<float *>(scale);
    a.channels = (int32_t)shape->channels;
    a.tiles = (a.channels + kChannels - 1) / kChannels;
    View *views[] = {&a.x};
    a.rows = rocket::rows_of(shape, views, 1);
    hipStream_t s = (hipStream_t)stream;
    if (shape->dtype == ROCKET_FLOAT32)
        launch<ROCKET_FLOAT32, RESTORE>(a, s);
    else if (shape->dtype == ROCKET_BFLOAT16)
        launch<ROCKET_BFLOAT16, RESTORE>(a, s);
    else
        launch<ROCKET_FLOAT16, RESTORE>(a, s);
    return rocket::launched();
}

}  // namespace

extern "C" rocket_status rocket_checkpoint(const rocket_sequence_shape *shape, const rocket_sequence *x, int8_t *q,
                                           float *scale, void *hip_stream) {
    return call<false>(shape, x, q, scale, hip_stream);
}

extern "C" rocket_status rocket_restore(const rocket_sequence_shape *shape, const int8_t *q, const float *scale,
                                        const rocket_sequence *x, void *hip_stream) {
    return call<true>(shape, x, q, scale, hip_stream);
}
