// Product of 8-bit rows with 8-bit weights.
//
//   y[t, m] = scale[t] wscale[m] (sum over k of q[t, k] p[m, k]) + bias[m]
//
// The sum is of whole numbers and exact: 32 bits hold it up to 131,072 columns.
// Scales and bias are fp32, the result is rounded once.
#include <algorithm>

#include "rows.h"
#include "stage.h"

namespace {

using rocket::Int4;

using rocket::Elem;
using rocket::Place;
using rocket::Rows;
using rocket::View;

typedef int Int16 __attribute__((ext_vector_type(16)));

struct ProductArgs {
    Rows rows;
    const int8_t *q, *p;
    const float *scale, *wscale, *bias;  // bias or null
    View y;
    int32_t columns;   // of q and p: a multiple of 64
    int32_t channels;  // of y
    int32_t tiles;     // along the channels
    int64_t first;     // the launch's first item
};

// Matrix instruction 32 x 32 x 32: the first operand's lane holds 16 bytes of row
// lane % 32, the second's of column lane % 32, both the half lane / 32 of the 32;
// result i of a lane is row 8 (i / 4) + 4 (lane / 32) + i % 4 of column lane % 32.
constexpr int kTile = 64, kStep = 64;
constexpr int kLine = kStep + 16;  // bytes of a row in shared memory

// The first operand is the weights, so that a lane has four channels in a row of
// one y row.
template <int DT>
__global__ __launch_bounds__(256) void product_kernel(ProductArgs a) {
    __shared__ __attribute__((aligned(16))) int8_t rows[kTile * kLine], weights[kTile * kLine];
    const int64_t item = a.first + rocket::item_of_block();
    const int64_t t0 = item / a.tiles * kTile;
    const int m0 = (int)(item % a.tiles) * kTile;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, wm = wave % 2 * 32, wt = wave / 2 * 32;
    const int line = threadIdx.x / 4, part = threadIdx.x % 4 * 16;
    const int64_t t = t0 + line;
    const bool has_t = t < a.rows.count, has_m = m0 + line < a.channels;
    Int16 sum = {};
    for (int k = 0; k < a.columns; k += kStep) {
        Int4 x = {}, w = {};
        if (has_t) x = *(const Int4 *)(a.q + t * a.columns + k + part);
        if (has_m) w = *(const Int4 *)(a.p + (int64_t)(m0 + line) * a.columns + k + part);
        __syncthreads();
        *(Int4 *)(rows + line * kLine + part) = x;
        *(Int4 *)(weights + line * kLine + part) = w;
        __syncthreads();
#pragma unroll
        for (int h = 0; h < kStep; h += 32) {
            const Int4 fa = *(const Int4 *)(weights + (wm + lane % 32) * kLine + h + lane / 32 * 16);
            const Int4 fb = *(const Int4 *)(rows + (wt + lane % 32) * kLine + h + lane / 32 * 16);
            sum = __builtin_amdgcn_mfma_i32_32x32x32_i8(fa, fb, sum, 0, 0, 0);
        }
    }
    const int64_t r = t0 + wt + lane % 32;
    if (r >= a.rows.count) return;
    const Place p = rocket::place_of(a.rows, r);
    using raw = typename Elem<DT>::raw;
    raw *y = (raw *)rocket::row_at(a.y, p);
    const float scale = p.live ? a.scale[r] : 0.0f;
#pragma unroll
    for (int i = 0; i < 16; i++) {
        const int m = m0 + wm + 8 * (i / 4) + 4 * (lane / 32) + i % 4;
        if (m >= a.channels) continue;
        const float v = __builtin_fmaf((float)sum[i], scale * a.wscale[m], a.bias ? a.bias[m] : 0.0f);
        y[m] = Elem<DT>::round(p.live ? v : 0.0f);
    }
}

// A tile of y by WM x WT wavefronts, each MT x NT matrices of 32 channels x 32 rows.
//
// A stage is 64 columns of the tile's weights and rows, 64 bytes a line in shared
// memory, a line's four pieces of 16 bytes moved by its number so that the reads of
// 32 lines meet every bank alike.  Four stages are there or on their way.  A stage
// is two steps of 32 columns; while the matrix unit works on one step's operands,
// the next step's are read into other registers, over the borders of stages too:
// what a barrier says is that the next stage has arrived and that this one has
// been read, and it stands where the matrix unit still has work.
template <int DT, int MT, int NT, int WM, int WT, int SLOTS>
__global__ __launch_bounds__(64 * WM * WT) void tile_kernel(ProductArgs a) {
    constexpr int kWaves = WM * WT, kM = 32 * MT * WM, kT = 32 * NT * WT, kSlots = SLOTS;
    constexpr int kLoadsM = kM / 16 / kWaves, kLoadsT = kT / 16 / kWaves, kLoads = kLoadsM + kLoadsT;
    constexpr int kStage = (kM + kT) * 64, kSteps = MT * NT, kReads = MT + NT;
    constexpr int kSize = Elem<DT>::kSize;
    typedef float Float4 __attribute__((ext_vector_type(4)));
    typedef uint32_t Words __attribute__((ext_vector_type(kSize)));   // four values
    static_assert(kLoadsM * kWaves * 16 == kM && kLoadsT * kWaves * 16 == kT, "whole loads");
    __shared__ __attribute__((aligned(1024))) char shared[kSlots * kStage + 8 * kM + 12 * kT];
    const uint32_t base = rocket::shared_address(shared);
    const int lane = threadIdx.x % 64, wave = rocket::uniform(threadIdx.x / 64);
    const int wm = wave % WM, wt = wave / WM, half = lane / 32;
    const int64_t item = a.first + rocket::item_of_block();
    const int64_t t0 = item / a.tiles * kT;
    const int m0 = (int)(item % a.tiles) * kM;
    const int stages = a.columns / 64;

    // where this lane's pieces of a stage come from
    const int64_t left_t = a.rows.count - t0;
    const int left_m = a.channels - m0;
    const Int4 weights = rocket::buffer_of(a.p + (int64_t)m0 * a.columns,
                                           (int64_t)(left_m < kM ? left_m : kM) * a.columns);
    const Int4 rows = rocket::buffer_of(a.q + t0 * a.columns, (left_t < kT ? left_t : kT) * a.columns);
    uint32_t from[kLoads];
#pragma unroll
    for (int k = 0; k < kLoads; k++) {
        const int line = (k < kLoadsM ? wave * kLoadsM + k : wave * kLoadsT + k - kLoadsM) * 16 + lane / 4;
        from[k] = line * a.columns + (lane % 4 ^ (line >> 2 & 3)) * 16;
    }
    // the tile's scales and bias, and where its rows lie, before the stages' loads: a
    // row that holds no data has its address's lowest bit set, one that is not there 0
    float *factors = (float *)(shared + kSlots * kStage), *row_scale = factors + 2 * kM;
    uint64_t *row_at = (uint64_t *)(row_scale + kT);
    for (int k = threadIdx.x; k < kM; k += 64 * kWaves) {
        factors[k] = k < left_m ? a.wscale[m0 + k] : 0.0f;
        factors[kM + k] = k < left_m && a.bias ? a.bias[m0 + k] : 0.0f;
    }
    for (int k = threadIdx.x; k < kT; k += 64 * kWaves) {
        const Place p = rocket::place_of(a.rows, t0 + (k < left_t ? k : 0));
        const uint64_t to = (uint64_t)(rocket::row_at(a.y, p) + (int64_t)m0 * kSize);
        row_scale[k] = k < left_t ? a.scale[t0 + k] : 0.0f;
        row_at[k] = k < left_t ? to | (p.live ? 0 : 1) : 0;
    }

    int asked = 0;
    uint32_t ask_at = 0, ask_to = base;
    auto open_stage = [&]() {
        ask_at = asked < stages ? asked * 64 : rocket::kNowhere;
        ask_to = base + asked % kSlots * kStage;
        asked++;
    };
    auto ask = [&](int k) {
        if (k < kLoadsM)
            rocket::load_stage16(weights, ask_to + (wave * kLoadsM + k) * 1024, from[k], ask_at);
        else
            rocket::load_stage16(rows, ask_to + kM * 64 + (wave * kLoadsT + k - kLoadsM) * 1024, from[k], ask_at);
    };

    // where it reads a stage: the second step's piece is the first one's with bit 1 turned
    typedef const __attribute__((address_space(3))) Int4 *SharedInt4;
    const uint32_t piece = (half ^ (lane >> 2 & 3)) * 16 + lane % 32 * 64;
    const uint32_t read_m = wm * MT * 2048 + piece, read_t = kM * 64 + wt * NT * 2048 + piece;
    Int16 sum[MT][NT] = {};
    Int4 fm[2][MT], ft[2][NT];
    auto read = [&](int step, uint32_t at, int k) {
        if (k < MT)
            fm[step][k] = *(SharedInt4)(rocket::shared_at((at + read_m) ^ step * 32) + k * 2048);
        else
            ft[step][k - MT] = *(SharedInt4)(rocket::shared_at((at + read_t) ^ step * 32) + (k - MT) * 2048);
    };
    // the k-th operand of a step in the order in which its products need them
    const auto order = [](int k) { return k == 0 ? 0 : k <= NT ? MT + k - 1 : k - NT; };
#pragma unroll
    for (int early = 0; early < kSlots; early++) {
        open_stage();
#pragma unroll
        for (int k = 0; k < kLoads; k++) ask(k);
    }
    rocket::wait_loads<(kSlots - 1) * kLoads>();
#pragma unroll
    for (int k = 0; k < kReads; k++) read(0, base, order(k));
    constexpr int kMeet = kSteps - 1 - kSteps / 4;   // the product after which the wavefronts meet
    for (int stage = 0; stage < stages; stage++) {
        const uint32_t at = base + stage % kSlots * kStage, next = base + (stage + 1) % kSlots * kStage;
#pragma unroll
        for (int k = 0; k < kSteps; k++) {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int r = k * kReads / (kMeet + 1); r < (k + 1) * kReads / (kMeet + 1) && r < kReads; r++)
                read(1, at, order(r));
            sum[k / NT][k % NT] =
                __builtin_amdgcn_mfma_i32_32x32x32_i8(fm[0][k / NT], ft[0][k % NT], sum[k / NT][k % NT], 0, 0, 0);
            if (k == kMeet) {
                __builtin_amdgcn_sched_barrier(0);
                rocket::wait_loads<(kSlots - 2) * kLoads>();
            }
        }
        open_stage();
#pragma unroll
        for (int k = 0; k < kSteps; k++) {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int r = k * kReads / kSteps; r < (k + 1) * kReads / kSteps; r++) read(0, next, order(r));
            sum[k / NT][k % NT] =
                __builtin_amdgcn_mfma_i32_32x32x32_i8(fm[1][k / NT], ft[1][k % NT], sum[k / NT][k % NT], 0, 0, 0);
#pragma unroll
            for (int l = k * kLoads / kSteps; l < (k + 1) * kLoads / kSteps; l++) ask(l);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    rocket::wait_loads<0>();

    // A lane has four channels in a row, eight apart, of one row of y.  32 rows at a
    // time go through shared memory, each wavefront's its own, so that a row's channels
    // are written side by side.
    constexpr int kRowBytes = 32 * MT * kSize, kLine = kRowBytes + 16, kLanes = kRowBytes / 16;
    static_assert(kWaves * 32 * kLine <= kSlots * kStage, "room for the rows");
    char *mine = shared + wave * 32 * kLine;
    const int part = lane % kLanes * 16, c = wm * 32 * MT + part / kSize;   // what it writes of a row
    constexpr int kEach = 16 / kSize;
#pragma unroll
    for (int y = 0; y < NT; y++) {
        const int t = (wt * NT + y) * 32;
        const float scale = row_scale[t + lane % 32];
        const uint32_t held = row_at[t + lane % 32] & 1 ? 0u : ~0u;
#pragma unroll
        for (int x = 0; x < MT; x++)
#pragma unroll
            for (int g = 0; g < 4; g++) {
                const int m = x * 32 + 8 * g + 4 * half;
                const Float4 s = *(const Float4 *)(factors + wm * 32 * MT + m);
                const Float4 b = *(const Float4 *)(factors + kM + wm * 32 * MT + m);
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; e++) v[e] = __builtin_fmaf((float)sum[x][y][4 * g + e], scale * s[e], b[e]);
                Words w;
#pragma unroll
                for (int e = 0; e < kSize; e++) w[e] = Elem<DT>::put(v + e * Elem<DT>::kPerWord) & held;
                *(Words *)(mine + lane % 32 * kLine + m * kSize) = w;
            }
#pragma unroll
        for (int k = 0; k < kLanes / 2; k++) {
            const int row = k * (64 / kLanes) + lane / kLanes;
            const uint32_t *from = (const uint32_t *)(mine + row * kLine + part);
            const Int4 v = *(const Int4 *)from;
            char *to = (char *)(row_at[t + row] & ~(uint64_t)1);
            if (!to || c >= left_m) continue;
            to += c * kSize;
            if (c + kEach <= left_m) {
                rocket::store_at(to, v);
            } else {
                using bits = typename Elem<DT>::bits;
                for (int e = 0; e < kEach && c + e < left_m; e++) ((bits *)to)[e] = ((const bits *)from)[e];
            }
        }
    }
}

// The tile: the largest of which there are enough to fill the chip.
template <int DT, int MT, int NT, int WM, int WT, int SLOTS = 4>
void tiles(ProductArgs a, hipStream_t s) {
    constexpr int kM = 32 * MT * WM, kT = 32 * NT * WT;
    a.tiles = (a.channels + kM - 1) / kM;
    const int64_t items = (a.rows.count + kT - 1) / kT * a.tiles;
    const int64_t most = rocket::most_groups(64 * WM * WT);
    for (a.first = 0; a.first < items; a.first += most)
        tile_kernel<DT, MT, NT, WM, WT, SLOTS><<<(uint32_t)std::min(items - a.first, most), 64 * WM * WT, 0, s>>>(a);
}

template <int DT>
void launch(ProductArgs a, hipStream_t s) {
    const int64_t big = (a.rows.count + 255) / 256 * ((a.channels + 255) / 256);
    const int64_t middle = (a.rows.count + 127) / 128 * ((a.channels + 127) / 128);
    if (big >= 200)
        tiles<DT, 4, 4, 2, 2>(a, s);
    else if (middle >= 200)
        tiles<DT, 2, 2, 2, 2>(a, s);
    else if (a.rows.count > 64)
        tiles<DT, 1, 1, 2, 2>(a, s);
    else {
        a.tiles = (a.channels + kTile - 1) / kTile;
        const int64_t items = (a.rows.count + kTile - 1) / kTile * a.tiles;
        product_kernel<DT><<<(uint32_t)items, 256, 0, s>>>(a);
    }
}

bool columns_ok(int64_t columns) { return columns > 0 && columns <= 131072 && columns % rocket::kPad8 == 0; }

}  // namespace

extern "C" rocket_status rocket_linear_bytes_workspace(const rocket_sequence_shape *shape, int64_t columns,
                                                  int64_t *bytes) {
    if (!bytes || !rocket::shape_ok(shape) || !columns_ok(columns)) return ROCKET_ERR_INVALID_ARG;
    *bytes = 0;
    return ROCKET_OK;
}

extern "C" rocket_status rocket_linear_bytes(const rocket_sequence_shape *shape, int64_t columns, const int8_t *q,
                                        const float *scale, const int8_t *weight, const float *weight_scale,
                                        const float *bias, const rocket_sequence *y, void *workspace,
                                        int64_t workspace_bytes, void *hip_stream) {
    if (!rocket::shape_ok(shape) || !columns_ok(columns) || !rocket::out_ok(y, shape)) return ROCKET_ERR_INVALID_ARG;
    if (rocket::empty(shape)) return ROCKET_OK;
    if (!rocket::bytes_ok(q) || !rocket::floats_ok(scale) || !rocket::bytes_ok(weight) ||
        !rocket::floats_ok(weight_scale) || (bias && !rocket::floats_ok(bias)))
        return ROCKET_ERR_INVALID_ARG;
    ProductArgs a = {};
    a.q = q, a.p = weight, a.scale = scale, a.wscale = weight_scale, a.bias = bias;
    a.y = rocket::view_of(y, shape->dtype);
    a.columns = (int32_t)columns, a.channels = (int32_t)shape->channels;
    View *views[] = {&a.y};
    a.rows = rocket::rows_of(shape, views, 1);
    hipStream_t s = (hipStream_t)hip_stream;
    if (shape->dtype == ROCKET_FLOAT32)
        launch<ROCKET_FLOAT32>(a, s);
    else if (shape->dtype == ROCKET_BFLOAT16)
        launch<ROCKET_BFLOAT16>(a, s);
    else
        launch<ROCKET_FLOAT16>(a, s);
    return rocket::launched();
}
