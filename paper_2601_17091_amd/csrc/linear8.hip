// Product of 8-bit rows with 8-bit weights.
//
//   y[t, m] = scale[t] wscale[m] (sum over k of q[t, k] p[m, k]) + bias[m]
//
// The sum is of whole numbers and exact: 32 bits hold it up to 131,072 columns.
// Scales and bias are fp32, the result is rounded once.
#include <algorithm>

#include "rows.h"

namespace {

using rocket::Elem;
using rocket::Place;
using rocket::Rows;
using rocket::View;

typedef int Int4 __attribute__((ext_vector_type(4)));
typedef int Int16 __attribute__((ext_vector_type(16)));

struct ProductArgs {
    Rows rows;
    const int8_t *q, *p;
    const float *scale, *wscale, *bias;  // bias or null
    View y;
    int32_t columns;   // of q and p: a multiple of 64
    int32_t channels;  // of y
    int32_t tiles;     // along the channels
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
    const int64_t item = rocket::item_of_block();
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

template <int DT>
void launch(ProductArgs a, hipStream_t s) {
    a.tiles = (a.channels + kTile - 1) / kTile;
    const int64_t items = (a.rows.count + kTile - 1) / kTile * a.tiles;
    product_kernel<DT><<<(uint32_t)items, 256, 0, s>>>(a);
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
