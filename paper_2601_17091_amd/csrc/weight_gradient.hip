// Gradient of a linear layer's weights from an 8-bit checkpoint of its rows.
//
//   dW[m, c] = sum over blocks b of scale[b, c] (sum over the block's rows t of dy[t, m] q[b, c, t])
//   db[m] = sum over rows of dy[t, m]
//
// A channel's scale is a factor of its block's sum, so nothing is rounded before
// the sums: q is exact in bf16 and fp16, dy is taken as it is (fp32 as the exact
// sum of three bf16 parts), and the matrix unit sums their products in fp32.
#include <algorithm>

#include "rows.h"

namespace {

using rocket::Elem;
using rocket::kKeepRows;
using rocket::Place;
using rocket::Rows;
using rocket::View;

typedef float Float16 __attribute__((ext_vector_type(16)));
typedef __bf16 Bf8 __attribute__((ext_vector_type(8)));
typedef _Float16 Half8 __attribute__((ext_vector_type(8)));

struct GradArgs {
    Rows rows;
    View dy;
    const int8_t *q;
    const float *scale;
    float *dweight;  // or the parts' sums [parts, m, c]
    float *dbias;    // or the parts' sums [parts, m]
    int64_t blocks, each;  // blocks of rows; of a part
    int32_t m, c;
};

constexpr int kTile = 64, kSteps = 64;

// Parts of a value that 16-bit operands hold: fp32 is the sum of three bf16.
template <int DT>
constexpr int kPlanes = DT == ROCKET_FLOAT32 ? 3 : 1;

template <int DT>
__device__ inline void split(typename Elem<DT>::raw x, uint16_t (&p)[kPlanes<DT>]) {
    if constexpr (DT == ROCKET_FLOAT32) {
        // 8 bits a part, cut off and not rounded: no part is larger than the value
        float rest = x;
#pragma unroll
        for (int k = 0; k < 3; k++) {
            p[k] = (uint16_t)(__builtin_bit_cast(uint32_t, rest) >> 16);
            rest -= Elem<ROCKET_BFLOAT16>::one(p[k]);
        }
        if (rocket::magnitude(x) >= rocket::kNotFinite) p[0] = Elem<ROCKET_BFLOAT16>::round(x), p[1] = p[2] = 0;
    } else {
        p[0] = x;
    }
}

// Matrix instruction 32 x 32 x 16: a lane holds 8 values of row (column) lane % 32,
// those of the half lane / 32; the result as in linear8.hip.
template <int DT>
__global__ __launch_bounds__(256) void gradient_kernel(GradArgs a) {
    using raw = typename Elem<DT>::raw;
    constexpr int kP = kPlanes<DT>;
    constexpr bool kHalf = DT == ROCKET_FLOAT16;
    __shared__ uint16_t dy[kP][kSteps][kTile];
    __shared__ __attribute__((aligned(8))) int8_t q[kTile][kSteps + 8];
    const uint32_t across = (a.c + kTile - 1) / kTile, down = (a.m + kTile - 1) / kTile;
    const uint32_t part_of = blockIdx.x / (across * down), tile = blockIdx.x % (across * down);
    const int m0 = tile / across * kTile, c0 = tile % across * kTile;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, wm = wave % 2 * 32, wc = wave / 2 * 32;
    const int line = threadIdx.x / 4, part = threadIdx.x % 4 * 16;
    const int c = c0 + wc + lane % 32;
    Float16 total = {};
    float bias = 0.0f;   // of channel m0 + threadIdx.x
    const int64_t begin = part_of * a.each, end = begin + a.each < a.blocks ? begin + a.each : a.blocks;
    for (int64_t b = begin; b < end; b++) {
        Float16 sum = {};
        for (int h = 0; h < kKeepRows; h += kSteps) {
            const int64_t r = b * kKeepRows + h + line;
            Place p = {};
            if (r < a.rows.count) p = rocket::place_of(a.rows, r);
            const raw *row = (const raw *)rocket::row_at(a.dy, p);
            __syncthreads();
            for (int e = 0; e < 16; e++) {
                const int m = m0 + part + e;
                uint16_t v[kP] = {};
                if (p.live && m < a.m) split<DT>(row[m], v);
#pragma unroll
                for (int k = 0; k < kP; k++) dy[k][line][part + e] = v[k];
            }
            for (int e = 0; e < 16; e += 8) {
                uint64_t v = 0;
                if (c0 + line < a.c) v = *(const uint64_t *)(a.q + (b * a.c + c0 + line) * kKeepRows + h + part + e);
                *(uint64_t *)&q[line][part + e] = v;
            }
            __syncthreads();
            if (threadIdx.x < kTile && c0 == 0)
                for (int t = 0; t < kSteps; t++)
#pragma unroll
                    for (int k = kP - 1; k >= 0; k--)
                        bias += kHalf ? Elem<ROCKET_FLOAT16>::one(dy[k][t][threadIdx.x])
                                      : Elem<ROCKET_BFLOAT16>::one(dy[k][t][threadIdx.x]);
            for (int t = 0; t < kSteps; t += 16) {
                const int t0 = t + lane / 32 * 8;
                float f[8];
#pragma unroll
                for (int e = 0; e < 8; e++) f[e] = (float)q[wc + lane % 32][t0 + e];
                if constexpr (kHalf) {
                    Half8 fa, fb;
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        fa[e] = __builtin_bit_cast(_Float16, dy[0][t0 + e][wm + lane % 32]);
                        fb[e] = (_Float16)f[e];
                    }
                    sum = __builtin_amdgcn_mfma_f32_32x32x16_f16(fa, fb, sum, 0, 0, 0);
                } else {
#pragma unroll
                    for (int k = kP - 1; k >= 0; k--) {
                        Bf8 fa, fb;
#pragma unroll
                        for (int e = 0; e < 8; e++) {
                            fa[e] = __builtin_bit_cast(__bf16, dy[k][t0 + e][wm + lane % 32]);
                            fb[e] = (__bf16)f[e];
                        }
                        sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa, fb, sum, 0, 0, 0);
                    }
                }
            }
        }
        const float scale = c < a.c ? a.scale[b * a.c + c] : 0.0f;
#pragma unroll
        for (int i = 0; i < 16; i++) total[i] = __builtin_fmaf(sum[i], scale, total[i]);
    }
    if (c < a.c)
#pragma unroll
        for (int i = 0; i < 16; i++) {
            const int m = m0 + wm + 8 * (i / 4) + 4 * (lane / 32) + i % 4;
            if (m < a.m) a.dweight[((int64_t)part_of * a.m + m) * a.c + c] = total[i];
        }
    if (a.dbias && c0 == 0 && threadIdx.x < kTile && m0 + (int)threadIdx.x < a.m)
        a.dbias[(int64_t)part_of * a.m + m0 + threadIdx.x] = bias;
}

// Sums of the parts, in their order.
__global__ __launch_bounds__(256) void join_kernel(const float *parts, float *sum, int64_t count, int32_t n) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= count) return;
    float v = 0.0f;
    for (int k = 0; k < n; k++) v += parts[k * count + i];
    sum[i] = v;
}

struct Cut {
    int64_t blocks, each, parts;
};

// Parts of the rows, so that the workgroups fill the chip.
Cut cut_of(const rocket_sequence_shape *s, int64_t channels) {
    Cut c;
    c.blocks = (s->n * s->steps + kKeepRows - 1) / kKeepRows;
    const int64_t tiles = ((s->channels + kTile - 1) / kTile) * ((channels + kTile - 1) / kTile);
    const int64_t parts = std::max<int64_t>(1, std::min<int64_t>({c.blocks, 1024 / std::max<int64_t>(tiles, 1), 64}));
    c.each = std::max<int64_t>(1, (c.blocks + parts - 1) / parts);
    c.parts = std::max<int64_t>(1, (c.blocks + c.each - 1) / c.each);
    return c;
}

bool sizes_ok(const rocket_sequence_shape *s, int64_t channels) {
    return rocket::shape_ok(s) && channels > 0 && channels <= (1 << 24) && s->channels * channels <= ((int64_t)1 << 34);
}

}  // namespace

extern "C" rocket_status rocket_linear_weight_gradient_workspace(const rocket_sequence_shape *shape, int64_t channels,
                                                                 int64_t *bytes) {
    if (!bytes || !sizes_ok(shape, channels)) return ROCKET_ERR_INVALID_ARG;
    const Cut cut = cut_of(shape, channels);
    *bytes = cut.parts > 1 ? (cut.parts * shape->channels * (channels + 1) * 4 + 7) / 8 * 8 : 0;
    return ROCKET_OK;
}

extern "C" rocket_status rocket_linear_weight_gradient(const rocket_sequence_shape *shape, int64_t channels,
                                                       const rocket_sequence *dy, const int8_t *q, const float *scale,
                                                       float *dweight, float *dbias, void *workspace,
                                                       int64_t workspace_bytes, void *hip_stream) {
    if (!sizes_ok(shape, channels) || !rocket::view_ok(dy, shape) || !rocket::floats_ok(dweight) ||
        (dbias && !rocket::floats_ok(dbias)))
        return ROCKET_ERR_INVALID_ARG;
    if (!rocket::empty(shape) && (!rocket::bytes_ok(q) || !rocket::floats_ok(scale))) return ROCKET_ERR_INVALID_ARG;
    int64_t need = 0;
    rocket_linear_weight_gradient_workspace(shape, channels, &need);
    if (need && (!workspace || (uintptr_t)workspace % 8 != 0 || workspace_bytes < need)) return ROCKET_ERR_INVALID_ARG;
    const Cut cut = cut_of(shape, channels);
    GradArgs a = {};
    a.dy = rocket::view_of(dy, shape->dtype);
    a.q = q, a.scale = scale;
    a.m = (int32_t)shape->channels, a.c = (int32_t)channels;
    a.blocks = cut.blocks, a.each = cut.each;
    const int64_t count = (int64_t)a.m * a.c;
    a.dweight = cut.parts > 1 ? (float *)workspace : dweight;
    a.dbias = !dbias ? nullptr : cut.parts > 1 ? (float *)workspace + cut.parts * count : dbias;
    View *views[] = {&a.dy};
    a.rows = rocket::rows_of(shape, views, 1);
    hipStream_t s = (hipStream_t)hip_stream;
    const uint32_t grid = (uint32_t)((a.c + kTile - 1) / kTile * ((a.m + kTile - 1) / kTile) * cut.parts);
    if (shape->dtype == ROCKET_FLOAT32)
        gradient_kernel<ROCKET_FLOAT32><<<grid, 256, 0, s>>>(a);
    else if (shape->dtype == ROCKET_BFLOAT16)
        gradient_kernel<ROCKET_BFLOAT16><<<grid, 256, 0, s>>>(a);
    else
        gradient_kernel<ROCKET_FLOAT16><<<grid, 256, 0, s>>>(a);
    if (cut.parts > 1) {
        join_kernel<<<(uint32_t)((count + 255) / 256), 256, 0, s>>>(a.dweight, dweight, count, (int32_t)cut.parts);
        if (dbias) join_kernel<<<(uint32_t)((a.m + 255) / 256), 256, 0, s>>>(a.dbias, dbias, a.m, (int32_t)cut.parts);
    }
    return rocket::launched();
}
