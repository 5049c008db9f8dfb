// Dropout whose mask is never stored.
//
//   y_i = r_i + (u_i < D ? 0 : x_i 65536 / (65536 - D)),   D = round(65536 p)
//
// u_i are 16-bit numbers of Philox4x32-10 (Salmon, Moraes, Dror and Shaw,
// SC 2011): the key is the seed, the counter (i / 8, call), and the block's
// 128 bits give the numbers of eight consecutive elements.  The gradient is
// the same map on dy without r, with the numbers computed again.
//
// Bound: HBM.  A 16-bit element moves 4 bytes (6 with the residual); its
// share of a block is 1/8 of ten rounds of two 32 x 32 -> 64 bit products.
// 16 bits per element and not 32: half the products, and p is met to 2^-17.
// One thread takes one block: 16-byte loads and stores of 16-bit elements.
// 500 x 1000 x 256, bf16, with the residual: 130 us, 5.9 TB/s (a copy of that
// size reaches 5.2 TB/s); 777 x 129 x 331, fp16: 21 us, 6.3 TB/s.
#include <algorithm>
#include <cmath>

#include "sequence.h"

namespace {

using rocket::Elem;

constexpr int kBlock = 8;  // elements of one Philox block
constexpr int kThreads = 256;

struct DropArgs {
    const void *x;
    const void *r;  // or null
    void *y;
    int64_t begin;        // the launch's first block
    int64_t rows, cols;
    int64_t xs, rs, ys;  // row strides, elements
    uint64_t seed, call;
    uint32_t threshold;
    float scale;
};

__device__ inline void philox(uint32_t (&c)[4], uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int round = 0; round < 10; round++) {
        uint64_t a = (uint64_t)0xD2511F53u * c[0];
        uint64_t b = (uint64_t)0xCD9E8D57u * c[2];
        c[0] = (uint32_t)(b >> 32) ^ c[1] ^ k0;
        c[1] = (uint32_t)b;
        c[2] = (uint32_t)(a >> 32) ^ c[3] ^ k1;
        c[3] = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
}

template <int DT>
__device__ inline void load8(const void *p, float (&f)[kBlock]) {
    constexpr int kWords = kBlock / Elem<DT>::kPerWord;
    typedef uint32_t vec __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int w = 0; w < kWords; w += 4) {
        vec v = rocket::load_at<vec>((const char *)p + 4 * w);
#pragma unroll
        for (int k = 0; k < 4; k++)
#pragma unroll
            for (int j = 0; j < Elem<DT>::kPerWord; j++) f[(w + k) * Elem<DT>::kPerWord + j] = Elem<DT>::get(v[k], j);
    }
}

template <int DT>
__device__ inline void store8(void *p, const float (&f)[kBlock]) {
    constexpr int kWords = kBlock / Elem<DT>::kPerWord;
    typedef uint32_t vec __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int w = 0; w < kWords; w += 4) {
        vec v;
#pragma unroll
        for (int k = 0; k < 4; k++) v[k] = Elem<DT>::put(f + (w + k) * Elem<DT>::kPerWord);
        rocket::store_at((char *)p + 4 * w, v);
    }
}

// Element i of the call is column i % cols of row i / cols.  STRIDED: rows
// apart from each other in some operand, else everything is one row.
template <int DT, bool STRIDED>
__global__ __launch_bounds__(kThreads) void dropout_kernel(DropArgs a) {
    using raw = typename Elem<DT>::raw;
    const int64_t block = a.begin + (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t first = block * kBlock, total = a.rows * a.cols;
    if (first >= total) return;
    uint32_t c[4] = {(uint32_t)block, (uint32_t)(block >> 32), (uint32_t)a.call, (uint32_t)(a.call >> 32)};
    int64_t row = 0, col = first;
    if (STRIDED) {
        row = first / a.cols;
        col = first - row * a.cols;
    }
    const raw *x = (const raw *)a.x + row * a.xs + col;
    const raw *r = a.r ? (const raw *)a.r + row * a.rs + col : nullptr;
    raw *y = (raw *)a.y + row * a.ys + col;
    if (col + kBlock <= a.cols) {
        float f[kBlock], g[kBlock];
        load8<DT>(x, f);
        if (r) load8<DT>(r, g);
        philox(c, (uint32_t)a.seed, (uint32_t)(a.seed >> 32));
#pragma unroll
        for (int e = 0; e < kBlock; e++) {
            uint32_t u = e & 1 ? c[e >> 1] >> 16 : c[e >> 1] & 0xffffu;
            f[e] = u < a.threshold ? 0.0f : f[e] * a.scale;
            if (r) f[e] += g[e];
        }
        store8<DT>(y, f);
        return;
    }
    philox(c, (uint32_t)a.seed, (uint32_t)(a.seed >> 32));
    const int count = (int)(total - first < kBlock ? total - first : kBlock);
    for (int e = 0; e < count; e++) {
        uint32_t word = e < 2 ? c[0] : e < 4 ? c[1] : e < 6 ? c[2] : c[3];
        uint32_t u = e & 1 ? word >> 16 : word & 0xffffu;
        float f = u < a.threshold ? 0.0f : Elem<DT>::one(*x) * a.scale;
        if (r) f += Elem<DT>::one(*r);
        *y = Elem<DT>::round(f);
        x++, y++, col++;
        if (r) r++;
        if (STRIDED && col == a.cols) {  // the next row
            col = 0;
            x += a.xs - a.cols;
            y += a.ys - a.cols;
            if (r) r += a.rs - a.cols;
        }
    }
}

template <int DT>
void launch(DropArgs a, bool strided, int64_t grid, hipStream_t s) {
    const int64_t most = rocket::most_groups(kThreads);
    for (int64_t at = 0; at < grid; at += most) {
        const uint32_t groups = (uint32_t)std::min(grid - at, most);
        a.begin = at * kThreads;
        if (strided)
            dropout_kernel<DT, true><<<groups, kThreads, 0, s>>>(a);
        else
            dropout_kernel<DT, false><<<groups, kThreads, 0, s>>>(a);
    }
}

bool rows_ok(const void *p, int64_t rows, int64_t cols, int64_t stride, int size) {
    int64_t e;
    return p && (uintptr_t)p % size == 0 && (rows <= 1 || stride >= cols) &&
           !__builtin_mul_overflow(rows, stride, &e) && e <= ((int64_t)1 << 58);
}

}  // namespace

extern "C" rocket_status rocket_dropout(const void *x, const void *residual, void *y, int64_t rows, int64_t cols,
                                        int64_t x_stride, int64_t residual_stride, int64_t y_stride, int32_t dtype,
                                        double p, uint64_t seed, uint64_t call, void *hip_stream) {
    if (rows < 0 || cols < 0 || !rocket::dtype_ok(dtype) || !(p >= 0.0 && p <= 1.0)) return ROCKET_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return ROCKET_OK;
    const int size = rocket::elem_size(dtype);
    int64_t total;
    if (__builtin_mul_overflow(rows, cols, &total) || total > ((int64_t)1 << 41)) return ROCKET_ERR_INVALID_ARG;
    if (!rows_ok(x, rows, cols, x_stride, size) || !rows_ok(y, rows, cols, y_stride, size) ||
        (residual && !rows_ok(residual, rows, cols, residual_stride, size)))
        return ROCKET_ERR_INVALID_ARG;
    DropArgs a = {};
    a.x = x, a.r = residual, a.y = y;
    a.rows = rows, a.cols = cols;
    a.xs = x_stride, a.rs = residual_stride, a.ys = y_stride;
    a.seed = seed, a.call = call;
    a.threshold = (uint32_t)std::floor(p * 65536.0 + 0.5);
    a.scale = a.threshold < 65536u ? (float)(65536.0 / (65536.0 - a.threshold)) : 0.0f;
    bool strided = rows > 1 && (x_stride != cols || y_stride != cols || (residual && residual_stride != cols));
    if (!strided) a.rows = 1, a.cols = total;
    int64_t blocks = (total + kBlock - 1) / kBlock, grid = (blocks + kThreads - 1) / kThreads;
    hipStream_t s = (hipStream_t)hip_stream;
    if (dtype == ROCKET_FLOAT32)
        launch<ROCKET_FLOAT32>(a, strided, grid, s);
    else if (dtype == ROCKET_BFLOAT16)
        launch<ROCKET_BFLOAT16>(a, strided, grid, s);
    else
        launch<ROCKET_FLOAT16>(a, strided, grid, s);
    return rocket::launched();
}
