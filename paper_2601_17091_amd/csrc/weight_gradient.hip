// Gradient of a linear layer's weights from an 8-bit checkpoint of its rows.
//
//   dW[m, c] = sum over blocks b of scale[b, c] (sum over the block's rows t of dy[t, m] q[b, c, t])
//   db[m] = sum over rows of dy[t, m]
//
// A channel's scale is a factor of its block's sum, so nothing is rounded before
// the sums: q is exact in bf16 and fp16, dy is taken as it is (fp32 as the exact
// sum of three bf16 parts), and the matrix unit sums their products in fp32.
//
// Bound: the matrix unit, 2 rows m c operations.  Many rows: tiles of 256 x 256 whose
// stages are on their way while others are read (staged_kernel).  The unit is busy for
// 46 % of the cycles at 2.0 to 2.1 GHz and wavefronts wait for 31 % of theirs; memory is
// no bound (3.2 GB read from L2, of which 84 % are there).  Whole versions that do not
// widen q or load nothing took 394 and 337 of 440 us: two wavefronts a SIMD do not cover
// loads, widening and barriers with the other's products.  Few rows: tiles of
// 64 x 64 straight from registers (gradient_kernel).  The rows are shared out where the
// tiles do not fill the chip, and the parts' sums joined in a fixed order.
// Measured (the same call differs by 6 % between cards):
//   64 x 1000 rows bf16, 1,536 by 2,000     405 to 430 us, 915 to 970 TFLOP/s
//   777 x 129 rows fp16, 993 by 924         263 to 275 us: 66 to lay out dy, whose rows have
//                                           odd places, 190 to 204 the product, 6 the join
//   20 x 1000 rows fp32, 768 by 2,000       232 to 238 us
//   64 rows fp32, 192 by 2,000              5.2 us
#include <algorithm>
#include <type_traits>

#include "rows.h"
#include "stage.h"

namespace {

using rocket::Int4;

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

constexpr int kTile = 64, kRows = 64;

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

typedef short Short4 __attribute__((ext_vector_type(4)));
typedef uint32_t Words4 __attribute__((ext_vector_type(4)));
typedef const __attribute__((address_space(3))) Words4 *SharedWords;
typedef _Float16 Half2 __attribute__((ext_vector_type(2)));

// Bytes 2 k and 2 k + 1 of four signed ones as two values of the operands' type,
// exactly.
template <bool HALF>
__device__ inline uint32_t widen(uint32_t b, int k) {
    if (HALF) {
        // 1024 + (q + 128) has q + 128 as its lowest bits
        const Half2 off = {(_Float16)-1152.0f, (_Float16)-1152.0f};
        const uint32_t pair = __builtin_amdgcn_perm(0x64646464u, b ^ 0x80808080u, k ? 0x04030402u : 0x04010400u);
        return __builtin_bit_cast(uint32_t, __builtin_bit_cast(Half2, pair) + off);
    }
    // whole numbers below 2^8 leave the lower half of an fp32 value empty
    const float x = (float)(int8_t)(b >> (16 * k)), y = (float)(int8_t)(b >> (16 * k + 8));
    return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, y), __builtin_bit_cast(uint32_t, x), 0x07060302u);
}

template <bool HALF>
__device__ inline float value16(uint32_t w, int j) {
    return HALF ? Elem<ROCKET_FLOAT16>::get(w, j) : Elem<ROCKET_BFLOAT16>::get(w, j);
}

// 8 values of one column of shared memory, four rows apart by `LINE` bytes and the
// next four: what a lane holds of the first operand.
template <int LINE>
__device__ inline Words4 turned(rocket::Shared p) {
    typedef __attribute__((address_space(3))) Short4 *Lds;
    const Short4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(p));
    const Short4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(p + 4 * LINE));
    const uint64_t w0 = __builtin_bit_cast(uint64_t, v0), w1 = __builtin_bit_cast(uint64_t, v1);
    return Words4{(uint32_t)w0, (uint32_t)(w0 >> 32), (uint32_t)w1, (uint32_t)(w1 >> 32)};
}

// ------------------------------------------------------------ few rows: direct tiles
// A tile of 64 x 64 by four wavefronts of one 32 x 32 matrix, 64 rows at a time: dy
// comes through registers, where it is taken apart, to shared memory as it lies, q to
// [c][64 rows]; the next rows are on their way meanwhile.  What bounds it is the way of
// one such step, so everything is one launch.
//
// Matrix instruction 32 x 32 x 16: a lane holds 8 values of row (column) lane % 32,
// those of the half lane / 32; the result as in linear8.hip.
template <int DT>
__global__ __launch_bounds__(256) void gradient_kernel(GradArgs a) {
    using raw = typename Elem<DT>::raw;
    constexpr int kP = kPlanes<DT>, kLineA = 2 * kTile + 16, kLineC = kRows + 16;
    constexpr bool kHalf = DT == ROCKET_FLOAT16;
    __shared__ __attribute__((aligned(16))) char dy[kP][kRows * kLineA], q[kTile * kLineC];
    const uint32_t across = (a.c + kTile - 1) / kTile, down = (a.m + kTile - 1) / kTile;
    const uint32_t part = blockIdx.x / (across * down), tile = blockIdx.x % (across * down);
    const int m0 = tile / across * kTile, c0 = tile % across * kTile;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, wm = wave % 2 * 32, wc = wave / 2 * 32;
    const int line = threadIdx.x / 4, piece = threadIdx.x % 4 * 16;
    const int group = lane / 16, in = lane % 16, half = lane / 32;
    const int c = c0 + wc + lane % 32;
    const int64_t begin = part * a.each, end = begin + a.each < a.blocks ? begin + a.each : a.blocks;
    const int64_t last = end * kKeepRows < a.rows.count ? end * kKeepRows : a.rows.count;
    raw x[16];
    Words4 b;
    const auto load = [&](int64_t row0) {
        const int64_t r = row0 + line;
        const int m = m0 + piece;
        Place p = {};
        if (r < a.rows.count) p = rocket::place_of(a.rows, r);
        const raw *row = (const raw *)rocket::row_at(a.dy, p) + m;
        if (p.live && m + 16 <= a.m) {
            __builtin_memcpy(x, row, sizeof(x));
        } else {
#pragma unroll
            for (int e = 0; e < 16; e++) x[e] = p.live && m + e < a.m ? row[e] : raw(0);
        }
        b = Words4{0, 0, 0, 0};
        if (c0 + line < a.c)
            b = *(const Words4 *)(a.q + (row0 / kKeepRows * a.c + c0 + line) * kKeepRows + row0 % kKeepRows + piece);
    };
    const rocket::Shared from_a = rocket::shared_at(rocket::shared_address(dy) + (8 * half + in / 4) * kLineA +
                                                    2 * (wm + 16 * (group & 1)) + in % 4 * 8);
    const char *from_c = q + (wc + lane % 32) * kLineC + 8 * half;
    Float16 total = {}, sum = {};
    float bias = 0.0f;
    if (begin * kKeepRows < last) load(begin * kKeepRows);
    for (int64_t row0 = begin * kKeepRows; row0 < last; row0 += kRows) {
        __syncthreads();
        uint32_t v[kP][8];
#pragma unroll
        for (int e = 0; e < 8; e++) {
            uint16_t lo[kP], hi[kP];
            split<DT>(x[2 * e], lo);
            split<DT>(x[2 * e + 1], hi);
#pragma unroll
            for (int k = 0; k < kP; k++) v[k][e] = lo[k] | (uint32_t)hi[k] << 16;
        }
#pragma unroll
        for (int k = 0; k < kP; k++)
#pragma unroll
            for (int e = 0; e < 8; e += 4)
                *(Words4 *)(dy[k] + line * kLineA + 2 * piece + 4 * e) =
                    Words4{v[k][e], v[k][e + 1], v[k][e + 2], v[k][e + 3]};
        *(Words4 *)(q + line * kLineC + piece) = b;
        __syncthreads();
        if (row0 + kRows < last) load(row0 + kRows);
#pragma unroll
        for (int t = 0; t < kRows; t += 16) {
            const uint64_t bytes = *(const uint64_t *)(from_c + t);
            Words4 fb;
#pragma unroll
            for (int k = 0; k < 4; k++) fb[k] = widen<kHalf>((uint32_t)(bytes >> (32 * (k / 2))), k % 2);
#pragma unroll
            for (int k = kP - 1; k >= 0; k--) {
                const Words4 fa = turned<kLineA>(from_a + k * kRows * kLineA + t * kLineA);
                if (a.dbias && c0 == 0 && wc == 0)
#pragma unroll
                    for (int e = 0; e < 8; e++) bias += value16<kHalf>(fa[e / 2], e % 2);
                if constexpr (kHalf)
                    sum = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(Half8, fa),
                                                                 __builtin_bit_cast(Half8, fb), sum, 0, 0, 0);
                else
                    sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(Bf8, fa),
                                                                  __builtin_bit_cast(Bf8, fb), sum, 0, 0, 0);
            }
        }
        if (row0 % kKeepRows == 0 && row0 + kRows < last) continue;
        const float scale = c < a.c ? a.scale[row0 / kKeepRows * a.c + c] : 0.0f;
#pragma unroll
        for (int i = 0; i < 16; i++) total[i] = __builtin_fmaf(sum[i], scale, total[i]);
        sum = Float16{};
    }
    if (c < a.c)
#pragma unroll
        for (int i = 0; i < 16; i++) {
            const int m = m0 + wm + 8 * (i / 4) + 4 * half + i % 4;
            if (m < a.m) a.dweight[((int64_t)part * a.m + m) * a.c + c] = total[i];
        }
    bias += __shfl_xor(bias, 32);
    const int m = m0 + wm + lane;
    if (a.dbias && c0 == 0 && wc == 0 && lane < 32 && m < a.m) a.dbias[(int64_t)part * a.m + m] = bias;
}

// ------------------------------------------------------- many rows: staged tiles
struct StagedArgs {
    const char *dy;       // rows of 16-bit values at one distance, 4-byte aligned
    int64_t dy_stride;    // bytes
    int64_t dy_plane;     // bytes between the parts of fp32 values
    const uint64_t *live; // a bit for each row, or null: all of them
    const int8_t *q;
    const float *scale;
    float *dweight, *dbias;  // the parts' sums, [parts, m, c] and [parts, tiles along c, m]
    int64_t rows, blocks, each;
    int32_t m, c, tiles_m, tiles_c;
    int32_t width;  // values of a row of dy: m, or m rounded up where it was laid out anew
};

// A tile of dW: WM x WC wavefronts, each MT x NT matrices of 32 x 32.  A stage is
// 64 rows: dy as it lies ([row][m], a row's 16-byte pieces moved by its number so
// that the transposing reads meet every bank alike) and q ([c][64 rows], moved
// alike), three stages in shared memory: while one is read, the next is there or
// on its way and the one after is asked for.
//
// The sum is kept in units of the current block's scale: at a block's first stage
// it is multiplied by (last scale / this scale), so that one set of registers
// holds it.  Where a scale is 2^20 or more from the one at which the sum began, the sum
// is added to `dweight` and begins anew: any two scales of a sum are so less than 2^40
// apart, and no term leaves fp32's range on its way (quotients of neighbours alone may
// be small and yet multiply to anything, as a channel fades).
//
// PLANES: parts of dy's values, the smallest first.
template <bool HALF, int PLANES, bool LIVE, int MT, int NT, int WM, int WC>
__global__ __launch_bounds__(64 * WM * WC) void staged_kernel(StagedArgs a) {
    constexpr int kWaves = WM * WC, kM = 32 * MT * WM, kC = 32 * NT * WC;
    constexpr int kPieces = kM / 8, kRowsA = 64 / kPieces;           // of a row; rows of a load
    constexpr int kTurn = kPieces >= 16 ? 3 : kPieces / 4 - 1;       // rows whose pieces are moved differently
    constexpr int kLoadsA = kM / 8 / kWaves, kLoadsC = kC / 16 / kWaves;
    constexpr int kBytesA = 64 * kM * 2, kBytesC = kC * 64, kBytesS = kWaves * 256;
    constexpr int kStage = kBytesA + kBytesC + kBytesS;
    constexpr int kLoads = kLoadsA + kLoadsC + 1;
    static_assert(kLoadsA * kWaves * 8 == kM && kLoadsC * kWaves * 16 == kC && NT <= 2, "whole loads");
    __shared__ __attribute__((aligned(1024))) char shared[3 * kStage];
    const uint32_t base = rocket::shared_address(shared);
    const int lane = threadIdx.x % 64, wave = rocket::uniform(threadIdx.x / 64);
    const int wm = wave % WM, wc = wave / WM;
    const uint32_t item = rocket::item_of_block(), tiles = a.tiles_m * a.tiles_c;
    const uint32_t part = item / tiles, tile = item % tiles;
    const int tile_c = tile % a.tiles_c;
    const int m0 = tile / a.tiles_c * kM, c0 = tile_c * kC;
    const int64_t first = part * a.each, last = first + a.each < a.blocks ? first + a.each : a.blocks;
    const int stages = (int)(last - first) * 2 * PLANES;

    // where this lane's pieces of a stage come from
    uint32_t from_a[kLoadsA], from_c[kLoadsC];
    int row_a[kLoadsA];
#pragma unroll
    for (int k = 0; k < kLoadsA; k++) {
        const int row = (wave * kLoadsA + k) * kRowsA + lane / kPieces;
        const int piece = lane % kPieces ^ (row & kTurn) << 2;
        row_a[k] = row;
        from_a[k] = (uint32_t)(row * a.dy_stride) + piece * 16;
    }
#pragma unroll
    for (int k = 0; k < kLoadsC; k++) {
        const int ch = (wave * kLoadsC + k) * 16 + lane / 4;
        from_c[k] = ch * kKeepRows + (lane % 4 ^ (ch >> 2 & 3)) * 16;
    }
    // The stage that is asked for next: its buffers, and then its loads one by one, so
    // that they find room between other work.
    const char *ask_dy = a.dy + first * kKeepRows * a.dy_stride + m0 * 2;
    const int8_t *ask_q = a.q + (first * a.c + c0) * kKeepRows;
    const float *ask_scale = a.scale + first * a.c + c0;
    int64_t ask_rows = a.rows - first * kKeepRows;
    int asked = 0, ask_place = 0;
    uint32_t ask_to = base;
    Int4 dy_buffer, q_buffer, scale_buffer;
    uint64_t live = 0;
    // of a stage's last row this tile's bytes, not those to the row's end: rows that are laid
    // out may be 2^25 bytes apart
    static_assert(63ll * (1 << 25) + kM * 2 <= INT32_MAX, "a stage of the widest rows");
    const int has_c = a.c - c0 < kC ? a.c - c0 : kC, row_bytes = (a.width - m0 < kM ? a.width - m0 : kM) * 2;
    auto open_stage = [&]() {
        const bool some = asked < stages;
        const int s = asked % (2 * PLANES), half = s / PLANES;
        const int rows = !some || ask_rows <= 0 ? 0 : ask_rows < 64 ? (int)ask_rows : 64;
        const int bytes = rows ? (rows - 1) * (int)a.dy_stride + row_bytes : 0;
        dy_buffer = rocket::buffer_of(ask_dy + (PLANES - 1 - s % PLANES) * a.dy_plane, bytes);
        q_buffer = rocket::buffer_of(ask_q + half * 64, some ? has_c * kKeepRows - half * 64 : 0);
        // the scale of the next stage's block: it is looked at before that begins
        const bool after = s == 2 * PLANES - 1;
        scale_buffer =
            rocket::buffer_of(ask_scale + (after ? a.c : 0), asked + (after ? 1 : 0) < stages ? has_c * 4 : 0);
        ask_to = base + ask_place * kStage;
        ask_place = ask_place == 2 ? 0 : ask_place + 1;
        if (LIVE) live = some ? a.live[(a.rows - ask_rows) / 64] : 0;
        if (s % PLANES == PLANES - 1) ask_dy += 64 * a.dy_stride, ask_rows -= 64;
        if (after) ask_q += (int64_t)a.c * kKeepRows, ask_scale += a.c;
        asked++;
    };
    auto ask = [&](int k) {
        if (k < kLoadsA) {
            uint32_t at = from_a[k];
            if (LIVE) at = live >> row_a[k] & 1 ? at : rocket::kNowhere;
            rocket::load_stage16(dy_buffer, ask_to + (wave * kLoadsA + k) * 1024, at);
        } else if (k < kLoadsA + kLoadsC) {
            const int l = k - kLoadsA;
            rocket::load_stage16(q_buffer, ask_to + kBytesA + (wave * kLoadsC + l) * 1024, from_c[l]);
        } else {
            rocket::load_stage4(scale_buffer, ask_to + kBytesA + kBytesC + wave * 256,
                                lane < 32 * NT ? (wc * 32 * NT + lane) * 4 : rocket::kNowhere);
        }
    };

    // where it reads a stage: groups of 16 lanes turn 4 rows of 16 values about
    const int group = lane / 16, in = lane % 16, half = lane / 32;
    uint32_t read_a[MT], read_c[NT];
    const auto place_a = [&](int matrix) {
        const int piece = matrix * 4 + (group & 1) * 2 + in % 4 / 2;
        return (16 * half + in / 4) * (kM * 2) + (piece ^ (in / 4 & kTurn) << 2) * 16 + in % 2 * 8;
    };
#pragma unroll
    for (int k = 0; k < MT; k++) read_a[k] = place_a(wm * MT + k);
    const uint32_t read_b = place_a(wm * MT + (wc < MT ? wc : 0));
#pragma unroll
    for (int k = 0; k < NT; k++) read_c[k] = kBytesA + ((wc * NT + k) * 32 + lane % 32) * 64;
    const int turn_c = lane % 32 >> 2 & 3;
    const uint32_t read_s = kBytesA + kBytesC + wave * 256 + lane % 32 * 4;

    Float16 sum[MT][NT] = {};
    float unit[NT], began[NT], bias = 0.0f;   // the block's scale, and the one at which the sum began
    uint32_t held[NT];
    const int64_t to0 = ((int64_t)part * a.m + m0 + wm * 32 * MT + 4 * half) * a.c + c0 + wc * 32 * NT + lane % 32;
    bool begun = false;   // whether dweight holds a sum already
    // A sum that was put aside begins at 0, and not as a product with 0, which would make a
    // NaN of an infinity.  The zeros are written where the sum lies: as values of the
    // language they make the compiler keep a second sum (50 registers spilled, 813 us in
    // place of 420), and chosen where the next block multiplies they take 444 us.  Of fp32's
    // three parts this here spills 139 registers, and the choice takes 2 % (228 us and 232).
    const auto zeroed = [](float v) {
        asm volatile("v_mov_b32 %0, 0" : "+v"(v));
        return v;
    };
    auto put = [&](bool add, auto anew) {
#pragma unroll
        for (int y = 0; y < NT; y++) {
            float *to = a.dweight + to0 + y * 32;
            int left = c0 + (wc * NT + y) * 32 + lane % 32 < a.c ? a.m - m0 - wm * 32 * MT - 4 * half : 0;
#pragma unroll
            for (int x = 0; x < MT; x++)
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    if (left > 0) *to = (add ? *to : 0.0f) + sum[x][y][i] * unit[y];
                    if constexpr (anew) sum[x][y][i] = zeroed(sum[x][y][i]);
                    to += i % 4 == 3 ? (int64_t)5 * a.c : (int64_t)a.c;
                    left -= i % 4 == 3 ? 5 : 1;
                    asm volatile("" : "+v"(to), "+v"(left)::"memory");   // one after the other: few registers
                }
        }
    };

    float factor[NT];
    bool anew = false;   // the sum was added to dweight and begins at 0
#pragma unroll
    for (int k = 0; k < NT; k++) {
        const int c = c0 + (wc * NT + k) * 32 + lane % 32;
        began[k] = unit[k] = c < a.c ? a.scale[first * a.c + c] : 0.0f;
        held[k] = unit[k] == 0.0f ? 0u : ~0u;
        factor[k] = 1.0f;
    }
#pragma unroll
    for (int early = 0; early < 2; early++) {
        open_stage();
#pragma unroll
        for (int k = 0; k < kLoads; k++) ask(k);
    }
    uint32_t at = base;
    constexpr int kTogether = PLANES == 1 ? 2 : 1;   // stages written out one after the other
    for (int block = 0; block < stages; block += 2 * PLANES) {
#pragma unroll kTogether
        for (int s = 0; s < 2 * PLANES; s++) {
            const int stage = block + s;
            rocket::wait_loads<kLoads>();
            rocket::Shared from[MT];
#pragma unroll
            for (int k = 0; k < MT; k++) from[k] = rocket::shared_at(at + read_a[k]);
            // 4 groups of 16 rows, MT steps each.  A matrix instruction keeps its unit for
            // 8 others' time, so between a step's two there is done what is wanted later:
            // the first operand is read two steps ahead, the second widened a group ahead,
            // the sum of the next step multiplied.
            constexpr int kSteps = 4 * MT;
            Words4 bytes[2][NT], fa[kSteps];
            uint32_t wide[2][NT][4];
#pragma unroll
            for (int k = 0; k < NT; k++)
                bytes[0][k] = *(SharedWords)rocket::shared_at(at + read_c[k] + (half ^ turn_c) * 16);
            const auto read_step = [&](int step) {
                const int g = step / MT;
                fa[step] = turned<kM * 2>(from[step % MT] + (32 * (g / 2) + 8 * (g % 2)) * (kM * 2));
            };
            read_step(0);
            read_step(1);
#pragma unroll
            for (int k = 0; k < NT; k++)
                bytes[1][k] = *(SharedWords)rocket::shared_at(at + read_c[k] + (2 + half ^ turn_c) * 16);
            open_stage();
            const auto widen_word = [&](int group, int k, int w) {
                wide[group % 2][k][w] = widen<HALF>(bytes[group / 2][k][group % 2 * 2 + w / 2] & held[k], w % 2);
            };
            const auto multiply = [&](int x) {
#pragma unroll
                for (int y = 0; y < NT; y++)
#pragma unroll
                    for (int i = 0; i < 16; i++)
                        sum[x][y][i] = PLANES > 1 && anew ? 0.0f : sum[x][y][i] * factor[y];
            };
            if (s == 0) multiply(0);
#pragma unroll
            for (int k = 0; k < NT; k++)
#pragma unroll
                for (int w = 0; w < 4; w++) widen_word(0, k, w);
#pragma unroll
            for (int step = 0; step < kSteps; step++) {
                const int group = step / MT, x = step % MT;
                __builtin_amdgcn_sched_barrier(0);
                if (step + 2 < kSteps) read_step(step + 2);
#pragma unroll
                for (int y = 0; y < NT; y++) {
                    const uint32_t *w = wide[group % 2][y];
                    const Words4 fb = {w[0], w[1], w[2], w[3]};
                    if constexpr (HALF)
                        sum[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(
                            __builtin_bit_cast(Half8, fa[step]), __builtin_bit_cast(Half8, fb), sum[x][y], 0, 0, 0);
                    else
                        sum[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                            __builtin_bit_cast(Bf8, fa[step]), __builtin_bit_cast(Bf8, fb), sum[x][y], 0, 0, 0);
                    if (group < 3)
#pragma unroll
                        for (int w4 = x * 4 / MT; w4 < (x + 1) * 4 / MT; w4++) widen_word(group + 1, y, w4);
                }
                if (s == 0 && step + 1 < MT) multiply(step + 1);
#pragma unroll
                for (int k = step * kLoads / kSteps; k < (step + 1) * kLoads / kSteps; k++) ask(k);
            }
            __builtin_amdgcn_sched_barrier(0);
            // dy's own sums: the tiles along c take the stages in turn, a wavefront one
            // matrix' rows
            if (a.dbias && stage / PLANES % a.tiles_c == tile_c && wc < MT)
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    const Words4 fa =
                        turned<kM * 2>(rocket::shared_at(at + read_b) + (32 * (k / 2) + 8 * (k % 2)) * (kM * 2));
#pragma unroll
                    for (int e = 0; e < 8; e++) bias += value16<HALF>(fa[e / 2], e % 2);
                }
            const uint32_t was = at;
            at = at == base + 2 * kStage ? base : at + kStage;
            if (s < 2 * PLANES - 1) continue;
            // the next block's scale
            float next[NT];
            bool far = false;
#pragma unroll
            for (int k = 0; k < NT; k++) {
                next[k] = *(const __attribute__((address_space(3))) float *)(rocket::shared_at(was + read_s) + k * 128);
                held[k] = next[k] == 0.0f ? 0u : ~0u;   // a scale of 0: whatever q holds counts nothing
                if (next[k] == 0.0f) next[k] = unit[k];
                factor[k] = unit[k] == 0.0f ? 1.0f : unit[k] / next[k];
                if (unit[k] == 0.0f) began[k] = next[k];   // all scales were 0: there is no sum yet
                const float from = __builtin_fabsf(began[k]), to = __builtin_fabsf(next[k]);
                far |= from > 0x1p20f * to || to > 0x1p20f * from;
            }
            anew = __any(far);
            if (anew) {
                // the matrix unit's last results are there before `zeroed`, which the compiler
                // does not see writing their registers, writes them
                asm volatile("s_nop 15\n\ts_nop 15");
                put(begun, std::bool_constant<PLANES == 1>());
                begun = true;
#pragma unroll
                for (int k = 0; k < NT; k++) factor[k] = 1.0f, began[k] = next[k];
            }
#pragma unroll
            for (int k = 0; k < NT; k++) unit[k] = next[k];
        }
    }
    rocket::wait_loads<0>();
    put(begun, std::false_type());
    if (a.dbias) {
        static_assert(MT <= WC, "a wavefront counts at most one matrix' rows");
        bias += __shfl_xor(bias, 32);
        const int m = m0 + (wm * MT + wc) * 32 + lane;
        if (wc < MT && lane < 32 && m < a.m)
            a.dbias[((int64_t)part * a.tiles_c + tile_c) * a.m + m] = bias;
    }
}

// A bit for each row: whether it holds data.
__global__ __launch_bounds__(256) void live_kernel(Rows rows, uint64_t *live) {
    for (int64_t first = (int64_t)blockIdx.x * 256; first < rows.count; first += (int64_t)gridDim.x * 256) {
        const int64_t r = first + threadIdx.x;
        const uint64_t bits = __ballot(r < rows.count && rocket::place_of(rows, r).live);
        if (threadIdx.x % 64 == 0 && r < rows.count) live[r / 64] = bits;
    }
}

// dy's rows laid out for the staged kernel: 16-bit parts, 16-byte aligned rows,
// zeros where a row holds no data.  A thread takes 8 columns.
template <int DT>
__global__ __launch_bounds__(256) void lay_kernel(Rows rows, View dy, int32_t m, int64_t pieces, uint16_t *to,
                                                  int64_t plane, int64_t begin) {
    const int64_t i = begin + (int64_t)blockIdx.x * 256 + threadIdx.x, r = i / pieces;
    if (r >= rows.count) return;
    const int c = (int)(i - r * pieces) * 8;
    using raw = typename Elem<DT>::raw;
    const Place p = rocket::place_of(rows, r);
    raw x[8] = {};
    if (p.live) {
        const raw *from = (const raw *)rocket::row_at(dy, p) + c;
        if (c + 8 <= m)
            __builtin_memcpy(x, from, sizeof(x));
        else
            for (int e = 0; e < 8; e++)
                if (c + e < m) x[e] = from[e];
    }
    uint16_t v[kPlanes<DT>][8];
#pragma unroll
    for (int e = 0; e < 8; e++) {
        uint16_t s[kPlanes<DT>];
        split<DT>(x[e], s);
#pragma unroll
        for (int k = 0; k < kPlanes<DT>; k++) v[k][e] = s[k];
    }
#pragma unroll
    for (int k = 0; k < kPlanes<DT>; k++) rocket::store_at(to + k * plane + i * 8, __builtin_bit_cast(Words4, v[k]));
}

// Sums of `n` parts of `count` values, in an order of their own: few parts by a thread
// a value, many parts (which are of few values: cut_parts) by 16 threads a value.
struct Sums {
    const float *parts;
    float *sum;
    int64_t count;
    int32_t n;
    uint32_t groups;   // workgroups that it takes
};

constexpr int kMany = 32;

Sums sums_of(const float *parts, float *sum, int64_t count, int64_t n) {
    const int64_t each = n > kMany ? 16 : 256;
    return Sums{parts, sum, count, (int32_t)n, n > 1 || parts != sum ? (uint32_t)((count + each - 1) / each) : 0};
}

// Two of them in one launch.
__global__ __launch_bounds__(256) void join_kernel(Sums a, Sums b) {
    __shared__ float shared[16][17];
    const bool second = blockIdx.x >= a.groups;
    const Sums s = second ? b : a;
    const int64_t group = second ? blockIdx.x - a.groups : blockIdx.x;
    if (s.n <= kMany) {
        const int64_t i = group * 256 + threadIdx.x;
        if (i >= s.count) return;
        float v = 0.0f;
        int k = 0;
        for (; k + 8 <= s.n; k += 8) {   // eight loads on their way
            float x[8];
#pragma unroll
            for (int u = 0; u < 8; u++) x[u] = s.parts[(k + u) * s.count + i];
#pragma unroll
            for (int u = 0; u < 8; u++) v += x[u];
        }
        for (; k < s.n; k++) v += s.parts[k * s.count + i];
        s.sum[i] = v;
        return;
    }
    const int col = threadIdx.x % 16, row = threadIdx.x / 16;
    const int64_t c = group * 16 + col;
    float v = 0.0f;
    if (c < s.count)
#pragma unroll 4
        for (int k = row; k < s.n; k += 16) v += s.parts[k * s.count + c];
    shared[row][col] = v;
    __syncthreads();
    if (threadIdx.x >= 16 || c >= s.count) return;
    float t = 0.0f;
#pragma unroll
    for (int k = 0; k < 16; k++) t += shared[k][col];
    s.sum[c] = t;
}

struct Cut {
    bool staged;
    bool lay;                // dy is laid out anew first
    int64_t blocks, each, parts;
    int32_t tile_m;          // channels of dy in a tile; 256 of the checkpoint
    int64_t tiles_m, tiles_c;
    int64_t stride;          // bytes of a laid row
    int64_t at_live, at_bias, at_dy, bytes;   // places in the workspace: after the parts of dW
};

constexpr int64_t kCus = 256;

// The parts of the rows that cost least: workgroups in rounds of `at_once`, a block's
// time in each, and the parts' sums' way through memory.  Times in microseconds.
template <class Time>
double cut_parts(Cut &c, Time time, double part_us) {
    double best = 1e300;
    for (int64_t p = 1; p <= std::min<int64_t>(std::max<int64_t>(c.blocks, 1), 1024); p += 1 + p / 8) {
        const int64_t each = std::max<int64_t>(1, (c.blocks + p - 1) / p);
        const int64_t parts = std::max<int64_t>(1, (c.blocks + each - 1) / each);
        const double us = time(each, parts) + (parts > 1 ? parts * (part_us + 0.02) + 6.0 : 0.0);
        if (us < best) best = us, c.each = each, c.parts = parts;
    }
    return best;
}

// Whether dy's rows are read as they lie: at one distance that lets no row reach into
// the next (those past the last one are told by where they would lie), 4-byte aligned.
bool fits(const rocket_sequence_shape *s, const View &dy) {
    const bool one = s->n == 1 || s->steps == 1 || dy.series == s->steps * dy.step;
    const int64_t step = s->steps == 1 ? dy.series : dy.step;
    return one && s->dtype != ROCKET_FLOAT32 && s->channels % 2 == 0 && step % 4 == 0 && step >= s->channels * 2 &&
           (uintptr_t)dy.data % 4 == 0 && step <= (1 << 24);
}

// How a call is cut.
Cut cut_of(const rocket_sequence_shape *s, int64_t channels, const View &dy) {
    Cut c = {};
    const int64_t rows = s->n * s->steps, m = s->channels;
    c.blocks = (rows + kKeepRows - 1) / kKeepRows;
    const int64_t planes = s->dtype == ROCKET_FLOAT32 ? 3 : 1;
    const double part_us = (double)m * channels * 8 / 4e6;
    // direct tiles: a block takes 1.7 us, or 1.05 us for each tile of a CU (1,000 rows of
    // 192 by 2,000 and of 1,536 by 2,000), of fp32 1.9 times that
    const int64_t tiles = ((m + kTile - 1) / kTile) * ((channels + kTile - 1) / kTile);
    const auto direct = [&](int64_t each, int64_t parts) {
        return 4.0 + each * (planes > 1 ? 1.9 : 1.0) * std::max(1.7, 1.05 * (double)(tiles * parts) / kCus);
    };
    const double direct_us = cut_parts(c, direct, part_us);
    // staged tiles: two workgroups of the smaller ones run beside each other on a CU
    Cut d = c;
    d.tile_m = m <= 32 ? 32 : m <= 64 ? 64 : m <= 128 ? 128 : 256;
    d.tiles_m = (m + d.tile_m - 1) / d.tile_m, d.tiles_c = (channels + 255) / 256;
    d.lay = !fits(s, dy);
    const int64_t at_once = d.tile_m <= 64 ? 2 * kCus : kCus;
    const double block_us = d.tile_m == 256 ? 4.2 : d.tile_m == 128 ? 2.2 : d.tile_m == 64 ? 2.4 : 2.0;
    const auto staged = [&](int64_t each, int64_t parts) {
        return (double)((d.tiles_m * d.tiles_c * parts + at_once - 1) / at_once) * (each * block_us * planes + 5.0);
    };
    // by the shape alone, not by whether these rows have to be laid out anew: results do
    // not change with strides and alignment
    const bool anew = planes > 1 || m % 2 != 0;
    const double staged_us = cut_parts(d, staged, part_us) + (anew ? 9.0 : 6.0);
    // no rows: the staged kernel would read the first block's scales, which is not there;
    // the direct one reads nothing and writes zeros
    if (rows > 0 && staged_us < direct_us) {
        c = d;
        c.staged = true;
        c.stride = (m + 7) / 8 * 16;
        c.at_bias = c.parts > 1 ? c.parts * m * channels * 4 : 0;
        c.at_live = (c.at_bias + c.parts * c.tiles_c * m * 4 + 15) / 16 * 16;
        c.at_dy = c.at_live + (c.blocks * 16 + 15) / 16 * 16;
        c.bytes = c.at_dy + (c.lay ? planes * rows * c.stride : 0);
    } else {
        c.at_bias = c.parts * m * channels * 4;
        c.bytes = c.parts > 1 ? c.at_bias + c.parts * m * 4 : 0;
    }
    c.bytes = (c.bytes + 7) / 8 * 8;
    return c;
}

template <bool HALF, int PLANES, int MT, int WM>
void staged_tiles(const StagedArgs &a, int64_t parts, hipStream_t s) {
    const uint32_t grid = (uint32_t)(parts * a.tiles_m * a.tiles_c), threads = 64 * WM * 4;
    if (a.live)
        staged_kernel<HALF, PLANES, PLANES == 1, MT, 2, WM, 4><<<grid, threads, 0, s>>>(a);
    else
        staged_kernel<HALF, PLANES, false, MT, 2, WM, 4><<<grid, threads, 0, s>>>(a);
}

template <bool HALF, int PLANES>
void staged_launch(const StagedArgs &a, const Cut &cut, hipStream_t s) {
    if (cut.tile_m == 32)
        staged_tiles<HALF, PLANES, 1, 1>(a, cut.parts, s);
    else if (cut.tile_m == 64)
        staged_tiles<HALF, PLANES, 2, 1>(a, cut.parts, s);
    else if (cut.tile_m == 128)
        staged_tiles<HALF, PLANES, 4, 1>(a, cut.parts, s);
    else
        staged_tiles<HALF, PLANES, 4, 2>(a, cut.parts, s);
}

bool sizes_ok(const rocket_sequence_shape *s, int64_t channels) {
    return rocket::shape_ok(s) && channels > 0 && channels <= (1 << 24) && s->channels * channels <= ((int64_t)1 << 34);
}

}  // namespace

extern "C" rocket_status rocket_linear_weight_gradient_workspace(const rocket_sequence_shape *shape, int64_t channels,
                                                                 const rocket_sequence *dy, int64_t *bytes) {
    if (!bytes || !sizes_ok(shape, channels) || !rocket::view_ok(dy, shape)) return ROCKET_ERR_INVALID_ARG;
    View view = rocket::view_of(dy, shape->dtype);
    *bytes = cut_of(shape, channels, view).bytes;
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
    View dy_view = rocket::view_of(dy, shape->dtype);
    const Cut cut = cut_of(shape, channels, dy_view);
    if (cut.bytes && (!workspace || (uintptr_t)workspace % 8 != 0 || workspace_bytes < cut.bytes))
        return ROCKET_ERR_INVALID_ARG;
    View *views[] = {&dy_view};
    const Rows rows = rocket::rows_of(shape, views, 1);
    const int32_t m = (int32_t)shape->channels, c = (int32_t)channels;
    const int64_t count = (int64_t)m * c;
    hipStream_t s = (hipStream_t)hip_stream;
    char *work = (char *)workspace;
    float *parts = cut.parts > 1 ? (float *)work : dweight;
    int64_t biases;
    if (cut.staged) {
        StagedArgs a = {};
        a.q = q, a.scale = scale, a.dweight = parts, a.dbias = dbias ? (float *)(work + cut.at_bias) : nullptr;
        a.rows = rows.count, a.blocks = cut.blocks, a.each = cut.each;
        a.m = m, a.c = c, a.tiles_m = (int32_t)cut.tiles_m, a.tiles_c = (int32_t)cut.tiles_c;
        biases = cut.parts * cut.tiles_c;
        a.width = cut.lay ? (int32_t)(cut.stride / 2) : m;
        if (!cut.lay) {
            a.dy = dy_view.data, a.dy_stride = shape->steps == 1 ? dy_view.series : dy_view.step;
            if (rows.lengths) {
                a.live = (const uint64_t *)(work + cut.at_live);
                const uint32_t grid = (uint32_t)std::min<int64_t>((rows.count + 255) / 256, 8 * kCus);
                live_kernel<<<grid, 256, 0, s>>>(rows, (uint64_t *)(work + cut.at_live));
            }
        } else {
            const int64_t pieces = cut.stride / 16, items = rows.count * pieces, most = rocket::most_groups(256) * 256;
            a.dy = work + cut.at_dy, a.dy_stride = cut.stride, a.dy_plane = rows.count * cut.stride;
            for (int64_t at = 0; at < items; at += most) {
                const uint32_t grid = (uint32_t)((std::min(items - at, most) + 255) / 256);
                uint16_t *to = (uint16_t *)(work + cut.at_dy);
                if (shape->dtype == ROCKET_FLOAT32)
                    lay_kernel<ROCKET_FLOAT32><<<grid, 256, 0, s>>>(rows, dy_view, m, pieces, to, a.dy_plane / 2, at);
                else  // 16-bit values are moved as they are
                    lay_kernel<ROCKET_BFLOAT16><<<grid, 256, 0, s>>>(rows, dy_view, m, pieces, to, a.dy_plane / 2, at);
            }
        }
        if (shape->dtype == ROCKET_FLOAT32)
            staged_launch<false, 3>(a, cut, s);
        else if (shape->dtype == ROCKET_BFLOAT16)
            staged_launch<false, 1>(a, cut, s);
        else
            staged_launch<true, 1>(a, cut, s);
    } else {
        GradArgs a = {};
        a.rows = rows, a.dy = dy_view, a.q = q, a.scale = scale, a.m = m, a.c = c;
        a.blocks = cut.blocks, a.each = cut.each, a.dweight = parts;
        a.dbias = !dbias ? nullptr : cut.parts > 1 ? (float *)(work + cut.at_bias) : dbias;
        biases = cut.parts;
        const uint32_t grid = (uint32_t)((c + kTile - 1) / kTile * ((m + kTile - 1) / kTile) * cut.parts);
        if (shape->dtype == ROCKET_FLOAT32)
            gradient_kernel<ROCKET_FLOAT32><<<grid, 256, 0, s>>>(a);
        else if (shape->dtype == ROCKET_BFLOAT16)
            gradient_kernel<ROCKET_BFLOAT16><<<grid, 256, 0, s>>>(a);
        else
            gradient_kernel<ROCKET_FLOAT16><<<grid, 256, 0, s>>>(a);
    }
    const Sums first = sums_of(parts, dweight, count, cut.parts);
    Sums second = {};
    if (dbias && (cut.staged || cut.parts > 1))
        second = sums_of((const float *)(work + cut.at_bias), dbias, m, biases);
    if (first.groups + second.groups > 0) join_kernel<<<first.groups + second.groups, 256, 0, s>>>(first, second);
    return rocket::launched();
}
