// Product of 8-bit rows with 8-bit weights.
//
//   y[t, m] = scale[t] wscale[m] (sum over k of q[t, k] p[m, k]) + bias[m]
//
// The sum is of whole numbers and exact: 32 bits hold it up to 131,072 columns (2^31 of
// -128 by -128 in all of them is told from -2^31, which no sum reaches).
// Scales and bias are fp32, the result is rounded once.
//
// Bound: few rows by reading the weights, many by the matrix unit (2,440 TOP/s in a
// library's product of 8,192) and its clock, which falls to 2.0 GHz and below under it.
// Measured, bf16 results where nothing else is said:
//   64 rows, 2,000 by 1,536 channels           7.6 us (a row by 192 channels: 3.9)
//   64 x 1000 rows, 2,000 by 1,536             211 to 225 us by the card, 1,750 to 1,860
//                                              TOP/s; without writing results 170
//   777 x 129 rows, half of them empty, 924 by 993, fp16    94 to 117 us, by how far the
//                                              tiles fill their three or four rounds, where
//                                              the 199 MB of results are in the last-level
//                                              cache already; 142 to 150 where they are not
#include <algorithm>

#include "rows.h"
#include "stage.h"
#include "walk.h"

namespace {

using rocket::Int4;

using rocket::Elem;
using rocket::Place;
using rocket::Rows;
using rocket::Tile;
using rocket::View;

typedef int Int16 __attribute__((ext_vector_type(16)));

// The most columns: 2^31 / 2^14.  The sum 2^31 arrives as -2^31, which stands for nothing
// else (128 * 127 * 131,072 is less); as 2^31 - 1 it is 2^31 again once it is fp32.
constexpr int kMostColumns = 131072;

__device__ inline int held_sum(int sum) { return sum == INT32_MIN ? INT32_MAX : sum; }

struct ProductArgs {
    Rows rows;
    const int8_t *q, *p;
    const float *scale, *wscale, *bias;  // bias or null
    View y;
    int32_t columns;   // of q and p: a multiple of 64
    int32_t channels;  // of y
    int32_t tiles;     // along the channels
    int32_t parts, each;   // of the columns' stages, and stages of a part
    int32_t *sums;         // [parts, rows, channels]
    const int32_t *order;  // [rows + 1]: order_kernel's
};

// Few rows: what bounds them is reading the weights, so a workgroup takes 16 channels
// and up to 64 rows, and its 16 wavefronts share the columns: each reads 64 columns
// at once straight into the operands' registers (16 lines of 64 bytes), several
// ahead; their sums meet in shared memory.  64 rows of 2,048 by 1,536 channels: 96
// workgroups.
//
// Matrix instruction 16 x 16 x 64: the first operand's lane holds 16 bytes of row
// lane % 16, the second's of column lane % 16, both the quarter lane / 16 of the 64;
// result i of a lane is row 4 (lane / 16) + i of column lane % 16.  The first operand
// is the weights.
constexpr int kFewRows = 64, kFewChannels = 16, kFewWaves = 16;

template <int DT, int NT>
__global__ __launch_bounds__(64 * kFewWaves) void few_kernel(ProductArgs a) {
    __shared__ int sums[kFewWaves][NT][kFewChannels][17];
    const int lane = threadIdx.x % 64, wave = rocket::uniform(threadIdx.x / 64);
    const int m0 = blockIdx.x * kFewChannels, m = m0 + lane % 16;
    // lines that are not there are read as the last one, and not written
    const int8_t *p = a.p + (int64_t)(m < a.channels ? m : a.channels - 1) * a.columns + lane / 16 * 16;
    const int8_t *q[NT];
#pragma unroll
    for (int y = 0; y < NT; y++) {
        const int64_t r = y * 16 + lane % 16;
        q[y] = a.q + (r < a.rows.count ? r : a.rows.count - 1) * a.columns + lane / 16 * 16;
    }
    Int4 sum[NT] = {};
    constexpr int kAhead = 4;
    const int stages = a.columns / 64;
    for (int k0 = wave; k0 < stages; k0 += kAhead * kFewWaves) {
        Int4 fm[kAhead], ft[kAhead][NT];
#pragma unroll
        for (int u = 0; u < kAhead; u++) {
            const int k = k0 + u * kFewWaves;
            if (k >= stages) continue;
            fm[u] = *(const Int4 *)(p + k * 64);
#pragma unroll
            for (int y = 0; y < NT; y++) ft[u][y] = *(const Int4 *)(q[y] + k * 64);
        }
#pragma unroll
        for (int u = 0; u < kAhead; u++) {
            if (k0 + u * kFewWaves >= stages) continue;
#pragma unroll
            for (int y = 0; y < NT; y++)
                sum[y] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fm[u], ft[u][y], sum[y], 0, 0, 0);
        }
    }
#pragma unroll
    for (int y = 0; y < NT; y++)
#pragma unroll
        for (int i = 0; i < 4; i++) sums[wave][y][4 * (lane / 16) + i][lane % 16] = sum[y][i];
    __syncthreads();
    const int c = threadIdx.x % 16, t = threadIdx.x / 16;
    if (t >= 16 * NT || t >= a.rows.count || m0 + c >= a.channels) return;
    uint32_t sum_of_waves = 0;
#pragma unroll
    for (int w = 0; w < kFewWaves; w++) sum_of_waves += (uint32_t)sums[w][t / 16][c][t % 16];
    const int total = held_sum((int)sum_of_waves);
    const Place place = rocket::place_of(a.rows, t);
    const float bias = a.bias ? a.bias[m0 + c] : 0.0f;
    const float v = place.live ? __builtin_fmaf((float)total, a.scale[t] * a.wscale[m0 + c], bias) : 0.0f;
    using raw = typename Elem<DT>::raw;
    ((raw *)rocket::row_at(a.y, place))[m0 + c] = Elem<DT>::round(v);
}

// Matrix instruction 32 x 32 x 32: the first operand's lane holds 16 bytes of row
// lane % 32, the second's of column lane % 32, both the half lane / 32 of the 32;
// result i of a lane is row 8 (i / 4) + 4 (lane / 32) + i % 4 of column lane % 32.
// The first operand is the weights, so that a lane has four channels in a row of one
// y row.

// A sum from an accumulation register, just where it is used: left to itself the
// compiler copies all of them at once and has to spill.
template <bool ACC>
__device__ inline int taken(int sum) {
    if (!ACC) return sum;
    int v;
    asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v) : "a"(sum));
    return v;
}

// Tiles of y by WM x WT wavefronts, each MT x NT matrices of 32 channels x 32 rows.
//
// A stage is 64 columns of the tile's weights and rows, 64 bytes a line in shared
// memory, a line's four pieces of 16 bytes moved by its number so that the reads of
// 32 lines meet every bank alike.  Three or four stages are there or on their way.  A stage
// is two steps of 32 columns; while the matrix unit works on one step's operands,
// the next step's are read into other registers, over the borders of stages too:
// what a barrier says is that the next stage has arrived and that this one has
// been read, and it stands where the matrix unit still has work.
//
// A workgroup goes from tile to tile, and the stages go on over their borders: while
// a tile's results are written, the next one's first stages arrive.
//
// SPLIT (of DT fp32): few tiles of many columns; a workgroup takes some of one tile's
// stages and leaves their sums, whole numbers, to finish_kernel.
//
// LIVE: the tiles are of the rows that hold data, one behind the other as order_kernel
// lists them; the others are zeroed at the end, most of them by the workgroups that have
// a tile less.  A row's place in q is looked up two tiles ahead, since the next tile's
// stages are on their way when this one's results are written; so a tile must have as
// many stages as there are slots.  777 series of up to 129 steps, half of the rows, of
// 960 columns by 993 channels, into one place: 111 us, and 172 where empty rows are
// multiplied like the others; where all rows hold data the list costs 6 us.
template <int DT, bool SPLIT, bool LIVE, int MT, int NT, int WM, int WT, int COLS, int SLOTS, int AT_ONCE>
__global__ __launch_bounds__(64 * WM * WT, AT_ONCE) void tile_kernel(ProductArgs a) {
    constexpr int kWaves = WM * WT, kThreads = 64 * kWaves, kM = 32 * MT * WM, kT = 32 * NT * WT, kSlots = SLOTS;
    constexpr int kPieces = COLS / 16, kLines = 64 / kPieces;   // of a line; lines of a load
    constexpr int kLoadsM = kM / kLines / kWaves, kLoadsT = kT / kLines / kWaves, kLoads = kLoadsM + kLoadsT;
    constexpr int kStage = (kM + kT) * COLS, kSteps = COLS / 32, kProducts = MT * NT, kReads = MT + NT;
    constexpr int kSize = Elem<DT>::kSize;
    // results on their way: 32 rows of 128 bytes (64 where there are no more) a wavefront
    constexpr int kAcross = kSize == 2 && MT > 1 ? 2 : 1, kRowBytes = 32 * kAcross * kSize, kLine = kRowBytes + 16;
    constexpr int kTable = 8 * kM + 12 * kT, kOut = kSlots * kStage, kTables = kOut + kWaves * 32 * kLine;
    typedef float Float4 __attribute__((ext_vector_type(4)));
    typedef uint32_t Words __attribute__((ext_vector_type(kSize)));   // four values
    static_assert(kLoadsM * kWaves * kLines == kM && kLoadsT * kWaves * kLines == kT, "whole loads");
    static_assert(kM <= kThreads && kT <= kThreads, "a thread for each line of a table");
    // Tiles that tell a sum of 2^31 from -2^31; cut_of gives the others no call of that many
    // columns.  The same in tiles of 256 x 256 spills 150 registers, and in those of 64 x 64
    // it takes 5 us (1,000 rows of 1,984 columns by 1,536 channels 14 us, 19 so); here nothing.
    constexpr bool kTellsMost = !SPLIT && !LIVE && kProducts == 4 && COLS == 64;
    constexpr int kSources = kTables + 2 * kTable;   // LIVE: where the lines of two tiles' rows lie in q
    __shared__ __attribute__((aligned(1024))) char shared[kSources + (LIVE ? 8 * kT : 0)];
    const uint32_t base = rocket::shared_address(shared);
    const int lane = threadIdx.x % 64, wave = rocket::uniform(threadIdx.x / 64);
    const int wm = wave % WM, wt = wave / WM, half = lane / 32;
    const int all_stages = (a.columns + COLS - 1) / COLS;
    const uint32_t group = rocket::item_of_block();
    const int part = SPLIT ? (int)(group % a.parts) : 0, stage0 = part * a.each;
    const int stages = SPLIT ? (all_stages - stage0 < a.each ? all_stages - stage0 : a.each) : all_stages;

    // tiles: this workgroup's first one, and the way to its next
    const int64_t first = SPLIT ? group / a.parts : group;
    const rocket::Steps steps = {SPLIT ? INT32_MAX : (int64_t)gridDim.x / a.tiles, (int)(gridDim.x % a.tiles), a.tiles};
    Tile tile = {first / a.tiles, (int)(first % a.tiles)};
    const int64_t count = LIVE ? a.order[a.rows.count] : a.rows.count, tiles_t = (count + kT - 1) / kT;

    // a line's pieces are moved by its number, so that 16 lines in a row meet every bank alike
    const auto turn_of = [](int line) { return COLS == 64 ? line >> 2 & 3 : line >> 1 & 7; };
    // the stage that is asked for next
    uint32_t from[kLoads];   // where this lane's pieces of a stage come from
#pragma unroll
    for (int k = 0; k < kLoads; k++) {
        const int line = (k < kLoadsM ? wave * kLoadsM + k : wave * kLoadsT + k - kLoadsM) * kLines + lane / kPieces;
        from[k] = line * a.columns + (lane % kPieces ^ turn_of(line)) * 16;
    }
    // 128 columns: the last stage may have 64, and the pieces past them read nothing
    uint32_t rest[2] = {0, 0}, past[2] = {0, 0};
    if (COLS == 128 && a.columns % COLS)
#pragma unroll
        for (int k = 0; k < 2; k++)
            rest[k] = (lane % kPieces ^ turn_of(k * kLines + lane / kPieces)) >= kPieces / 2 ? rocket::kNowhere : 0;
    rocket::Asked asked = {tile, 0, true};
    int ask_slot = 0, ask_turn = 0;
    uint32_t ask_at = 0, ask_to = base;
    Int4 weights, rows;
    const auto open_tile = [&]() {
        const int64_t first_t = asked.tile.t * kT, first_m = (int64_t)asked.tile.m * kM;
        asked.there = first_t < count;
        weights = rocket::buffer_of(a.p + first_m * a.columns,
                                    asked.there ? rocket::bytes_of_lines(a.channels, first_m, kM, a.columns) : 0);
        if (LIVE) {
            rows = rocket::buffer_of(a.q, a.rows.count * a.columns);
            const uint32_t *sources = (const uint32_t *)(shared + kSources) + ask_turn * kT;
            ask_turn ^= 1;
#pragma unroll
            for (int k = 0; k < kLoadsT; k++) {
                const int line = (wave * kLoadsT + k) * kLines + lane / kPieces;
                from[kLoadsM + k] = sources[line] + (lane % kPieces ^ turn_of(line)) * 16;
            }
        } else {
            rows = rocket::buffer_of(a.q + first_t * a.columns, rocket::bytes_of_lines(count, first_t, kT, a.columns));
        }
    };
    const auto open_stage = [&]() {
        if (asked.crosses(stages, steps)) open_tile();
        ask_at = asked.next(stage0, COLS);
        if (COLS == 128)
            for (int k = 0; k < 2; k++) past[k] = stage0 + asked.stage == all_stages ? rest[k] : 0;
        ask_to = base + ask_slot * kStage;
        ask_slot = (ask_slot + 1) % kSlots;
    };
    const auto ask = [&](int k) {
        if (k < kLoadsM)
            rocket::load_stage16(weights, ask_to + (wave * kLoadsM + k) * 1024, from[k] | past[k % 2], ask_at);
        else
            rocket::load_stage16(rows, ask_to + kM * COLS + (wave * kLoadsT + k - kLoadsM) * 1024,
                                 from[k] | past[k % 2], ask_at);
    };

    // a tile's scales, bias and where its rows lie: a row that holds no data has its
    // address's lowest bit set, one that is not there is 0
    struct Table {
        float wscale, bias, scale;
        uint64_t at;
    };
    const auto row_of = [&](Tile x) -> int64_t {   // -1: not there
        const int64_t r = x.t * kT + threadIdx.x;
        return threadIdx.x >= kT || r >= count ? -1 : LIVE ? a.order[r] : r;
    };
    const auto look_up = [&](Tile x, int64_t r) {
        Table v = {};
        const int k = threadIdx.x, m = x.m * kM + k;
        if (!SPLIT && k < kM && m < a.channels) v.wscale = a.wscale[m], v.bias = a.bias ? a.bias[m] : 0.0f;
        if (r >= 0) {
            const Place p = rocket::place_of(a.rows, r);
            v.scale = SPLIT ? 0.0f : a.scale[r];
            char *to = SPLIT ? (char *)(a.sums + (part * a.rows.count + r) * a.channels) : rocket::row_at(a.y, p);
            v.at = (uint64_t)(to + (int64_t)x.m * kM * kSize) | (SPLIT || LIVE || p.live ? 0 : 1);
        }
        return v;
    };
    const auto write_table = [&](const Table &v, int turn) {
        float *to = (float *)(shared + kTables + turn * kTable);
        const int k = threadIdx.x;
        if (k < kM) to[k] = v.wscale, to[kM + k] = v.bias;
        if (k < kT) to[2 * kM + k] = v.scale, ((uint64_t *)(to + 2 * kM + kT))[k] = v.at;
    };
    const auto write_sources = [&](int64_t r, int turn) {
        if (threadIdx.x < kT)
            ((uint32_t *)(shared + kSources))[turn * kT + threadIdx.x] =
                r < 0 ? rocket::kNowhere : (uint32_t)r * (uint32_t)a.columns;
    };
    int64_t coming = row_of(tile);
    write_table(look_up(tile, coming), 0);
    if (LIVE) {
        write_sources(coming, 0);
        coming = row_of(steps.after(tile));
        write_sources(coming, 1);
        __syncthreads();
    }

    // where it reads a stage: a step's pieces are the first one's with the higher bits turned
    typedef const __attribute__((address_space(3))) Int4 *SharedInt4;
    const uint32_t piece = (half ^ turn_of(lane % 32)) * 16 + lane % 32 * COLS;
    const uint32_t read_m = wm * MT * 32 * COLS + piece, read_t = (kM + wt * NT * 32) * COLS + piece;
    Int16 sum[MT][NT];
    Int4 fm[2][MT], ft[2][NT];
    const auto read = [&](int step, uint32_t at, int k) {
        if (k < MT)
            fm[step % 2][k] = *(SharedInt4)(rocket::shared_at((at + read_m) ^ step * 32) + k * 32 * COLS);
        else
            ft[step % 2][k - MT] = *(SharedInt4)(rocket::shared_at((at + read_t) ^ step * 32) + (k - MT) * 32 * COLS);
    };
    // the k-th operand of a step in the order in which its products need them
    const auto order = [](int k) { return k == 0 ? 0 : k <= NT ? MT + k - 1 : k - NT; };
    open_tile();
#pragma unroll
    for (int early = 0; early < kSlots; early++) {
        open_stage();
#pragma unroll
        for (int k = 0; k < kLoads; k++) ask(k);
    }
    rocket::wait_loads<(kSlots - 1) * kLoads>();
#pragma unroll
    for (int k = 0; k < kReads; k++) read(0, base, order(k));
    constexpr int kMeet = kProducts - 1 - kProducts / 4;   // the product after which the wavefronts meet
    int slot = 0;
    for (int turn = 0; tile.t < tiles_t; turn ^= 1) {
#pragma unroll
        for (int x = 0; x < MT; x++)
#pragma unroll
            for (int y = 0; y < NT; y++) sum[x][y] = Int16{};
        for (int stage = 0; stage < stages; stage++) {
            const uint32_t at = base + slot * kStage;
            slot = (slot + 1) % kSlots;
            const uint32_t next = base + slot * kStage;
#pragma unroll
            for (int step = 0; step < kSteps; step++) {
                // the wavefronts meet in the last step but one, which reads the last one's operands
                const bool meets = step == kSteps - 2, ends = step == kSteps - 1;
                const int within = meets ? kMeet + 1 : kProducts;
                if (ends) open_stage();
#pragma unroll
                for (int k = 0; k < kProducts; k++) {
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int r = k * kReads / within; r < (k + 1) * kReads / within && r < kReads; r++)
                        read(ends ? 0 : step + 1, ends ? next : at, order(r));
                    sum[k / NT][k % NT] = __builtin_amdgcn_mfma_i32_32x32x32_i8(
                        fm[step % 2][k / NT], ft[step % 2][k % NT], sum[k / NT][k % NT], 0, 0, 0);
                    if (meets && k == kMeet) {
                        __builtin_amdgcn_sched_barrier(0);
                        rocket::wait_loads<(kSlots - 2) * kLoads>();
                    }
                    if (ends)
#pragma unroll
                        for (int l = k * kLoads / kProducts; l < (k + 1) * kLoads / kProducts; l++) ask(l);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }

        // A lane has four channels in a row, eight apart, of one row of y.  They go through
        // shared memory, each wavefront's its own, so that a row's channels are written side
        // by side.
        // (the matrix unit's last results reach their registers 18 cycles after they are asked
        // for, which the compiler does not see that `taken` reads)
        asm volatile("s_nop 15\n\ts_nop 15");
        if (kTellsMost && a.columns == kMostColumns)
#pragma unroll
            for (int x = 0; x < MT; x++)
#pragma unroll
                for (int y = 0; y < NT; y++)
#pragma unroll
                    for (int i = 0; i < 16; i++) sum[x][y][i] = held_sum(sum[x][y][i]);
        const Tile following = steps.after(tile);
        const Table table = look_up(following, LIVE ? coming : row_of(following));
        if (LIVE) coming = row_of(steps.after(following));
        const float *factors = (const float *)(shared + kTables + turn * kTable), *row_scale = factors + 2 * kM;
        const uint64_t *row_at = (const uint64_t *)(row_scale + kT);
        const int left_m = a.channels - tile.m * kM;
        constexpr int kLanes = kRowBytes / 16, kEach = 16 / kSize;   // lanes that write a row; values of a lane
        char *mine = shared + kOut + wave * 32 * kLine;
#pragma unroll
        for (int x0 = 0; x0 < MT; x0 += kAcross) {
            const int m0 = (wm * MT + x0) * 32, c = m0 + lane % kLanes * kEach;
            Float4 wscale[kAcross][4], bias[kAcross][4];
#pragma unroll
            for (int x = 0; x < kAcross; x++)
#pragma unroll
                for (int g = 0; g < 4; g++) {
                    wscale[x][g] = *(const Float4 *)(factors + m0 + x * 32 + 8 * g + 4 * half);
                    bias[x][g] = *(const Float4 *)(factors + kM + m0 + x * 32 + 8 * g + 4 * half);
                }
#pragma unroll
            for (int y = 0; y < NT; y++) {
                const int t = (wt * NT + y) * 32;
                const float scale = row_scale[t + lane % 32];
                const uint32_t held = row_at[t + lane % 32] & 1 ? 0u : ~0u;
#pragma unroll
                for (int x = 0; x < kAcross; x++)
#pragma unroll
                    for (int g = 0; g < 4; g++) {
                        float v[4];
#pragma unroll
                        for (int e = 0; e < 4; e++)
                            v[e] = __builtin_fmaf((float)taken<kProducts >= 16>(sum[x0 + x][y][4 * g + e]),
                                                  scale * wscale[x][g][e], bias[x][g][e]);
                        Words w;
#pragma unroll
                        for (int e = 0; e < kSize; e++)
                            w[e] = SPLIT ? (uint32_t)taken<kProducts >= 16>(sum[x0 + x][y][4 * g + e])
                                         : Elem<DT>::put(v + e * Elem<DT>::kPerWord) & held;
                        *(Words *)(mine + lane % 32 * kLine + (x * 32 + 8 * g + 4 * half) * kSize) = w;
                    }
#pragma unroll
                for (int k = 0; k < kLanes / 2; k++) {
                    const int row = k * (64 / kLanes) + lane / kLanes;
                    const uint32_t *own = (const uint32_t *)(mine + row * kLine + lane % kLanes * 16);
                    const Int4 v = *(const Int4 *)own;
                    char *to = (char *)(row_at[t + row] & ~(uint64_t)1);
                    if (!to || c >= left_m) continue;
                    to += c * kSize;
                    if (c + kEach <= left_m) {
                        rocket::store_at(to, v);
                    } else {
                        using bits = typename Elem<DT>::bits;
                        for (int e = 0; e < kEach && c + e < left_m; e++) ((bits *)to)[e] = ((const bits *)own)[e];
                    }
                }
            }
        }
        write_table(table, turn ^ 1);
        if (LIVE) write_sources(coming, turn);
        tile = following;
    }
    if (LIVE) {
        // a wavefront takes some rows at a time, whose places its lanes look up at once
        constexpr int kSome = 16, kEach = 16 / kSize;
        const Int4 zero = {0, 0, 0, 0};
        const int64_t some = (a.rows.count - count + kSome - 1) / kSome;
        // workgroups with a tile more, and what a tile is worth in zeros
        const int64_t more = tiles_t * a.tiles % gridDim.x, fewer = gridDim.x - more;
        const int64_t worth = more ? ((int64_t)stages * COLS * kM * kT / 400 + kM * kT * 2) / (kSome * kSize * a.channels) : 0;
        const int64_t each = some > fewer * worth ? (some - fewer * worth) / gridDim.x : 0;   // of those with more
        const int64_t rest = some - more * each, mine = (rest + fewer - 1) / fewer;
        const int64_t from_some = group < more ? rest + group * each : (group - more) * mine;
        const int64_t to_some = group < more ? from_some + each : std::min(from_some + mine, rest);
        for (int64_t u = from_some + wave; u < to_some; u += kWaves) {
            const int64_t d = count + u * kSome;
            const int places = (int)std::min<int64_t>(kSome, a.rows.count - d);
            const int32_t r = a.order[d + std::min(lane, places - 1)];
            for (int k = 0; k < places; k++) {
                char *to = rocket::row_at(a.y, rocket::place_of(a.rows, __builtin_amdgcn_readlane(r, k)));
                for (int c = lane * kEach; c < a.channels; c += 64 * kEach) {
                    if (c + kEach <= a.channels) {
                        rocket::store_at(to + (int64_t)c * kSize, zero);
                    } else {
                        using bits = typename Elem<DT>::bits;
                        for (int e = c; e < a.channels; e++) ((bits *)to)[e] = 0;
                    }
                }
            }
        }
    }
    rocket::wait_loads<0>();
}

// Rows that hold data, then those that do not, each in their order, and how many do: a
// workgroup some series, after it has counted the rows before them.
__global__ __launch_bounds__(256) void order_kernel(Rows rows, int32_t each, int32_t *order) {
    __shared__ int32_t counts[2][4];
    const int first = blockIdx.x * each, end = std::min(first + each, rows.n);
    const auto held = [&](int i) { return std::max(0, std::min(rows.lengths[i], rows.steps)); };
    int32_t all = 0, before = 0;
    for (int i = threadIdx.x; i < rows.n; i += 256) {
        const int32_t here = held(i);
        all += here;
        if (i < first) before += here;
    }
#pragma unroll
    for (int k = 32; k; k /= 2) all += __shfl_xor(all, k), before += __shfl_xor(before, k);
    if (threadIdx.x % 64 == 0) counts[0][threadIdx.x / 64] = all, counts[1][threadIdx.x / 64] = before;
    __syncthreads();
    all = counts[0][0] + counts[0][1] + counts[0][2] + counts[0][3];
    before = counts[1][0] + counts[1][1] + counts[1][2] + counts[1][3];
    for (int i = first; i < end; i++) {
        const int32_t here = held(i), row = i * rows.steps, dead = all + row - before;
        for (int t = threadIdx.x; t < rows.steps; t += 256)
            order[t < here ? before + t : dead + t - here] = row + t;
        before += here;
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) order[rows.count] = all;
}

// The results of split tiles: a thread an element, in the order of the sums.
template <int DT>
__global__ __launch_bounds__(256) void finish_kernel(ProductArgs a) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, r = i / a.channels, count = a.rows.count * a.channels;
    if (r >= a.rows.count) return;
    const int m = (int)(i - r * a.channels);
    uint32_t sum_of_parts = 0;
    for (int k = 0; k < a.parts; k++) sum_of_parts += (uint32_t)a.sums[k * count + i];
    const int total = held_sum((int)sum_of_parts);
    const Place place = rocket::place_of(a.rows, r);
    const float bias = a.bias ? a.bias[m] : 0.0f;
    const float v = place.live ? __builtin_fmaf((float)total, a.scale[r] * a.wscale[m], bias) : 0.0f;
    using raw = typename Elem<DT>::raw;
    ((raw *)rocket::row_at(a.y, place))[m] = Elem<DT>::round(v);
}

constexpr int64_t kCus = 256;

// How a call is cut, by what each way costs: rounds of workgroups, each with its
// stages of 64 columns and the writing of its results (microseconds as measured with
// 128 to 2,048 columns and 256 to 1,536 channels on 1,000 to 300,000 rows).
enum Way { kFew, kBig, kTall, kMiddle, kMiddleTwice, kSmall, kSplit };

struct Cut {
    Way way;
    int32_t parts, each;
    int64_t bytes;
    bool live;   // where lengths are given, the rows that hold data are listed first
};

constexpr int64_t kMostSeries = 4096;   // that order_kernel's workgroups count, each all of them

Cut cut_of(const rocket_sequence_shape *s, int64_t columns) {
    const int64_t rows = s->n * s->steps, channels = s->channels, steps = s->steps;
    Cut c = {kFew, 1, 0, 0, false};
    if (rows <= kFewRows) return c;
    struct Cost {
        Way way;
        int m, t, at_once;
        double stage, end;
    };
    constexpr Cost kCosts[] = {{kBig, 256, 256, 1, 0.80, 8.0},   {kTall, 256, 128, 1, 0.52, 3.8},
                               {kMiddle, 128, 128, 1, 0.285, 2.3}, {kMiddleTwice, 128, 128, 2, 0.56, 3.2},
                               {kSmall, 64, 64, 2, 0.26, 1.1}};
    const double stages = (double)(columns / 64);
    double best = 1e300;
    int64_t rounds = 0;
    for (const Cost &k : kCosts) {
        if (columns == kMostColumns && k.way != kMiddleTwice) continue;   // kTellsMost
        const int64_t tiles = (rows + k.t - 1) / k.t * ((channels + k.m - 1) / k.m), all = k.at_once * kCus;
        // two on a CU: a last round of few tiles goes faster
        const double rest = (double)(tiles % all) / (double)all;
        const double last = k.at_once == 1 ? 1.0 : std::min(1.0, 0.4 + 2.0 * rest);
        const double us = ((double)(tiles / all) + (rest > 0.0 ? last : 0.0)) * (stages * k.stage + k.end);
        if (us < best) best = us, c.way = k.way, rounds = (tiles + all - 1) / all;
    }
    const int64_t series = rows / steps;
    // rows that hold data are listed where that takes less than what empty rows would cost,
    // were they half of them: a round and the product's share, which falls with the columns
    // (100 x 1000 by 512 columns and 192 channels 31.7 us, else 50.1; 4000 x 50 by 256
    // columns and channels 47, else 38)
    const int64_t least = c.way == kMiddleTwice ? 3 * 64 : 2 * 128;   // columns of a way's slots
    c.live = (c.way == kBig || c.way == kTall || c.way == kMiddleTwice) && rounds > 1 && columns >= least &&
             best * std::min(1.0, stages / 8.0) > 20.0 && series > 1 && series <= kMostSeries && steps > 1 &&
             rows * columns <= INT32_MAX && columns != kMostColumns;
    if (c.live) c.bytes = (rows + 1) * 4;
    const int64_t tiles = (rows + 127) / 128 * ((channels + 127) / 128), lines = (columns + 127) / 128;
    for (int64_t p = 2; p <= lines / 2 && tiles * p <= 4 * kCus; p += 1 + p / 8) {
        const int64_t each = (lines + p - 1) / p, parts = (lines + each - 1) / each;
        const double us = (double)((tiles * parts + kCus - 1) / kCus) * (each * 0.56 + 2.0) + 6.0 +
                          (double)(parts * rows * channels) * 8e-6 / 4.0;
        if (us < best) best = us, c = Cut{kSplit, (int32_t)parts, (int32_t)each, parts * rows * channels * 4, false};
    }
    return c;
}

template <int DT, bool SPLIT, bool LIVE, int MT, int NT, int WM, int WT, int COLS, int SLOTS, int AT_ONCE>
void tiles(ProductArgs a, hipStream_t s) {
    constexpr int kM = 32 * MT * WM, kT = 32 * NT * WT;
    a.tiles = (a.channels + kM - 1) / kM;
    const int64_t items = (a.rows.count + kT - 1) / kT * a.tiles;
    const int64_t groups = SPLIT ? items * a.parts : std::min(items, AT_ONCE * kCus);
    tile_kernel<DT, SPLIT, LIVE, MT, NT, WM, WT, COLS, SLOTS, AT_ONCE><<<(uint32_t)groups, 64 * WM * WT, 0, s>>>(a);
}

template <int DT, int MT, int NT, int COLS, int SLOTS, int AT_ONCE>
void listed(ProductArgs a, const Cut &cut, hipStream_t s) {
    if (cut.live && a.rows.lengths) {
        const int32_t each = (int32_t)((a.rows.n + kCus - 1) / kCus);
        order_kernel<<<(uint32_t)((a.rows.n + each - 1) / each), 256, 0, s>>>(a.rows, each, a.sums);
        a.order = a.sums;
        tiles<DT, false, true, MT, NT, 2, 2, COLS, SLOTS, AT_ONCE>(a, s);
    } else {
        tiles<DT, false, false, MT, NT, 2, 2, COLS, SLOTS, AT_ONCE>(a, s);
    }
}

template <int DT>
void launch(ProductArgs a, const Cut &cut, hipStream_t s) {
    a.parts = cut.parts, a.each = cut.each;
    switch (cut.way) {
    case kFew: {
        const uint32_t groups = (uint32_t)((a.channels + kFewChannels - 1) / kFewChannels);
        if (a.rows.count <= 16)
            few_kernel<DT, 1><<<groups, 64 * kFewWaves, 0, s>>>(a);
        else if (a.rows.count <= 32)
            few_kernel<DT, 2><<<groups, 64 * kFewWaves, 0, s>>>(a);
        else
            few_kernel<DT, 4><<<groups, 64 * kFewWaves, 0, s>>>(a);
        break;
    }
    case kBig: listed<DT, 4, 4, 128, 2, 1>(a, cut, s); break;
    case kTall: listed<DT, 4, 2, 128, 2, 1>(a, cut, s); break;
    case kMiddle: tiles<DT, false, false, 2, 2, 2, 2, 128, 3, 1>(a, s); break;
    case kMiddleTwice: listed<DT, 2, 2, 64, 3, 2>(a, cut, s); break;
    case kSmall: tiles<DT, false, false, 1, 1, 2, 2, 64, 4, 2>(a, s); break;
    case kSplit: {
        tiles<ROCKET_FLOAT32, true, false, 2, 2, 2, 2, 128, 3, 1>(a, s);
        finish_kernel<DT><<<(uint32_t)((a.rows.count * a.channels + 255) / 256), 256, 0, s>>>(a);
        break;
    }
    }
}

bool columns_ok(int64_t columns) { return columns > 0 && columns <= kMostColumns && columns % rocket::kPad8 == 0; }

}  // namespace

extern "C" rocket_status rocket_linear_bytes_workspace(const rocket_sequence_shape *shape, int64_t columns,
                                                  int64_t *bytes) {
    if (!bytes || !rocket::shape_ok(shape) || !columns_ok(columns)) return ROCKET_ERR_INVALID_ARG;
    *bytes = rocket::empty(shape) ? 0 : (cut_of(shape, columns).bytes + 7) / 8 * 8;
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
    const Cut cut = cut_of(shape, columns);
    if (cut.bytes && (!workspace || (uintptr_t)workspace % 8 != 0 || workspace_bytes < cut.bytes))
        return ROCKET_ERR_INVALID_ARG;
    ProductArgs a = {};
    a.sums = (int32_t *)workspace;
    a.q = q, a.p = weight, a.scale = scale, a.wscale = weight_scale, a.bias = bias;
    a.y = rocket::view_of(y, shape->dtype);
    a.columns = (int32_t)columns, a.channels = (int32_t)shape->channels;
    View *views[] = {&a.y};
    a.rows = rocket::rows_of(shape, views, 1);
    hipStream_t s = (hipStream_t)hip_stream;
    if (shape->dtype == ROCKET_FLOAT32)
        launch<ROCKET_FLOAT32>(a, cut, s);
    else if (shape->dtype == ROCKET_BFLOAT16)
        launch<ROCKET_BFLOAT16>(a, cut, s);
    else
        launch<ROCKET_FLOAT16>(a, cut, s);
    return rocket::launched();
}
