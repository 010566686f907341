// Products of matrices in 8-bit floating point with a scale for each block of 128.  The definitions stand in include/enec_lowbit.h.
#include "enec_lowbit.h"
#include "lowbit_fp8.hpp"
#include "lowbit_product.hpp"

#include <atomic>

namespace enec {
namespace lowbit {

using f32x4_a4 = f32x4 __attribute__((aligned(4)));

struct Product8 {
    const uint8_t *x, *x_scales, *w, *w_scales;         // (x: 16-bit values, where the kernel brings them into 8 bits)
    void *y;
    size_t x_stride, y_stride, part_row;                // elements
    float *parts;
    uint32_t m, n, k, groups, scale_row;                // groups of 128 columns; bytes between rows of scales
    uint32_t n_tiles, m_tiles, split_stages;
    int y_dtype;
};

__device__ __forceinline__ i32x8 halves(const u32x4 &a, const u32x4 &b)
{
    return i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
}

// The 8-bit matrix instructions align the products of eight columns (consecutive ones, as they are read here) to the largest of them and drop what
// lies below 2^-13 of its power of two; beyond that they sum in 32 bits.  For y in bf16 that is far below its own rounding: 1.5e-5 of the norm for normal
// values, 4e-5 where some channels stand out, bf16's rounding 1.7e-3.  An fp16 y is rounded to 2.1e-4, and would show it.  For y in fp16 and fp32 (EXACT) codes become
// bf16 values, which is exact from scale bytes of 3 on, and bf16 instructions, which sum in 32 bits, multiply them at half the rate.
template <bool HIGH> __device__ __forceinline__ uint32_t two_values(int codes, float scale)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)codes, scale, HIGH));
}
// columns 8 q ... 8 q + 7 of a lane's 32, as bf16 values
__device__ __forceinline__ bf16x8 eight_values(const i32x8 &v, int q, int byte)
{
    const float scale = f32_of_bits((uint32_t)byte << 23);          // (only its exponent counts, 0 is 2^-127 and 255 makes each NaN)
    return __builtin_bit_cast(bf16x8, u32x4{two_values<false>(v[2 * q], scale), two_values<true>(v[2 * q], scale), two_values<false>(v[2 * q + 1], scale),
                                            two_values<true>(v[2 * q + 1], scale)});
}

// A workgroup has 32 RA WA rows of weights and 32 RB WB tokens, a wave 32 RA rows and 32 RB tokens of them.  The matrix instruction multiplies 32 rows and 32
// tokens over 64 columns and takes a scale for each row and token; as all of a block's columns have the same scale, any assignment of columns to
// lanes is right that is the same for both operands.  A stage is one block of 128 columns, which the memory unit brings into LDS, BUFFERS stages in
// turn: a row's eight chunks of 16 bytes lie side by side, chunk i at place i ^ (row div 2 mod 8), so that the sixteen lanes of a read's quarter find
// sixteen different places of 256 bytes.  A wave reads the next half stage into registers while it multiplies this one; the only barrier of a stage is between
// its halves, when all waves have the second half in registers: the stage's buffer is free then, and the next stage has landed.
// Bound by the matrix unit's power and the way of the tiles into LDS: 4096 x 28672 x 8192 (tokens, rows, columns) takes 715 to 747 us by the card and its warmth, 2580 to 2690 TFLOP/s, with the unit
// busy for 65 to 70 % of the cycles, at a clock that its power brings down to 1.5 to 1.8 GHz, and no read meeting another one's bank; the copies alone take 536 us of it (620 before lines
// were touched ahead).  2048 x 11008 x 4096: 88 us, 2100 TFLOP/s, 473 tiles of 256 x 192 in two rounds.  EXACT: 96 x 4096 x 11008 22 us with its splits' join, 4096 x 28672 x 8192
// 1740 to 1840, 1050 to 1110 TFLOP/s: each wave makes bf16 values of all codes that it uses.
template <bool EXACT, int RA, int RB, int WA, int WB, int BUFFERS>
__global__ void __launch_bounds__(64 * WA * WB, RA * RB >= 8 ? 1 : 2) fp8_tile_kernel(Product8 a)
{
    constexpr uint32_t THREADS = 64 * WA * WB, ROWS = 32 * RA * WA, TOKENS = 32 * RB * WB, ALL = ROWS + TOKENS, STAGE = ALL * 128;
    constexpr uint32_t W_COPIES = ROWS * 8 / THREADS, COPIES = ALL * 8 / THREADS, SCALES = (ALL + 63) / 64 * 256;      // (copied by 64)
    static_assert(ROWS * 8 % THREADS == 0 && TOKENS * 8 % THREADS == 0 && THREADS % 128 == 0 && ROWS % 64 == 0, "whole copies of a wave");
    static_assert(BUFFERS >= 2 && BUFFERS <= 9, "scales land within seven stages");
    extern __shared__ __attribute__((aligned(16))) uint8_t shared[];
    uint8_t *scale_bytes = shared + BUFFERS * STAGE;        // of four stages, three in turn: four bytes of each row, then of each token
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 5, c = lane & 31;
    const uint32_t wa = wave % WA, wb = wave / WA;
    // Workgroups are dealt out to the eight dies one by one: each die takes a run of tiles, in bands of tiles of tokens (see product_tile_kernel).
    // 4096 x 8192 x 28672 took 946 us with bands of one, 730 of four, 744 of six, 735 of eight, 745 of twelve.
    constexpr uint32_t BAND = 4;
    const uint32_t tiles = a.n_tiles * a.m_tiles, per_die = (tiles + 7) / 8, tile = blockIdx.x % 8 * per_die + blockIdx.x / 8;
    if (blockIdx.x / 8 >= per_die || tile >= tiles) return;
    const uint32_t before = tile / (BAND * a.n_tiles) * BAND, band = a.m_tiles - before < BAND ? a.m_tiles - before : BAND;
    const uint32_t within = tile - before * a.n_tiles, n0 = within / band * ROWS, m0 = (before + within % band) * TOKENS;
    const uint32_t rows = a.n - n0 < ROWS ? a.n - n0 : ROWS, tokens = a.m - m0 < TOKENS ? a.m - m0 : TOKENS;
    const uint32_t pitch = a.groups * 128;
    const uint8_t *w = a.w + (size_t)n0 * pitch, *x = a.x + (size_t)m0 * pitch;
    const Range w_scales = range_of(a.w_scales + (size_t)n0 * a.scale_row, rows * a.scale_row);
    const Range x_scales = range_of(a.x_scales + (size_t)m0 * a.scale_row, tokens * a.scale_row);
    const uint32_t first = blockIdx.y * a.split_stages, end = first + a.split_stages < a.groups ? first + a.split_stages : a.groups;

    const uint32_t from = threadIdx.x / 8 * pitch + 16 * ((threadIdx.x ^ threadIdx.x >> 4) & 7);
    auto fetch_one = [&](uint32_t stage, uint32_t slot, uint32_t r) {       // (behind the end: nothing is read, but as many copies are counted)
        const uint32_t there = stage < end ? pitch : 0;
        const Range of = r < W_COPIES ? range_of(w, rows * there) : range_of(x, tokens * there);
        copy_to_lds<16>(of, from + (r < W_COPIES ? r : r - W_COPIES) * (THREADS / 8) * pitch + stage * 128, shared + slot * STAGE + wave * 1024 + r * (THREADS * 16));
    };
    auto fetch = [&](uint32_t stage, uint32_t slot) {
#pragma unroll
        for (uint32_t r = 0; r < COPIES; ++r) fetch_one(stage, slot, r);
    };
    auto fetch_scales = [&](uint32_t block) {
        uint8_t *to = scale_bytes + block % 3 * SCALES;
#pragma unroll
        for (uint32_t r = 0; r < ALL; r += THREADS) {
            const uint32_t begin = r + wave * 64, row = begin + lane;
            if (begin >= ALL) continue;
            if (begin < ROWS) copy_to_lds<4>(w_scales, row * a.scale_row + block * 4, to + begin * 4);
            else copy_to_lds<4>(x_scales, (row - ROWS) * a.scale_row + block * 4, to + begin * 4);
        }
    };

    // Large tiles have room for one or two stages ahead, which is less than the way from memory takes: a stage's lines are asked for TOUCH stages before its copies, four
    // bytes each, into LDS that nobody reads, so that the copies find them in the die's cache.  A wave touches 64 rows, a workgroup half of the tile's weights and half of its
    // tokens; its neighbours, which work on the same rows, touch the others.
    constexpr uint32_t TOUCH = RA * RB > 8 ? 2 : 0;
    uint8_t *junk = scale_bytes + 3 * SCALES + wave * 256;
    const bool alone = band < 2;
    const uint32_t touched = (alone ? wave * 64 : (wave & 1) * 64 + (wave < 2 ? within % band : within / band) % 2 * 128) + lane;
    auto touch = [&](uint32_t stage) {
        const uint32_t there = stage < end ? pitch : 0;
        const Range of = alone || wave < 2 ? range_of(w, rows * there) : range_of(x, tokens * there);
        copy_to_lds<4>(of, touched * pitch + stage * 128, junk);
    };

    // where this lane's chunks lie: of rows c, 32 + c, ..., half a stage has two of them for a lane
    uint32_t w_at[4], x_at[4];
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) {
        const uint32_t chunk = (((j >> 1) * 4 + 2 * g + (j & 1)) ^ (c >> 1 & 7)) * 16;
        w_at[j] = (wa * (32 * RA) + c) * 128 + chunk;
        x_at[j] = (ROWS + wb * (32 * RB) + c) * 128 + chunk;
    }
    const uint32_t ws_at = (wa * (32 * RA) + c) * 4, xs_at = (ROWS + wb * (32 * RB) + c) * 4;

    i32x8 wv[2][RA], xv[2][RB];
    int ws[2][RA], xs[2][RB];                               // scales, by the stage's parity
    auto read = [&](int i, uint32_t slot, int half) {       // operand i of a half stage
        const uint8_t *t = shared + slot * STAGE;
        if (i < RA) {
            wv[half][i] = halves(*reinterpret_cast<const u32x4 *>(t + w_at[2 * half] + i * 4096), *reinterpret_cast<const u32x4 *>(t + w_at[2 * half + 1] + i * 4096));
        } else {
            const int u = i - RA;
            xv[half][u] = halves(*reinterpret_cast<const u32x4 *>(t + x_at[2 * half] + u * 4096), *reinterpret_cast<const u32x4 *>(t + x_at[2 * half + 1] + u * 4096));
        }
    };
    auto read_scales = [&](uint32_t stage, int parity) {
        const uint8_t *t = scale_bytes + (stage >> 2) % 3 * SCALES + (stage & 3);
#pragma unroll
        for (int i = 0; i < RA; ++i) ws[parity][i] = t[ws_at + i * 128];
#pragma unroll
        for (int i = 0; i < RB; ++i) xs[parity][i] = t[xs_at + i * 128];
    };
    // A wave's copies are counted, and done in the order in which they were issued: with at most AHEAD left, those of the next stage are in LDS.  Then all
    // waves' are, and this stage's second half is in everybody's registers.
    constexpr int AHEAD = (BUFFERS - 2) * COPIES + (TOUCH ? BUFFERS - 1 : 0);
    auto meet = [&] {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(AHEAD) : "memory");
        __builtin_amdgcn_sched_barrier(0);
    };

    f32x16 acc[RA][RB] = {};
    fetch_scales(first / 4), fetch_scales(first / 4 + 1);   // (a split begins with such a block)
#pragma unroll
    for (int b = 0; b < BUFFERS; ++b) {
        fetch(first + b, b);
        if constexpr (TOUCH != 0) touch(first + BUFFERS + b);
    }
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((BUFFERS - 1) * COPIES + (TOUCH ? BUFFERS : 0)) : "memory");
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < RA + RB; ++i) read(i, 0, 0);
    read_scales(first, 0);
    uint32_t slot = 0;
    auto step = [&](uint32_t s, int parity) {
        const uint32_t next_slot = slot + 1 == BUFFERS ? 0 : slot + 1;
        constexpr int TILES = RA * RB;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            if (half == 1) {
                meet();
                if ((s & 3) == 0) fetch_scales(s / 4 + 2);
                if constexpr (EXACT) fetch(s + BUFFERS, slot);
                read_scales(s + 1, parity ^ 1);
            }
            if constexpr (EXACT) {
#pragma unroll
                for (int o = 0; o < RA + RB; ++o) read(o, half == 0 ? slot : next_slot, half ^ 1);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    bf16x8 wq[RA], xq[RB];
#pragma unroll
                    for (int t = 0; t < RA; ++t) wq[t] = eight_values(wv[half][t], q, ws[parity][t]);
#pragma unroll
                    for (int u = 0; u < RB; ++u) xq[u] = eight_values(xv[half][u], q, xs[parity][u]);
#pragma unroll
                    for (int t = 0; t < RA; ++t)
#pragma unroll
                        for (int u = 0; u < RB; ++u) acc[t][u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wq[t], xq[u], acc[t][u], 0, 0, 0);
                }
            } else {
                // the other half's operands, and the next stage's copies, are asked for one by one between the products
                constexpr int STEPS = TILES > 8 ? TILES / 2 : TILES;
#pragma unroll
                for (int i = 0; i < TILES; ++i) {
#pragma unroll
                    for (int o = i * (RA + RB) / STEPS; o < (i + 1) * (RA + RB) / STEPS; ++o)
                        if (o < RA + RB) read(o, half == 0 ? slot : next_slot, half ^ 1);
                    if (half == 1) {
#pragma unroll
                        for (int r = i * (int)COPIES / TILES; r < (i + 1) * (int)COPIES / TILES; ++r) fetch_one(s + BUFFERS, slot, r);
                    }
                    const int t = i / RB, u = i % RB;
                    acc[t][u] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wv[half][t], xv[half][u], acc[t][u], 0, 0, 0, ws[parity][t], 0, xs[parity][u]);
                    if (TOUCH != 0 && half == 1 && i == TILES - 1) touch(s + BUFFERS + TOUCH);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        slot = next_slot;
    };
    uint32_t s = first;
    for (; s + 1 < end; s += 2) {
        step(s, 0);
        step(s + 1, 1);
    }
    if (s < end) step(s, 0);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");        // (no copy may come after the workgroup, nor into what follows)
    constexpr bool ONLY_16 = RA * RB >= 8;                  // tiles that are never split, of y in bf16
    if (ONLY_16 || ((!EXACT || a.y_dtype == FP16) && !a.parts)) {
        // 16-bit values by way of LDS, a token's rows side by side there: a lane's four rows of a token would be stores of 8 bytes, 32 tokens apart
        constexpr uint32_t PITCH = ROWS * 2 + 16, CHUNKS = ROWS / 8;
        __syncthreads();
#pragma unroll
        for (int u = 0; u < RB; ++u)
#pragma unroll
            for (int t = 0; t < RA; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const f32x16 &v = acc[t][u];
                    constexpr int Y = EXACT ? FP16 : BF16;
                    const u32x2 w = {pack2<Y>(v[4 * e], v[4 * e + 1]), pack2<Y>(v[4 * e + 2], v[4 * e + 3])};
                    *reinterpret_cast<u32x2 *>(shared + (wb * (32 * RB) + 32 * u + c) * PITCH + (wa * (32 * RA) + 32 * t + 8 * e + 4 * g) * 2) = w;
                }
        __syncthreads();
#pragma unroll 4
        for (uint32_t i = threadIdx.x; i < TOKENS * CHUNKS; i += THREADS) {
            const uint32_t token = i / CHUNKS, r = i % CHUNKS * 8;
            if (token >= tokens || r >= rows) continue;
            const u32x4 v = *reinterpret_cast<const u32x4 *>(shared + token * PITCH + r * 2);
            uint16_t *to = static_cast<uint16_t *>(a.y) + (size_t)(m0 + token) * a.y_stride + n0 + r;
            if (r + 8 <= rows) {
                *reinterpret_cast<u32x4_a2 *>(to) = v;
            } else {
#pragma unroll
                for (uint32_t j = 0; j < 7; ++j)
                    if (r + j < rows) to[j] = (uint16_t)(v[j >> 1] >> (16 * (j & 1)));
            }
        }
        return;
    }
    if constexpr (!ONLY_16) {
        // 32-bit values: four rows of a token are 16 bytes
        float *to = a.parts ? a.parts + (size_t)blockIdx.y * a.m * a.part_row : static_cast<float *>(a.y);
        const size_t stride = a.parts ? a.part_row : a.y_stride;
#pragma unroll
        for (int u = 0; u < RB; ++u) {
            const uint32_t token = m0 + wb * (32 * RB) + 32 * u + c;
            if (token >= a.m) continue;
#pragma unroll
            for (int t = 0; t < RA; ++t) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t r = n0 + wa * (32 * RA) + 32 * t + 8 * e + 4 * g;
                    const f32x4 v = {acc[t][u][4 * e], acc[t][u][4 * e + 1], acc[t][u][4 * e + 2], acc[t][u][4 * e + 3]};
                    if (r + 4 <= a.n) {
                        *reinterpret_cast<f32x4_a4 *>(to + (size_t)token * stride + r) = v;
                    } else {
#pragma unroll
                        for (uint32_t j = 0; j < 3; ++j)
                            if (r + j < a.n) to[(size_t)token * stride + r + j] = v[j];
                    }
                }
            }
        }
    }
}

// Up to 16 XT tokens: bound by the weights' way from memory.  A workgroup has sixteen rows of weights; its waves take units of four blocks of 128 columns in turn,
// each through a ring of its own in LDS that the memory unit fills, so that no wave waits for another one before their sums meet.  The instruction here
// multiplies sixteen rows and sixteen tokens over a whole block: a lane has row (or token) lane mod 16 and chunks 2 g and 2 g + 1 of its eight, g = lane div 16.
// Chunk i lies at place i ^ turn(row): the sixteen lanes of a read's quarter are rows {0-3, 12-15} of one g and {4-11} of the next, and find sixteen places.
// With X_INSIDE the workgroup brings the few tokens' 16-bit values into 8 bits itself, while its first weights are on their way.
// 1 token x 28672 x 8192: 43 to 48 us, 5.5 to 4.9 TB/s; x 11008 x 4096 12.2 to 12.6, 3.7 TB/s; 1024 x 1024, a launch's start, one way from memory and the join of the waves' sums, 3.4.
__device__ __forceinline__ uint32_t thin_turn(uint32_t r) { return (r >> 1 & 1) | (r >> 1 & 4); }
constexpr uint32_t X_EACH = 4;                  // vectors of the tokens that a thread brings into 8 bits, at most
template <bool EXACT, int X_INSIDE, int XT, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, 2) fp8_thin_kernel(Product8 a)
{
    constexpr uint32_t W_SIZE = 16 * 128, STAGE = X_INSIDE ? W_SIZE : (1 + XT) * W_SIZE, COPIES = STAGE / 1024;
    static_assert(!X_INSIDE || XT == 1, "few tokens");
    extern __shared__ __attribute__((aligned(16))) uint8_t shared[];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, c = lane & 15;
    uint8_t *ring = shared + wave * (4 * STAGE), *x_codes = shared + WAVES * (4 * STAGE), *x_bytes = x_codes + a.m * a.groups * 128;
    const uint32_t n0 = blockIdx.x * 16, pitch = a.groups * 128, rows = a.n - n0 < 16 ? a.n - n0 : 16;
    const uint8_t *w = a.w + (size_t)n0 * pitch;
    // rows and tokens that are not there take the last one's scale, and their sums go nowhere
    uint32_t token[XT];
#pragma unroll
    for (uint32_t u = 0; u < XT; ++u) token[u] = 16 * u + c < a.m ? 16 * u + c : a.m - 1;
    const uint32_t *w_scales = reinterpret_cast<const uint32_t *>(a.w_scales + (size_t)(n0 + (c < rows ? c : rows - 1)) * a.scale_row);
    const uint32_t units = (a.groups + 3) / 4;
    const uint32_t from = lane / 8 * pitch + 16 * ((lane & 7) ^ thin_turn(lane / 8)), from8 = (8 + lane / 8) * pitch + 16 * ((lane & 7) ^ thin_turn(8 + lane / 8));
    auto fetch = [&](uint32_t stage, uint32_t slot) {       // (behind the end: nothing is read, but as many copies are counted)
        const uint32_t there = stage < a.groups ? pitch : 0;
        const Range wr = range_of(w, rows * there);
        copy_to_lds<16>(wr, from + stage * 128, ring + slot * STAGE);
        copy_to_lds<16>(wr, from8 + stage * 128, ring + slot * STAGE + 1024);
        if constexpr (!X_INSIDE) {
            const Range xr = range_of(a.x, a.m * there);
#pragma unroll
            for (uint32_t u = 0; u < XT; ++u) {
                copy_to_lds<16>(xr, from + 16 * u * pitch + stage * 128, ring + slot * STAGE + (1 + u) * W_SIZE);
                copy_to_lds<16>(xr, from8 + 16 * u * pitch + stage * 128, ring + slot * STAGE + (1 + u) * W_SIZE + 1024);
            }
        }
    };
    auto scale_at = [&](const uint32_t *p, uint32_t i) { return p[i < units ? i : units - 1]; };
    auto x_scale_at = [&](uint32_t u, uint32_t i) {
        return X_INSIDE ? 0 : scale_at(reinterpret_cast<const uint32_t *>(a.x_scales + (size_t)token[u] * a.scale_row), i);
    };
    uint32_t ws = scale_at(w_scales, wave), xs[XT], next_xs[XT];
#pragma unroll
    for (uint32_t u = 0; u < XT; ++u) xs[u] = x_scale_at(u, wave);
    // The tokens' values: sixteen threads a block, eight values each, asked for before any weights.
    constexpr int DT = X_INSIDE ? X_INSIDE - 1 : 0;
    const uint32_t per_row = a.groups * 16, all = X_INSIDE ? a.m * per_row : 0;
    auto load_x = [&](uint32_t i, float (&v)[8]) {
        const uint32_t r = i / per_row, col = (i - r * per_row) * 8;
        const size_t at = (size_t)r * a.x_stride + col;
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) v[j] = 0.0f;
        if (i >= all) return;
        if (col + 8 <= a.k) {
            load8<DT>(a.x, at, v);
        } else if (col < a.k) {                             // (loads that do not wait for one another)
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) v[j] = load1<DT>(a.x, at + (col + j < a.k ? j : a.k - 1 - col));
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) v[j] = col + j < a.k ? v[j] : 0.0f;
        }
    };
    auto store_x = [&](uint32_t i, const float (&v)[8]) {
        if (i >= all) return;
        const uint32_t r = i / per_row, col = (i - r * per_row) * 8, byte = block_byte(v);
        // (a block's chunks turned by its row, as the ring's)
        *reinterpret_cast<u32x2 *>(x_codes + r * pitch + (col & ~127u) + ((col >> 4 & 7) ^ thin_turn(r)) * 16 + (col & 8)) = fp8_codes(v, byte);
        if ((i & 15) == 0) x_bytes[r * a.groups + (col >> 7)] = (uint8_t)byte;
    };
    float x_values[X_EACH][8];
    if constexpr (X_INSIDE != 0) {
#pragma unroll
        for (uint32_t u = 0; u < X_EACH; ++u) load_x(threadIdx.x + u * 64 * WAVES, x_values[u]);
        __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) fetch(4 * wave + j, j);
    if constexpr (X_INSIDE != 0) {
#pragma unroll
        for (uint32_t u = 0; u < X_EACH; ++u) store_x(threadIdx.x + u * 64 * WAVES, x_values[u]);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }
    const uint32_t low = ((2 * g) ^ thin_turn(c)) * 16, high = ((2 * g + 1) ^ thin_turn(c)) * 16;
    f32x4 acc[XT] = {};
    for (uint32_t i = wave; i < units; i += WAVES) {
        const uint32_t next_ws = scale_at(w_scales, i + WAVES);
#pragma unroll
        for (uint32_t u = 0; u < XT; ++u) next_xs[u] = x_scale_at(u, i + WAVES);
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            const uint32_t stage = 4 * i + j < a.groups ? 4 * i + j : a.groups - 1;
            // A wave's copies are done in the order in which they were issued: three stages' may be left
            __builtin_amdgcn_sched_barrier(0);
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(3 * COPIES) : "memory");
            __builtin_amdgcn_sched_barrier(0);
            const uint8_t *t = ring + j * STAGE + c * 128;
            const i32x8 wv = halves(*reinterpret_cast<const u32x4 *>(t + low), *reinterpret_cast<const u32x4 *>(t + high));
            i32x8 xv[XT];
            uint32_t xb[XT];
#pragma unroll
            for (uint32_t u = 0; u < XT; ++u) {
                // (a token that is not there: the last one's codes, of its tile in the ring; turns go by the row within a tile)
                const uint32_t r = X_INSIDE ? token[u] : token[u] & 15;
                const uint8_t *x = X_INSIDE ? x_codes + r * pitch + stage * 128 : ring + j * STAGE + (1 + (token[u] >> 4)) * W_SIZE + r * 128;
                xv[u] = halves(*reinterpret_cast<const u32x4 *>(x + ((2 * g) ^ thin_turn(r)) * 16), *reinterpret_cast<const u32x4 *>(x + ((2 * g + 1) ^ thin_turn(r)) * 16));
                xb[u] = X_INSIDE ? x_bytes[r * a.groups + stage] : xs[u] >> (8 * j) & 255;
            }
            __builtin_amdgcn_sched_barrier(0);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
            fetch(4 * (i + WAVES) + j, j);
            if (4 * i + j >= a.groups) continue;
            const int wb = (int)(ws >> (8 * j) & 255);
#pragma unroll
            for (uint32_t u = 0; u < XT; ++u) {
                if constexpr (EXACT) {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        acc[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(eight_values(wv, q, wb), eight_values(xv[u], q, (int)xb[u]), acc[u], 0, 0, 0);
                } else {
                    acc[u] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv, xv[u], acc[u], 0, 0, 0, wb, 0, (int)xb[u]);
                }
            }
        }
        ws = next_ws;
#pragma unroll
        for (uint32_t u = 0; u < XT; ++u) xs[u] = next_xs[u];
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");        // (no copy may come into what the sums take)
    __syncthreads();
    f32x4 *sums = reinterpret_cast<f32x4 *>(shared);
    if (wave != 0) {
#pragma unroll
        for (uint32_t u = 0; u < XT; ++u) sums[(wave * XT + u) * 64 + lane] = acc[u];
    }
    __syncthreads();
    if (wave != 0) return;
    const uint32_t r = n0 + 4 * g;
#pragma unroll
    for (uint32_t u = 0; u < XT; ++u) {
#pragma unroll
        for (int k = 1; k < WAVES; ++k) acc[u] += sums[(k * XT + u) * 64 + lane];
        if (16 * u + c < a.m && r < a.n) store4(a.y, a.y_dtype, (size_t)(16 * u + c) * a.y_stride + r, a.n - r, acc[u]);
    }
}

}  // namespace lowbit
}  // namespace enec

namespace {

using namespace enec::lowbit;

inline bool aligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// The tiles there are.  With one on every compute unit a stage takes `us`, with two on each, where two fit, `us_two`; the same for y in fp16 and fp32.  (These and plan_of's constants are
// fitted to the times of 500 products of 1 to 4096 tokens with eighteen matrices from 1024 x 4096 to 28672 x 8192, y in bf16 and fp32, every tile and split forced; its choices
// are 0.6 % above the best ones in the mean and 26 % at worst, and of 252 other products 1.3 %, 16 of them more than 5 %, and 23 % at worst.)
struct Shape {
    uint32_t rows, tokens;
    double us, us_two, us_exact, us_exact_two;
};
constexpr int SHAPES = 7, FIRST_EXACT = 3;
constexpr Shape SHAPE[SHAPES] = {{256, 256, 1.30, 0, 0, 0},      {256, 192, 1.08, 0, 0, 0},        {256, 128, 0.79, 0, 0, 0},        {128, 128, 0.585, 0, 0.91, 0},
                                 {128, 64, 0.40, 0.69, 0.53, 0.95}, {64, 64, 0.25, 0.40, 0.35, 0.555}, {64, 32, 0.215, 0.305, 0.34, 0.46}};
constexpr uint32_t THIN = 64;                       // tokens at most of the kernel for few
constexpr uint32_t UNITS = 256;                     // compute units
constexpr uint32_t MOST_SPLITS = 16, UNIT = 4;      // a split is whole blocks of scales: so many stages, or a multiple
constexpr uint32_t MOST_SPLIT_TILES = 320;          // tiles and splits together, where there are splits

// How a product is cut up: the tile (-1: the kernel for few tokens), and the splits of the columns where tiles alone leave the card empty.
struct Plan {
    int shape;
    uint32_t splits, split_stages;
};
inline bool too_large(const Shape &s, uint32_t m) { return s.tokens > 32 && s.tokens >= 2 * up(m, 16) * 16; }      // half of the tile or more would be empty

inline uint32_t thin_tiles(uint32_t m) { return m <= 16 ? 1 : m <= 32 ? 2 : 4; }
inline uint32_t thin_waves(uint32_t tiles, uint32_t groups) { return groups <= 32 || tiles > 2 ? 2 : 4; }

Plan plan_of(uint32_t m, uint32_t n, uint32_t groups, bool exact)
{
    Plan p{-1, 1, up(groups, UNIT) * UNIT};
    const double matrix = (double)n * groups * 128, from_memory = matrix / 6.1e6 + 1.5;
    // the weights' way from memory and the units' work overlap in part
    const auto both = [&](double us) { return us > from_memory ? us + 0.38 * from_memory : from_memory + 0.38 * us; };
    double best = 1e300;
    if (m <= THIN) {
        // every sixteen rows read all tokens again; the unit with the most rows, or a wave's units one after the other, take the time
        const uint32_t tiles = thin_tiles(m);
        const double read = (double)up(up(n, 16), UNITS) * UNITS * 16 * groups * 128 * (1 + tiles) / (exact ? 13.8e6 : 19e6);
        const double chain = up(up(groups, UNIT), thin_waves(tiles, groups)) * (exact ? 0.14 : 0.23) * (1 + tiles) / 2;
        best = both(2 + (read > chain ? read : chain));
    }
    for (int i = exact ? FIRST_EXACT : 0; i < SHAPES; ++i) {
        const Shape &s = SHAPE[i];
        if (too_large(s, m)) continue;
        const uint64_t tiles = (uint64_t)up(n, s.rows) * up(m, s.tokens);
        const bool splittable = i >= FIRST_EXACT && (uint64_t)m * up(n, 4) < 1u << 31;
        const double one = exact ? s.us_exact : s.us, two = exact ? s.us_exact_two : s.us_two, start = exact ? 3.1 : i >= FIRST_EXACT ? 2.3 : 6.8;
        const uint32_t places = two > 0 ? 2 * UNITS : UNITS;
        for (uint32_t splits = 1; splits == 1 || (splittable && splits <= MOST_SPLITS && splits * UNIT <= groups && tiles * splits <= MOST_SPLIT_TILES); ++splits) {
            const uint32_t each = up(up(groups, splits), UNIT) * UNIT, count = up(groups, each);
            const uint64_t all = tiles * count, full = all / places, rest = all % places;
            // whole rounds and what is left (units that have none leave the others more of the memory); joining is a launch, the sums' way out and back, one split after the other
            double us = (double)full * (each * (two > 0 ? two : one) + start);
            if (rest > UNITS) us += each * two + start;
            else if (rest) us += each * one * (rest <= 192 ? 0.92 : 1) + start;
            us = both(us) + (count > 1 ? 1.7 + 0.27 * count + (double)count * m * n * 8 / 5.4e6 : 0);
            if (us < best) best = us, p.shape = i, p.splits = count, p.split_stages = each;
        }
    }
    return p;
}

// Bytes for the sums of the splits: of no more than m tokens, however few, so that one piece serves products of any number of them (fewer may be split
// more).  The number of splits and tiles is bounded, which bounds the splits' tokens by the tile's.
size_t parts_of(uint32_t m, uint32_t n, uint32_t groups)
{
    const uint32_t by_columns = groups / UNIT < MOST_SPLITS ? groups / UNIT : MOST_SPLITS;
    uint64_t most = 0;
    for (int i = FIRST_EXACT; i < SHAPES && by_columns > 1; ++i) {
        const Shape &s = SHAPE[i];
        if (too_large(s, m)) continue;
        const uint64_t by_tiles = (uint64_t)s.tokens * (MOST_SPLIT_TILES / up(n, s.rows)), by_splits = (uint64_t)by_columns * m, rows = by_tiles < by_splits ? by_tiles : by_splits;
        most = most > rows ? most : rows;
    }
    return most * part_row(n) * sizeof(float);
}

template <bool EXACT, int RA, int RB, int WA, int WB, int BUFFERS> bool launch_tile(Product8 a, uint32_t splits, hipStream_t s)
{
    constexpr size_t ROWS = 32 * RA * WA, TOKENS = 32 * RB * WB, LDS = (ROWS + TOKENS) * 128 * BUFFERS + (ROWS + TOKENS + 63) / 64 * 768 + (RA * RB > 8 ? WA * WB * 256 : 0);
    static_assert(LDS <= 160 * 1024, "LDS of a compute unit");
    static std::atomic<uint64_t> allowed{0};
    const auto kernel = fp8_tile_kernel<EXACT, RA, RB, WA, WB, BUFFERS>;
    if (LDS > 65536 && !allow_lds((const void *)kernel, LDS, allowed)) return false;
    a.n_tiles = up(a.n, ROWS), a.m_tiles = up(a.m, TOKENS);
    kernel<<<dim3(up(a.n_tiles * a.m_tiles, 8) * 8, splits), 64 * WA * WB, LDS, s>>>(a);
    return true;
}

template <bool EXACT> bool launch_shape(const Product8 &a, const Plan &p, hipStream_t s)
{
    if constexpr (!EXACT) {
        switch (p.shape) {
        case 0: return launch_tile<false, 4, 4, 2, 2, 2>(a, p.splits, s);
        case 1: return launch_tile<false, 4, 3, 2, 2, 2>(a, p.splits, s);
        case 2: return launch_tile<false, 4, 2, 2, 2, 3>(a, p.splits, s);
        }
    }
    switch (p.shape) {
    case 3: return launch_tile<EXACT, 2, 2, 2, 2, 4>(a, p.splits, s);
    case 4: return launch_tile<EXACT, 2, 1, 2, 2, 3>(a, p.splits, s);
    case 5: return launch_tile<EXACT, 1, 1, 2, 2, 4>(a, p.splits, s);
    default: return launch_tile<EXACT, 1, 1, 2, 1, 5>(a, p.splits, s);
    }
}

// Waves of a workgroup for few tokens: with more of them more weights are on their way and fewer units follow one another in a wave, but more wait for one
// another at the end.  With the tokens brought into 8 bits inside, which more threads do faster, 1 token x 4096 x 1024 / 2048 / 4096 / 8192 took 3.7 / 4.8 / 7.7 / 14.1 us with
// two waves, 3.8 / 4.2 / 6.2 / 10.5 with four and 4.0 / 4.4 / 6.4 / 10.0 with eight; without, 8 tokens x 11008 x 4096 / 8192 14.8 / 22.3 with two, 16.4 / 24.8 with four, x 28672 x 8192
// 51 and 49, x 4096 x 8192 13.7 and 12.9.
// Up to 2048 columns two waves are better where there are many workgroups, up to 4096 four are: with weights from memory 1 token x 4096 / 9216 / 11008 / 16384 / 32003 x 2048 took
// 4.0 / 7.1 / 7.2 / 8.7 / 14.9 us with four and 4.2 / 6.8 / 7.1 / 8.8 / 13.6 with two, x 11008 x 2560 8.3 and 8.1, x 11008 / 12288 x 3328 9.6 / 10.1 and 10.1 / 10.7,
// x 8192 / 9216 / 11008 / 12288 / 16384 / 32003 x 4096 10.1 / 11.7 / 12.2 / 13.0 / 16.2 / 27.5 and 10.7 / 11.6 / 12.7 / 13.6 / 17.4 / 29.9.  (From the last-level cache, where a model's
// weights do not lie, 11008 x 4096 took 11.7 and 10.8.)
// Bringing them into 8 bits inside saves a launch and costs every workgroup the work again: where four vectors a thread are enough, 1 token x 11008 x 4096 took 12.8 us
// against 14.4, 4 tokens x 4096 x 2048 5.4 against 6.4, 2 tokens x 32003 x 4096, the worst found, 31.1 against 30.9; with eight a thread 2 tokens x 4096 x 4096 took 9.9
// against 8.6, with thirty-two 16 tokens x 32003 x 2048 65 against 20.
inline uint32_t waves_inside(uint32_t n, uint32_t groups)
{
    const uint32_t per_unit = up(up(n, 16), UNITS);
    return groups <= 8 ? 2 : groups <= 16 ? (per_unit <= 2 ? 4 : 2) : groups <= 32 ? 4 : 8;
}
inline bool x_inside(uint32_t m, uint32_t n, uint32_t groups) { return m <= 16 && (uint64_t)m * groups * 16 <= X_EACH * 64 * waves_inside(n, groups); }

template <bool EXACT, int X_INSIDE, int XT, int WAVES> bool launch_thin_of(const Product8 &a, hipStream_t s)
{
    static std::atomic<uint64_t> allowed{0};
    constexpr size_t RINGS = WAVES * 4 * (X_INSIDE ? 2048 : 2048 * (1 + XT));
    const size_t lds = RINGS + (X_INSIDE ? (size_t)a.m * a.groups * 129 : 0);
    const auto kernel = fp8_thin_kernel<EXACT, X_INSIDE, XT, WAVES>;
    if (lds > 65536 && !allow_lds((const void *)kernel, RINGS + (X_INSIDE ? X_EACH * 64 * WAVES * 8 * 129 / 128 : 0), allowed)) return false;
    kernel<<<up(a.n, 16), 64 * WAVES, lds, s>>>(a);
    return true;
}
template <int DT> bool launch_thin_inside(const Product8 &a, hipStream_t s)
{
    constexpr bool EXACT = DT == FP16;
    const uint32_t waves = waves_inside(a.n, a.groups);
    return waves == 2 ? launch_thin_of<EXACT, DT + 1, 1, 2>(a, s) : waves == 4 ? launch_thin_of<EXACT, DT + 1, 1, 4>(a, s) : launch_thin_of<EXACT, DT + 1, 1, 8>(a, s);
}
template <bool EXACT, int XT> bool launch_thin(const Product8 &a, hipStream_t s)
{
    constexpr int MOST = XT > 2 ? 2 : 4;
    return thin_waves(XT, a.groups) == 2 ? launch_thin_of<EXACT, 0, XT, 2>(a, s) : launch_thin_of<EXACT, 0, XT, MOST>(a, s);
}

template <bool EXACT> int launch(Product8 a, void *parts, hipStream_t s)
{
    if (a.groups == 0) {
        const uint32_t per_row = up(a.n, 4);
        join_kernel<<<up(a.m * per_row, 256), 256, 0, s>>>(nullptr, 0, a.m, a.n, 0, divide_by(per_row), a.y, a.y_stride, a.y_dtype);
        return hipGetLastError() == hipSuccess ? ENEC_OK : ENEC_E_HIP;
    }
    bool ok = true;
    const Plan p = plan_of(a.m, a.n, a.groups, EXACT);
    if (p.shape < 0) {
        const uint32_t tiles = thin_tiles(a.m);
        ok = tiles == 1 ? launch_thin<EXACT, 1>(a, s) : tiles == 2 ? launch_thin<EXACT, 2>(a, s) : launch_thin<EXACT, 4>(a, s);
    } else {
        a.split_stages = p.split_stages;
        if (p.splits > 1) a.parts = static_cast<float *>(parts), a.part_row = part_row(a.n);
        ok = launch_shape<EXACT>(a, p, s);
        if (ok && p.splits > 1) {
            const uint32_t per_row = up(a.n, 4);
            join_kernel<<<up(a.m * per_row, 256), 256, 0, s>>>(a.parts, p.splits, a.m, a.n, a.part_row, divide_by(per_row), a.y, a.y_stride, a.y_dtype);
        }
    }
    return ok && hipGetLastError() == hipSuccess ? ENEC_OK : ENEC_E_HIP;
}

// sizes that every kernel here can count with: offsets inside a tile have 31 bits, and so have the counts of vectors that are laid out and of tiles
inline bool sizes_ok(size_t m, size_t n, size_t k)
{
    return m <= (1u << 21) && n <= (1u << 26) && k <= (1u << 21) && m * k <= (size_t)1 << 34 && m * n <= (size_t)1 << 40 && fp8_fits(m, k) && fp8_fits(n, k)
           && (k != 0 || m * n < (size_t)1 << 33);
}

inline bool exact_of(int y_dtype) { return y_dtype != ENEC_BF16; }

// a linear layer's activations in 8 bits, codes and scales
inline size_t codes_space(size_t m, size_t k) { return m * fp8_padded(k); }
inline size_t scales_space(size_t m, size_t k) { return (m * fp8_scale_row(k) + 15) / 16 * 16; }

}  // namespace

extern "C" {

size_t enec_fp8_linear_workspace(size_t m, size_t n, size_t k)
{
    if (!sizes_ok(m, n, k) || m == 0 || n == 0 || k == 0) return 0;
    return codes_space(m, k) + scales_space(m, k) + enec_fp8_matmul_workspace(m, n, k);
}
size_t enec_fp8_matmul_workspace(size_t m, size_t n, size_t k)
{
    if (!sizes_ok(m, n, k) || m == 0 || n == 0 || k == 0) return 0;
    return parts_of((uint32_t)m, (uint32_t)n, (uint32_t)((k + 127) / 128));
}

int enec_fp8_linear(const void *x, size_t m, size_t x_stride, int dtype, const void *codes, const void *scales, size_t n, size_t k, void *y, size_t y_stride,
                    void *workspace, size_t workspace_bytes, void *stream)
{
    if (dtype != ENEC_BF16 && dtype != ENEC_FP16) return ENEC_E_DTYPE;
    if (!sizes_ok(m, n, k)) return ENEC_E_ARG;
    if (m == 0 || n == 0) return ENEC_OK;
    if (!y || !aligned(y, 2) || y_stride < n) return ENEC_E_ARG;
    if (k != 0 && (!x || !codes || !scales || !aligned(x, 2) || !aligned(codes, 16) || !aligned(scales, 4) || x_stride < k)) return ENEC_E_ARG;
    const size_t need = enec_fp8_linear_workspace(m, n, k);
    if (workspace_bytes < need || (need && !workspace)) return ENEC_E_CAPACITY;
    if (need && !aligned(workspace, 16)) return ENEC_E_ARG;
    const hipStream_t s = (hipStream_t)stream;
    uint8_t *x_codes = static_cast<uint8_t *>(workspace), *x_scales = x_codes + codes_space(m, k), *parts = x_scales + scales_space(m, k);
    Product8 a{x_codes, x_scales, static_cast<const uint8_t *>(codes), static_cast<const uint8_t *>(scales), y, x_stride, y_stride, 0, nullptr, (uint32_t)m, (uint32_t)n,
               (uint32_t)k, (uint32_t)((k + 127) / 128), (uint32_t)fp8_scale_row(k), 0, 0, 0, dtype};
    if (k != 0 && x_inside(a.m, a.n, a.groups)) {
        a.x = static_cast<const uint8_t *>(x);
        const bool ok = dtype == ENEC_BF16 ? launch_thin_inside<BF16>(a, s) : launch_thin_inside<FP16>(a, s);
        return ok && hipGetLastError() == hipSuccess ? ENEC_OK : ENEC_E_HIP;
    }
    if (k != 0)
        if (const int rc = quantize_to_fp8(x, m, k, x_stride, dtype, x_codes, x_scales, s)) return rc;
    return exact_of(dtype) ? launch<true>(a, parts, s) : launch<false>(a, parts, s);
}

int enec_fp8_matmul(const void *x_codes, const void *x_scales, size_t m, const void *codes, const void *scales, size_t n, size_t k, void *y, size_t y_stride,
                    int dtype, void *workspace, size_t workspace_bytes, void *stream)
{
    if (dtype != ENEC_BF16 && dtype != ENEC_FP16 && dtype != ENEC_FP32) return ENEC_E_DTYPE;
    if (!sizes_ok(m, n, k)) return ENEC_E_ARG;
    if (m == 0 || n == 0) return ENEC_OK;
    if (!y || !aligned(y, dtype == ENEC_FP32 ? 4 : 2) || y_stride < n) return ENEC_E_ARG;
    if (k != 0 && (!x_codes || !x_scales || !codes || !scales || !aligned(x_codes, 16) || !aligned(x_scales, 4) || !aligned(codes, 16) || !aligned(scales, 4)))
        return ENEC_E_ARG;
    const size_t need = enec_fp8_matmul_workspace(m, n, k);
    if (workspace_bytes < need || (need && !workspace)) return ENEC_E_CAPACITY;
    if (need && !aligned(workspace, 16)) return ENEC_E_ARG;
    const Product8 a{static_cast<const uint8_t *>(x_codes), static_cast<const uint8_t *>(x_scales), static_cast<const uint8_t *>(codes),
                     static_cast<const uint8_t *>(scales), y, 0, y_stride, 0, nullptr, (uint32_t)m, (uint32_t)n, (uint32_t)k, (uint32_t)((k + 127) / 128),
                     (uint32_t)fp8_scale_row(k), 0, 0, 0, dtype};
    const hipStream_t s = (hipStream_t)stream;
    return exact_of(dtype) ? launch<true>(a, workspace, s) : launch<false>(a, workspace, s);
}

#ifdef ENEC_TEST_HOOKS
// What a call of these sizes launches: the tile's number, -1 for the kernel for few tokens, -2 for the one that brings them into 8 bits itself; splits; the latter two kernels' waves,
// and their tiles of sixteen tokens.
void enec_test_fp8_plan(size_t m, size_t n, size_t k, int y_dtype, int linear, int32_t *out)
{
    const uint32_t groups = (uint32_t)((k + 127) / 128), tiles = thin_tiles((uint32_t)m);
    if (linear && x_inside((uint32_t)m, (uint32_t)n, groups)) {
        out[0] = -2, out[1] = 1, out[2] = (int32_t)waves_inside((uint32_t)n, groups), out[3] = 1;
        return;
    }
    const Plan p = plan_of((uint32_t)m, (uint32_t)n, groups, exact_of(y_dtype));
    out[0] = p.shape, out[1] = (int32_t)p.splits, out[2] = p.shape < 0 ? (int32_t)thin_waves(tiles, groups) : 0, out[3] = p.shape < 0 ? (int32_t)tiles : 0;
}
#endif

}  // extern "C"
