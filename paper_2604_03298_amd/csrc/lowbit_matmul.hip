// Products with weights in microscaled 4-bit floating point.  The definitions stand in include/enec_lowbit.h.
#include "enec_lowbit.h"
#include "lowbit_product.hpp"

#include <atomic>

namespace enec {
namespace lowbit {

enum { MX4 = 3 };                       // activations in 4 bits, beside BF16 and FP16

struct Product {
    const void *x;                      // activations: 16-bit values, or codes
    const uint8_t *x_scales, *codes, *scales;
    void *y;
    size_t x_stride, y_stride;          // elements
    uint32_t m, n, k, groups;           // groups of 128 columns
    int y_dtype;
    // bytes between rows of x, and of a row; the tiles; the stages of a split and where their sums go
    size_t x_row, part_row;
    uint32_t x_bytes, n_tiles, m_tiles, split_stages;
    float *parts;
};

// The instruction takes one of the four scale bytes of a register; which one is part of the instruction.
template <int S> __device__ __forceinline__ f32x4 mfma_mx4_byte(const u32x4 &a, const u32x4 &b, const f32x4 &c, int sa, int sb)
{
    const i32x8 x = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0}, y = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, S, sa, S, sb);
}
__device__ __forceinline__ f32x4 mfma_mx4(int s, const u32x4 &a, const u32x4 &b, const f32x4 &c, int sa, int sb)
{
    return s == 0   ? mfma_mx4_byte<0>(a, b, c, sa, sb)
           : s == 1 ? mfma_mx4_byte<1>(a, b, c, sa, sb)
           : s == 2 ? mfma_mx4_byte<2>(a, b, c, sa, sb)
                    : mfma_mx4_byte<3>(a, b, c, sa, sb);
}
// eight codes as bf16 values: at most two significant bits and the scale's power of two, so exact; a scale of infinity makes each NaN
__device__ __forceinline__ bf16x8 values_of(uint32_t codes, float scale)
{
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// The same as fp16 values without their scale, whose range is bf16's and not fp16's: each block's sum takes it instead, which is five instructions for
// a matrix instruction.  (fp16 activations as the sum of two bf16 numbers need none, but twice the matrix instructions: 2048 tokens x 4096 x 11008
// 300 us instead of 255, one token x 8192 x 28672 41 instead of 28.)
__device__ __forceinline__ f16x8 unscaled_values_of(uint32_t codes)
{
    const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, 1.0f, 1);
    const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, 1.0f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, 1.0f, 3);
    return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// Word j of the four lanes sixteen apart becomes lane j's, in the order of the lanes: exchanges of halves, then of quarters.  As instructions of their own,
// see over_groups_max in lowbit_attention.hip.
__device__ __forceinline__ void exchange_words(u32x4 &v)
{
    uint32_t a = v[0], b = v[1], c = v[2], d = v[3];
    asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %2\n\tv_permlane32_swap_b32 %1, %3\n\ts_nop 1\n\tv_permlane16_swap_b32 %0, %1\n\tv_permlane16_swap_b32 %2, %3"
        : "+v"(a), "+v"(b), "+v"(c), "+v"(d));
    v = u32x4{a, b, c, d};
}
// 2^(byte - 127), byte j of a word; 255: infinity
__device__ __forceinline__ float scale_of(uint32_t bytes, int j)
{
    const uint32_t e = (j < 3 ? bytes << (23 - 8 * j) : bytes >> 1) & 0x7F800000u;
    return f32_of_bits(e > 0x00400000u ? e : 0x00400000u);
}
// How a stage lies in LDS.  A row (of weights, or a token's) is a run of chunks of 16 bytes, chunk i at place i ^ turn(row).  A wave reads 16 bytes a lane
// in four goes of sixteen lanes, lanes {0-3, 12-15, 20-27} the first: rows {0-3, 12-15} of one lane group and rows {4-11} of its neighbour.  Each
// turn puts such sixteen chunks into the sixteen different places of 256 bytes, so that no bank is asked twice:
//   256 bytes a row: the groups' chunks four apart (bf16 activations), or one apart (fp16, where a step is one block: the turn is the row itself)
//   128 bytes, one apart (4-bit ones, and their weights); 64 bytes, one apart
template <int ROW> __device__ __forceinline__ uint32_t turn(uint32_t r)
{
    if constexpr (ROW == 256) return (r & 3) + 12 * (r >> 3 & 1);
    if constexpr (ROW == 128) return (r & 2) + 4 * (r >> 3 & 1);
    return 2 * (r >> 3 & 1);
}

// Weights are the left operand of the matrix instructions, activations the right one (fp16: the other way round).
// A workgroup has 16 RT WN rows of weights and 16 MT WM tokens; a wave 16 RT rows and 16 MT tokens of them.  Where there are few tokens the rows of a
// workgroup are few too, so that all compute units have some, and KG groups of waves take its stages in turn; their sums meet in LDS (128 tokens x 4096
// x 11008 bf16: two groups 19 us, one 22; one token x 8192 x 28672: four groups 22, one 41).  A stage is 128 columns (4-bit activations: 256), whose
// codes, scales and activations the memory unit brings into LDS, BUFFERS stages in turn.  Loads straight into registers were slower: a lane has a row of
// its own there, so that each lane's 16 bytes are an access by themselves to the vector cache, where four neighbouring lanes of a copy make one
// (2048 tokens x 4096 x 16384: 125 million accesses and 272 us then; the cache takes about one in a cycle).
// As left operand a lane has row lane mod 16, and of a stage's blocks of 32 columns block lane / 16 (or 4 s + lane / 16 at step s).
// Few tokens: bound by the weights' way from memory, of which too little is asked for at a time: a stage is 2 KB of weights for 32 rows and 4 KB of
// activations, mostly of tokens that are not there.  4096 x 11008 bf16 with one token 7.3 us a call (3.3 TB/s; 7.0 to 8.2 the kernel, 6.4 to 6.6 with 4-bit
// activations, whose stages are twice as long), 32 tokens 8.0, 8192 x 28672 with one token 22 (5.7 TB/s).
// Many: by the matrix unit and the waits of two stages, at whose ends all copies have to be in LDS and all waves meet: matrix instructions take 48 % of the
// cycles (bf16) and 44 (4 bits), waits 28 and 32 % of the waves' time.  4096 tokens x 8192 x 28672 bf16 1420 to 1440 us (1340 TFLOP/s; a large library product of bf16 reaches 1378 on this card), fp16 238 to 268 us
// for 2048 x 4096 x 11008 (690 to 775 TFLOP/s; five vector instructions scale each block's sum), 4-bit activations 490 to 527 us for 4096 x 8192 x 28672 (3650
// to 3930 TFLOP/s).
template <int ACT, int RT, int MT, int WN, int WM, int KG, int BUFFERS>
__global__ void __launch_bounds__(64 * WN * WM * KG, RT * MT > 32 ? 1 : 2) product_tile_kernel(Product a)
{
    constexpr int THREADS = 64 * WN * WM, ALL = THREADS * KG, TOKENS = 16 * MT * WM, ROWS = 16 * RT * WN;
    constexpr int X_ROW = ACT == MX4 ? 128 : 256, W_ROW = ACT == MX4 ? 128 : 64, X_CHUNKS = X_ROW / 16, W_CHUNKS = W_ROW / 16;
    constexpr int X_SIZE = TOKENS * X_ROW, W_SIZE = ROWS * W_ROW, S_SIZE = ROWS * 16, XS_SIZE = ACT == MX4 ? TOKENS * 16 : 0;
    constexpr uint32_t S_STAGES = ACT == MX4 ? 2 : 4;                    // that sixteen bytes of scales are for
    constexpr int BLOCKS = KG > (int)S_STAGES ? KG / S_STAGES : 1;       // of scales that a round of stages needs
    constexpr int X_COPIES = X_SIZE / 16 / THREADS, W_COPIES = W_SIZE / 16 / THREADS;
    static_assert(KG == 1 || KG % S_STAGES == 0 || S_STAGES % KG == 0, "rounds and blocks of scales end together");
    static_assert(ACT != FP16 || MT <= 4, "all tokens' tiles at once");
    static_assert(X_SIZE % (16 * THREADS) == 0 && W_SIZE % (16 * THREADS) == 0 && S_SIZE % 256 == 0 && XS_SIZE % 256 == 0, "whole copies of a wave");
    constexpr int U = MT < 4 ? MT : 4, STEPS = ACT == MX4 ? 2 : 4, UNITS = STEPS * (MT / U);
    extern __shared__ __attribute__((aligned(16))) uint8_t shared[];
    uint8_t *x_stages = shared, *w_stages = shared + BUFFERS * KG * X_SIZE;
    uint8_t *scale_bytes = w_stages + BUFFERS * KG * W_SIZE;           // two of BLOCKS (S_SIZE + XS_SIZE), in turn
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, c = lane & 15;
    const uint32_t kg = wave / (WN * WM), mate = wave % (WN * WM), thread = threadIdx.x % THREADS;      // wave and thread of the group
    const uint32_t wn = mate % WN, wm = mate / WN;
    // Workgroups are dealt out to the eight dies one by one.  Each die takes a run of tiles, tokens first, in bands of six tiles of tokens: the tiles that
    // it works on at a time are about as many rows of weights as of activations, and it reads the fewest of both (4096 tokens x 8192 x 28672: 1400 us,
    // all tokens in one band 1520, bands of one 1460; in 4 bits 490, 520, 520).
    constexpr uint32_t BAND = 6;
    const uint32_t tiles = a.n_tiles * a.m_tiles, per_die = (tiles + 7) / 8, tile = blockIdx.x % 8 * per_die + blockIdx.x / 8;
    if (tile >= tiles) return;
    const uint32_t before = tile / (BAND * a.n_tiles) * BAND, band = a.m_tiles - before < BAND ? a.m_tiles - before : BAND;
    const uint32_t within = tile - before * a.n_tiles, n0 = within / band * ROWS, m0 = (before + within % band) * TOKENS;
    const uint32_t rows = a.n - n0 < ROWS ? a.n - n0 : ROWS, tokens = a.m - m0 < TOKENS ? a.m - m0 : TOKENS;
    const uint32_t w_pitch = a.groups * 64, s_pitch = a.groups * 4, x_pitch = (uint32_t)a.x_row;
    const Range codes = range_of(a.codes + (size_t)n0 * w_pitch, rows * w_pitch), scales = range_of(a.scales + (size_t)n0 * s_pitch, rows * s_pitch);
    const Range x = range_of(static_cast<const uint8_t *>(a.x) + (size_t)m0 * a.x_row, (tokens - 1) * x_pitch + a.x_bytes);
    const Range x_scales = range_of(ACT == MX4 ? a.x_scales + (size_t)m0 * s_pitch : a.scales, ACT == MX4 ? tokens * s_pitch : 0);

    const uint32_t first = blockIdx.y * a.split_stages, stages = ACT == MX4 ? (a.groups + 1) / 2 : a.groups;
    const uint32_t end = first + a.split_stages < stages ? first + a.split_stages : stages;

    // the chunk of row r that belongs to this thread's place
    auto x_turn = [](uint32_t r) { return ACT == FP16 ? r : turn<X_ROW>(r); };
    auto x_from = [&](uint32_t r) { return r * x_pitch + 16 * ((thread % X_CHUNKS) ^ x_turn(r & 15)); };
    auto w_from = [&](uint32_t r) { return r * w_pitch + 16 * ((thread % W_CHUNKS) ^ turn<W_ROW>(r & 15)); };
    const uint32_t s_from = threadIdx.x / 4 * s_pitch + 4 * (threadIdx.x % 4);
    auto copy = [&](uint32_t i, uint32_t buffer) {
        uint8_t *x_to = x_stages + (buffer * KG + kg) * X_SIZE, *w_to = w_stages + (buffer * KG + kg) * W_SIZE;
#pragma unroll
        for (int r = 0; r < X_COPIES; ++r)
            copy_to_lds<16>(x, x_from(thread / X_CHUNKS + r * (THREADS / X_CHUNKS)) + i * X_ROW, x_to + (r * THREADS + mate * 64) * 16);
#pragma unroll
        for (int r = 0; r < W_COPIES; ++r)
            copy_to_lds<16>(codes, w_from(thread / W_CHUNKS + r * (THREADS / W_CHUNKS)) + i * W_ROW, w_to + (r * THREADS + mate * 64) * 16);
    };
    // Scales come for several stages at once, sixteen bytes of each row: four lanes' words are one access.
    auto copy_scales = [&](uint32_t block, uint32_t turn_of) {
#pragma unroll
        for (int k = 0; k < BLOCKS; ++k) {
            uint8_t *to = scale_bytes + ((turn_of & 1) * BLOCKS + k) * (S_SIZE + XS_SIZE);
#pragma unroll
            for (int r = 0; r * ALL * 4 < S_SIZE; ++r)
                if ((r * ALL + wave * 64) * 4 < S_SIZE)
                    copy_to_lds<4>(scales, s_from + r * (ALL / 4) * s_pitch + (block + k) * 16, to + (r * ALL + wave * 64) * 4);
#pragma unroll
            for (int r = 0; r * ALL * 4 < XS_SIZE; ++r)
                if ((r * ALL + wave * 64) * 4 < XS_SIZE)
                    copy_to_lds<4>(x_scales, s_from + r * (ALL / 4) * s_pitch + (block + k) * 16, to + S_SIZE + (r * ALL + wave * 64) * 4);
        }
    };
    // A wave's copies are counted, and done in the order in which they were issued: with at most AHEAD left, those before them are in LDS.  Then
    // all waves' are, and nobody reads the stage before any more.
    constexpr int AHEAD = (BUFFERS - 2) * (X_COPIES + W_COPIES);         // at least so many copies are of the next round
    auto landed = [&](bool last) {
        __builtin_amdgcn_sched_barrier(0);
        if (AHEAD == 0 || last) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(AHEAD) : "memory");
        __builtin_amdgcn_sched_barrier(0);
    };

    // where this lane's chunks lie: of tokens c, 16 + c, ..., and of rows c, 16 + c, ...
    uint32_t x_at[STEPS], w_at[2];
#pragma unroll
    for (int j = 0; j < STEPS; ++j) x_at[j] = (wm * (16 * MT) + c) * X_ROW + (((ACT != BF16 ? 4 * j + g : 4 * g + j) ^ x_turn(c)) << 4);
#pragma unroll
    for (int j = 0; j < 2; ++j) w_at[j] = (wn * (16 * RT) + c) * W_ROW + (((ACT == MX4 ? 4 * j + g : g) ^ turn<W_ROW>(c)) << 4);
    auto x_chunk = [&](const uint8_t *t, int j, int u) { return *reinterpret_cast<const u32x4 *>(t + x_at[j] + u * (16 * X_ROW)); };
    auto w_chunk = [&](const uint8_t *t, int j, int r) { return *reinterpret_cast<const u32x4 *>(t + w_at[j] + r * (16 * W_ROW)); };

    f32x4 acc[RT][MT] = {};
    // Group kg takes stages first + kg, first + KG + kg, ..., in rounds that all groups begin together.
    constexpr uint32_t ROUND = KG > 1 ? KG : 1;
    const uint32_t rounds = (end - first + ROUND - 1) / ROUND, per_block = KG > 1 ? (S_STAGES > KG ? S_STAGES / KG : 1) : S_STAGES;
    auto stage_of = [&](uint32_t round) { return first + round * ROUND + (KG > 1 ? kg : 0); };
    auto fetch = [&](uint32_t round) {
        const uint32_t i = stage_of(round);
        copy(i < end ? i : end - 1, round % BUFFERS);
    };
    copy_scales(first / S_STAGES, 0);                       // (a split begins with such a block)
    fetch(0);
    if (BUFFERS == 3 && rounds > 1) fetch(1);
    for (uint32_t round = 0; round < rounds; ++round) {
        landed(round + 1 >= rounds);
        const uint32_t i = stage_of(round);
        if (round % per_block == 0 && round + per_block < rounds) copy_scales(first / S_STAGES + (round / per_block + 1) * BLOCKS, round / per_block + 1);
        if (round + BUFFERS - 1 < rounds) fetch(round + BUFFERS - 1);
        if (KG > 1 && i >= end) continue;
        const uint8_t *x_now = x_stages + (round % BUFFERS * KG + kg) * X_SIZE, *w_now = w_stages + (round % BUFFERS * KG + kg) * W_SIZE;
        const uint8_t *ws_now = scale_bytes + ((round / per_block & 1) * BLOCKS + (KG > 1 ? kg / S_STAGES : 0)) * (S_SIZE + XS_SIZE) + (16 / S_STAGES) * (i % S_STAGES);
        // tokens' tiles are taken U at a time; the next ones' chunks are asked for before these are multiplied, and no earlier
        u32x4 xv[2][U];
        if constexpr (ACT == MX4) {
            u32x4 w[2][RT];
            uint32_t ws[RT], xs[MT];
            const uint32_t pick = 0x0c0c0400u + 0x101u * g;              // of a row's eight bytes this lane's block's two
#pragma unroll
            for (int t = 0; t < RT; ++t) w[0][t] = w_chunk(w_now, 0, t);
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                const u32x2 v = *reinterpret_cast<const u32x2 *>(ws_now + (wn * (16 * RT) + 16 * t + c) * 16);
                ws[t] = __builtin_amdgcn_perm(v[1], v[0], pick);
            }
#pragma unroll
            for (int u = 0; u < MT; ++u) {
                const u32x2 v = *reinterpret_cast<const u32x2 *>(ws_now + S_SIZE + (wm * (16 * MT) + 16 * u + c) * 16);
                xs[u] = __builtin_amdgcn_perm(v[1], v[0], pick);
            }
            if (i == a.groups / 2) {                                     // one group only: the other's bytes are not this row's
#pragma unroll
                for (int t = 0; t < RT; ++t) ws[t] &= 255;
#pragma unroll
                for (int u = 0; u < MT; ++u) xs[u] &= 255;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) xv[0][u] = x_chunk(x_now, 0, u);
#pragma unroll
            for (int k = 0; k < UNITS; ++k) {
                const int s = k / (MT / U), b = k % (MT / U), next = k + 1;
                __builtin_amdgcn_sched_barrier(0);
                if (next < UNITS) {
#pragma unroll
                    for (int u = 0; u < U; ++u) xv[next & 1][u] = x_chunk(x_now, next / (MT / U), next % (MT / U) * U + u);
                }
                if (k == 0) {
#pragma unroll
                    for (int t = 0; t < RT; ++t) w[1][t] = w_chunk(w_now, 1, t);
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int t = 0; t < RT; ++t) acc[t][b * U + u] = mfma_mx4(s, w[s][t], xv[k & 1][u], acc[t][b * U + u], (int)ws[t], (int)xs[b * U + u]);
            }
        } else if constexpr (ACT == FP16) {
            // A step is a block of 32 columns.  Weights are the right operand here: all sums of a lane are of one row, and so is the scale.
            u32x4 w[RT];
            uint32_t ws[RT];
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                w[t] = w_chunk(w_now, 0, t);
                ws[t] = *reinterpret_cast<const uint32_t *>(ws_now + (wn * (16 * RT) + 16 * t + c) * 16);
                if ((ws[t] >> (8 * g) & 255) == 255) w[t] = u32x4{};    // 0 * infinity, whatever the codes are
                exchange_words(w[t]);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) xv[0][u] = x_chunk(x_now, 0, u);
#pragma unroll
            for (int j = 0; j < STEPS; ++j) {
                __builtin_amdgcn_sched_barrier(0);
                if (j + 1 < STEPS) {
#pragma unroll
                    for (int u = 0; u < U; ++u) xv[(j + 1) & 1][u] = x_chunk(x_now, j + 1, u);
                }
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    const f16x8 wv = unscaled_values_of(w[t][j]);
                    const float by = scale_of(ws[t], j);
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const f32x4 sum = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, xv[j & 1][u]), wv, f32x4{}, 0, 0, 0);
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[t][u][e] = __builtin_fmaf(sum[e], by, acc[t][u][e]);
                    }
                }
            }
        } else {
            u32x4 w[RT];
            uint32_t ws[RT];
            bf16x8 wv[2][RT];
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                w[t] = w_chunk(w_now, 0, t);
                ws[t] = ws_now[(wn * (16 * RT) + 16 * t + c) * 16 + g];
            }
#pragma unroll
            for (int u = 0; u < U; ++u) xv[0][u] = x_chunk(x_now, 0, u);
#pragma unroll
            for (int t = 0; t < RT; ++t) wv[0][t] = values_of(w[t][0], f32_of_bits(ws[t] << 23));
#pragma unroll
            for (int k = 0; k < UNITS; ++k) {
                const int j = k / (MT / U), b = k % (MT / U), next = k + 1;
                __builtin_amdgcn_sched_barrier(0);
                if (next < UNITS) {
#pragma unroll
                    for (int u = 0; u < U; ++u) xv[next & 1][u] = x_chunk(x_now, next / (MT / U), next % (MT / U) * U + u);
                }
                if (b == MT / U - 1 && j < 3) {
#pragma unroll
                    for (int t = 0; t < RT; ++t) wv[(j + 1) & 1][t] = values_of(w[t][j + 1], f32_of_bits(ws[t] << 23));
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int t = 0; t < RT; ++t)
                        acc[t][b * U + u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[j & 1][t], __builtin_bit_cast(bf16x8, xv[k & 1][u]), acc[t][b * U + u], 0, 0, 0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (KG > 1) {                                 // the groups' sums, in their order; LDS is free now
        f32x4 *sums = reinterpret_cast<f32x4 *>(shared);
        __syncthreads();
        if (kg != 0) {
#pragma unroll
            for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int u = 0; u < MT; ++u) sums[(((kg - 1) * WN * WM + mate) * RT * MT + t * MT + u) * 64 + lane] = acc[t][u];
        }
        __syncthreads();
        if (kg != 0) return;
#pragma unroll
        for (int k = 1; k < KG; ++k)
#pragma unroll
            for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int u = 0; u < MT; ++u) acc[t][u] += sums[(((k - 1) * WN * WM + mate) * RT * MT + t * MT + u) * 64 + lane];
    }
    if constexpr (ACT == FP16) {                            // four tokens of a row
#pragma unroll
        for (int u = 0; u < MT; ++u)
#pragma unroll
            for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t token = m0 + wm * (16 * MT) + 16 * u + 4 * g + e, r = n0 + 16 * (wn * RT + t) + c;
                    if (token >= a.m || r >= a.n) continue;
                    if (a.parts) a.parts[((size_t)blockIdx.y * a.m + token) * a.part_row + r] = acc[t][u][e];
                    else static_cast<_Float16 *>(a.y)[(size_t)token * a.y_stride + r] = (_Float16)acc[t][u][e];
                }
        return;
    }
#pragma unroll
    for (int u = 0; u < MT; ++u) {
        const uint32_t token = m0 + wm * (16 * MT) + 16 * u + c;
        if (token >= a.m) continue;
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const uint32_t r = n0 + 16 * (wn * RT + t) + 4 * g;
            if (r >= a.n) continue;
            if (a.parts) *reinterpret_cast<f32x4 *>(a.parts + ((size_t)blockIdx.y * a.m + token) * a.part_row + r) = acc[t][u];
            else store4(a.y, a.y_dtype, (size_t)token * a.y_stride + r, a.n - r, acc[t][u]);
        }
    }
}

// Activations as the kernel above copies them: rows of a multiple of 128 columns, zeros behind the last one.
__global__ void __launch_bounds__(256) lay_out_kernel(const uint16_t *__restrict__ x, size_t x_stride, uint32_t k, Divide per_row, uint32_t n_vec,
                                                      u32x4 *__restrict__ out)
{
    const uint32_t at = blockIdx.x * 256u + threadIdx.x;
    if (at >= n_vec) return;
    const uint32_t row = quotient(at, per_row), col = (at - row * per_row.by) * 8u;
    const uint16_t *p = x + (size_t)row * x_stride + col;
    u32x4 v = {};
    if (col + 8 <= k) {
        v = *reinterpret_cast<const u32x4_a2 *>(p);
    } else if (col < k) {                                   // (loads that do not wait for one another)
        uint32_t e[8];
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) e[i] = p[col + i < k ? i : k - 1 - col];
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) v[i >> 1] |= (col + i < k ? e[i] : 0) << (16 * (i & 1));
    }
    out[at] = v;
}

}  // namespace lowbit
}  // namespace enec

namespace {

using namespace enec::lowbit;

inline bool aligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// The tiles there are.  `resident` workgroups of one fit a compute unit (by LDS), and with all of them there a round of stages, `stages` of them, takes
// `us` (fitted to times of 1 to 4096 tokens with matrices of 4096 x 1024 to 8192 x 28672, as are the constants of plan_of; of 104 products over 12 us, with
// every tile and split forced, the choice is within 5 % of the best for 82, within 10 % for 93, and a third off for the worst).
struct Shape {
    uint32_t rows, tokens, resident, stages;
    double us;
};
constexpr Shape SHAPES[3][7] = {
    {{256, 128, 1, 1, 1.72}, {256, 64, 2, 1, 1.90}, {128, 64, 3, 1, 1.48}, {128, 32, 3, 1, 1.20}, {64, 32, 1, 4, 0.70},
     {32, 16, 2, 4, 0.60}, {128, 64, 1, 2, 1.08}},
    {{256, 128, 1, 1, 2.75}, {256, 64, 2, 1, 2.80}, {128, 64, 3, 1, 2.10}, {128, 32, 3, 1, 1.45}, {64, 32, 1, 4, 0.90},
     {32, 16, 2, 4, 0.75}, {128, 64, 1, 2, 1.80}},
    {{256, 256, 1, 1, 2.49}, {128, 128, 2, 1, 1.40}, {128, 64, 2, 1, 1.39}, {128, 32, 2, 1, 0.90}, {64, 32, 1, 4, 0.80},
     {32, 16, 2, 4, 0.50}, {128, 64, 1, 2, 1.10}},
};
constexpr double THIN[3] = {0.05, 0.10, 0.05};      // what a workgroup that is not there costs of the time saved: less overlaps
constexpr const Shape *shapes_of(int act) { return SHAPES[act == MX4 ? 2 : act]; }
static_assert(BF16 == 0 && FP16 == 1, "the tables' order");
constexpr uint32_t UNITS = 256;                     // compute units

// How a product is cut up: the tile, and the splits of the columns where tiles alone leave the card empty.
struct Plan {
    int shape;
    uint32_t splits, split_stages;
};
constexpr uint32_t MOST_SPLITS = 16, UNIT = 4;      // a split is whole blocks of scales and whole rounds: so many stages, or a multiple

inline uint32_t stages_of(uint32_t k, int act) { return act == MX4 ? up(up(k, 128), 2) : up(k, 128); }

Plan plan_of(uint32_t m, uint32_t n, uint32_t k, int act)
{
    Plan p{};
    const bool mx4 = act == MX4;
    const uint32_t stages = stages_of(k, act);
    double best = 1e300;
    for (int i = 0; i < 7; ++i) {
        const Shape &s = shapes_of(act)[i];
        if (s.tokens > 16 && s.tokens >= 2 * up(m, 16) * 16) continue;       // half of the tile or more would be empty
        const uint64_t tiles = (uint64_t)up(n, s.rows) * up(m, s.tokens), full = UNITS * s.resident;
        const bool splittable = (uint64_t)m * up(n, 4) < 1u << 31;
        for (uint32_t splits = 1; splits == 1 || (splittable && splits <= MOST_SPLITS && splits * UNIT <= stages && tiles * (splits / 2) < full); splits *= 2) {
            const uint32_t each = up(up(stages, splits), UNIT) * UNIT, count = up(stages, each);
            // The busiest compute unit has `most` workgroups.  Fewer than fit take their share of the time and some more; where one fits and not all
            // units have one, memory has less to do; past that the units drift apart, and half of the last round's waste goes.  A workgroup's start and end are
            // 3 us, and joining is a launch, the sums' way out and back.
            const uint64_t all = tiles * count, most = (all + UNITS - 1) / UNITS, left = most % s.resident;
            double turns = (double)(most / s.resident) + (left ? (double)left / s.resident + (s.resident - left) * THIN[mx4 ? 2 : act] : 0);
            if (s.resident == 1 && all * 4 < most * UNITS * 3) turns *= 0.88;
            if (turns > 2 || (s.resident > 1 && all > UNITS)) turns = (turns + (double)all / full) / 2;
            const double us = turns * (up(each, s.stages) * s.us + 3) + (count > 1 ? 4 + (double)count * m * n * 8 / 4e6 : 0);
            if (us < best) best = us, p.shape = i, p.splits = count, p.split_stages = each;
        }
    }
    return p;
}

// Bytes for the sums of the splits: of no more than m tokens, however few, so that one piece serves products of any number of them (fewer may be split
// more).  Splits and tiles together are below twice what the card holds, which bounds the splits' tokens by the tile's.
size_t parts_of(uint32_t m, uint32_t n, uint32_t k, int act)
{
    uint32_t splits = 1;
    while (splits < MOST_SPLITS && splits * 2 * UNIT <= stages_of(k, act)) splits *= 2;
    uint64_t most = 0;
    for (int i = 0; i < 7 && splits > 1; ++i) {
        const Shape &s = shapes_of(act)[i];
        if (s.tokens > 16 && s.tokens >= 2 * up(m, 16) * 16) continue;
        const uint64_t full = UNITS * s.resident, by_tiles = s.tokens * (2 * (full - 1) / up(n, s.rows)), by_splits = (uint64_t)splits * m;
        const uint64_t rows = by_tiles < by_splits ? by_tiles : by_splits;
        most = most > rows ? most : rows;
    }
    return most * part_row(n) * sizeof(float);
}

// A copy of the activations, and the sums.  (It is the same for both formats, and for activations that need no copy.)
inline size_t laid_out_bytes(uint32_t m, uint32_t k) { return 2 * (size_t)m * (up(k, 128) * 128); }
size_t linear_space(uint32_t m, uint32_t n, uint32_t k)
{
    const size_t a = parts_of(m, n, k, BF16), b = parts_of(m, n, k, FP16);
    return laid_out_bytes(m, k) + (a > b ? a : b);
}

template <int ACT, int RT, int MT, int WN, int WM, int KG, int BUFFERS> bool launch_tile(const Product &a, uint32_t splits, hipStream_t s)
{
    constexpr size_t TOKENS = 16 * MT * WM, ROWS = 16 * RT * WN;
    static std::atomic<uint64_t> allowed{0};
    constexpr size_t STAGES = KG * BUFFERS * (TOKENS * (ACT == MX4 ? 128 : 256) + ROWS * (ACT == MX4 ? 128 : 64));
    constexpr size_t BLOCKS = ACT == MX4 && KG == 4 ? 2 : 1, LDS = STAGES + 2 * BLOCKS * 16 * (ACT == MX4 ? TOKENS + ROWS : ROWS);
    static_assert(LDS <= 160 * 1024 && (KG - 1) * 4 * TOKENS * ROWS <= LDS, "LDS of a compute unit; the groups' sums take the stages' place");
    const auto kernel = product_tile_kernel<ACT, RT, MT, WN, WM, KG, BUFFERS>;
    if (LDS > 65536 && !allow_lds((const void *)kernel, LDS, allowed)) return false;
    kernel<<<dim3(up(a.n_tiles * a.m_tiles, 8) * 8, splits), 64 * WN * WM * KG, LDS, s>>>(a);
    return true;
}

template <int ACT> int launch(Product a, const Plan &p, void *workspace, hipStream_t s)
{
    if (a.k == 0) {
        const uint32_t per_row = up(a.n, 4);
        join_kernel<<<up(a.m * per_row, 256), 256, 0, s>>>(nullptr, 0, a.m, a.n, 0, divide_by(per_row), a.y, a.y_stride, a.y_dtype);
        return hipGetLastError() == hipSuccess ? ENEC_OK : ENEC_E_HIP;
    }
    const Shape &shape = shapes_of(ACT)[p.shape];
    if constexpr (ACT == MX4) {
        a.x_row = a.x_bytes = a.groups * 64;
    } else if (a.k % 128 == 0 && a.x_stride % 8 == 0 && a.x_stride <= (1u << 22) && aligned(a.x, 16)) {
        a.x_row = a.x_stride * 2, a.x_bytes = a.k * 2;
    } else {
        const uint32_t cols = up(a.k, 128) * 128, n_vec = a.m * (cols / 8);
        lay_out_kernel<<<up(n_vec, 256), 256, 0, s>>>(static_cast<const uint16_t *>(a.x), a.x_stride, a.k, divide_by(cols / 8), n_vec,
                                                      static_cast<u32x4 *>(workspace));
        a.x = workspace;
        a.x_row = a.x_bytes = cols * 2;
    }
    a.n_tiles = up(a.n, shape.rows), a.m_tiles = up(a.m, shape.tokens), a.split_stages = p.split_stages;
    if (p.splits > 1) a.parts = reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) + (ACT == MX4 ? 0 : laid_out_bytes(a.m, a.k))), a.part_row = part_row(a.n);
    bool ok;
    switch (p.shape) {
    case 0: ok = launch_tile<ACT, 4, ACT == MX4 ? 8 : 4, 4, 2, 1, 2>(a, p.splits, s); break;
    case 1: ok = launch_tile<ACT, 4, 4, ACT == MX4 ? 2 : 4, ACT == MX4 ? 2 : 1, 1, 2>(a, p.splits, s); break;
    case 2: ok = launch_tile<ACT, 2, 4, 4, 1, 1, 2>(a, p.splits, s); break;
    case 3: ok = launch_tile<ACT, 2, 2, 4, 1, 1, 3>(a, p.splits, s); break;
    case 4: ok = launch_tile<ACT, 1, 2, 4, 1, 4, 2>(a, p.splits, s); break;
    case 5: ok = launch_tile<ACT, 1, 1, 2, 1, 4, 3>(a, p.splits, s); break;
    default: ok = launch_tile<ACT, 2, 4, 4, 1, 2, 2>(a, p.splits, s); break;
    }
    if (!ok) return ENEC_E_HIP;
    if (p.splits > 1) {
        const uint32_t per_row = up(a.n, 4);
        join_kernel<<<up(a.m * per_row, 256), 256, 0, s>>>(a.parts, p.splits, a.m, a.n, a.part_row, divide_by(per_row), a.y, a.y_stride, a.y_dtype);
    }
    return hipGetLastError() == hipSuccess ? ENEC_OK : ENEC_E_HIP;
}

// sizes that every kernel here can count with: offsets inside a tile have 31 bits, and so have the counts of vectors that are laid out and of tiles
inline bool sizes_ok(size_t m, size_t n, size_t k)
{
    return m <= (1u << 21) && n <= (1u << 26) && k <= (1u << 21) && m * k <= (size_t)1 << 34 && m * n <= (size_t)1 << 40 && (k != 0 || m * n < (size_t)1 << 33);
}

}  // namespace

extern "C" {

size_t enec_mx4_linear_workspace(size_t m, size_t n, size_t k)
{
    if (!sizes_ok(m, n, k) || m == 0 || n == 0 || k == 0) return 0;
    return linear_space((uint32_t)m, (uint32_t)n, (uint32_t)k);
}
size_t enec_mx4_matmul_workspace(size_t m, size_t n, size_t k)
{
    if (!sizes_ok(m, n, k) || m == 0 || n == 0 || k == 0) return 0;
    return parts_of((uint32_t)m, (uint32_t)n, (uint32_t)k, MX4);
}

int enec_mx4_linear(const void *x, size_t m, size_t x_stride, int dtype, const void *codes, const void *scales, size_t n, size_t k, void *y,
                    size_t y_stride, void *workspace, size_t workspace_bytes, void *stream)
{
    if (dtype != ENEC_BF16 && dtype != ENEC_FP16) return ENEC_E_DTYPE;
    if (!sizes_ok(m, n, k)) return ENEC_E_ARG;
    if (m == 0 || n == 0) return ENEC_OK;
    if (!y || !aligned(y, 2) || y_stride < n) return ENEC_E_ARG;
    if (k != 0 && (!x || !codes || !scales || !aligned(x, 2) || !aligned(codes, 16) || !aligned(scales, 4) || x_stride < k)) return ENEC_E_ARG;
    const Plan p = k == 0 ? Plan{} : plan_of((uint32_t)m, (uint32_t)n, (uint32_t)k, dtype);
    const size_t need = k == 0 ? 0 : linear_space((uint32_t)m, (uint32_t)n, (uint32_t)k);
    if (workspace_bytes < need || (need && !workspace)) return ENEC_E_CAPACITY;
    if (need && !aligned(workspace, 16)) return ENEC_E_ARG;
    const Product a{x, nullptr, static_cast<const uint8_t *>(codes), static_cast<const uint8_t *>(scales), y, x_stride, y_stride,
                    (uint32_t)m, (uint32_t)n, (uint32_t)k, (uint32_t)((k + 127) / 128), dtype, 0, 0, 0, 0, 0, 0, nullptr};
    return dtype == ENEC_BF16 ? launch<BF16>(a, p, workspace, (hipStream_t)stream) : launch<FP16>(a, p, workspace, (hipStream_t)stream);
}

int enec_mx4_matmul(const void *x_codes, const void *x_scales, size_t m, const void *codes, const void *scales, size_t n, size_t k, void *y,
                    size_t y_stride, int dtype, void *workspace, size_t workspace_bytes, void *stream)
{
    if (dtype != ENEC_BF16 && dtype != ENEC_FP16 && dtype != ENEC_FP32) return ENEC_E_DTYPE;
    if (!sizes_ok(m, n, k)) return ENEC_E_ARG;
    if (m == 0 || n == 0) return ENEC_OK;
    if (!y || !aligned(y, dtype == ENEC_FP32 ? 4 : 2) || y_stride < n) return ENEC_E_ARG;
    if (k != 0 && (!x_codes || !x_scales || !codes || !scales || !aligned(x_codes, 16) || !aligned(x_scales, 4) || !aligned(codes, 16) || !aligned(scales, 4)))
        return ENEC_E_ARG;
    const Plan p = k == 0 ? Plan{} : plan_of((uint32_t)m, (uint32_t)n, (uint32_t)k, MX4);
    const size_t need = k == 0 ? 0 : parts_of((uint32_t)m, (uint32_t)n, (uint32_t)k, MX4);
    if (workspace_bytes < need || (need && !workspace)) return ENEC_E_CAPACITY;
    if (need && !aligned(workspace, 16)) return ENEC_E_ARG;
    const Product a{x_codes, static_cast<const uint8_t *>(x_scales), static_cast<const uint8_t *>(codes), static_cast<const uint8_t *>(scales), y, 0, y_stride,
                    (uint32_t)m, (uint32_t)n, (uint32_t)k, (uint32_t)((k + 127) / 128), dtype, 0, 0, 0, 0, 0, 0, nullptr};
    return launch<MX4>(a, p, workspace, (hipStream_t)stream);
}

}  // extern "C"
