// Products with weights in microscaled 4-bit floating point.  The definitions stand in include/enec_lowbit.h.
#include "enec_lowbit.h"
#include "lowbit.hpp"

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
    // for many tokens: bytes between rows of x, and between its planes; the tiles; the stages of a split and where their sums go
    size_t x_row, part_row;
    uint32_t x_bytes, x_plane, n_tiles, m_tiles, split_stages;
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
// eight codes as bf16 values: at most two significant bits and the scale's power of two, so exact
__device__ __forceinline__ bf16x8 values_of(uint32_t codes, float scale)
{
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// An fp16 value is the sum of two bf16 values, exactly: eight of its eleven bits and the rest, whose exponents bf16 has room for.  The weights' scales
// have bf16's range and not fp16's, so fp16 activations are multiplied as these two.
__device__ __forceinline__ void split_fp16(const u32x4 &v, bf16x8 &hi, bf16x8 &lo)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const f32x2 f = unpack2<FP16>(v[j]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const __bf16 h = (__bf16)f[i];
            hi[2 * j + i] = h;
            lo[2 * j + i] = __builtin_isinf(f[i]) ? (__bf16)0.0f : (__bf16)(f[i] - (float)h);
        }
    }
}

__device__ __forceinline__ void store4(void *y, int dtype, size_t at, uint32_t valid, const f32x4 &v)
{
    if (dtype == FP32) {
        for (uint32_t i = 0; i < 4; ++i)
            if (i < valid) static_cast<float *>(y)[at + i] = v[i];
        return;
    }
    const u32x2 w = dtype == BF16 ? u32x2{pack2<BF16>(v[0], v[1]), pack2<BF16>(v[2], v[3])} : u32x2{pack2<FP16>(v[0], v[1]), pack2<FP16>(v[2], v[3])};
    uint16_t *p = static_cast<uint16_t *>(y) + at;
    if (valid >= 4) {
        *reinterpret_cast<u32x2_a2 *>(p) = w;
    } else {
        for (uint32_t i = 0; i < 4; ++i)
            if (i < valid) p[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
    }
}

// Weights are the left operand, 16 rows, activations the right one, 16 tokens.  A product over a row does not care about the order of
// its columns, so they are dealt out for the loads: of 512 columns a lane takes 128 in a row, four blocks, whose codes are 64
// consecutive bytes and whose scales are one word; at step s it multiplies with its block s.
// The waves of a workgroup share the rows and split the columns; their sums meet in LDS, in a fixed order.
template <int ACT, int RT, int MT, int W>
__global__ void __launch_bounds__(64 * W) product_few_kernel(Product a)
{
    __shared__ f32x4 sums[W][RT * MT][64];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, c = lane & 15;
    const uint32_t n0 = blockIdx.x * (16 * RT), m0 = blockIdx.y * (16 * MT);
    f32x4 acc[RT][MT] = {};
    const uint32_t steps = (a.groups + 3) / 4;
    for (uint32_t step = wave; step < steps; step += W) {
        const uint32_t group = 4 * step + g;
        const bool in = group < a.groups;
        u32x4 w[RT][4] = {};
        uint32_t ws[RT] = {};
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const uint32_t row = n0 + 16 * t + c;
            if (in && row < a.n) {
                const size_t at = (size_t)row * a.groups + group;
                ws[t] = reinterpret_cast<const uint32_t *>(a.scales)[at];
#pragma unroll
                for (int s = 0; s < 4; ++s) w[t][s] = reinterpret_cast<const u32x4 *>(a.codes)[at * 4 + s];
            }
        }
        if constexpr (ACT == MX4) {
            u32x4 x[MT][4] = {};
            uint32_t xs[MT] = {};
#pragma unroll
            for (int u = 0; u < MT; ++u) {
                const uint32_t token = m0 + 16 * u + c;
                if (in && token < a.m) {
                    const size_t at = (size_t)token * a.groups + group;
                    xs[u] = reinterpret_cast<const uint32_t *>(a.x_scales)[at];
#pragma unroll
                    for (int s = 0; s < 4; ++s) x[u][s] = static_cast<const u32x4 *>(a.x)[at * 4 + s];
                }
            }
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int t = 0; t < RT; ++t)
#pragma unroll
                    for (int u = 0; u < MT; ++u) acc[t][u] = mfma_mx4(s, w[t][s], x[u][s], acc[t][u], (int)ws[t], (int)xs[u]);
        } else {
            const uint16_t *x = static_cast<const uint16_t *>(a.x);
#pragma unroll
            for (int s = 0; s < 4; ++s) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t col = group * 128 + s * 32 + j * 8;
                    bf16x8 wv[RT];
#pragma unroll
                    for (int t = 0; t < RT; ++t) wv[t] = values_of(w[t][s][j], power_of(ws[t] >> (8 * s) & 255));
#pragma unroll
                    for (int u = 0; u < MT; ++u) {
                        const uint32_t token = m0 + 16 * u + c;
                        u32x4 v = {};
                        if (token < a.m) {
                            const uint16_t *p = x + (size_t)token * a.x_stride + col;
                            if (col + 8 <= a.k) {
                                v = *reinterpret_cast<const u32x4_a2 *>(p);
                            } else {
                                for (uint32_t i = 0; i < 8; ++i)
                                    if (col + i < a.k) v[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
                            }
                        }
                        if constexpr (ACT == BF16) {
                            const bf16x8 xv = __builtin_bit_cast(bf16x8, v);
#pragma unroll
                            for (int t = 0; t < RT; ++t) acc[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[t], xv, acc[t][u], 0, 0, 0);
                        } else {
                            bf16x8 hi, lo;
                            split_fp16(v, hi, lo);
#pragma unroll
                            for (int t = 0; t < RT; ++t) {
                                acc[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[t], lo, acc[t][u], 0, 0, 0);
                                acc[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[t], hi, acc[t][u], 0, 0, 0);
                            }
                        }
                    }
                }
            }
        }
    }
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int u = 0; u < MT; ++u) sums[wave][t * MT + u][lane] = acc[t][u];
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < RT * MT * 64; i += 64 * W) {
        const uint32_t tile = i >> 6, l = i & 63;
        f32x4 v = sums[0][tile][l];
        for (int w = 1; w < W; ++w) v += sums[w][tile][l];
        const uint32_t row = n0 + 16 * (tile / MT) + 4 * (l >> 4), token = m0 + 16 * (tile % MT) + (l & 15);
        if (token < a.m && row < a.n) store4(a.y, a.y_dtype, (size_t)token * a.y_stride + row, a.n - row, v);
    }
}

// ---- many tokens -------------------------------------------------------------------------------------------------------

// LDS rows of 256 bytes a token, sixteen chunks of 16 bytes; chunk i of token t lies at place i ^ (t mod 16), so that sixteen tokens'
// chunks of one number are in sixteen places and a wave's reads meet no bank twice.
constexpr int STAGE_ROW = 256;

// Memory through a descriptor, whose range the memory unit checks: what lies outside reads as zeros, so that neither the last rows nor the last
// columns need a branch.  Offsets are 32 bits wide, from a tile's first row; an offset of NOWHERE plus any inside a tile lies outside.
using Range = __amdgpu_buffer_rsrc_t;
constexpr uint32_t NOWHERE = 0x80000000u;
__device__ __forceinline__ Range range_of(const void *p, uint32_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, (int)bytes, 0x00020000);
}
__device__ __forceinline__ u32x4 read16(Range r, uint32_t at) { return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)at, 0, 0)); }
__device__ __forceinline__ uint32_t read4(Range r, uint32_t at) { return (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(r, (int)at, 0, 0); }
__device__ __forceinline__ uint32_t read2(Range r, uint32_t at) { return (uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(r, (int)at, 0, 0); }
// 16 bytes a lane into LDS, the lanes' side by side
__device__ __forceinline__ void copy_to_lds(Range r, uint32_t at, uint8_t *to)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void *)to, 16, (int)at, 0, 0, 0);
}

// A workgroup has 16 RT WN rows of weights and 16 MT WM tokens; a wave 16 RT rows and 16 MT tokens of them.  Activations of a stage go into LDS by the
// memory unit, two stages in turn, for all waves; weights go from memory into the registers of the waves that multiply with them, a stage ahead: at 4 bits
// they are a quarter of the bytes, and WM = 1 brings each of them to one wave only, which makes 16-bit values of it once.
// A stage is 256 bytes of a token.  16-bit activations: 128 columns, the halves of the four double blocks of 256 columns (a lane takes
// 32 bytes of codes in a row from a double block: whole lines of memory); 4-bit ones: 512 columns, as in the kernel above.
template <int ACT, int RT, int MT, int WN, int WM>
__global__ void __launch_bounds__(64 * WN * WM, 2) product_tile_kernel(Product a)
{
    constexpr int THREADS = 64 * WN * WM, TOKENS = 16 * MT * WM, ROWS = 16 * RT * WN, COPIES = TOKENS * STAGE_ROW / (16 * THREADS), U = MT == 4 ? 4 : 2;
    constexpr int UNITS = 4 * (MT / U), PLANES = ACT == FP16 ? 2 : 1;
    __shared__ __attribute__((aligned(16))) uint8_t stage[2][TOKENS * STAGE_ROW];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, c = lane & 15;
    const uint32_t wn = wave % WN, wm = wave / WN;
    // Workgroups are dealt out to the eight dies one by one.  Each die takes a run of tiles, tokens first, so that it reads few rows of weights.
    const uint32_t tiles = a.n_tiles * a.m_tiles, per_die = (tiles + 7) / 8, tile = blockIdx.x % 8 * per_die + blockIdx.x / 8;
    if (tile >= tiles) return;
    const uint32_t n0 = tile / a.m_tiles * ROWS, m0 = tile % a.m_tiles * TOKENS;
    const uint32_t rows = a.n - n0 < ROWS ? a.n - n0 : ROWS, tokens = a.m - m0 < TOKENS ? a.m - m0 : TOKENS;
    const uint32_t pitch = a.groups * 64;
    const Range codes = range_of(a.codes + (size_t)n0 * pitch, rows * pitch), scales = range_of(a.scales + (size_t)n0 * (a.groups * 4), rows * a.groups * 4);
    const Range x = range_of(static_cast<const uint8_t *>(a.x) + (size_t)m0 * a.x_row, (tokens - 1) * (uint32_t)a.x_row + a.x_bytes);

    const uint32_t stages = ACT == MX4 ? (a.groups + 3) / 4 : (a.groups + 1) / 2 * 2;      // (of one plane)
    const uint32_t first = blockIdx.y * a.split_stages, end = first + a.split_stages < stages ? first + a.split_stages : stages;

    uint32_t from[COPIES];
    const uint32_t chunk = (threadIdx.x & 15) ^ (threadIdx.x >> 4 & 15);
#pragma unroll
    for (int r = 0; r < COPIES; ++r) {
        const uint32_t token = r * (THREADS / 16) + (threadIdx.x >> 4);
        from[r] = (token < tokens ? token : tokens - 1) * (uint32_t)a.x_row + (ACT == MX4 ? 16 * chunk : 128 * (chunk >> 2) + 16 * (chunk & 3));
    }
    auto copy = [&](uint32_t i, uint32_t plane) {
        const uint32_t at = ACT == MX4 ? (4 * i + (chunk >> 2) < a.groups ? 256 * i : NOWHERE) : 256 * (i & ~1u) + 64 * (i & 1) + plane * a.x_plane;
        uint8_t *to = stage[(i * PLANES + plane) & 1] + wave * 1024;
#pragma unroll
        for (int r = 0; r < COPIES; ++r) copy_to_lds(x, at + from[r], to + r * (THREADS * 16));
    };
    // where this lane's chunks of its tokens lie: chunk 4 g + j of tokens c, 16 + c, ...
    uint32_t read[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) read[j] = (wm * (16 * MT) + c) * STAGE_ROW + (((4 * g + j) ^ c) << 4);
    auto chunk_at = [&](const uint8_t *s, int j, int u) { return *reinterpret_cast<const u32x4 *>(s + read[j] + u * (16 * STAGE_ROW)); };

    uint32_t row[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) row[t] = (16 * (wn * RT + t) + c) * a.groups;
    f32x4 acc[RT][MT] = {};
    uint32_t ws[RT], next_ws[RT];
    auto landed = [&]() {                                   // this wave's copies and loads are there, and then all waves' copies are
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };

    // In units of U tokens' tiles: the next unit's chunks are asked for before this one's are multiplied, and no earlier.
    if constexpr (ACT == MX4) {
        const Range x_scales = range_of(a.x_scales + (size_t)m0 * (a.groups * 4), tokens * a.groups * 4);
        u32x4 w[RT][4];
        uint32_t xs[MT], next_xs[MT];
        auto fetch = [&](uint32_t i, int s) {
            const uint32_t at = 4 * i + g < a.groups ? 256 * i + 64 * g + 16 * s : NOWHERE;
#pragma unroll
            for (int t = 0; t < RT; ++t) w[t][s] = read16(codes, row[t] * 64 + at);
        };
        auto fetch_scales = [&](uint32_t i) {
            const uint32_t at = 4 * i + g < a.groups ? 16 * i + 4 * g : NOWHERE;
#pragma unroll
            for (int t = 0; t < RT; ++t) next_ws[t] = read4(scales, row[t] * 4 + at);
#pragma unroll
            for (int u = 0; u < MT; ++u) next_xs[u] = read4(x_scales, (wm * (16 * MT) + 16 * u + c) * (a.groups * 4) + at);
        };
        copy(first, 0);
        fetch_scales(first);
#pragma unroll
        for (int s = 0; s < 4; ++s) fetch(first, s);
        for (uint32_t i = first; i < end; ++i) {
            landed();
#pragma unroll
            for (int t = 0; t < RT; ++t) ws[t] = next_ws[t];
#pragma unroll
            for (int u = 0; u < MT; ++u) xs[u] = next_xs[u];
            if (i + 1 < end) copy(i + 1, 0);
            fetch_scales(i + 1);
            const uint8_t *now = stage[i & 1];
            u32x4 xv[2][U];
#pragma unroll
            for (int u = 0; u < U; ++u) xv[0][u] = chunk_at(now, 0, u);
#pragma unroll
            for (int unit = 0; unit < UNITS; ++unit) {
                const int s = unit / (MT / U), b = unit % (MT / U), next = unit + 1;
                __builtin_amdgcn_sched_barrier(0);
                if (next < UNITS) {
#pragma unroll
                    for (int u = 0; u < U; ++u) xv[next & 1][u] = chunk_at(now, next / (MT / U), next % (MT / U) * U + u);
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int t = 0; t < RT; ++t) acc[t][b * U + u] = mfma_mx4(s, w[t][s], xv[unit & 1][u], acc[t][b * U + u], (int)ws[t], (int)xs[b * U + u]);
                if (b == MT / U - 1) fetch(i + 1, s);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    } else {
        u32x4 w[RT][2];
        auto fetch = [&](uint32_t i, int h) {                // the codes of stage i + h, i even
            const uint32_t at = 2 * i + g < 2 * a.groups ? 64 * i + 32 * g + 16 * h : NOWHERE;
#pragma unroll
            for (int t = 0; t < RT; ++t) w[t][h] = read16(codes, row[t] * 64 + at);
        };
        auto fetch_scales = [&](uint32_t i) {                // of stages i and i + 1
            const uint32_t at = 2 * i + g < 2 * a.groups ? 4 * i + 2 * g : NOWHERE;
#pragma unroll
            for (int t = 0; t < RT; ++t) next_ws[t] = read2(scales, row[t] * 4 + at);
        };
        copy(first, 0);
        fetch_scales(first);
        fetch(first, 0);
        fetch(first, 1);
        for (uint32_t i = first; i < end; i += 2) {          // (first and end are even)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int p = 0; p < PLANES; ++p) {
                    landed();
                    if (h == 0 && p == 0) {
#pragma unroll
                        for (int t = 0; t < RT; ++t) ws[t] = next_ws[t];
                        fetch_scales(i + 2);
                    }
                    if (p + 1 < PLANES) copy(i + h, p + 1);
                    else if (i + h + 1 < end) copy(i + h + 1, 0);
                    const uint8_t *now = stage[(h * PLANES + p) & 1];
                    u32x4 xv[2][U];
                    bf16x8 wv[RT];
#pragma unroll
                    for (int u = 0; u < U; ++u) xv[0][u] = chunk_at(now, 0, u);
#pragma unroll
                    for (int unit = 0; unit < UNITS; ++unit) {
                        const int j = unit / (MT / U), b = unit % (MT / U), next = unit + 1;
                        __builtin_amdgcn_sched_barrier(0);
                        if (b == 0) {
#pragma unroll
                            for (int t = 0; t < RT; ++t) wv[t] = values_of(w[t][h][j], f32_of_bits((ws[t] >> (8 * h) & 255) << 23));
                        }
                        if (next < UNITS) {
#pragma unroll
                            for (int u = 0; u < U; ++u) xv[next & 1][u] = chunk_at(now, next / (MT / U), next % (MT / U) * U + u);
                        }
#pragma unroll
                        for (int u = 0; u < U; ++u)
#pragma unroll
                            for (int t = 0; t < RT; ++t)
                                acc[t][b * U + u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[t], __builtin_bit_cast(bf16x8, xv[unit & 1][u]), acc[t][b * U + u], 0, 0, 0);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                fetch(i + 2, h);
            }
        }
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

// Activations as the kernel above copies them: bf16, rows of a multiple of 256 columns, zeros behind the last one; of fp16 two
// such rows one behind the other, the values' parts.
template <int DT>
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
    } else {
        for (uint32_t i = 0; i < 8; ++i)
            if (col + i < k) v[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
    }
    if constexpr (DT == BF16) {
        out[at] = v;
    } else {
        bf16x8 hi, lo;
        split_fp16(v, hi, lo);
        out[(size_t)row * (2 * per_row.by) + (at - row * per_row.by)] = __builtin_bit_cast(u32x4, hi);
        out[(size_t)row * (2 * per_row.by) + (at - row * per_row.by) + per_row.by] = __builtin_bit_cast(u32x4, lo);
    }
}

// The sums of the splits, in their order.
__global__ void __launch_bounds__(256) join_kernel(const float *__restrict__ parts, uint32_t splits, uint32_t m, uint32_t n, size_t part_row, Divide per_row,
                                                   void *y, size_t y_stride, int y_dtype)
{
    const uint32_t at = blockIdx.x * 256u + threadIdx.x, token = quotient(at, per_row), r = (at - token * per_row.by) * 4u;
    if (token >= m) return;
    const float *p = parts + (size_t)token * part_row + r;
    f32x4 v = *reinterpret_cast<const f32x4 *>(p);
    for (uint32_t i = 1; i < splits; ++i) v += *reinterpret_cast<const f32x4 *>(p + i * (m * part_row));
    store4(y, y_dtype, (size_t)token * y_stride + r, n - r, v);
}

}  // namespace lowbit
}  // namespace enec

namespace {

using namespace enec::lowbit;

inline bool aligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// How a product is cut up: the tile, and the splits of the columns where tiles alone leave the card empty.
struct Plan {
    int kind;                           // 0: the kernel for few tokens
    uint32_t rows, tokens, splits, split_stages;
    size_t laid_out, parts;             // bytes of the workspace
};

constexpr uint32_t MOST_COLUMNS = 1u << 21;         // offsets inside a tile are 31 bits wide

inline uint32_t up(uint32_t v, uint32_t by) { return (v + by - 1) / by; }
inline size_t part_row(uint32_t n) { return ((size_t)n + 15) / 16 * 16; }

Plan plan_of(uint32_t m, uint32_t n, uint32_t k, bool mx4)
{
    static const uint32_t shapes[][2] = {{256, 128}, {128, 128}, {256, 64}, {128, 64}, {128, 32}};
    Plan p{};
    // (the counts of vectors that are laid out, and of tiles, have 31 bits)
    if (m <= 16 || k > MOST_COLUMNS || k == 0 || (uint64_t)m * up(k, 256) >= 1u << 26 || (uint64_t)up(n, 128) * up(m, 32) >= 1u << 27) return p;
    const uint32_t groups = up(k, 128), unit = mx4 ? 1 : 2, stages = mx4 ? up(groups, 4) : up(groups, 2) * 2;
    double best = 1e300;
    for (int kind = 1; kind <= 5; ++kind) {
        const uint32_t rows = shapes[kind - 1][0], tokens = shapes[kind - 1][1];
        if (tokens > 32 && m <= tokens / 2) continue;
        const uint64_t tiles = (uint64_t)up(n, rows) * up(m, tokens);
        for (uint32_t splits = 1; splits <= 16 && splits * unit <= stages && (splits == 1 || (uint64_t)m * up(n, 4) < 1u << 31); splits *= 2) {
            const uint32_t each = up(up(stages, splits), unit) * unit;
            const uint64_t rounds = (tiles * up(stages, each) + 511) / 512;
            // a stage costs its matrix instructions, or bringing its bytes; joining costs the sums' way out and back
            const double stage = (double)rows * tokens / 128 / 128 + 0.5 + 0.25 * rows / 128;
            const double cost = rounds * (each + 4.0) * stage + (splits > 1 ? 8 + (double)splits * m * n * 8 / 4e6 : 0);
            if (cost < best) best = cost, p = {kind, rows, tokens, up(stages, each), each, 0, 0};
        }
    }
    if (!mx4) p.laid_out = 4 * (size_t)m * (up(k, 256) * 256);
    if (p.splits > 1) p.parts = p.splits * (size_t)m * part_row(n) * sizeof(float);
    return p;
}

template <int ACT, int RT, int MT, int WN, int WM> void launch_tile(const Product &a, uint32_t splits, hipStream_t s)
{
    product_tile_kernel<ACT, RT, MT, WN, WM><<<dim3(up(a.n_tiles * a.m_tiles, 8) * 8, splits), 64 * WN * WM, 0, s>>>(a);
}

template <int ACT> int launch(Product a, void *workspace, hipStream_t s)
{
    const Plan p = plan_of(a.m, a.n, a.k, ACT == MX4);
    if (p.kind == 0) {
        const uint32_t rows = up(a.n, 16);
        if (a.m <= 16) product_few_kernel<ACT, 1, 1, 4><<<dim3(rows, 1), 256, 0, s>>>(a);
        else product_few_kernel<ACT, 1, 4, 4><<<dim3(rows, up(a.m, 64)), 256, 0, s>>>(a);
        return hipGetLastError() == hipSuccess ? ENEC_OK : ENEC_E_HIP;
    }
    if constexpr (ACT == MX4) {
        a.x_row = a.x_bytes = a.groups * 64;
    } else if (ACT == BF16 && a.k % 256 == 0 && a.x_stride % 8 == 0 && a.x_stride <= MOST_COLUMNS && aligned(a.x, 16)) {
        a.x_row = a.x_stride * 2, a.x_bytes = a.k * 2;
    } else {
        const uint32_t cols = up(a.k, 256) * 256, n_vec = a.m * (cols / 8);
        lay_out_kernel<ACT><<<up(n_vec, 256), 256, 0, s>>>(static_cast<const uint16_t *>(a.x), a.x_stride, a.k, divide_by(cols / 8), n_vec,
                                                           static_cast<u32x4 *>(workspace));
        a.x = workspace;
        a.x_plane = cols * 2;
        a.x_row = a.x_bytes = ACT == FP16 ? 2 * a.x_plane : a.x_plane;
    }
    a.n_tiles = up(a.n, p.rows), a.m_tiles = up(a.m, p.tokens), a.split_stages = p.split_stages;
    if (p.splits > 1) a.parts = reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) + p.laid_out), a.part_row = part_row(a.n);
    switch (p.kind) {
    case 1: launch_tile<ACT, 4, 8, 4, 1>(a, p.splits, s); break;
    case 2: launch_tile<ACT, 4, 4, 2, 2>(a, p.splits, s); break;
    case 3: launch_tile<ACT, 4, 4, 4, 1>(a, p.splits, s); break;
    case 4: launch_tile<ACT, 2, 4, 4, 1>(a, p.splits, s); break;
    default: launch_tile<ACT, 2, 2, 4, 1>(a, p.splits, s); break;
    }
    if (p.splits > 1) {
        const uint32_t per_row = up(a.n, 4);
        join_kernel<<<up(a.m * per_row, 256), 256, 0, s>>>(a.parts, p.splits, a.m, a.n, a.part_row, divide_by(per_row), a.y, a.y_stride, a.y_dtype);
    }
    return hipGetLastError() == hipSuccess ? ENEC_OK : ENEC_E_HIP;
}

// sizes that every kernel here can count with: columns in 32 bits with the padding, tokens and rows in a grid
inline bool sizes_ok(size_t m, size_t n, size_t k) { return m <= (1u << 21) && n <= (1u << 30) && k <= (1u << 30); }

}  // namespace

extern "C" {

size_t enec_mx4_linear_workspace(size_t m, size_t n, size_t k)
{
    if (!sizes_ok(m, n, k) || m == 0 || n == 0) return 0;
    const Plan p = plan_of((uint32_t)m, (uint32_t)n, (uint32_t)k, false);
    return p.laid_out + p.parts;
}
size_t enec_mx4_matmul_workspace(size_t m, size_t n, size_t k)
{
    if (!sizes_ok(m, n, k) || m == 0 || n == 0) return 0;
    const Plan p = plan_of((uint32_t)m, (uint32_t)n, (uint32_t)k, true);
    return p.laid_out + p.parts;
}

int enec_mx4_linear(const void *x, size_t m, size_t x_stride, int dtype, const void *codes, const void *scales, size_t n, size_t k, void *y,
                    size_t y_stride, void *workspace, size_t workspace_bytes, void *stream)
{
    if (dtype != ENEC_BF16 && dtype != ENEC_FP16) return ENEC_E_DTYPE;
    if (!sizes_ok(m, n, k)) return ENEC_E_ARG;
    if (m == 0 || n == 0) return ENEC_OK;
    if (!y || !aligned(y, 2) || y_stride < n) return ENEC_E_ARG;
    if (k != 0 && (!x || !codes || !scales || !aligned(x, 2) || !aligned(codes, 16) || !aligned(scales, 4) || x_stride < k)) return ENEC_E_ARG;
    const size_t need = enec_mx4_linear_workspace(m, n, k);
    if (workspace_bytes < need || (need && !workspace)) return ENEC_E_CAPACITY;
    if (need && !aligned(workspace, 16)) return ENEC_E_ARG;
    const Product a{x, nullptr, static_cast<const uint8_t *>(codes), static_cast<const uint8_t *>(scales), y, x_stride, y_stride,
                    (uint32_t)m, (uint32_t)n, (uint32_t)k, (uint32_t)((k + 127) / 128), dtype, 0, 0, 0, 0, 0, 0, 0, nullptr};
    return dtype == ENEC_BF16 ? launch<BF16>(a, workspace, (hipStream_t)stream) : launch<FP16>(a, workspace, (hipStream_t)stream);
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
    const size_t need = enec_mx4_matmul_workspace(m, n, k);
    if (workspace_bytes < need || (need && !workspace)) return ENEC_E_CAPACITY;
    if (need && !aligned(workspace, 16)) return ENEC_E_ARG;
    const Product a{x_codes, static_cast<const uint8_t *>(x_scales), static_cast<const uint8_t *>(codes), static_cast<const uint8_t *>(scales), y, 0, y_stride,
                    (uint32_t)m, (uint32_t)n, (uint32_t)k, (uint32_t)((k + 127) / 128), dtype, 0, 0, 0, 0, 0, 0, 0, nullptr};
    return launch<MX4>(a, workspace, (hipStream_t)stream);
}

}  // extern "C"
