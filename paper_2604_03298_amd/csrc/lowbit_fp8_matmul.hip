// Products of matrices in 8-bit floating point with a scale for each block of 128.  The definitions stand in include/enec_lowbit.h.
#include "enec_lowbit.h"
#include "lowbit_fp8.hpp"
#include "lowbit_product.hpp"

#include <atomic>

namespace enec {
namespace lowbit {

struct Product8 {
    const uint8_t *x, *x_scales, *w, *w_scales;
    void *y;
    size_t y_stride, part_row;
    float *parts;
    uint32_t m, n, groups, scale_row;   // groups of 128 columns; bytes between rows of scales
    uint32_t n_tiles, m_tiles, split_stages;
    int y_dtype;
};

__device__ __forceinline__ i32x8 halves(const u32x4 &a, const u32x4 &b)
{
    return i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
}

// The 8-bit matrix instructions align the products of eight columns (consecutive ones, as they are read here) to the largest of them and drop what
// lies below 2^-13 of its power of two; beyond that they sum in 32 bits.  For y in 16 bits that is far below its own rounding: 1.5e-5 of the norm for normal
// values, bf16's rounding 1.7e-3.  For y in 32 bits (EXACT) codes become bf16 values, which is exact from scale bytes of 3 on, and bf16 instructions,
// which sum in 32 bits, multiply them at half the rate.
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
template <bool EXACT, int RA, int RB, int WA, int WB, int BUFFERS>
__global__ void __launch_bounds__(64 * WA * WB, RA * RB > 8 ? 1 : 2) fp8_tile_kernel(Product8 a)
{
    constexpr uint32_t THREADS = 64 * WA * WB, ROWS = 32 * RA * WA, TOKENS = 32 * RB * WB, ALL = ROWS + TOKENS, STAGE = ALL * 128;
    constexpr uint32_t W_COPIES = ROWS * 8 / THREADS, COPIES = ALL * 8 / THREADS;
    static_assert(ROWS * 8 % THREADS == 0 && TOKENS * 8 % THREADS == 0 && THREADS % 128 == 0 && ROWS % 64 == 0, "whole copies of a wave");
    static_assert(BUFFERS >= 2 && BUFFERS <= 5, "scales land within three stages");
    extern __shared__ __attribute__((aligned(16))) uint8_t shared[];
    uint8_t *scale_bytes = shared + BUFFERS * STAGE;        // of four stages, two in turn: four bytes of each row, then of each token
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 5, c = lane & 31;
    const uint32_t wa = wave % WA, wb = wave / WA;
    // Workgroups are dealt out to the eight dies one by one: each die takes a run of tiles, in bands of tiles of tokens (see product_tile_kernel).
    constexpr uint32_t BAND = 6;
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
        uint8_t *to = scale_bytes + (block & 1) * (ALL * 4);
#pragma unroll
        for (uint32_t r = 0; r < ALL; r += THREADS) {
            const uint32_t begin = r + wave * 64, row = begin + lane;
            if (begin >= ALL) continue;
            if (begin < ROWS) copy_to_lds<4>(w_scales, row * a.scale_row + block * 4, to + begin * 4);
            else copy_to_lds<4>(x_scales, (row - ROWS) * a.scale_row + block * 4, to + begin * 4);
        }
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
        const uint8_t *t = scale_bytes + (stage >> 2 & 1) * (ALL * 4) + (stage & 3);
#pragma unroll
        for (int i = 0; i < RA; ++i) ws[parity][i] = t[ws_at + i * 128];
#pragma unroll
        for (int i = 0; i < RB; ++i) xs[parity][i] = t[xs_at + i * 128];
    };
    // A wave's copies are counted, and done in the order in which they were issued: with at most AHEAD left, those of the next stage are in LDS.  Then all
    // waves' are, and this stage's second half is in everybody's registers.
    constexpr int AHEAD = (BUFFERS - 2) * COPIES;
    auto meet = [&] {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(AHEAD) : "memory");
        __builtin_amdgcn_sched_barrier(0);
    };

    f32x16 acc[RA][RB] = {};
    fetch_scales(first / 4);                                // (a split begins with such a block)
#pragma unroll
    for (int b = 0; b < BUFFERS; ++b) fetch(first + b, b);
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((BUFFERS - 1) * COPIES) : "memory");
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
                if ((s & 3) == 0) fetch_scales(s / 4 + 1);
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
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");        // (no copy may come after the workgroup)
#pragma unroll
    for (int u = 0; u < RB; ++u) {
        const uint32_t token = m0 + wb * (32 * RB) + 32 * u + c;
        if (token >= a.m) continue;
#pragma unroll
        for (int t = 0; t < RA; ++t) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t r = n0 + wa * (32 * RA) + 32 * t + 8 * e + 4 * g;
                if (r >= a.n) continue;
                const f32x4 v = {acc[t][u][4 * e], acc[t][u][4 * e + 1], acc[t][u][4 * e + 2], acc[t][u][4 * e + 3]};
                if (a.parts) *reinterpret_cast<f32x4 *>(a.parts + ((size_t)blockIdx.y * a.m + token) * a.part_row + r) = v;
                else store4(a.y, a.y_dtype, (size_t)token * a.y_stride + r, a.n - r, v);
            }
        }
    }
}

// Up to sixteen tokens: bound by the weights' way from memory.  A workgroup has sixteen rows of weights, and its waves take units of 512 columns in turn, straight
// into registers, the next unit asked for before this one is multiplied; the waves' sums meet in LDS, in their order.
template <bool EXACT, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) fp8_thin_kernel(Product8 a)
{
    __shared__ f32x4 sums[WAVES][64];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, c = lane & 15;
    const uint32_t n0 = blockIdx.x * 16, pitch = a.groups * 128;
    // rows and tokens that are not there read the last one's, and their sums go nowhere
    const uint32_t row = n0 + c < a.n ? n0 + c : a.n - 1, token = c < a.m ? c : a.m - 1;
    const uint8_t *w = a.w + (size_t)row * pitch + 32 * g, *x = a.x + (size_t)token * pitch + 32 * g;
    const uint32_t *w_scales = reinterpret_cast<const uint32_t *>(a.w_scales + (size_t)row * a.scale_row);
    const uint32_t *x_scales = reinterpret_cast<const uint32_t *>(a.x_scales + (size_t)token * a.scale_row);
    const uint32_t units = (a.groups + 3) / 4;
    struct Unit {
        u32x4 w[8], x[8];
        uint32_t ws, xs;
    };
    auto load = [&](uint32_t i, Unit &v) {
        v.ws = w_scales[i], v.xs = x_scales[i];
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            if (4 * i + j >= a.groups) continue;
            const u32x4 *p = reinterpret_cast<const u32x4 *>(w + (size_t)(4 * i + j) * 128), *q = reinterpret_cast<const u32x4 *>(x + (size_t)(4 * i + j) * 128);
            v.w[2 * j] = __builtin_nontemporal_load(p), v.w[2 * j + 1] = __builtin_nontemporal_load(p + 1);
            v.x[2 * j] = q[0], v.x[2 * j + 1] = q[1];
        }
    };
    f32x4 acc = {};
    Unit v[2];
    if (wave < units) load(wave, v[0]);
    auto step = [&](uint32_t i, const Unit &now, Unit &next) {
        if (i + WAVES < units) load(i + WAVES, next);
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            if (4 * i + j >= a.groups) continue;
            const i32x8 wv = halves(now.w[2 * j], now.w[2 * j + 1]), xv = halves(now.x[2 * j], now.x[2 * j + 1]);
            const int ws = (int)(now.ws >> (8 * j)), xs = (int)(now.xs >> (8 * j));
            if constexpr (EXACT) {
#pragma unroll
                for (int q = 0; q < 4; ++q) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(eight_values(wv, q, ws & 255), eight_values(xv, q, xs & 255), acc, 0, 0, 0);
            } else {
                acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv, xv, acc, 0, 0, 0, ws, 0, xs);
            }
        }
    };
    for (uint32_t i = wave; i < units; i += 2 * WAVES) {
        step(i, v[0], v[1]);
        if (i + WAVES < units) step(i + WAVES, v[1], v[0]);
    }
    if (wave != 0) sums[wave][lane] = acc;
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int k = 1; k < WAVES; ++k) acc += sums[k][lane];
    const uint32_t r = n0 + 4 * g;
    if (c < a.m && r < a.n) store4(a.y, a.y_dtype, (size_t)c * a.y_stride + r, a.n - r, acc);
}

}  // namespace lowbit
}  // namespace enec

namespace {

using namespace enec::lowbit;

inline bool aligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

struct Shape {
    uint32_t rows, tokens;
};
constexpr Shape SHAPES[] = {{256, 256}, {128, 128}, {64, 64}};
constexpr uint32_t THIN = 16;                       // tokens at most

int shape_of(uint32_t m, uint32_t n)
{
    if (m > 128 && n > 128) return 0;
    return m > 64 ? 1 : 2;
}

template <bool EXACT, int RA, int RB, int WA, int WB, int BUFFERS> bool launch_tile(Product8 a, uint32_t splits, hipStream_t s)
{
    constexpr size_t ROWS = 32 * RA * WA, TOKENS = 32 * RB * WB, LDS = (ROWS + TOKENS) * (128 * BUFFERS + 8);
    static_assert(LDS <= 160 * 1024, "LDS of a compute unit");
    static std::atomic<uint64_t> allowed{0};
    const auto kernel = fp8_tile_kernel<EXACT, RA, RB, WA, WB, BUFFERS>;
    if (LDS > 65536 && !allow_lds((const void *)kernel, LDS, allowed)) return false;
    a.n_tiles = up(a.n, ROWS), a.m_tiles = up(a.m, TOKENS);
    kernel<<<dim3(up(a.n_tiles * a.m_tiles, 8) * 8, splits), 64 * WA * WB, LDS, s>>>(a);
    return true;
}

template <bool EXACT> int launch(Product8 a, hipStream_t s)
{
    if (a.groups == 0) {
        const uint32_t per_row = up(a.n, 4);
        join_kernel<<<up(a.m * per_row, 256), 256, 0, s>>>(nullptr, 0, a.m, a.n, 0, divide_by(per_row), a.y, a.y_stride, a.y_dtype);
        return hipGetLastError() == hipSuccess ? ENEC_OK : ENEC_E_HIP;
    }
    a.split_stages = up(a.groups, 4) * 4;
    bool ok = true;
    if (a.m <= THIN) {
        fp8_thin_kernel<EXACT, 8><<<up(a.n, 16), 512, 0, s>>>(a);
    } else {
        const int shape = shape_of(a.m, a.n);
        if constexpr (EXACT) {
            ok = shape < 2 ? launch_tile<true, 2, 2, 2, 2, 2>(a, 1, s) : launch_tile<true, 1, 1, 2, 2, 4>(a, 1, s);
        } else {
            ok = shape == 0   ? launch_tile<false, 4, 4, 2, 2, 2>(a, 1, s)
                 : shape == 1 ? launch_tile<false, 2, 2, 2, 2, 2>(a, 1, s)
                              : launch_tile<false, 1, 1, 2, 2, 4>(a, 1, s);
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

// a linear layer's activations in 8 bits, codes and scales
inline size_t codes_space(size_t m, size_t k) { return m * fp8_padded(k); }
inline size_t scales_space(size_t m, size_t k) { return (m * fp8_scale_row(k) + 15) / 16 * 16; }

}  // namespace

extern "C" {

size_t enec_fp8_linear_workspace(size_t m, size_t n, size_t k)
{
    if (!sizes_ok(m, n, k) || m == 0 || n == 0 || k == 0) return 0;
    return codes_space(m, k) + scales_space(m, k);
}
size_t enec_fp8_matmul_workspace(size_t m, size_t n, size_t k)
{
    if (!sizes_ok(m, n, k) || m == 0 || n == 0 || k == 0) return 0;
    return 0;
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
    uint8_t *x_codes = static_cast<uint8_t *>(workspace), *x_scales = x_codes + codes_space(m, k);
    if (k != 0)
        if (const int rc = quantize_to_fp8(x, m, k, x_stride, dtype, x_codes, x_scales, (hipStream_t)stream)) return rc;
    const Product8 a{x_codes, x_scales, static_cast<const uint8_t *>(codes), static_cast<const uint8_t *>(scales), y, y_stride, 0, nullptr, (uint32_t)m, (uint32_t)n,
                     (uint32_t)((k + 127) / 128), (uint32_t)fp8_scale_row(k), 0, 0, 0, dtype};
    return launch<false>(a, (hipStream_t)stream);
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
                     static_cast<const uint8_t *>(scales), y, y_stride, 0, nullptr, (uint32_t)m, (uint32_t)n, (uint32_t)((k + 127) / 128),
                     (uint32_t)fp8_scale_row(k), 0, 0, 0, dtype};
    return dtype == ENEC_FP32 ? launch<true>(a, (hipStream_t)stream) : launch<false>(a, (hipStream_t)stream);
}

}  // extern "C"
