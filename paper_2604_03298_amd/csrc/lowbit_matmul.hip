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

}  // namespace lowbit
}  // namespace enec

namespace {

using namespace enec::lowbit;

inline bool aligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

template <int ACT> int launch(const Product &a, hipStream_t s)
{
    const uint32_t rows = (a.n + 15) / 16;
    if (a.m <= 16) product_few_kernel<ACT, 1, 1, 4><<<dim3(rows, 1), 256, 0, s>>>(a);
    else product_few_kernel<ACT, 1, 4, 4><<<dim3(rows, (a.m + 63) / 64), 256, 0, s>>>(a);
    return hipGetLastError() == hipSuccess ? ENEC_OK : ENEC_E_HIP;
}

// sizes that every kernel here can count with: columns in 32 bits with the padding, tokens and rows in a grid
inline bool sizes_ok(size_t m, size_t n, size_t k) { return m <= (1u << 21) && n <= (1u << 30) && k <= (1u << 30); }

}  // namespace

extern "C" {

size_t enec_mx4_linear_workspace(size_t, size_t, size_t) { return 0; }
size_t enec_mx4_matmul_workspace(size_t, size_t, size_t) { return 0; }

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
                    (uint32_t)m, (uint32_t)n, (uint32_t)k, (uint32_t)((k + 127) / 128), dtype};
    return dtype == ENEC_BF16 ? launch<BF16>(a, (hipStream_t)stream) : launch<FP16>(a, (hipStream_t)stream);
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
                    (uint32_t)m, (uint32_t)n, (uint32_t)k, (uint32_t)((k + 127) / 128), dtype};
    return launch<MX4>(a, (hipStream_t)stream);
}

}  // extern "C"
