// 8-bit floating point with a scale for each block of 128: a matrix into codes and scales, and back.  The format stands in include/enec_lowbit.h.
#include "enec_lowbit.h"
#include "lowbit_fp8.hpp"

namespace enec {
namespace lowbit {

// Bound by HBM: 3.01 bytes a bf16 value, each moved once.  A thread has eight consecutive values (one 16-byte load, one 8-byte store), sixteen
// threads a block of 128; the largest magnitude of a block takes four moves between lanes (through LDS instead they cost 0.3 us of 4 x 4096).  It is found on the bits: magnitudes of
// floats order as whole numbers do, and a NaN or an infinity has the exponent field 255.  The scale is a power of two, so the division is exact
// wherever its result is not below all of E4M3's values, and nearest even is the instruction's rounding.
// 28672 x 8192 bf16: 113 us, 6.3 TB/s; 2048 x 4096 6.9; 4 x 4096 2.15.
template <int DT, int U>
__global__ void __launch_bounds__(256) fp8_quantize_kernel(const void *__restrict__ in, uint32_t cols, size_t stride, Divide per_row, uint32_t n_vec,
                                                           uint32_t scale_row, u32x2 *__restrict__ codes, uint8_t *__restrict__ scales)
{
    float v[U][8];
    const uint32_t first = blockIdx.x * (256u * U) + threadIdx.x;
    for (int u = 0; u < U; ++u) {
        const uint32_t at = first + u * 256u;
        const uint32_t row = quotient(at, per_row), col = (at - row * per_row.by) * 8u;
        const size_t i = (size_t)row * stride + col;
        if (at < n_vec && col + 8 <= cols) {
            load8<DT>(in, i, v[u]);
        } else if (at < n_vec && col < cols) {              // (loads that do not wait for one another)
            for (int j = 0; j < 8; ++j) v[u][j] = load1<DT>(in, i + (col + j < cols ? j : cols - 1 - col));
            for (int j = 0; j < 8; ++j) v[u][j] = col + j < cols ? v[u][j] : 0.0f;
        } else {
            for (int j = 0; j < 8; ++j) v[u][j] = 0.0f;
        }
    }
    for (int u = 0; u < U; ++u) {
        const uint32_t at = first + u * 256u;
        if (at >= n_vec) return;                            // (blocks are whole: sixteen lanes go or stay)
        const uint32_t byte = block_byte(v[u]);
        codes[at] = fp8_codes(v[u], byte);
        if ((at & 15) == 0) {
            const uint32_t row = quotient(at, per_row), group = (at - row * per_row.by) >> 4, groups = per_row.by >> 4;
            uint8_t *to = scales + (size_t)row * scale_row;
            to[group] = (uint8_t)byte;
            if (group + 1 == groups)
                for (uint32_t g = groups; g < scale_row; ++g) to[g] = 0;
        }
    }
}

// The way back: eight bytes of codes and a scale in, eight values out.  Bound by HBM as well: the same matrix 117 us, 6.0 TB/s.
template <int DT, int U>
__global__ void __launch_bounds__(256) fp8_dequantize_kernel(const u32x2 *__restrict__ codes, const uint8_t *__restrict__ scales, uint32_t cols, size_t stride,
                                                             Divide per_row, uint32_t n_vec, uint32_t scale_row, void *__restrict__ out)
{
    const uint32_t first = blockIdx.x * (256u * U) + threadIdx.x;
    u32x2 c[U];
    uint32_t byte[U];
    for (int u = 0; u < U; ++u) {
        const uint32_t at = first + u * 256u, row = quotient(at, per_row), group = (at - row * per_row.by) >> 4;
        c[u] = at < n_vec ? codes[at] : u32x2{};
        byte[u] = at < n_vec ? scales[(size_t)row * scale_row + group] : 0;
    }
    for (int u = 0; u < U; ++u) {
        const uint32_t at = first + u * 256u;
        const uint32_t row = quotient(at, per_row), col = (at - row * per_row.by) * 8u;
        const size_t i = (size_t)row * stride + col;
        const float scale = power_of(byte[u]);
        float v[8];
        for (int j = 0; j < 2; ++j) {
            const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(c[u][j], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(c[u][j], true);
            v[4 * j] = lo[0] * scale, v[4 * j + 1] = lo[1] * scale, v[4 * j + 2] = hi[0] * scale, v[4 * j + 3] = hi[1] * scale;
        }
        if (at < n_vec && col + 8 <= cols) {
            store8<DT>(out, i, v);
        } else {
            for (int j = 0; j < 8; ++j)
                if (at < n_vec && col + j < cols) store1<DT>(out, i + j, v[j]);
        }
    }
}

namespace {
constexpr int UNROLL = 2;               // of the way back (one vector a thread: 2048 x 4096 5.4 us instead of 5.0)
inline bool aligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
}  // namespace

int quantize_to_fp8(const void *in, size_t rows, size_t cols, size_t row_stride, int dtype, void *codes, void *scales, hipStream_t s)
{
    const uint32_t vectors = (uint32_t)(fp8_padded(cols) / 8), n_vec = (uint32_t)(rows * vectors);
    // One vector a thread, and two for large matrices: 4 x 4096 took 2.15 and 2.35 us, 256 x 4096 2.6 and 2.95, 4096 x 4096 11.9 and 12.3, there and back 11008 x 4096 45.4 and 44.2,
    // 28672 x 8192 230 and 228.
    const uint32_t each = n_vec <= 1u << 22 ? 1 : 2;
    auto kernel = dtype == ENEC_BF16   ? (each == 1 ? fp8_quantize_kernel<BF16, 1> : fp8_quantize_kernel<BF16, 2>)
                  : dtype == ENEC_FP16 ? (each == 1 ? fp8_quantize_kernel<FP16, 1> : fp8_quantize_kernel<FP16, 2>)
                                       : (each == 1 ? fp8_quantize_kernel<FP32, 1> : fp8_quantize_kernel<FP32, 2>);
    kernel<<<dim3((n_vec - 1) / (256 * each) + 1), 256, 0, s>>>(in, (uint32_t)cols, row_stride, divide_by(vectors), n_vec, (uint32_t)fp8_scale_row(cols),
                                                                  static_cast<u32x2 *>(codes), static_cast<uint8_t *>(scales));
    return hipGetLastError() == hipSuccess ? ENEC_OK : ENEC_E_HIP;
}

}  // namespace lowbit
}  // namespace enec

using namespace enec::lowbit;

extern "C" {

int enec_fp8_bytes(size_t rows, size_t cols, size_t *code_bytes, size_t *scale_bytes)
{
    if (!fp8_fits(rows, cols)) return ENEC_E_ARG;
    if (code_bytes) *code_bytes = rows * fp8_padded(cols);
    if (scale_bytes) *scale_bytes = rows * fp8_scale_row(cols);
    return ENEC_OK;
}

int enec_fp8_quantize(const void *in, size_t rows, size_t cols, size_t row_stride, int dtype, void *codes, void *scales, void *stream)
{
    if (dtype != ENEC_BF16 && dtype != ENEC_FP16 && dtype != ENEC_FP32) return ENEC_E_DTYPE;
    if (!fp8_fits(rows, cols)) return ENEC_E_ARG;
    if (rows == 0 || cols == 0) return ENEC_OK;
    if (!in || !codes || !scales || !aligned(codes, 16) || !aligned(scales, 4) || !aligned(in, dtype == ENEC_FP32 ? 4 : 2) || row_stride < cols)
        return ENEC_E_ARG;
    return quantize_to_fp8(in, rows, cols, row_stride, dtype, codes, scales, (hipStream_t)stream);
}

int enec_fp8_dequantize(const void *codes, const void *scales, size_t rows, size_t cols, void *out, size_t row_stride, int dtype, void *stream)
{
    if (dtype != ENEC_BF16 && dtype != ENEC_FP16 && dtype != ENEC_FP32) return ENEC_E_DTYPE;
    if (!fp8_fits(rows, cols)) return ENEC_E_ARG;
    if (rows == 0 || cols == 0) return ENEC_OK;
    if (!out || !codes || !scales || !aligned(codes, 16) || !aligned(scales, 4) || !aligned(out, dtype == ENEC_FP32 ? 4 : 2) || row_stride < cols)
        return ENEC_E_ARG;
    const uint32_t vectors = (uint32_t)(fp8_padded(cols) / 8), n_vec = (uint32_t)(rows * vectors);
    auto kernel = dtype == ENEC_BF16   ? fp8_dequantize_kernel<BF16, UNROLL>
                  : dtype == ENEC_FP16 ? fp8_dequantize_kernel<FP16, UNROLL>
                                       : fp8_dequantize_kernel<FP32, UNROLL>;
    kernel<<<dim3((n_vec - 1) / (256 * UNROLL) + 1), 256, 0, (hipStream_t)stream>>>(static_cast<const u32x2 *>(codes), static_cast<const uint8_t *>(scales),
                                                                                    (uint32_t)cols, row_stride, divide_by(vectors), n_vec,
                                                                                    (uint32_t)fp8_scale_row(cols), out);
    return hipGetLastError() == hipSuccess ? ENEC_OK : ENEC_E_HIP;
}

}  // extern "C"
