// Microscaled 4-bit floating point: a matrix into codes and scales, and back.  The format stands in include/enec_lowbit.h.
#include "enec_lowbit.h"
#include "lowbit.hpp"

namespace enec {
namespace lowbit {

// Bound by HBM: 2.53 bytes a bf16 value, each moved once, and about fifteen instructions for eight values.  A thread has eight
// consecutive values (one 16-byte load, one 4-byte store), four threads a block of 32, so a wave's accesses are whole lines both
// ways; the largest magnitude of a block takes two exchanges between neighbouring lanes.  It is found on the bits: magnitudes of
// floats order as whole numbers do, and a NaN or an infinity has the exponent field 255.  U vectors per thread are asked for
// before the first is used: 11008 x 4096 bf16 took 21.5 us with two, 24 with four, 27.6 with eight; with stores that stream past the cache 17.6
// (6.5 TB/s: the matrix fits the last-level cache).  One row of 4096 takes 1.9 us, and its call 5.4 on the host.
template <int DT, int U>
__global__ void __launch_bounds__(256) mx4_quantize_kernel(const void *__restrict__ in, uint32_t cols, size_t stride, Divide per_row,
                                                           uint32_t n_vec, uint32_t *__restrict__ codes, uint8_t *__restrict__ scales)
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
        uint32_t a = 0;
        for (int j = 0; j < 8; ++j) {
            const uint32_t b = bits_of(v[u][j]) & 0x7FFFFFFFu;
            a = a > b ? a : b;
        }
        for (int k = 1; k < 4; k *= 2) {
            const uint32_t b = __shfl_xor(a, k);
            a = a > b ? a : b;
        }
        const uint32_t e = a >> 23, byte = e == 255 ? 255 : e > 2 ? e - 2 : 0;
        const float scale = power_of(byte);
        uint32_t c = 0;
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[u][0], v[u][1], scale, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[u][2], v[u][3], scale, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[u][4], v[u][5], scale, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[u][6], v[u][7], scale, 3);
        if (at < n_vec) {
            codes[at] = byte == 255 ? 0 : c;
            if ((at & 3) == 0) scales[at >> 2] = (uint8_t)byte;
        }
    }
}

// The way back: four bytes of codes and a scale in, eight values out.  Bound by HBM as well: 11008 x 4096 bf16 16.5 us (6.9 TB/s).
template <int DT, int U>
__global__ void __launch_bounds__(256) mx4_dequantize_kernel(const uint32_t *__restrict__ codes, const uint8_t *__restrict__ scales, uint32_t cols,
                                                             size_t stride, Divide per_row, uint32_t n_vec, void *__restrict__ out)
{
    const uint32_t first = blockIdx.x * (256u * U) + threadIdx.x;
    uint32_t c[U], byte[U];
    for (int u = 0; u < U; ++u) {
        const uint32_t at = first + u * 256u;
        c[u] = at < n_vec ? codes[at] : 0;
        byte[u] = at < n_vec ? scales[at >> 2] : 0;
    }
    for (int u = 0; u < U; ++u) {
        const uint32_t at = first + u * 256u;
        const uint32_t row = quotient(at, per_row), col = (at - row * per_row.by) * 8u;
        const size_t i = (size_t)row * stride + col;
        const float scale = power_of(byte[u]);
        float v[8];
        const f32x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[u], scale, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[u], scale, 1);
        const f32x2 p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[u], scale, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[u], scale, 3);
        v[0] = p0[0], v[1] = p0[1], v[2] = p1[0], v[3] = p1[1], v[4] = p2[0], v[5] = p2[1], v[6] = p3[0], v[7] = p3[1];
        if (at < n_vec && col + 8 <= cols) {
            store8<DT>(out, i, v);
        } else {
            for (int j = 0; j < 8; ++j)
                if (at < n_vec && col + j < cols) store1<DT>(out, i + j, v[j]);
        }
    }
}

}  // namespace lowbit
}  // namespace enec

namespace {

using namespace enec::lowbit;

constexpr size_t MAX_VALUES = (size_t)1 << 34;      // as enec.h's tensors; vectors of eight stay below 2^31
constexpr int UNROLL = 2;

inline size_t padded(size_t cols) { return (cols + ENEC_MX4_ROW_GROUP - 1) / ENEC_MX4_ROW_GROUP * ENEC_MX4_ROW_GROUP; }
inline bool fits(size_t rows, size_t cols) { return cols <= (size_t)1 << 31 && (cols == 0 || rows <= MAX_VALUES / padded(cols)); }
inline bool aligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

}  // namespace

extern "C" {

int enec_mx4_bytes(size_t rows, size_t cols, size_t *code_bytes, size_t *scale_bytes)
{
    if (!fits(rows, cols)) return ENEC_E_ARG;
    if (code_bytes) *code_bytes = rows * padded(cols) / 2;
    if (scale_bytes) *scale_bytes = rows * padded(cols) / ENEC_MX4_BLOCK;
    return ENEC_OK;
}

int enec_mx4_quantize(const void *in, size_t rows, size_t cols, size_t row_stride, int dtype, void *codes, void *scales, void *stream)
{
    if (dtype != ENEC_BF16 && dtype != ENEC_FP16 && dtype != ENEC_FP32) return ENEC_E_DTYPE;
    if (!fits(rows, cols)) return ENEC_E_ARG;
    if (rows == 0 || cols == 0) return ENEC_OK;
    if (!in || !codes || !scales || !aligned(codes, 16) || !aligned(scales, 4) || !aligned(in, dtype == ENEC_FP32 ? 4 : 2) || row_stride < cols)
        return ENEC_E_ARG;
    const Divide per_row = divide_by((uint32_t)(padded(cols) / 8));
    const uint32_t n_vec = (uint32_t)(rows * (padded(cols) / 8));
    const dim3 grid((n_vec + 256 * UNROLL - 1) / (256 * UNROLL));
    hipStream_t s = (hipStream_t)stream;
    auto kernel = dtype == ENEC_BF16   ? mx4_quantize_kernel<BF16, UNROLL>
                  : dtype == ENEC_FP16 ? mx4_quantize_kernel<FP16, UNROLL>
                                       : mx4_quantize_kernel<FP32, UNROLL>;
    kernel<<<grid, 256, 0, s>>>(in, (uint32_t)cols, row_stride, per_row, n_vec, static_cast<uint32_t *>(codes), static_cast<uint8_t *>(scales));
    return hipGetLastError() == hipSuccess ? ENEC_OK : ENEC_E_HIP;
}

int enec_mx4_dequantize(const void *codes, const void *scales, size_t rows, size_t cols, void *out, size_t row_stride, int dtype, void *stream)
{
    if (dtype != ENEC_BF16 && dtype != ENEC_FP16 && dtype != ENEC_FP32) return ENEC_E_DTYPE;
    if (!fits(rows, cols)) return ENEC_E_ARG;
    if (rows == 0 || cols == 0) return ENEC_OK;
    if (!out || !codes || !scales || !aligned(codes, 16) || !aligned(scales, 4) || !aligned(out, dtype == ENEC_FP32 ? 4 : 2) || row_stride < cols)
        return ENEC_E_ARG;
    const Divide per_row = divide_by((uint32_t)(padded(cols) / 8));
    const uint32_t n_vec = (uint32_t)(rows * (padded(cols) / 8));
    const dim3 grid((n_vec + 256 * UNROLL - 1) / (256 * UNROLL));
    hipStream_t s = (hipStream_t)stream;
    auto kernel = dtype == ENEC_BF16   ? mx4_dequantize_kernel<BF16, UNROLL>
                  : dtype == ENEC_FP16 ? mx4_dequantize_kernel<FP16, UNROLL>
                                       : mx4_dequantize_kernel<FP32, UNROLL>;
    kernel<<<grid, 256, 0, s>>>(static_cast<const uint32_t *>(codes), static_cast<const uint8_t *>(scales), (uint32_t)cols, row_stride, per_row,
                                n_vec, out);
    return hipGetLastError() == hipSuccess ? ENEC_OK : ENEC_E_HIP;
}

}  // extern "C"
