// Parts that the products of lowbit_matmul.hip and lowbit_fp8_matmul.hip share: copies into LDS, outputs, the sums of splits.
#pragma once

#include "lowbit.hpp"

namespace enec {
namespace lowbit {

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

// Memory through a descriptor, whose range the memory unit checks: rows behind a matrix's last one need no branch.  Offsets are 32 bits wide,
// from a tile's first row.
using Range = __amdgpu_buffer_rsrc_t;
__device__ __forceinline__ Range range_of(const void *p, uint32_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, (int)bytes, 0x00020000);
}
// 16 or 4 bytes a lane into LDS, the lanes' side by side
template <int BYTES> __device__ __forceinline__ void copy_to_lds(Range r, uint32_t at, uint8_t *to)
{
    const auto lds = (__attribute__((address_space(3))) void *)to;
    if constexpr (BYTES == 16) __builtin_amdgcn_raw_ptr_buffer_load_lds(r, lds, 16, (int)at, 0, 0, 0);
    else __builtin_amdgcn_raw_ptr_buffer_load_lds(r, lds, 4, (int)at, 0, 0, 0);
}

// The sums of the splits, in their order (none, where there are no columns: zeros).
static __global__ void __launch_bounds__(256) join_kernel(const float *__restrict__ parts, uint32_t splits, uint32_t m, uint32_t n, size_t part_row, Divide per_row,
                                                   void *y, size_t y_stride, int y_dtype)
{
    const uint32_t at = blockIdx.x * 256u + threadIdx.x, token = quotient(at, per_row), r = (at - token * per_row.by) * 4u;
    if (token >= m) return;
    const float *p = parts + (size_t)token * part_row + r;
    f32x4 v = {};
    for (uint32_t i = 0; i < splits; ++i) v += *reinterpret_cast<const f32x4 *>(p + i * (m * part_row));
    store4(y, y_dtype, (size_t)token * y_stride + r, n - r, v);
}

inline uint32_t up(uint32_t v, uint32_t by) { return (v + by - 1) / by; }
inline size_t part_row(uint32_t n) { return ((size_t)n + 15) / 16 * 16; }

}  // namespace lowbit
}  // namespace enec
