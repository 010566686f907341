// 8-bit floating point with a scale for each block of 128, as its kernels and the products' share it.
#pragma once

#include "lowbit.hpp"

namespace enec {
namespace lowbit {

constexpr size_t FP8_BLOCK = 128;
inline size_t fp8_padded(size_t cols) { return (cols + FP8_BLOCK - 1) / FP8_BLOCK * FP8_BLOCK; }
inline size_t fp8_scale_row(size_t cols) { return (fp8_padded(cols) / FP8_BLOCK + 3) / 4 * 4; }
// as enec.h's tensors; vectors of eight are at most 2^31
inline bool fp8_fits(size_t rows, size_t cols) { return cols <= (size_t)1 << 31 && (cols == 0 || rows <= ((size_t)1 << 34) / fp8_padded(cols)); }

template <int CONTROL> __device__ __forceinline__ uint32_t larger_moved(uint32_t a)
{
    const uint32_t b = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, CONTROL, 15, 15, true);
    return a > b ? a : b;
}
// The scale's byte of a block of which this thread and the others of its sixteen have eight values each.
__device__ __forceinline__ uint32_t block_byte(const float (&v)[8])
{
    uint32_t a = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t b = bits_of(v[j]) & 0x7FFFFFFFu;
        a = a > b ? a : b;
    }
    // (by lane moves: from the neighbour, from the other pair, from the half row's other four, from the row's other eight)
    a = larger_moved<0xB1>(a), a = larger_moved<0x4E>(a), a = larger_moved<0x141>(a), a = larger_moved<0x140>(a);
    return a >= 0x7F800000u ? 255 : scale_byte(a);
}
// eight values as E4M3 codes of v / 2^(byte - 127); zeros if the byte says that the block has no values
__device__ __forceinline__ u32x2 fp8_codes(const float (&v)[8], uint32_t byte)
{
    const float inverse = byte == 255 ? 0.0f : power_of(254 - byte);
    u32x2 r = {};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        uint32_t w = 0;
        w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * j] * inverse, v[4 * j + 1] * inverse, w, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * j + 2] * inverse, v[4 * j + 3] * inverse, w, true);
        r[j] = byte == 255 ? 0 : w;
    }
    return r;
}

// `in` into `codes` and `scales`, whose sizes and alignment have been checked; rows and cols are not zero
int quantize_to_fp8(const void *in, size_t rows, size_t cols, size_t row_stride, int dtype, void *codes, void *scales, hipStream_t s);

}  // namespace lowbit
}  // namespace enec
