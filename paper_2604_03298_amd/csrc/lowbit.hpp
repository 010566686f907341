// Shared parts of the low-bit kernels: vector types, format conversions, unaligned access, the pages of a batch.
#pragma once

#include <hip/hip_runtime.h>
#include <atomic>
#include <cstdint>

namespace enec {
namespace lowbit {

using f32x2 = float __attribute__((ext_vector_type(2)));
using f32x4 = float __attribute__((ext_vector_type(4)));
using f32x16 = float __attribute__((ext_vector_type(16)));
using u32x2 = uint32_t __attribute__((ext_vector_type(2)));
using u32x4 = uint32_t __attribute__((ext_vector_type(4)));
using i32x8 = int __attribute__((ext_vector_type(8)));
using bf16x2 = __bf16 __attribute__((ext_vector_type(2)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using f16x2 = _Float16 __attribute__((ext_vector_type(2)));
using f16x8 = _Float16 __attribute__((ext_vector_type(8)));
using i16x2 = short __attribute__((ext_vector_type(2)));

// Tensors come with any stride, so a run of values starts at any multiple of an element.  The memory unit takes such
// addresses; the types only keep the compiler from assuming more.
using u32_a2 = uint32_t __attribute__((aligned(2)));
using u32x2_a2 = u32x2 __attribute__((aligned(2)));
using u32x4_a2 = u32x4 __attribute__((aligned(2)));
using u32x4_a4 = u32x4 __attribute__((aligned(4)));

enum { BF16 = 0, FP16 = 1, FP32 = 2 };
template <int DT> constexpr int SIZE = DT == FP32 ? 4 : 2;

__device__ __forceinline__ float f32_of_bits(uint32_t v) { return __builtin_bit_cast(float, v); }
__device__ __forceinline__ uint32_t bits_of(float v) { return __builtin_bit_cast(uint32_t, v); }
// two values packed in a word, as the format DT of 16 bits
template <int DT> __device__ __forceinline__ f32x2 unpack2(uint32_t v)
{
    if constexpr (DT == BF16) return f32x2{f32_of_bits(v << 16), f32_of_bits(v & 0xFFFF0000u)};
    const f16x2 h = __builtin_bit_cast(f16x2, v);
    return f32x2{(float)h[0], (float)h[1]};
}
template <int DT> __device__ __forceinline__ uint32_t pack2(float a, float b)
{
    if constexpr (DT == BF16) return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
    return __builtin_bit_cast(uint32_t, f16x2{(_Float16)a, (_Float16)b});
}
template <int DT> __device__ __forceinline__ float load1(const void *p, size_t i)
{
    if constexpr (DT == FP32) return static_cast<const float *>(p)[i];
    if constexpr (DT == BF16) return f32_of_bits((uint32_t) static_cast<const uint16_t *>(p)[i] << 16);
    return (float)static_cast<const _Float16 *>(p)[i];
}
template <int DT> __device__ __forceinline__ void store1(void *p, size_t i, float v)
{
    if constexpr (DT == FP32) static_cast<float *>(p)[i] = v;
    else if constexpr (DT == BF16) static_cast<__bf16 *>(p)[i] = (__bf16)v;
    else static_cast<_Float16 *>(p)[i] = (_Float16)v;
}
// eight consecutive values from element i on
template <int DT> __device__ __forceinline__ void load8(const void *p, size_t i, float (&v)[8])
{
    if constexpr (DT == FP32) {
        const u32x4_a4 *q = reinterpret_cast<const u32x4_a4 *>(static_cast<const float *>(p) + i);
        const u32x4 a = q[0], b = q[1];
        for (int j = 0; j < 4; ++j) v[j] = f32_of_bits(a[j]), v[4 + j] = f32_of_bits(b[j]);
    } else {
        const u32x4 a = *reinterpret_cast<const u32x4_a2 *>(static_cast<const uint16_t *>(p) + i);
        for (int j = 0; j < 4; ++j) {
            const f32x2 t = unpack2<DT>(a[j]);
            v[2 * j] = t[0], v[2 * j + 1] = t[1];
        }
    }
}
// (past the caches: 90 MB of bf16 read back from 4 bits take 17.0 us, 22.1 with plain stores; plain loads are as fast as such loads)
template <int DT> __device__ __forceinline__ void store8(void *p, size_t i, const float (&v)[8])
{
    if constexpr (DT == FP32) {
        u32x4_a4 *q = reinterpret_cast<u32x4_a4 *>(static_cast<float *>(p) + i);
        u32x4 a, b;
        for (int j = 0; j < 4; ++j) a[j] = bits_of(v[j]), b[j] = bits_of(v[4 + j]);
        __builtin_nontemporal_store(a, q), __builtin_nontemporal_store(b, q + 1);
    } else {
        u32x4 a;
        for (int j = 0; j < 4; ++j) a[j] = pack2<DT>(v[2 * j], v[2 * j + 1]);
        __builtin_nontemporal_store(a, reinterpret_cast<u32x4_a2 *>(static_cast<uint16_t *>(p) + i));
    }
}

// 2^(byte - 127); 255 is NaN
__device__ __forceinline__ float power_of(uint32_t byte)
{
    return f32_of_bits(byte == 255 ? 0x7FC00000u : byte == 0 ? 1u << 22 : byte << 23);
}

// E4M3 codes: the byte of the smallest power of two 2^e with a <= 448 2^e, a given by its bits, 448 = 1.75 * 2^8: one exponent more where the mantissa is over 1.75.
// Below 2^-126 the exponent field says 0 where the exponent is smaller still; both give the least scale.
__device__ __forceinline__ uint32_t scale_byte(uint32_t a)
{
    const int32_t e = (int32_t)(a >> 23) - 8 + ((a & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return e > 0 ? (uint32_t)e : 0;
}

// v / d for v < 2^31: (v * mul) >> shift with mul = ceil(2^(31 + s) / d), s = ceil(log2 d); exact, as the error of mul is below d <= 2^s
struct Divide {
    uint32_t mul, shift, by;
};
inline Divide divide_by(uint32_t d)
{
    uint32_t s = 0;
    while (((uint64_t)1 << s) < d) ++s;
    return {(uint32_t)((((uint64_t)1 << (31 + s)) + d - 1) / d), 31 + s, d};
}
__device__ __forceinline__ uint32_t quotient(uint32_t v, const Divide &d)
{
    return (uint32_t)(((uint64_t)v * d.mul) >> d.shift);
}

// More LDS than 64 KB has to be allowed, once for a kernel and device; `allowed` keeps a bit for each device that it is on.
inline bool allow_lds(const void *kernel, size_t bytes, std::atomic<uint64_t> &allowed)
{
    int device = 0;
    if (hipGetDevice(&device) != hipSuccess) return false;
    const uint64_t bit = device < 64 ? (uint64_t)1 << device : 0;
    if (allowed.load(std::memory_order_relaxed) & bit) return true;
    if (hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != hipSuccess) return false;
    allowed.fetch_or(bit, std::memory_order_relaxed);
    return true;
}

}  // namespace lowbit
}  // namespace enec
