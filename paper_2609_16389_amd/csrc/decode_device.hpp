// Device helpers shared by the kernels around a decoding step (products with
// 4-bit weights, layers of experts, log probabilities).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace xdecode_dev {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// c + a * b on the matrix units, 16 x 16 over 32 k: lane l holds row (a) or
// column (b) l % 16 and eight of the k; rows 4 (l / 16) .. + 3 of column
// l % 16 of c.  DT 0: bfloat16, 1: binary16.
template <int DT>
__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c)
{
    if constexpr (DT == 0)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c,
                                                       0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0,
                                                      0, 0);
}

// Loads at any byte alignment (the memory path takes them as they are).
template <class T>
__device__ __forceinline__ T load_any(const void *p)
{
    struct __attribute__((packed, aligned(1))) any {
        T v;
    };
    return ((const any *)p)->v;
}

template <class T>
__device__ __forceinline__ void store_any(void *p, T v)
{
    struct __attribute__((packed, aligned(1))) any {
        T v;
    };
    ((any *)p)->v = v;
}

// Values of storage type DT (0: bfloat16, 1: binary16) to fp32 and back,
// rounded to nearest even.
template <int DT>
__device__ __forceinline__ float to_float(uint16_t b)
{
    if constexpr (DT == 0)
        return __builtin_bit_cast(float, (uint32_t)b << 16);
    else
        return (float)__builtin_bit_cast(_Float16, b);
}

template <int DT>
__device__ __forceinline__ uint16_t from_float(float v)
{
    if constexpr (DT == 0)
        return __builtin_bit_cast(uint16_t, (__bf16)v);
    else
        return __builtin_bit_cast(uint16_t, (_Float16)v);
}

// Eight 16-bit values from k of a row of n (zeros past its end).
__device__ __forceinline__ u32x4 load8_guarded(const uint16_t *row, int64_t k, int64_t n)
{
    if (k + 8 <= n)
        return load_any<u32x4>(row + k);
    u32x4 v = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (k + j < n)
            v[j / 2] |= (uint32_t)row[k + j] << (16 * (j & 1));
    return v;
}

}  // namespace xdecode_dev
