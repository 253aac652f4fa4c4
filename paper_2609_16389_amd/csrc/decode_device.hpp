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

// The same from a place that all lanes share (kept in scalar registers, which
// the empty asm forces) and a lane's own distance from it.
template <class T>
__device__ __forceinline__ T load_at(const void *base, uint32_t off)
{
    struct __attribute__((packed, aligned(1))) any {
        T v;
    };
    typedef const __attribute__((address_space(1))) char *gptr;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)base);
    const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)((uintptr_t)base >> 32));
    gptr b = (gptr)((uintptr_t)hi << 32 | lo);
    asm("" : "+s"(b));
    return ((const __attribute__((address_space(1))) any *)(b + off))->v;
}
template <class T>
__device__ __forceinline__ T load_at(const void *base, int64_t off)
{
    return load_any<T>((const char *)base + off);
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

// `v` moved down by `bytes` (0 .. 16), zeros entering at the top.
__device__ __forceinline__ u32x4 shift_down(u32x4 v, int bytes)
{
    uint64_t lo = v[0] | (uint64_t)v[1] << 32, hi = v[2] | (uint64_t)v[3] << 32;
    if (bytes >= 8) {
        lo = bytes >= 16 ? 0 : hi;
        hi = 0;
    }
    const int b = 8 * (bytes & 7);
    lo = lo >> b | (b ? hi << (64 - b) : 0);
    hi >>= b;
    u32x4 r = {(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
    return r;
}

// 16 bytes of a row of `n` (> 0) bytes from byte `at`, zeros past its end: the
// row's last 16 moved into place, without a branch on the lane.
__device__ __forceinline__ u32x4 load16_end(const void *row, int64_t at, int64_t n)
{
    if (n >= 16) {
        const int64_t from = min(at, n - 16);
        return shift_down(load_any<u32x4>((const char *)row + from), (int)min(at - from, (int64_t)16));
    }
    u32x4 v = {0u, 0u, 0u, 0u};
#pragma unroll 1
    for (int j = 0; j < (int)n; ++j) {   // a row shorter than that, from its last byte down
        const uint32_t b = ((const uint8_t *)row)[n - 1 - j];
        v[3] = v[3] << 8 | v[2] >> 24;
        v[2] = v[2] << 8 | v[1] >> 24;
        v[1] = v[1] << 8 | v[0] >> 24;
        v[0] = v[0] << 8 | b;
    }
    return shift_down(v, (int)min(at, (int64_t)16));
}

// Partial sums between workgroups: 16 bytes at a distance of at most 2^32 from
// `base`, at device scope (sc1).  Such a store, once complete, is visible to
// such loads from every XCD.
constexpr int kDeviceScope = 1 << 4;
__device__ __forceinline__ void store4_device(void *base, uint32_t off, f32x4 v)
{
    __builtin_amdgcn_raw_buffer_store_b128(
        __builtin_bit_cast(u32x4, v), __builtin_amdgcn_make_buffer_rsrc(base, (short)0, (int)0xffffffff, 0x00020000), off,
        0, kDeviceScope);
}
__device__ __forceinline__ f32x4 load4_device(void *base, uint32_t off)
{
    return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                         __builtin_amdgcn_make_buffer_rsrc(base, (short)0, (int)0xffffffff, 0x00020000),
                                         off, 0, kDeviceScope));
}

}  // namespace xdecode_dev
