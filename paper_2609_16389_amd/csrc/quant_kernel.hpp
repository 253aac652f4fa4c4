// y = x * W^T for a few rows x and 4-bit weights with group scales.
//
//     y[m][n] = sum over k of x[m][k] * s[n][k / group] * (q[n][k] - z[n][k / group])
//
// x and s are 16-bit floating point, q holds two values a byte (even k in the
// low half), z is a byte (8 where there is none).
//
// A weight becomes a 16-bit float with one shift and one bit-field insert for
// two: the four bits go to the top of the mantissa of 16, which makes 16 + q
// exactly.  The matrix units then form, for every group,
//     P = sum of x (16 + q)     S = sum of x (a product with ones)
// in fp32, and the group adds s (P - (16 + z) S) to the output.  (16 and not a
// larger power of two: the part that cancels is 24 on average against |q - 8|
// of 4, which costs two bits of fp32; 128 + q would cost five.)
//
// Layout: the weights are the matrix units' second operand, lane l holding
// column n = l % 16, so that a lane needs one scale a group.  A wave takes
// every kWaves-th unit of 256 k: per column 128 bytes, one cache line, in two
// 16-byte loads a lane.  Lane group g (l / 16) holds k 32 g .. + 31 of a block
// of 128; any assignment of k to lanes is valid as long as x is loaded alike.
// Groups smaller than 128 need each product inside one group: there the four
// dwords are transposed between the lane groups (four lane swaps), so that
// dword i holds k 32 i + 8 g .. + 7.
// Within a dword the bit-field inserts pair value i with i + 4; x is permuted
// to match, once for all columns.
// The waves of a workgroup split K and add their blocks through LDS in
// ascending order.
#pragma once

#include "decode_device.hpp"

namespace xquant_dev {

using namespace xdecode_dev;

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / 64;
constexpr int kUnit = 256;  // k per unit of a wave: two blocks of 128

struct QuantParams {
    const uint16_t *x;
    const uint8_t *q;
    const uint16_t *s;
    const uint8_t *z;  // null: 8 everywhere
    void *y;
    int64_t ldx, ldq, lds, ldz, ldy;  // elements (q: bytes)
    int M, N, K, group;
    int out16;         // y in the type of x, else fp32
};

// Two weights of a dword as 16-bit floats 16 + q: values i and i + 4.
template <int DT, int I>
__device__ __forceinline__ uint32_t widen2(uint32_t w)
{
    constexpr int at = DT == 0 ? 3 : 6;  // lowest bit of the mantissa's top four
    constexpr uint32_t mask = DT == 0 ? 0x00780078u : 0x03c003c0u;
    constexpr uint32_t base = DT == 0 ? 0x41804180u : 0x4c004c00u;
    constexpr int up = at - 4 * I;
    const uint32_t t = up >= 0 ? w << (up & 31) : w >> (-up & 31);
    return (t & mask) | base;
}

template <int DT>
__device__ __forceinline__ u32x4 widen8(uint32_t w)
{
    u32x4 r = {widen2<DT, 0>(w), widen2<DT, 1>(w), widen2<DT, 2>(w), widen2<DT, 3>(w)};
    return r;
}

// x in the order of widen8's values: 0, 4, 1, 5, 2, 6, 3, 7.
__device__ __forceinline__ u32x4 pair_up(u32x4 v)
{
    u32x4 r = {__builtin_amdgcn_perm(v[2], v[0], 0x05040100u), __builtin_amdgcn_perm(v[2], v[0], 0x07060302u),
               __builtin_amdgcn_perm(v[3], v[1], 0x05040100u), __builtin_amdgcn_perm(v[3], v[1], 0x07060302u)};
    return r;
}

// Dword i of lane group g to dword g of lane group i.
__device__ __forceinline__ u32x4 transpose_groups(u32x4 v)
{
    const auto a = __builtin_amdgcn_permlane32_swap(v[0], v[2], false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(v[1], v[3], false, false);
    const auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
    const auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    u32x4 r = {c[0], c[1], d[0], d[1]};
    return r;
}

// 16 bytes of a row of `n` from byte `at` (zeros past its end).
__device__ __forceinline__ u32x4 load16_guarded(const uint8_t *row, int64_t at, int64_t n)
{
    if (at + 16 <= n)
        return load_any<u32x4>(row + at);
    u32x4 v = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int j = 0; j < 16; ++j)
        if (at + j < n)
            v[j / 4] |= (uint32_t)row[at + j] << (8 * (j & 3));
    return v;
}

// Workgroup (blockIdx.x, blockIdx.y): columns from 16 NT blockIdx.x, rows from
// 16 MT blockIdx.y.  SMALL: groups of 32 or 64, else a multiple of 128.
template <int DT, int MT, int NT, bool SMALL>
__global__ void __launch_bounds__(kThreads)
quant_kernel(QuantParams p)
{
    __shared__ float red[kWaves * MT * NT * 256];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int c = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * 16 * NT, m0 = blockIdx.y * 16 * MT;
    const int64_t width = ((int64_t)p.K + 1) / 2;

    const uint8_t *qrow[NT];
    const uint16_t *srow[NT];
    const uint8_t *zrow[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int64_t n = min(n0 + 16 * j + c, p.N - 1);
        qrow[j] = p.q + n * p.ldq;
        srow[j] = p.s + n * p.lds;
        zrow[j] = p.z ? p.z + n * p.ldz : nullptr;
    }
    const uint16_t *xrow[MT];
    bool live[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int m = m0 + 16 * i + c;
        live[i] = m < p.M;
        xrow[i] = p.x + (int64_t)min(m, p.M - 1) * p.ldx;
    }
    const uint32_t one = DT == 0 ? 0x3f803f80u : 0x3c003c00u;
    const u32x4 ones = {one, one, one, one};
    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};

    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
            acc[i][j] = zero;

    for (int64_t k0 = (int64_t)wave * kUnit; k0 < p.K; k0 += kWaves * kUnit) {
        const bool whole = k0 + kUnit <= p.K;
        u32x4 w[2][NT];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const int64_t at = k0 / 2 + 64 * b + 16 * g;
                w[b][j] = whole ? load_any<u32x4>(qrow[j] + at) : load16_guarded(qrow[j], at, width);
                if (SMALL)
                    w[b][j] = transpose_groups(w[b][j]);
            }
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int64_t kb = k0 + 128 * b;
            f32x4 P[MT][NT], S[MT];
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                const int64_t k = SMALL ? kb + 32 * d + 8 * g : kb + 32 * g + 8 * d;
                const bool first = SMALL ? p.group == 32 || d % 2 == 0 : d == 0;
                const bool last = SMALL ? p.group == 32 || d % 2 == 1 : d == 3;
                u32x4 a[MT];
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    u32x4 v = {0u, 0u, 0u, 0u};
                    if (live[i])
                        v = whole ? load_any<u32x4>(xrow[i] + k) : load8_guarded(xrow[i], k, p.K);
                    a[i] = pair_up(v);
                    S[i] = mfma16<DT>(a[i], ones, first ? zero : S[i]);
                }
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    const u32x4 f = widen8<DT>(w[b][j][d]);
#pragma unroll
                    for (int i = 0; i < MT; ++i)
                        P[i][j] = mfma16<DT>(a[i], f, first ? zero : P[i][j]);
                }
                // the group's first k, which may lie past K
                const int64_t kg = SMALL ? kb + 32 * (p.group == 32 ? d : d & 2) : kb;
                if (last && kg < p.K) {
                    const int64_t gi = kg / p.group;
#pragma unroll
                    for (int j = 0; j < NT; ++j) {
                        const float s = to_float<DT>(srow[j][gi]);
                        const float off = 16.0f + (p.z ? (float)zrow[j][gi] : 8.0f);
#pragma unroll
                        for (int i = 0; i < MT; ++i)
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                acc[i][j][r] = fmaf(s, fmaf(-off, S[i][r], P[i][j][r]), acc[i][j][r]);
                    }
                }
            }
        }
    }

    // the waves' blocks, added in ascending order
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                red[((wave * MT * NT + i * NT + j) * 4 + r) * 64 + lane] = acc[i][j][r];
    __syncthreads();
    for (int o = tid; o < MT * NT * 256; o += kThreads) {
        const int tile = o >> 8, r = o >> 6 & 3, l = o & 63;
        const int m = m0 + 16 * (tile / NT) + 4 * (l >> 4) + r, n = n0 + 16 * (tile % NT) + (l & 15);
        if (m >= p.M || n >= p.N)
            continue;
        float v = red[o];
#pragma unroll
        for (int w = 1; w < kWaves; ++w)
            v += red[w * MT * NT * 256 + o];
        if (p.out16)
            ((uint16_t *)p.y)[(int64_t)m * p.ldy + n] = from_float<DT>(v);
        else
            ((float *)p.y)[(int64_t)m * p.ldy + n] = v;
    }
}

}  // namespace xquant_dev
