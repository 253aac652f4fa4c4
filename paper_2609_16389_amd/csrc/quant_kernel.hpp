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
// bfloat16 reaches as far as fp32, so that 128 products x (16 + q), or x 271 with
// the largest z, would leave fp32's range for an x of 1e35: there the weights,
// and the ones, are held times 2^-16, and the output is multiplied by 2^16.
//
// Layout: the weights are the matrix units' second operand, lane l holding
// column n = l % 16, so that a lane needs one scale a group.  A wave takes a
// range of K in units of one or two blocks of 128 k: per column and unit of two
// blocks 128 bytes, one cache line, in two 16-byte loads a lane.  Lane group g
// (l / 16) holds k 32 g .. + 31 of a block; any assignment of k to lanes is
// valid as long as x is loaded alike.
// Groups smaller than 128 need each product inside one group: there the four
// dwords are transposed between the lane groups (four lane swaps), so that
// dword i holds k 32 i + 8 g .. + 7.
// Within a dword the bit-field inserts pair value i with i + 4; x is permuted
// to match, once for all columns.
// The waves of a workgroup split K and add their blocks through LDS in
// ascending order.
//
// What bounds it: with one row the bytes of q and a launch's latency (bfloat16,
// groups of 128: 1 x 4096 x 4096 4.2 us in a stream of calls, 1 x 14336 x 4096
// with groups of 64 and zero points 9.7 us or 3.4 TB/s); with many rows the
// time of a unit, a chain of a barrier, reads of x, widening, products and
// scaling that no unit of the CU fills (64 x 16384 x 16384 75 us: matrix units 27%
// busy, vector instructions 36%; a wave taking two tiles of 16 columns, which
// halves its reads of x and saves a quarter of the products, gained 4%).
#pragma once

#include <utility>

#include "decode_device.hpp"

namespace xquant_dev {

using namespace xdecode_dev;


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

// The masks of widen8, hidden from the compiler so that it keeps them in
// registers and masks and inserts in one instruction.
struct Masks {
    uint32_t mask, base;
};

template <int DT>
__device__ __forceinline__ Masks masks()
{
    Masks m;
    asm("v_mov_b32 %0, %1" : "=v"(m.mask) : "i"(DT == 0 ? 0x00780078u : 0x03c003c0u));
    asm("s_mov_b32 %0, %1" : "=s"(m.base) : "i"(DT == 0 ? 0x39803980u : 0x4c004c00u));
    return m;
}

// Two weights of a dword as 16-bit floats 16 + q (bfloat16: times 2^-16): values
// I and I + 4.
template <int DT, int I>
__device__ __forceinline__ uint32_t widen2(uint32_t w, Masks m)
{
    constexpr int up = (DT == 0 ? 3 : 6) - 4 * I;   // to the mantissa's top four bits
    const uint32_t t = up >= 0 ? w << (up & 31) : w >> (-up & 31);
    return (t & m.mask) | m.base;
}

template <int DT>
__device__ __forceinline__ u32x4 widen8(uint32_t w, Masks m)
{
    u32x4 r = {widen2<DT, 0>(w, m), widen2<DT, 1>(w, m), widen2<DT, 2>(w, m), widen2<DT, 3>(w, m)};
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

// f.operator()<0>() ... <N - 1>(): a loop unrolled in the source, so that no
// array of registers is ever indexed.
template <int N, class F>
__device__ __forceinline__ void repeat(F &&f)
{
    [&]<int... I>(std::integer_sequence<int, I...>) {
        (f.template operator()<I>(), ...);
    }(std::make_integer_sequence<int, N>{});
}

// LDS of a workgroup of WN x WK waves of CT column tiles for rows R and units
// of BL blocks.
template <int R, int WN, int WK, int CT, int BL>
struct QuantLds {
    static constexpr int MT = (R + 15) / 16;
    static constexpr int XPART = BL * (R < 16 ? 16 * R * 16 : MT * 4096);   // x of one unit of k
    static constexpr int BUFS = WN == 1 ? 1 : 2;
    static constexpr int PIECES = R * 16 * BL / (WN * 64);   // 16-byte pieces of it that a thread brings in
    static constexpr int AHEAD = PIECES <= 2 ? 2 : 1;   // units of x on their way to registers
    __attribute__((aligned(16))) union {
        struct {
            char x[WK][BUFS][XPART];
            float2 scale[WK * WN][CT][16][16];   // {s, 16 + z} of 16 groups of 16 columns
        };
        float red[WK][WN * CT][MT][256];
    };
    // the weights of the unit that K ends in, in the place of x of the first
    // ranges; the last range's holds x of that unit
    static_assert((WK - 1) * BUFS * XPART >= 16 * WN * CT * 64 * BL, "room for the last unit's weights");
    __device__ __forceinline__ uint8_t *wend() { return (uint8_t *)x; }
};

// The waves of a workgroup: WN take CT tiles of 16 columns each, WK a range of
// k each, in units of BL blocks of 128.
// Workgroup (blockIdx.x, blockIdx.y): columns from 16 WN CT blockIdx.x, rows from
// R blockIdx.y (R: 2 WN, or a multiple of 16).  GS: groups of 32 or 64, or 128
// for any multiple of that.  off_t holds the distance of a lane's row of q from
// its tile's first: 32 bits where leading dimensions allow.
//
// Per unit a wave waits for x and then for its weights, while the weights of
// the next unit and x of the next two are on their way.  Loads return in
// order, so one that may or may not have been issued would make every wait
// behind it a wait for all: the loop's loads of x and weights are unconditional,
// past the end they repeat the last unit's, and the unit that K ends in comes
// after it.  Those of the scales come once in CHUNK units, and the wait for x
// behind them allows for both: it leaves two loads on their way, not more.
//
// With WN == 1 a wave alone writes and reads its x, and always its scales: its
// LDS accesses complete in order, and the compiler keeps those of one array at
// places it cannot tell apart in order, so there is no barrier between them.
// (A fence at wavefront scope there moves the loads too: 5 x 4097 x 2047 8.3 us
// without, 11.1 with.)
template <int DT, int R, int WN, int WK, int CT, int BL, int GS, class off_t>
__global__ void __launch_bounds__(64 * WN * WK, R < 16 || WN * WK > 8 ? 4 : 2)
quant_kernel(QuantParams p)
{
    typedef QuantLds<R, WN, WK, CT, BL> Lds;
    constexpr int kUnit = 128 * BL;
    constexpr int MT = Lds::MT, THREADS = 64 * WN * WK, NP = Lds::PIECES, XA = Lds::AHEAD;
    constexpr int GROUPS = 128 / GS;            // of a block
    constexpr int CHUNK = 16 * GS / kUnit;      // units that 16 groups cover
    __shared__ Lds sh;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wn = wave % WN, wk = wave / WN;
    const int c = lane & 15, g = lane >> 4;
    const int m0 = blockIdx.y * R, rows = min(R, p.M - m0);
    const int nw = blockIdx.x * 16 * WN * CT, n0 = nw + 16 * CT * wn;

    // this wave's whole units of k (WK is a power of two)
    const int units = p.K / kUnit;
    const int u0 = wk * (units / WK) + min(wk, units % WK), mine = units / WK + (wk < units % WK);
    const int steps = (units + WK - 1) / WK;    // of the longest range

    // columns past N are read from the last one, never stored
    const int nb = min(n0, p.N - 1);
    int nl[CT];
    off_t qoff[CT];
    repeat<CT>([&]<int t>() {
        nl[t] = min(16 * t + c, p.N - 1 - nb);
        qoff[t] = (off_t)nl[t] * (off_t)p.ldq + 16 * g;
    });
    const uint8_t *const qbase = p.q + (int64_t)nb * p.ldq;
    u32x4 w[2][CT][BL];
    auto load_w = [&](u32x4 (&to)[CT][BL], int t) {
        const uint8_t *const q = qbase + (int64_t)(u0 + min(t, mine - 1)) * (kUnit / 2);
        repeat<CT * BL>([&]<int i>() { to[i / BL][i % BL] = load_at<u32x4>(q + 64 * (i % BL), qoff[i / BL]); });
    };

    // x: of a unit, thread t of the WN waves of a range brings in pieces t, t +
    // 64 WN, ...: piece i is 8 k from 8 (i % PR) of row i / PR (rows past M
    // repeat the last one)
    constexpr int PR = 16 * BL;
    const int xi = wn * 64 + lane;
    const uint16_t *const xbase = p.x + (int64_t)m0 * p.ldx + 8 * (xi % PR);
    u32x4 xr[XA][NP];
    auto load_x = [&](u32x4 (&to)[NP], int t) {
        const int64_t k = (int64_t)(u0 + min(t, mine - 1)) * kUnit;
#pragma unroll
        for (int q = 0; q < NP; ++q)
            to[q] = load_any<u32x4>(xbase + min(xi / PR + 64 / PR * WN * q, rows - 1) * p.ldx + k);
    };
    // where 8 k of a row lie in LDS: piece kc of a block of 128 goes to lane
    // group kg of product kd; 16 rows are swizzled so that neither the pieces of
    // a row nor the rows of a piece share a bank
    auto x_place = [&](int row, int b, int kc) {
        const int kd = GS < 128 ? kc >> 2 : kc & 3, kg = GS < 128 ? kc & 3 : kc >> 2;
        return R < 16 ? (((b * 4 + kd) * 4 + kg) * R + row) * 16
                      : ((b * 4 + kd) * MT + (row >> 4)) * 1024 + kg * 256 + ((row ^ (4 * kd + kg)) & 15) * 16;
    };
    auto store_x = [&](const u32x4 (&from)[NP], int buf) {
#pragma unroll
        for (int q = 0; q < NP; ++q)
            *(u32x4 *)(sh.x[wk][buf] + x_place(xi / PR + 64 / PR * WN * q, xi % PR >> 4, xi & 15)) = pair_up(from[q]);
    };

    // scales and zero points of 16 groups (of GS k) from group q0 on: lane
    // group g brings in four of column c of each tile
    const int groups = (p.K - 1) / p.group + 1;
    uint64_t sr[CT];
    uint32_t zr[CT];
    auto load_scales = [&](int q0) {
        repeat<CT>([&]<int t>() {
            const uint16_t *const sbase = p.s + (int64_t)(nb + nl[t]) * p.lds;
            const uint8_t *const zbase = p.z ? p.z + (int64_t)(nb + nl[t]) * p.ldz : nullptr;
            zr[t] = 0x08080808u;
            if (p.group == GS && groups >= 4) {
                // (at the end of a row its last four, moved down: what lies past it
                // meets x of zero or no product at all)
                const int q = q0 + 4 * g, at = min(q, groups - 4), past = min(q - at, 3);
                sr[t] = load_any<uint64_t>(sbase + at) >> (16 * past);
                if (p.z)
                    zr[t] = load_any<uint32_t>(zbase + at) >> (8 * past);
            } else {
                uint64_t sv = 0;
                uint32_t zv = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int at = min((int)((uint32_t)(q0 + 4 * g + e) * GS / (uint32_t)p.group), groups - 1);
                    sv |= (uint64_t)sbase[at] << (16 * e);
                    if (p.z)
                        zv |= (uint32_t)zbase[at] << (8 * e);
                }
                sr[t] = sv;
                if (p.z)
                    zr[t] = zv;
            }
        });
    };
    auto store_scales = [&] {
        repeat<CT * 4>([&]<int i>() {
            constexpr int t = i / 4, e = i % 4;
            sh.scale[wave][t][4 * g + e][c] = float2{to_float<DT>((uint16_t)(sr[t] >> (16 * e))),
                                                     16.0f + (float)(zr[t] >> (8 * e) & 255u)};
        });
    };

    const Masks widen = masks<DT>();
    const uint32_t one = DT == 0 ? 0x37803780u : 0x3c003c00u;   // (bfloat16: 2^-16)
    const u32x4 ones = {one, one, one, one};
    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    f32x4 acc[CT][MT];
    repeat<CT * MT>([&]<int i>() { acc[i / MT][i % MT] = zero; });

    // one unit: the products of every group, scaled into the outputs; the sum of
    // x serves all of the wave's tiles
    auto compute = [&](const u32x4 (&from)[CT][BL], int buf, int q0) __attribute__((always_inline)) {
        repeat<BL>([&]<int b>() __attribute__((always_inline)) {
            u32x4 v[CT];
            repeat<CT>([&]<int t>() { v[t] = GS < 128 ? transpose_groups(from[t][b]) : from[t][b]; });
            f32x4 P[CT][MT], S[MT];
            repeat<4>([&]<int d>() __attribute__((always_inline)) {
                constexpr bool first = d % (GS / 32) == 0, last = d % (GS / 32) == GS / 32 - 1;
                u32x4 f[CT];
                repeat<CT>([&]<int t>() { f[t] = widen8<DT>(v[t][d], widen); });
                repeat<MT>([&]<int i>() __attribute__((always_inline)) {
                    const u32x4 a = *(const u32x4 *)(sh.x[wk][buf] + x_place(R < 16 ? min(c, R - 1) : 16 * i + c, b,
                                                                             GS < 128 ? 4 * d + g : 4 * g + d));
                    S[i] = mfma16<DT>(a, ones, first ? zero : S[i]);
                    repeat<CT>([&]<int t>() { P[t][i] = mfma16<DT>(a, f[t], first ? zero : P[t][i]); });
                });
                if constexpr (last)
                    repeat<CT>([&]<int t>() {
                        const float2 sc = sh.scale[wave][t][q0 + b * GROUPS + d / (GS / 32)][c];
                        repeat<MT * 4>([&]<int j>() {
                            constexpr int i = j / 4, r = j % 4;
                            acc[t][i][r] = fmaf(sc.x, fmaf(-sc.y, S[i][r], P[t][i][r]), acc[t][i][r]);
                        });
                    });
                if constexpr (MT * CT > 4)
                    __builtin_amdgcn_sched_barrier(0);   // (reads of x moved up from the next product would not fit)
            });
        });
    };
    auto sync = [&] {
        __builtin_amdgcn_s_waitcnt(15 | (3 << 14) | (7 << 4));  // lgkmcnt(0)
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    if (mine > 0) {
        load_scales(u0 * (kUnit / GS));
#pragma unroll
        for (int a = 0; a < XA; ++a)
            load_x(xr[a], a);
        load_w(w[0], 0);
        load_w(w[1], 1);
        auto step = [&]<int B>(int t) {
            const int buf = WN == 1 ? 0 : B;
            if (B == 0 && t % CHUNK == 0) {
                store_scales();
                load_scales((u0 + min(t + CHUNK, mine - 1) / CHUNK * CHUNK) * (kUnit / GS));
            }
            store_x(xr[B % XA], buf);
            load_x(xr[B % XA], t + XA);
            if (WN > 1)
                sync();
            compute(w[B], buf, t % CHUNK * (kUnit / GS));
            load_w(w[B], t + 2);
        };
        for (int t = 0;;) {
            step.template operator()<0>(t);
            if (++t == mine)
                break;
            step.template operator()<1>(t);
            if (++t == mine)
                break;
        }
    }
    if (WN > 1 && mine < steps)
        sync();   // (ranges differ by one unit)
    if (p.K % kUnit) {
        // the unit that K ends in: padded with zeros on its way through LDS, and
        // taken by the last range's waves
        const int kend = units * kUnit;
        sync();   // (x is done with)
        char *const to = sh.x[WK - 1][0];
        for (int o = tid; o < 16 * WN * CT * 4 * BL; o += THREADS)
            *(u32x4 *)(sh.wend() + 16 * o) =
                load16_end(p.q + (int64_t)min(nw + o / (4 * BL), p.N - 1) * p.ldq, kend / 2 + 16 * (o % (4 * BL)),
                           ((int64_t)p.K + 1) / 2);
        for (int o = tid; o < R * PR; o += THREADS) {
            const int row = o / PR;
            const u32x4 v = load16_end(p.x + (int64_t)(m0 + min(row, rows - 1)) * p.ldx,
                                       2 * ((int64_t)kend + 8 * (o % PR)), 2 * (int64_t)p.K);
            *(u32x4 *)(to + x_place(row, o % PR >> 4, o & 15)) = pair_up(v);
        }
        if (wk == WK - 1) {
            load_scales(units * (kUnit / GS));
            store_scales();
        }
        sync();
        if (wk == WK - 1) {
            repeat<CT * BL>([&]<int i>() {
                w[0][i / BL][i % BL] = *(const u32x4 *)(sh.wend() + (16 * (CT * wn + i / BL) + c) * 64 * BL +
                                                        64 * (i % BL) + 16 * g);
            });
            compute(w[0], 0, 0);
        }
    }
    sync();   // (x and the scales are done with)

    // the ranges' sums, added in ascending order
    repeat<CT * MT * 4>([&]<int j>() {
        constexpr int t = j / (4 * MT), i = j / 4 % MT, r = j % 4;
        sh.red[wk][CT * wn + t][i][64 * r + lane] = acc[t][i][r];
    });
    sync();
    for (int o = tid; o < WN * CT * MT * 256; o += THREADS) {
        const int j = o / (MT * 256), i = (o >> 8) % MT, r = o >> 6 & 3, l = o & 63;
        const int row = 16 * i + 4 * (l >> 4) + r, n = nw + 16 * j + (l & 15);
        if (row >= rows || n >= p.N)
            continue;
        float v = sh.red[0][j][i][o & 255];
#pragma unroll
        for (int w = 1; w < WK; ++w)
            v += sh.red[w][j][i][o & 255];
        if (DT == 0)
            v *= 0x1p16f;
        const int64_t at = (int64_t)(m0 + row) * p.ldy + n;
        if (p.out16)
            ((uint16_t *)p.y)[at] = from_float<DT>(v);
        else
            ((float *)p.y)[at] = v;
    }
}

}  // namespace xquant_dev
