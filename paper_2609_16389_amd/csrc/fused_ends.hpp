// What becomes of the sums of a tile (fused_tile.hpp): the ends of the 8-bit
// products, the gated feed-forward block, the log probabilities of a head and
// their gradients' products.
//
// An End takes four neighbouring columns of a row at a time (quad), from the
// registers of the product or, where k was split over workgroups (kJoins), from
// the sums of its parts (join_parts, in ascending order).
#pragma once

#include "fused_tile.hpp"

namespace xfused_dev {

constexpr float kLog2e = 1.44269504088896340736f;

// Four values of a row from column `col` of `n`, rounded to the type that
// `kind` names (kBf16, kFp16 or kFp32).
constexpr int kFp32 = 2;
__device__ __forceinline__ void store_quad(void *row, int kind, int col, int n, f32x4 v)
{
    if (kind == kFp32) {
        float *const q = (float *)row + col;
        if (col + 4 <= n) {
            store_any<f32x4>(q, v);
        } else {
#pragma unroll
            for (int k = 0; k < 3; ++k)
                if (col + k < n)
                    q[k] = v[k];
        }
        return;
    }
    uint16_t h[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
        h[k] = kind == kBf16 ? from_float<kBf16>(v[k]) : from_float<kFp16>(v[k]);
    uint16_t *const q = (uint16_t *)row + col;
    if (col + 4 <= n) {
        store_any<uint64_t>(q, (uint64_t)(h[0] | (uint32_t)h[1] << 16) | (uint64_t)(h[2] | (uint32_t)h[3] << 16) << 32);
    } else {
#pragma unroll
        for (int k = 0; k < 3; ++k)
            if (col + k < n)
                q[k] = h[k];
    }
}
__device__ __forceinline__ void *row_at(void *base, int64_t ld, int row, int kind)
{
    return (char *)base + (int64_t)row * ld * (kind == kFp32 ? 4 : 2);
}

// Calls f(row, col, i, j) for the blocks of a wave that hold rows of the result.
template <int TM, int TN, int FM, int FN, class F>
__device__ __forceinline__ void each_quad(int M, int N, int m0, int n0, int wm, int wn, int lane, F f)
{
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const int row = m0 + wm * TM + i * 16 + (lane & 15);
        if (row < M) {
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                const int col = n0 + wn * TN + j * 16 + (lane >> 4) * 4;
                if (col < N)
                    f(row, col, i, j);
            }
        }
    }
}

// The wave's block of the result from (row0, col0) on, rounded to the 16-bit type
// that `kind` names, through LDS (the wave's own, TM x TN values), so that a store is
// 16 bytes a lane of whole rows of the block: 128 bytes of a row where TN is 64.
// (Straight from the accumulators it is 8 bytes a lane, 32 of 16 rows: 8-bit 4096 x
// 14336 x 4096 279 us in place of 255, gated_grad 333 x 1001 x 2731 59 in place of 54.)  f(i, j, row,
// col): the four values of a quad; N: columns that are stored.
template <int TM, int TN, int FM, int FN, class F>
__device__ __forceinline__ void store_block(char *sh, uint16_t *out, int64_t ld, int kind, int M, int N, int row0, int col0,
                                            int lane, F f)
{
    constexpr int CH = TN / 8, ROWS = 64 / CH;   // chunks of a row, rows of a store
    const int r = lane & 15, g = lane >> 4;
    asm volatile("" ::: "memory");
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const f32x4 v = f(i, j, row0 + i * 16 + r, col0 + j * 16 + g * 4);
            uint16_t h[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                h[k] = kind == kBf16 ? from_float<kBf16>(v[k]) : from_float<kFp16>(v[k]);
            const int row = i * 16 + r, c = (j * 2 + (g >> 1)) ^ (row & (CH - 1));
            *(uint64_t *)(sh + row * TN * 2 + c * 16 + (g & 1) * 8) =
                (uint64_t)(h[0] | (uint32_t)h[1] << 16) | (uint64_t)(h[2] | (uint32_t)h[3] << 16) << 32;
        }
    asm volatile("" ::: "memory");   // (what other lanes have written is read: a wave's LDS accesses stay in order)
#pragma unroll
    for (int t = 0; t < TM / ROWS; ++t) {
        const int row = t * ROWS + lane / CH, c = lane % CH, col = col0 + c * 8;
        const u32x4 v = *(const u32x4 *)(sh + row * TN * 2 + ((c ^ (row & (CH - 1))) << 4));
        if (row0 + row < M && col < N) {
            uint16_t *const to = out + (int64_t)(row0 + row) * ld + col;
            if (col + 8 <= N) {
                store_any<u32x4>(to, v);
            } else {
#pragma unroll
                for (int k = 0; k < 7; ++k)
                    if (col + k < N)
                        to[k] = (uint16_t)(v[k / 2] >> (16 * (k & 1)));
            }
        }
    }
    asm volatile("" ::: "memory");
}

// Sums of a range of k, as they are: part [ks][M][ld] (4 bytes a value), for a
// gated tile with the second matrix's columns from ld / 2 on.
template <int TYPE, bool GATED>
struct PartEnd {
    static constexpr bool kGated = GATED, kStages = true;   // (of an End that does)
    struct Params {
        char *part;
        int ld;   // a multiple of 4, of 8 where gated
    };
    template <int BM, int BN, int TM, int TN, int FM, int FN, int WN, class Acc>
    static __device__ __forceinline__ void finish(const TileParams &p, const Params &e, Acc &acc, char *, int m0, int n0,
                                                  int wm, int wn, int, int ks, int lane)
    {
        char *const base = e.part + (int64_t)ks * p.M * e.ld * 4;
        if constexpr (GATED) {
            each_quad<TM, TN / 2, FM, FN / 2>(p.M, p.N, m0, n0, wm, wn, lane, [&](int row, int col, int i, int j) {
                char *const q = base + ((int64_t)row * e.ld + col) * 4;
                *(u32x4 *)q = __builtin_bit_cast(u32x4, acc[i][j]);
                *(u32x4 *)(q + e.ld / 2 * 4) = __builtin_bit_cast(u32x4, acc[i][j + FN / 2]);
            });
        } else {
            each_quad<TM, TN, FM, FN>(p.M, p.N, m0, n0, wm, wn, lane, [&](int row, int col, int i, int j) {
                *(u32x4 *)(base + ((int64_t)row * e.ld + col) * 4) = __builtin_bit_cast(u32x4, acc[i][j]);
            });
        }
    }
};

// Slopes of a gradient in binary16 have one factor that takes the largest of the matrix
// to 2^14, and a row whose largest is more than 2^kRoom below that would lose bits and
// then vanish.  Its slopes are raised by a power of two to where a row 2^kRoom below
// has them: its row of d_x, which no other row takes part in, is divided by that again,
// and in the weights' gradient, a sum over the rows, it meets a row of x that has been
// divided by it.  So slopes are off by at most 2^-28 of their row's largest beside half a
// step, whatever the sizes of the rows; what x loses is at most 2^-33 of the largest
// slope of all, in terms that small beside it.  (More room leaves less to the small
// slopes of a row, less of it takes bits from x in more rows.)
constexpr int kRoom = 10, kMostRaise = 100;

// The exponent, from the bits of the largest magnitudes of the row and of all.
__device__ __forceinline__ int raise_of(uint32_t row, uint32_t most)
{
    return row == 0 ? 0 : min(max((int)(most >> 23) - (int)(row >> 23) - kRoom, 0), kMostRaise);
}
__device__ __forceinline__ float power_of_two(int n) { return __builtin_bit_cast(float, (uint32_t)(127 + n) << 23); }
// 1 over a power of two, exactly.
__device__ __forceinline__ float over(float power)
{
    return __builtin_bit_cast(float, (254u << 23) - __builtin_bit_cast(uint32_t, power));
}

// Rows of binary16 values, 16 bytes of them at a time, as copies whose rows are whole
// chunks.
struct RaisedCopy {
    const char *from;
    char *to;                        // null: no copies
    int64_t ld, bytes, rows, chunks;
    int times;                       // the copies stand one after another
};
// One row, over 2^n (n < 0: zeros), by a wave.
__device__ __forceinline__ void copy_lowered(const RaisedCopy &m, int64_t row, int n, int lane)
{
    const char *const from = m.from + row * m.ld;
    const float by = power_of_two(-max(n, 0));
#pragma unroll 2
    for (int64_t c = lane; c < m.chunks; c += 64) {
        u32x4 v = {0, 0, 0, 0};
        if (n >= 0)
            v = c * 16 + 16 <= m.bytes ? sixteen<true>(from + c * 16) : load16_end(from, c * 16, m.bytes);
        if (n > 0)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                v[j] = from_float<kFp16>(to_float<kFp16>((uint16_t)(v[j] & 0xffffu)) * by) |
                       (uint32_t)from_float<kFp16>(to_float<kFp16>((uint16_t)(v[j] >> 16)) * by) << 16;
        for (int k = 0; k < m.times; ++k)
            *(u32x4 *)(m.to + ((k * m.rows + row) * m.chunks + c) * 16) = v;
    }
}

// A product as it is: out = sum * scale + add, rounded to out's type.  RAISED: rows
// are sums of raised slopes (see there), and each is divided by its power of two.
struct StoreParams {
    void *out;
    int64_t ld;
    int kind;
    const float *scale;   // a number in memory; null: 1
    const float *add;     // what earlier parts of k left (leading dimension ld_add); null: nothing
    int64_t ld_add;
    const float *raise;   // null: 1
};
template <bool RAISED>
struct StoreEndOf {
    static constexpr bool kGated = false, kJoins = true, kStages = false;
    typedef StoreParams Params;
    typedef float value_t;
    static __device__ __forceinline__ f32x4 value(const Params &e, int row, int col, int M, int N, f32x4 v)
    {
        if (e.scale) {
            const float s = *e.scale;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                v[k] *= s;
        }
        if constexpr (RAISED) {
            if (e.raise && row < M) {
                const float r = over(e.raise[row]);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    v[k] *= r;
            }
        }
        if (e.add && row < M) {
            const float *const q = e.add + (int64_t)row * e.ld_add + col;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (col + k < N)
                    v[k] += q[k];
        }
        return v;
    }
    static __device__ __forceinline__ void quad(const Params &e, int row, int col, int N, f32x4 v, f32x4)
    {
        store_quad(row_at(e.out, e.ld, row, e.kind), e.kind, col, N, value(e, row, col, row + 1, N, v));
    }
    template <int BM, int BN, int TM, int TN, int FM, int FN, int WN, class Acc>
    static __device__ __forceinline__ void finish(const TileParams &p, const Params &e, Acc &acc, char *smem, int m0,
                                                  int n0, int wm, int wn, int, int, int lane)
    {
        if (e.kind != kFp32)
            store_block<TM, TN, FM, FN>(smem + (wm * WN + wn) * TM * TN * 2, (uint16_t *)e.out, e.ld, e.kind, p.M, p.N,
                                        m0 + wm * TM, n0 + wn * TN, lane, [&](int i, int j, int row, int col) {
                                            return value(e, row, col, p.M, p.N, acc[i][j]);
                                        });
        else
            each_quad<TM, TN, FM, FN>(p.M, p.N, m0, n0, wm, wn, lane, [&](int row, int col, int i, int j) {
                quad(e, row, col, p.N, acc[i][j], acc[i][j]);
            });
    }
};
typedef StoreEndOf<false> StoreEnd;

// 8-bit products: out = (sum * scale of the row) * scale of the column.  The sum
// is exact in 32 bits (|sum| <= 2^14 K < 2^31).
struct ScaledEnd {
    static constexpr bool kGated = false, kJoins = true, kStages = true;
    struct Params {
        const float *row_scale, *col_scale;
        void *out;
        int64_t ld;
        int kind;
    };
    typedef int value_t;
    static __device__ __forceinline__ f32x4 value(const Params &e, int row, int col, int M, int N, i32x4 s)
    {
        const float r = row < M ? e.row_scale[row] : 0.0f;
        f32x4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            v[k] = (float)s[k] * r * (col + k < N ? e.col_scale[col + k] : 0.0f);
        return v;
    }
    static __device__ __forceinline__ void quad(const Params &e, int row, int col, int N, i32x4 s, i32x4)
    {
        store_quad(row_at(e.out, e.ld, row, e.kind), e.kind, col, N, value(e, row, col, row + 1, N, s));
    }
    template <int BM, int BN, int TM, int TN, int FM, int FN, int WN, class Acc>
    static __device__ __forceinline__ void finish(const TileParams &p, const Params &e, Acc &acc, char *smem, int m0,
                                                  int n0, int wm, int wn, int, int, int lane)
    {
        if (e.kind != kFp32)
            store_block<TM, TN, FM, FN>(smem + (wm * WN + wn) * TM * TN * 2, (uint16_t *)e.out, e.ld, e.kind, p.M, p.N,
                                        m0 + wm * TM, n0 + wn * TN, lane, [&](int i, int j, int row, int col) {
                                            return value(e, row, col, p.M, p.N, acc[i][j]);
                                        });
        else
            each_quad<TM, TN, FM, FN>(p.M, p.N, m0, n0, wm, wn, lane, [&](int row, int col, int i, int j) {
                quad(e, row, col, p.N, acc[i][j], acc[i][j]);
            });
    }
};

// Activations and their slopes.  Far from zero they are a or 0 to the last bit:
// the argument of the exponentials is held to where that is so, which keeps
// infinities out of the products (a NaN stays).
enum { kSilu = 0, kGelu = 1, kGeluTanh = 2 };

__device__ __forceinline__ float hold(float a, float most) { return a > most ? most : a < -most ? -most : a; }
__device__ __forceinline__ float exp_of(float a) { return __builtin_amdgcn_exp2f(a * kLog2e); }

// 1 / (1 + e), to an ulp or two
__device__ __forceinline__ float logistic(float e) { return __builtin_amdgcn_rcpf(1.0f + e); }

// the share p of a in act(a) = a p
__device__ __forceinline__ float share(int act, float a)
{
    if (act == kSilu)
        return logistic(exp_of(-a));
    if (act == kGelu) {
        // (1 + erf(a / sqrt 2)) / 2: its left tail is exp(-b^2 / 2) t P(t) with b = |a| and t =
        // 1 / (1 + b / 4), P of degree 9 fitted to the scaled complementary error function
        // for the least relative error over b in 0 .. 4000, 1.2e-7 in fp32
        const float b = fabsf(hold(a, 40.0f)), t = __builtin_amdgcn_rcpf(__builtin_fmaf(b, 0.25f, 1.0f));
        float v = 0.01981145516037941f;
        v = __builtin_fmaf(v, t, -0.08100754022598267f);
        v = __builtin_fmaf(v, t, 0.09583782404661179f);
        v = __builtin_fmaf(v, t, -0.03195888549089432f);
        v = __builtin_fmaf(v, t, 0.06384158879518509f);
        v = __builtin_fmaf(v, t, 0.0589248463511467f);
        v = __builtin_fmaf(v, t, 0.08161342144012451f);
        v = __builtin_fmaf(v, t, 0.09346522390842438f);
        v = __builtin_fmaf(v, t, 0.09973648935556412f);
        v = __builtin_fmaf(v, t, 0.0997355654835701f);
        const float tail = exp_of(-0.5f * b * b) * (t * v);
        return a < 0.0f ? tail : 1.0f - tail;
    }
    const float b = hold(a, 16.0f);
    return logistic(exp_of(-1.59576912160573071176f * (b + 0.044715f * b * b * b)));
}
__device__ __forceinline__ float act_of(int act, float a) { return a * share(act, a); }

__device__ __forceinline__ void act_slope(int act, float a, float &value, float &slope)
{
    const float p = share(act, a);
    value = a * p;
    if (act == kSilu) {
        const float b = hold(a, 200.0f);
        slope = p * (1.0f + b * logistic(exp_of(b)));
    } else if (act == kGelu) {
        const float b = hold(a, 40.0f);
        slope = p + b * (0.39894228040143267794f * exp_of(-0.5f * b * b));
    } else {
        const float b = hold(a, 16.0f);
        const float rest = logistic(exp_of(1.59576912160573071176f * (b + 0.044715f * b * b * b)));   // 1 - p
        slope = p + b * (p * rest) * (1.59576912160573071176f * (1.0f + 0.134145f * b * b));
    }
}

// A gated block: out = act(gate) * lift, and both before it (pre) if wanted.
template <int DT>
struct GatedEnd {
    static constexpr bool kGated = true, kJoins = true, kStages = true;
    struct Params {
        void *out;
        int64_t ld;
        int kind, act;
        uint16_t *pre;   // null: not wanted
        int64_t ldp;
        int64_t lift;    // columns of pre from the gate to the lift
    };
    typedef float value_t;
    static __device__ __forceinline__ void quad(const Params &e, int row, int col, int N, f32x4 g, f32x4 u)
    {
        f32x4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            v[k] = act_of(e.act, g[k]) * u[k];
        store_quad(row_at(e.out, e.ld, row, e.kind), e.kind, col, N, v);
        if (e.pre) {
            uint16_t *const q = e.pre + (int64_t)row * e.ldp;
            store_quad(q, DT, col, N, g);
            store_quad(q + e.lift, DT, col, N, u);
        }
    }
    template <int BM, int BN, int TM, int TN, int FM, int FN, int WN, class Acc>
    static __device__ __forceinline__ void finish(const TileParams &p, const Params &e, Acc &acc, char *smem, int m0,
                                                  int n0, int wm, int wn, int, int, int lane)
    {
        constexpr int TH = TN / 2, FH = FN / 2;
        char *const sh = smem + (wm * WN + wn) * TM * TH * 2;
        auto store = [&](void *out, int64_t ld, int kind, auto f) {
            store_block<TM, TH, FM, FH>(sh, (uint16_t *)out, ld, kind, p.M, p.N, m0 + wm * TM, n0 + wn * TH, lane,
                                        [&](int i, int j, int, int) { return f(i, j); });
        };
        auto inner = [&](int i, int j) {
            f32x4 v;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                v[k] = act_of(e.act, acc[i][j][k]) * acc[i][j + FH][k];
            return v;
        };
        if (e.pre) {
            store(e.pre, e.ldp, DT, [&](int i, int j) { return acc[i][j]; });
            store(e.pre + e.lift, e.ldp, DT, [&](int i, int j) { return acc[i][j + FH]; });
        }
        if (e.kind != kFp32)
            store(e.out, e.ld, e.kind, inner);
        else
            each_quad<TM, TH, FM, FH>(p.M, p.N, m0, n0, wm, wn, lane, [&](int row, int col, int i, int j) {
                store_quad(row_at(e.out, e.ld, row, e.kind), e.kind, col, p.N, inner(i, j));
            });
    }
};

// Logits of a head: per row and tile the largest and the sum of the exponentials
// relative to it, and the target's logit.
struct StatsEnd {
    static constexpr bool kGated = false, kJoins = false, kStages = true;
    struct Params {
        const int64_t *targets;   // null: none wanted
        float2 *stat;             // [tile of columns][M]
        float *at;                // [M]
    };
    template <int BM, int BN, int TM, int TN, int FM, int FN, int WN, class Acc>
    static __device__ __forceinline__ void finish(const TileParams &p, const Params &e, Acc &acc, char *smem, int m0,
                                                  int n0, int wm, int wn, int tn, int, int lane)
    {
        float2 *const meet_at = (float2 *)smem;   // [BM][WN]
        const bool edge = n0 + BN > p.N;
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const int r = wm * TM + i * 16 + (lane & 15), row = m0 + r, first = n0 + wn * TN + (lane >> 4) * 4;
            // the target's place among this lane's columns (j * 16 + k)
            const int64_t hot = (e.targets && row < p.M ? e.targets[row] : -1) - first;
            const bool mine = hot >= 0 && hot < TN;
            if (__any(mine)) {
#pragma unroll
                for (int j = 0; j < FN; ++j)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (mine && hot == j * 16 + k)
                            e.at[row] = acc[i][j][k];
            }
            if (edge) {
#pragma unroll
                for (int j = 0; j < FN; ++j)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (first + j * 16 + k >= p.N)
                            acc[i][j][k] = -INFINITY;
            }
            float most = -INFINITY;
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    most = fmaxf(most, acc[i][j][k]);
            most = fmaxf(most, __shfl_xor(most, 16));
            most = fmaxf(most, __shfl_xor(most, 32));
            // Relative to the largest.  Times log2 e it is rounded as a logit is, and what that
            // left (`off`) is taken out of the sum again; far from zero that would be more than
            // an exponent, and the difference is taken first.  (A NaN or +inf makes the sum NaN.)
            const float ref = most > -INFINITY ? most : 0.0f;
            float sum = 0.0f;
            if (__any(fabsf(ref) > 0x1p20f)) {
#pragma unroll
                for (int j = 0; j < FN; ++j)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        sum += exp_of(acc[i][j][k] - ref);
            } else {
                const float times = -kLog2e * ref, off = __builtin_fmaf(ref, kLog2e, times);
#pragma unroll
                for (int j = 0; j < FN; ++j)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        sum += __builtin_amdgcn_exp2f(__builtin_fmaf(acc[i][j][k], kLog2e, times));
                sum *= __builtin_amdgcn_exp2f(-off);
            }
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            if (lane < 16)
                meet_at[r * WN + wn] = make_float2(most, sum);
        }
        __syncthreads();
        for (int r = threadIdx.x; r < BM; r += blockDim.x) {
            if (m0 + r >= p.M)
                break;
            float most = -INFINITY, sum = 0.0f;
#pragma unroll
            for (int k = 0; k < WN; ++k)
                most = fmaxf(most, meet_at[r * WN + k].x);
#pragma unroll
            for (int k = 0; k < WN; ++k) {
                const float2 s = meet_at[r * WN + k];
                sum += s.x > -INFINITY || !(s.y == s.y) ? s.y * exp_of(s.x - most) : 0.0f;
            }
            e.stat[(int64_t)tn * p.M + m0 + r] = make_float2(most, sum);
        }
    }
};

// Slopes between the products of a gradient are rounded to 16 bits, as many as
// the products' results are: over many rows the roundings of both add up like
// independent ones.  Few rows, where one slope may decide a whole result, are
// kept in two parts (the rounded value, and what the rounding left), which cost
// nothing beside the weights that are read for them.
template <int DT>
__device__ __forceinline__ float left_of(float v)
{
    const float r = v - to_float<DT>(from_float<DT>(v));
    return fabsf(r) < INFINITY ? r : 0.0f;   // (of an infinity or a NaN the first part says it all)
}

// What the gradient of a head's log probabilities takes of each row.
struct HeadRows {
    const int64_t *targets;
    const float *lse, *d_logprob, *d_lse;   // d_logprob, d_lse: null: zero
    int64_t V;

    // Those from row r on.
    HeadRows from(int64_t r) const
    {
        return {targets ? targets + r : nullptr, lse ? lse + r : nullptr, d_logprob ? d_logprob + r : nullptr,
                d_lse ? d_lse + r : nullptr, V};
    }
    // The factors of the target's place and of p (minus d_logprob plus d_lse), and
    // whether the row takes part: one of nothing but -inf does not, nor does one without
    // factors, whatever its lse.
    __device__ __forceinline__ bool factors(int64_t row, int64_t &target, float &dl, float &dp) const
    {
        target = d_logprob ? targets[row] : -1;
        dl = target < 0 ? 0.0f : d_logprob[row];
        if (target >= V)
            dl = NAN;
        dp = (d_lse ? d_lse[row] : 0.0f) - dl;
        return !(lse[row] == -INFINITY || (dl == 0.0f && dp == 0.0f));
    }
    // Bits of the largest of the finite factors.
    __device__ __forceinline__ uint32_t size(int64_t row) const
    {
        const uint32_t a = d_logprob && targets[row] >= 0 ? __builtin_bit_cast(uint32_t, d_logprob[row]) & 0x7fffffffu : 0u;
        const uint32_t b = d_lse ? __builtin_bit_cast(uint32_t, d_lse[row]) & 0x7fffffffu : 0u;
        return max(a < 0x7f800000u ? a : 0u, b < 0x7f800000u ? b : 0u);
    }
};

// The gradient in a head's logits, d_logprob (hot - p) + d_lse p, as the operand
// of the products that follow, times a factor that takes the largest |d_logprob| or
// |d_lse| to 1 (binary16: 2^14, since p / rows would fall below its smallest numbers;
// a slope is at most twice that): with equal d_logprob, as of a mean, the slope of a
// token that the model gives little is then 1, not a rounded 1 / rows that is off by
// as much in every row.
template <int DT>
struct SlopeEnd {
    static constexpr bool kGated = false, kJoins = false, kStages = false;
    struct Params {
        HeadRows of;
        const float *scale;
        const float *raise;                     // binary16: of each row
        uint16_t *out, *rest;                   // rest: of two parts the second; null: one part
        int64_t ld;     // a multiple of 8; columns up to a multiple of 8 are written
        int64_t first;  // the target of column 0
    };
    template <int BM, int BN, int TM, int TN, int FM, int FN, int WN, class Acc>
    static __device__ __forceinline__ void finish(const TileParams &p, const Params &e, Acc &acc, char *smem, int m0,
                                                  int n0, int wm, int wn, int, int, int lane)
    {
        const float scale = *e.scale;
        const int padded = (p.N + 7) / 8 * 8;
        const bool edge = n0 + BN > p.N;
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            __builtin_amdgcn_sched_barrier(0);   // (rows one after another: the registers are full)
            const int row = min(m0 + wm * TM + i * 16 + (lane & 15), p.M - 1);
            int64_t target;
            float dl, dp;
            const bool empty = !e.of.factors(row, target, dl, dp);
            const float lse = e.of.lse[row];
            // the target's place among this lane's columns (j * 16 + k)
            const int first = n0 + wn * TN + (lane >> 4) * 4;
            const int64_t hot = target - e.first - first;
            const bool mine = hot >= 0 && hot < TN && !empty;
            float dps = empty ? 0.0f : dp * scale, dls = dl * scale;
            if constexpr (DT == kFp16) {
                dps *= e.raise[row];
                dls *= e.raise[row];
            }
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                const int col = first + j * 16;
                f32x4 v;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    v[k] = empty ? 0.0f : exp_of(acc[i][j][k] - lse) * dps;
                if (mine) {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        v[k] += hot == j * 16 + k ? dls : 0.0f;
                }
                if (edge) {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        v[k] = col + k < p.N ? v[k] : 0.0f;
                }
                acc[i][j] = v;
            }
        }
        auto store = [&](uint16_t *out, auto f) {
            store_block<TM, TN, FM, FN>(smem + (wm * WN + wn) * TM * TN * 2, out, e.ld, DT, p.M, padded, m0 + wm * TM,
                                        n0 + wn * TN, lane, [&](int i, int j, int, int) { return f(acc[i][j]); });
        };
        store(e.out, [](f32x4 v) { return v; });
        if (e.rest)
            store(e.rest, [](f32x4 v) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float x = v[k];
                    asm("" : "+v"(x));   // (rounded again rather than kept from the first part)
                    v[k] = left_of<DT>(x);
                }
                return v;
            });
    }
};

// ---------------------------------------------------------------------------
// around the products
// ---------------------------------------------------------------------------

// The parts of sums split over k, and the end of the product: four columns a
// thread, `quads` of them a row.
template <class End>
__global__ void __launch_bounds__(256) join_parts(const char *part, int split, int M, int N, int ld, int64_t quads,
                                                  typename End::Params e)
{
    typedef typename End::value_t value_t;
    typedef value_t quad_t __attribute__((ext_vector_type(4)));
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int row = (int)(at / quads), col = (int)(at % quads) * 4;
    if (row >= M)
        return;
    quad_t s[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
    for (int k = 0; k < split; ++k) {
        const char *const q = part + (((int64_t)k * M + row) * ld + col) * 4;
        s[0] += *(const quad_t *)q;
        if constexpr (End::kGated)
            s[1] += *(const quad_t *)(q + ld / 2 * 4);
    }
    End::quad(e, row, col, N, s[0], s[1]);
}

// Copies of matrices whose rows are not whole 16-byte chunks at such addresses: rows
// of `bytes` bytes, at any alignment, to rows of `chunks` x 16, zeros after the
// end, `times` one after another.  Four rows a workgroup, 64 lanes along each.
// Up to two matrices a launch (for a few megabytes a launch takes as long as
// the copy).  `part`: rows that take none in a head's gradient are zeros.
struct CopyParams {
    struct {
        const char *from;
        char *to;
        int64_t ld, bytes, rows, chunks, blocks;
        int times;
        bool part;
    } m[2];
    HeadRows of;
};
__device__ __forceinline__ void copy_block(const CopyParams &p, int64_t block)
{
    const bool second = block >= p.m[0].blocks;
    const auto &m = p.m[second];
    const int64_t row = (block - (second ? p.m[0].blocks : 0)) * 4 + (threadIdx.x >> 6);
    if (row >= m.rows)
        return;
    const char *const from = m.from + row * m.ld;
    int64_t target;
    float dl, dp;
    const bool none = m.part && !p.of.factors(row, target, dl, dp);
    for (int64_t c = threadIdx.x & 63; c < m.chunks; c += 64) {
        const u32x4 v = none                    ? u32x4{0, 0, 0, 0}
                        : c * 16 + 16 <= m.bytes ? sixteen<true>(from + c * 16)
                                                 : load16_end(from, c * 16, m.bytes);
        for (int k = 0; k < m.times; ++k)
            *(u32x4 *)(m.to + ((k * m.rows + row) * m.chunks + c) * 16) = v;
    }
}
__global__ void __launch_bounds__(256) copy_rows(CopyParams p) { copy_block(p, blockIdx.x); }

// Per row of K values: scale = max |x| * (1 / 127) (at least 2^-126), q = x / scale
// rounded to the nearest whole number, ties to even.  A row that holds a NaN or
// an infinity: scale NaN, q = 0.  One workgroup a row, read twice (the second
// time from the caches).  Values up to `padded` are written, zeros past K.
template <int DT>
__device__ __forceinline__ float value_at(const char *x, int64_t k)
{
    if constexpr (DT == kFp32)
        return ((const float *)x)[k];
    else
        return to_float<DT>(((const uint16_t *)x)[k]);
}

template <int DT>
__device__ __forceinline__ void eight(const char *x, int64_t k, int64_t K, float (&v)[8])
{
    if (k + 8 <= K) {
        if constexpr (DT == kFp32) {
            const f32x4 a = load_any<f32x4>(x + k * 4), b = load_any<f32x4>(x + k * 4 + 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[j] = a[j];
                v[j + 4] = b[j];
            }
        } else {
            const u32x4 a = load_any<u32x4>(x + k * 2);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[2 * j] = to_float<DT>((uint16_t)(a[j] & 0xffffu));
                v[2 * j + 1] = to_float<DT>((uint16_t)(a[j] >> 16));
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            v[j] = k + j < K ? value_at<DT>(x, k + j) : 0.0f;
    }
}

__device__ __forceinline__ uint32_t most_of(uint32_t v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1)
        v = max(v, (uint32_t)__shfl_xor((int)v, d));
    return v;
}

__device__ __forceinline__ float row_scale(uint32_t most)
{
    return most >= 0x7f800000u ? NAN : fmaxf(__builtin_bit_cast(float, most) * (1.0f / 127.0f), 0x1p-126f);
}

// Eight values over `scale`, rounded.  v * (1 / scale) is within 2.3e-5 of the
// quotient in fp32 (three roundings of 127 at most), so that both round alike unless it
// is as near to the middle between two whole numbers; then the quotient itself is
// taken (a division costs as much as all the rest).
__device__ __forceinline__ uint64_t eight_bytes(const float (&v)[8], float scale)
{
    if (!(scale == scale))
        return 0;
    const float inverse = 1.0f / scale;
    float n[8], off = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float r = v[j] * inverse;
        n[j] = rintf(r);
        off = fmaxf(off, fabsf(r - n[j]));
    }
    if (off > 0.5f - 0x1p-15f)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            n[j] = rintf(v[j] / scale);
    uint32_t q[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        q[j / 4] |= ((uint32_t)(int)fminf(fmaxf(n[j], -127.0f), 127.0f) & 0xffu) << (8 * (j & 3));
    return q[0] | (uint64_t)q[1] << 32;
}

// HELD: rows of up to kHeld values, which stay in registers between the passes.  4096
// rows of 4096 bfloat16 values 12.4 us (4.1 TB/s; with a division for each value and the
// row read twice 17).
constexpr int kHeld = 256 * 8 * 4;
template <int DT, bool HELD>
__global__ void __launch_bounds__(256) scale_rows(const char *x, int64_t ldx, int64_t K, int8_t *q, int64_t ldq,
                                                  int64_t padded, float *scales)
{
    __shared__ uint32_t share_most[4];
    const int64_t row = blockIdx.x;
    const char *const r = x + row * ldx * (DT == kFp32 ? 4 : 2);
    float held[4][8];
    uint32_t most = 0;
    auto look = [&](float (&v)[8], int64_t k) {
        eight<DT>(r, k, K, v);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            most = max(most, __builtin_bit_cast(uint32_t, v[j]) & 0x7fffffffu);
    };
    if constexpr (HELD) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (threadIdx.x * 8 + i * 2048 < K)
                look(held[i], threadIdx.x * 8 + i * 2048);
    } else {
        for (int64_t k = threadIdx.x * 8; k < K; k += 2048)
            look(held[0], k);
    }
    most = most_of(most);
    if ((threadIdx.x & 63) == 0)
        share_most[threadIdx.x >> 6] = most;
    __syncthreads();
    most = max(max(share_most[0], share_most[1]), max(share_most[2], share_most[3]));
    const float scale = row_scale(most);
    if (threadIdx.x == 0)
        scales[row] = scale;
    auto write = [&](const float (&v)[8], int64_t k) {
        const uint64_t b = eight_bytes(v, scale);
        int8_t *const to = q + row * ldq + k;
        if (k + 8 <= padded) {
            store_any<uint64_t>(to, b);
        } else {
#pragma unroll
            for (int j = 0; j < 7; ++j)
                if (k + j < padded)
                    to[j] = (int8_t)(b >> (8 * j));
        }
    };
    if constexpr (HELD) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t k = threadIdx.x * 8 + i * 2048;
            if (k < padded) {
                if (k >= K)
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        held[i][j] = 0.0f;
                write(held[i], k);
            }
        }
    } else {
        for (int64_t k = threadIdx.x * 8; k < padded; k += 2048) {
            eight<DT>(r, k, K, held[0]);
            write(held[0], k);
        }
    }
}

// A power of two that takes the finite value with bits `most` to 2^14 .. 2^15.
__device__ __forceinline__ float lift_of(uint32_t most)
{
    const int e = (int)(most >> 23) - 127;   // (a subnormal one counts as 2^-127)
    return most == 0 ? 1.0f : __builtin_ldexpf(1.0f, min(max(14 - e, -126), 126));
}

// The first workgroup: scales[0] takes the largest finite |d_logprob| (where there
// is a target) or |d_lse| to `to`, scales[1] is its inverse.  The next `copy_blocks`:
// copies of what the products read.  Those after them (binary16), a wave a row: the
// powers of two by which rows are raised, and the copies of x that the weights' gradient
// multiplies, zeros where a row takes no part.  Each finds the largest for itself, while
// the first does: a launch of their own took 5 us.
__global__ void __launch_bounds__(256) slope_scale(CopyParams copies, int copy_blocks, RaisedCopy x, HeadRows of, int64_t rows,
                                                   float to, float *scales, float *raise)
{
    if (blockIdx.x > 0 && blockIdx.x <= copy_blocks)
        return copy_block(copies, blockIdx.x - 1);
    __shared__ uint32_t share_most[4];
    uint32_t most = 0;
#pragma unroll 8
    for (int64_t r = threadIdx.x; r < rows; r += 256)
        most = max(most, of.size(r));
    most = most_of(most);
    if ((threadIdx.x & 63) == 0)
        share_most[threadIdx.x >> 6] = most;
    __syncthreads();
    most = max(max(share_most[0], share_most[1]), max(share_most[2], share_most[3]));
    if (blockIdx.x == 0) {
        if (threadIdx.x == 0) {
            // (a smaller factor for what is next to fp32's ends, where it or its inverse would be no normal number)
            const float m = fminf(fmaxf(__builtin_bit_cast(float, most), to * 0x1p-126f), to * 0x1p126f);
            scales[0] = most == 0 ? 1.0f : to / m;
            scales[1] = most == 0 ? 1.0f : m / to;
        }
        return;
    }
    const int lane = threadIdx.x & 63;
    const int64_t before = 1 + (int64_t)copy_blocks;
    for (int64_t row = (blockIdx.x - before) * 4 + (threadIdx.x >> 6); row < rows; row += (gridDim.x - before) * 4) {
        int64_t target;
        float dl, dp;
        const bool part = of.factors(row, target, dl, dp);
        const int n = raise_of(of.size(row), most);
        if (lane == 0)
            raise[row] = power_of_two(n);
        if (x.to)
            copy_lowered(x, row, part ? n : -1, lane);
    }
}

// The gradient in a gated block's projections, [d lift act'(gate) | d act(gate)],
// as the operand of the products that follow.  In binary16 times a power of two
// that takes the largest of them to 2^14, rows of small ones raised: a first launch (MOST)
// finds the largest of each block and unit.
// Eight columns a thread, the padding after 2 I zeros.  HBM is the bound: 4096 x 14336
// bfloat16 100 us, 5.9 TB/s, binary16 128 and 140 us with the copy of 4096 x 4096 values of
// x; for a megabyte or two the launch and a chain of latencies.
struct GatedSlopeParams {
    const uint16_t *pre, *d;
    int64_t ldp, ldd;
    uint16_t *out;   // M x ld, ld a multiple of 8 of at least 2 I
    int64_t rest;    // values from there to the second of two parts; 0: one part
    int64_t ld;
    int I, act;
    int chunks;       // of 8 in I columns
    int64_t rows, units;   // rows times 64 chunks
    uint32_t *most;   // bits of each block's largest (binary16)
    int blocks;       // that find them
    uint32_t *unit_most;   // and of each unit's
    int copies;       // the first blocks copy what the products read
    float *inverse;   // of the power of two
    float *raise;     // of each row
    RaisedCopy x;     // binary16, by the last launch
};
constexpr int kMostBlocks = 1020;

template <int DT>
__device__ __forceinline__ void store_eight(uint16_t *to, int n, const float (&v)[8])
{
    if (n >= 8) {
        u32x4 b;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            b[j] = from_float<DT>(v[2 * j]) | (uint32_t)from_float<DT>(v[2 * j + 1]) << 16;
        store_any<u32x4>(to, b);
    } else {
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (j < n)
                to[j] = from_float<DT>(v[j]);
    }
}

template <int DT, bool MOST>
__global__ void __launch_bounds__(256) gated_slope(GatedSlopeParams p, CopyParams copies)
{
    constexpr bool kRaised = DT == kFp16 && !MOST;
    const bool copying = blockIdx.x < p.copies;
    if (!kRaised && copying)
        return copy_block(copies, blockIdx.x);
    // a wave takes 512 columns of a row at a time
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t groups = (p.chunks + 63) / 64;
    const int64_t block = blockIdx.x - p.copies, blocks = gridDim.x - p.copies;
    // (where rows are raised a wave's units are neighbours, of a row or two)
    const int64_t each = kRaised ? (p.units + blocks * 4 - 1) / (blocks * 4) : 1;
    auto row_of = [&](int64_t unit) -> int64_t { return unit < ((int64_t)1 << 32) ? (uint32_t)unit / groups : unit / groups; };
    // the largest of a row, from its units'
    auto row_most = [&](int64_t row) {
        uint32_t v = 0;
        for (uint32_t g = lane; g < groups; g += 64)
            v = max(v, p.unit_most[row * groups + g]);
        return (uint32_t)__builtin_amdgcn_readfirstlane(most_of(v));
    };
    __shared__ uint32_t share_most[4];
    uint32_t most = 0, row_size = 0;   // row_size: of the first row
    float s = 1.0f;
    if constexpr (kRaised) {
        for (int b = threadIdx.x; b < p.blocks; b += 256)
            most = max(most, p.most[b]);
        const int64_t row = copying ? (int64_t)blockIdx.x * 4 + wave : row_of((block * 4 + wave) * each);
        if (row < (copying ? p.x.rows : p.rows))
            row_size = row_most(row);
        most = most_of(most);
        if (lane == 0)
            share_most[wave] = most;
        __syncthreads();
        most = __builtin_amdgcn_readfirstlane(max(max(share_most[0], share_most[1]), max(share_most[2], share_most[3])));
        s = lift_of(most);
        if (blockIdx.x == p.copies && threadIdx.x == 0)
            *p.inverse = 1.0f / s;
        if (copying) {
            for (int64_t row = (int64_t)blockIdx.x * 4 + wave; row < p.x.rows; row += (int64_t)p.copies * 4) {
                copy_lowered(p.x, row, raise_of(row_size, most), lane);
                if (row + (int64_t)p.copies * 4 < p.x.rows)
                    row_size = row_most(row + (int64_t)p.copies * 4);
            }
            return;
        }
    }
    const int64_t first = (block * 4 + wave) * each;
    for (int64_t unit = first; unit < (kRaised ? min(first + each, p.units) : p.units); unit += kRaised ? 1 : blocks * 4) {
        const int64_t row = row_of(unit);
        const int group = (int)(unit - row * groups), col = (group * 64 + lane) * 8;
        float raise = 1.0f;
        if constexpr (kRaised) {
            if (group == 0 && unit > first)
                row_size = row_most(row);
            raise = power_of_two(raise_of(row_size, most));
            if (group == 0 && lane == 0)
                p.raise[row] = raise;
        }
        const bool inside = col < p.I;
        float g[8], u[8], d[8], dg[8], du[8];
        const uint16_t *const pre = p.pre + row * p.ldp;
        if (inside) {
            eight<DT>((const char *)pre, col, p.I, g);
            eight<DT>((const char *)(pre + p.I), col, p.I, u);
            eight<DT>((const char *)(p.d + row * p.ldd), col, p.I, d);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float value, slope;
                act_slope(p.act, g[j], value, slope);
                dg[j] = d[j] * u[j] * slope * s;
                du[j] = d[j] * value * s;
                if constexpr (kRaised) {
                    dg[j] *= raise;
                    du[j] *= raise;
                }
            }
        }
        if constexpr (MOST) {
            uint32_t here = 0;
            if (inside) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint32_t a = __builtin_bit_cast(uint32_t, dg[j]) & 0x7fffffffu;
                    const uint32_t b = __builtin_bit_cast(uint32_t, du[j]) & 0x7fffffffu;
                    here = max(here, max(a < 0x7f800000u ? a : 0u, b < 0x7f800000u ? b : 0u));
                }
            }
            here = most_of(here);
            if (lane == 0)
                p.unit_most[unit] = here;
            most = max(most, here);
        } else if (inside) {
            const int n = p.I - col;
            auto store = [&](uint16_t *out) {
                store_eight<DT>(out + col, n, dg);
                store_eight<DT>(out + p.I + col, n, du);
                if (n <= 8)
                    for (int c = 2 * p.I; c < (2 * p.I + 7) / 8 * 8; ++c)
                        out[c] = 0;
            };
            uint16_t *const out = p.out + row * p.ld;
            store(out);
            if (p.rest) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    dg[j] = left_of<DT>(dg[j]);
                    du[j] = left_of<DT>(du[j]);
                }
                store(out + p.rest);
            }
        }
    }
    if constexpr (MOST) {
        // (atomics on one address take 15 ns each: the blocks of the next launch look at
        // all the places instead)
        if (lane == 0)
            share_most[wave] = most;
        __syncthreads();
        if (threadIdx.x == 0)
            p.most[block] = max(max(share_most[0], share_most[1]), max(share_most[2], share_most[3]));
    }
}

// Log probabilities from the tiles' statistics: kJoinRows rows a workgroup, each by
// 64 threads.  (16 rows and 16 threads took 10 us for 77 rows of 391 tiles.)
constexpr int kJoinRows = 4, kJoinThreads = 256 / kJoinRows;
__global__ void __launch_bounds__(256) head_join(const float2 *stat, int tiles, int64_t rows, const float *at,
                                                 const int64_t *targets, int64_t V, float *lse, float *logprob)
{
    __shared__ float2 part[kJoinRows][kJoinThreads + 1];
    const int r = threadIdx.x % kJoinRows, t0 = threadIdx.x / kJoinRows;
    const int64_t row = (int64_t)blockIdx.x * kJoinRows + r;
    float most = -INFINITY, sum = 0.0f;
    auto add = [&](float m, float s) {
        const float both = fmaxf(most, m);
        // (a part of nothing but -inf has no sum; one with a NaN or +inf has a NaN)
        const float a = most > -INFINITY || !(sum == sum) ? sum * exp_of(most - both) : 0.0f;
        const float b = m > -INFINITY || !(s == s) ? s * exp_of(m - both) : 0.0f;
        most = both;
        sum = a + b;
    };
    // (eight loads at a time: the tiles are few, and their latency is the time)
    if (row < rows)
        for (int t = t0; t < tiles; t += 8 * kJoinThreads) {
            float2 s[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int at_t = t + k * kJoinThreads;
                s[k] = at_t < tiles ? stat[(int64_t)at_t * rows + row] : make_float2(-INFINITY, 0.0f);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k)
                add(s[k].x, s[k].y);
        }
    part[r][t0] = make_float2(most, sum);
    __syncthreads();
    // (in halves, as a tree)
    for (int n = kJoinThreads / 2; n; n /= 2) {
        if (t0 < n) {
            add(part[r][t0 + n].x, part[r][t0 + n].y);
            part[r][t0] = make_float2(most, sum);
        }
        __syncthreads();
    }
    if (t0 > 0 || row >= rows)
        return;
    const bool bad = !(sum == sum), empty = most == -INFINITY;
    const float log_sum = logf(sum);
    if (lse)
        lse[row] = bad ? NAN : empty ? -INFINITY : most + log_sum;
    if (logprob) {
        const int64_t t = targets[row];
        logprob[row] = t < 0 ? 0.0f : t >= V || bad ? NAN : empty ? -INFINITY : (at[row] - most) - log_sum;
    }
}

}  // namespace xfused_dev
