// A mixture-of-experts layer for a few tokens, from the router's scores to the
// weighted sum of its experts, in two launches.
//
//     chosen(t) = the `top` experts of the largest scores (equal ones: the lower index first)
//     w[t][j]   = exp(score of choice j - largest) / (the same summed over the choices, or over all experts)
//     h[t][j]   = silu(gate_e x_t) * (up_e x_t),  e = choice j of t,  silu(a) = a / (1 + exp(-a))
//     y[t]      = sum over j of w[t][j] down_e h[t][j]
//
// What bounds it: the bytes of the chosen experts' weights, each read once
// however many tokens chose it.  So the work is laid out by expert, not by
// token: a slot is one chosen expert with the tokens that chose it (up to 64,
// in blocks of the 16 rows of a matrix instruction).  There are
// min(tokens * top, experts) slots: with few tokens slot s is choice s % top of
// token s / top, left empty when an earlier token has chosen that expert too;
// with many, slot s is expert s, left empty when nobody has.
//
// First launch (route_up): one workgroup a slot and 16 or 64 of the inner
// columns.  It works out its slot from the scores by itself (a comparison of
// every score with the expert's own, per token, which costs less than a
// launch), then forms its gate and up columns for the slot's tokens, 16 of
// each a wave, and writes h.  With up to 16 tokens its waves split the hidden
// dimension, with more they take columns and share x through LDS.  The first
// workgroup of a slot also writes the slot's tokens and weights.
// Second launch (down_sum): the slots' inner dimensions, one after the other in
// units of 64, are cut into even ranges; a range forms its part of 16 columns
// of y a wave, for every token, in LDS.  With one or two tokens the waves of a
// workgroup take a range each, else they take the same range and 16 columns
// each, sharing h through LDS (each workgroup reads all of h, which with 16
// columns would be more than the weights).  The ranges' sums are added in
// ascending order, by whichever workgroup is the last to finish: no float
// atomics, one order of summation.
//
// In both, a wave brings its rows of x or h in through LDS, the pieces of a
// unit arranged so that the matrix operand is one conflict-free 16-byte read,
// and keeps two units of weights on their way.  The loops' loads are
// unconditional (past the end they repeat the last unit's): loads return in
// order, and one that may not have been issued turns the waits behind it into
// waits for all.
//
// The second product needs h on the matrix units, which take 16 bits.  Rounded
// to 16 bits h would lose more than the rounding of y does, so it is written as
// 16-bit parts, and multiplied as that many products (the matrix units are
// idle most of the time): three, which hold its 24 bits, or for binary16 with a
// y of 16 bits two, which hold 23 (its y has 11; with three of them 64 tokens, 2
// of 8 experts of 4096 x 14336 take 590 us instead of 561).
//   bfloat16: h = a + b + c, each part the rounding of what the ones before leave.
//   binary16, whose range is short: h = 2^e (a + 2^-11 (b + 2^-11 c)), with e such
//   that the largest h of a token's 16 columns has an a between 2^14 and 2^15.
//   The second launch brings the four e of a unit to their largest, E, as it
//   puts the parts in LDS, and multiplies the unit's sums by 2^E.  So h may have
//   any size that fp32 holds.  Brought to E, the least that a resolves is 2^-39
//   of the largest of the 64 columns, and h keeps its bits down to 2^-25 of that.
//
// Measured, first and second launch: 64 tokens, 2 of 8 experts of 4096 x 14336
// (hidden x inner, every expert read) 342 us at 5.6 TB/s and 201 us at 5.0 TB/s;
// 16 tokens, 6 of 64 of 2048 x 1408 111 us at 5.4 TB/s and 64 us at 4.8 TB/s.
// With one token the chain of launch, routing, first loads and joins is as long
// as the reading: 8 of 128 of 2048 x 768 17 us for 50 MB and 12 us for 25 MB.
#pragma once

#include <type_traits>

#include "decode_device.hpp"

namespace xexperts_dev {

using namespace xdecode_dev;

constexpr int kMaxTokens = 64;    // tokens of a launch
constexpr int kMaxExperts = 1024;
constexpr int kMaxTop = 32;
// k per unit of a wave.  (128 in the first product: 16 tokens, 6 of 64 experts
// of 2048 x 1408 212 us against 190: the registers of two units then leave two
// workgroups a CU.)
constexpr int kUpUnit = 64, kDownUnit = 64;
constexpr int kPad = kDownUnit;   // inner columns of h are padded to this
constexpr int kMaxParts = 32;     // ranges of the second product that workgroups take

struct ExpertsParams {
    const uint16_t *x;
    const float *scores;
    const uint16_t *up, *down;
    void *y;
    int64_t ldx, lds, ldu, su, ldd, sd, ldy;  // elements
    int T, E, top, H, I, Ip;                  // Ip: I rounded up to kPad
    int slots;
    int renormalize, out16;
    int parts;
    int *expert;      // [slots]: the slot's expert, -1: empty
    int *count;       // [slots]: its tokens
    uint16_t *pair;   // [slots][kMaxTokens]: token * top + choice
    float *weight;    // [T * top]: exp(score - largest), over the whole softmax's sum without renormalize
    uint16_t *h;      // [parts of h][T * top][Ip]
    int8_t *scale;    // [T * top][Ip / 16]: e of 16 columns of h (binary16)
    float *part;      // [parts][T][H rounded up to whole workgroups], where parts > 1
    int *done;        // [workgroups of a range], zero between launches
};

// Where 8 k of a row (piece kc of the row's unit, 8 kc .. + 7) lie in LDS, for
// R rows: lane group kc % 4 of product kc / 4.  16 rows are swizzled so that
// neither the pieces of a row nor the rows of a piece share a bank.
template <int R>
__device__ __forceinline__ int place(int row, int kc)
{
    constexpr int MT = (R + 15) / 16;
    return R < 16 ? (kc * R + row) * 16
                  : ((kc >> 2) * MT + (row >> 4)) * 1024 + (kc & 3) * 256 + ((row ^ kc) & 15) * 16;
}
template <int R>
constexpr int unit_bytes(int unit)
{
    return R < 16 ? unit * R * 2 : (R + 15) / 16 * 16 * unit * 2;
}

// A score as a whole number in the same order: NaN above all, the two zeros
// alike.
__device__ __forceinline__ uint32_t order_of(float v)
{
    if (v != v)
        return 0xffffffffu;
    const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.0f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}

// The parts of h (see above), of binary16 once it is divided by 2^e.
template <int DT, int PL>
__device__ __forceinline__ void split_parts(float v, uint16_t (&part)[PL])
{
    constexpr float step = DT == 0 ? 1.0f : 0x1p11f;
    float r = v;
#pragma unroll
    for (int i = 0; i < PL; ++i) {
        part[i] = from_float<DT>(r);
        const float got = to_float<DT>(part[i]);
        r = (r - got) * step;
        if (!(__builtin_fabsf(got) < __builtin_inff()))   // nothing is left of what has overflowed
            r = 0.0f;
    }
}

// 2^n, n from -126 to 127.
__device__ __forceinline__ float power2(int n) { return __builtin_bit_cast(float, (127 + n) << 23); }

// e of the 16 lanes' values (a row of lanes), -112 .. 114.  (An infinity or a
// NaN among them leaves nothing of the others, nor do they count.)
__device__ __forceinline__ int row_exponent(float v)
{
    int m = __builtin_bit_cast(int, v) & 0x7fffffff;
    m = max(m, __builtin_amdgcn_update_dpp(0, m, 0x128, 0xf, 0xf, false));   // row_ror 8
    m = max(m, __builtin_amdgcn_update_dpp(0, m, 0x124, 0xf, 0xf, false));   // row_ror 4
    m = max(m, __builtin_amdgcn_update_dpp(0, m, 0x122, 0xf, 0xf, false));   // row_ror 2
    m = max(m, __builtin_amdgcn_update_dpp(0, m, 0x121, 0xf, 0xf, false));   // row_ror 1
    return max((m >> 23) - 141, -112);
}

// Eight binary16 values times 2^-d, d >= 0.
__device__ __forceinline__ u32x4 scale_down(u32x4 v, int d)
{
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    auto times = [&](int n) {
        const _Float16 f = (_Float16)power2(-n);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t two = v[i];
            v[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, two) * f16x2{f, f});
        }
    };
    times(min(d, 24));   // 2^-24 is the least that binary16 holds
    if (d > 24)
        times(min(d - 24, 100));
    return v;
}

// exp of a score against the largest; a score of -inf has no weight.
__device__ __forceinline__ float score_exp(float v, float largest)
{
    return v == -__builtin_inff() ? 0.0f : expf(v - largest);
}

// 16 values of a row, kept as they were loaded: at an address that is 2 mod 4 the
// 16-byte loads begin a value earlier, in the same four bytes, and `end` is the
// last value.  (16-byte loads at 2 mod 4 take more than twice as long as at 0 mod
// 4.  25 tokens, 1 of 8 experts of 1855 x 3961: 175 us with them, 124 so; 7 tokens,
// 3 of 13 of 1001 x 777 36 and 28.)
struct Odd16 {
    u32x4 v[2];
    uint32_t end;
    __device__ __forceinline__ void load(const uint16_t *p)
    {
        const uint16_t *const from = p - ((uintptr_t)p >> 1 & 1);
        v[0] = load_any<u32x4>(from);
        v[1] = load_any<u32x4>(from + 8);
        end = p[15];
    }
    // moved into place, for an address that is `mis` (0 or 2) mod 4
    __device__ __forceinline__ void align(uint32_t mis)
    {
        const uint32_t d[9] = {v[0][0], v[0][1], v[0][2], v[0][3], v[1][0], v[1][1], v[1][2], v[1][3], end};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i >> 2][i & 3] = __builtin_amdgcn_alignbyte(d[i + 1], d[i], mis);
    }
    // moved down by n (0 .. 16) values, zeros entering at the top
    __device__ __forceinline__ void drop(int n)
    {
        uint32_t d[17] = {v[0][0], v[0][1], v[0][2], v[0][3], v[1][0], v[1][1], v[1][2], v[1][3]};
#pragma unroll
        for (int by = 8; by >= 1; by /= 2)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                d[i] = n >> 1 & by ? d[i + by] : d[i];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i >> 2][i & 3] = __builtin_amdgcn_alignbyte(d[i + 1], d[i], 2 * (n & 1));
    }
};

// The piece of a row (8 k) that product d takes from lane group g, as d 4 + g:
// with Odd16 a lane group holds 16 k in a row.
template <bool ODD>
__device__ __forceinline__ int piece_at(int kc)
{
    return ODD ? (kc & 1) * 4 + (kc >> 1) : kc;
}

__device__ __forceinline__ void sync_lds()
{
    __builtin_amdgcn_s_waitcnt(15 | (3 << 14) | (7 << 4));  // lgkmcnt(0)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// R: rows of a slot that the launch provides for (2, or a multiple of 16); PL:
// parts of h; WN waves take 16 columns each, or (WN == 1) WK waves a range of k
// each.  ODD: rows of weights may begin at addresses that are 2 mod 4.
template <int DT, int R, int PL, int WN, int WK, bool ODD>
__global__ void __launch_bounds__(64 * WN * WK, R <= 16 ? 4 : 3)
route_up(ExpertsParams p)
{
    static_assert(WN == 1 || WK == 1, "a barrier is the whole workgroup's");
    constexpr int MTS = (R + 15) / 16, THREADS = 64 * WN * WK, BUFS = WN == 1 ? 1 : 2;
    __shared__ __attribute__((aligned(16))) union {
        uint32_t key[kMaxExperts];
        char x[WK][BUFS][unit_bytes<R>(kUpUnit)];
        float red[WK > 1 ? WK * MTS * 512 : 1];
    } sh;
    __shared__ int sh_expert, sh_count, sh_first;
    __shared__ uint8_t sh_rank[kMaxTokens];
    __shared__ uint16_t sh_pair[kMaxTokens];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wn = wave % WN, wk = wave / WN;
    const int slot = blockIdx.y, i0 = 16 * (WN * blockIdx.x + wn);

    // the slot's expert: the one of rank j among its token's scores
    const bool by_choice = p.slots < p.E;
    const int t0 = by_choice ? slot / p.top : 0;
    if (by_choice) {
        const int j = slot - t0 * p.top;
        const float *const row = p.scores + t0 * p.lds;
        for (int e = tid; e < p.E; e += THREADS)
            sh.key[e] = order_of(row[e]);
        __syncthreads();
        int per = 32;   // lanes an expert
        while (per > 1 && THREADS / per < p.E)
            per /= 2;
        for (int e0 = 0; e0 < p.E; e0 += THREADS / per) {
            const int e = e0 + tid / per;
            const uint32_t mine = sh.key[min(e, p.E - 1)];
            int rank = 0;
            for (int o = tid & (per - 1); o < p.E; o += per)
                rank += sh.key[o] > mine || (sh.key[o] == mine && o < e);
            for (int d = per / 2; d >= 1; d /= 2)
                rank += __shfl_xor(rank, d, 64);
            if (rank == j && e < p.E)
                sh_expert = e;
        }
        __syncthreads();
    }
    const int expert = __builtin_amdgcn_readfirstlane(by_choice ? sh_expert : slot);

    // its rank among each token's scores, `per` lanes a token, and, for the
    // first workgroup of a slot, its weight
    auto ranks = [&](bool weigh) {
        int per = 64;
        while (per > THREADS / kMaxTokens && THREADS / per < p.T)
            per /= 2;
        const int tok = tid / per, sub = tid & (per - 1);
        const float *const row = p.scores + (int64_t)min(tok, p.T - 1) * p.lds;
        const float own = row[expert];
        const uint32_t mine = order_of(own);
        int rank = 0;
        float largest = -__builtin_inff();
#pragma unroll 4
        for (int o = sub; o < p.E; o += per) {
            const float v = row[o];
            const uint32_t k = order_of(v);
            rank += k > mine || (k == mine && o < expert);
            largest = fmaxf(largest, v);
        }
        for (int d = per / 2; d >= 1; d /= 2) {
            rank += __shfl_xor(rank, d, 64);
            largest = fmaxf(largest, __shfl_xor(largest, d, 64));
        }
        const bool chosen = rank < p.top && tok < p.T;
        if (tok < kMaxTokens && sub == 0)
            sh_rank[tok] = chosen ? (uint8_t)rank : 255;
        if (weigh) {
            float w = score_exp(own, largest);
            if (!p.renormalize) {
                float all = 0.0f;
                for (int o = sub; o < p.E; o += per)
                    all += score_exp(row[o], largest);
                for (int d = per / 2; d >= 1; d /= 2)
                    all += __shfl_xor(all, d, 64);
                w = all == 0.0f ? 0.0f : w / all;
            }
            if (chosen && sub == 0)
                p.weight[tok * p.top + rank] = w;
        }
    };
    // (one token's slots hold that token: its weights can wait)
    const bool one = p.T == 1 && by_choice;
    int count = 1;
    if (one) {
        if (tid == 0) {
            sh_pair[0] = (uint16_t)slot;
            if (blockIdx.x == 0) {
                p.expert[slot] = expert;
                p.count[slot] = 1;
                p.pair[slot * kMaxTokens] = (uint16_t)slot;
            }
        }
        __syncthreads();
    } else {
        ranks(blockIdx.x == 0);
        __syncthreads();
        if (wave == 0) {
            const int rank = lane < p.T ? sh_rank[lane] : 255;
            const uint64_t mask = __ballot(rank != 255);
            if (rank != 255)
                sh_pair[__popcll(mask & ((1ull << lane) - 1))] = (uint16_t)(lane * p.top + rank);
            if (lane == 0) {
                sh_count = __popcll(mask);
                sh_first = mask ? __builtin_ctzll(mask) : -1;
            }
        }
        __syncthreads();
        count = __builtin_amdgcn_readfirstlane(sh_count);
        const bool empty = count == 0 || (by_choice && sh_first != t0);
        if (blockIdx.x == 0) {
            if (tid == 0) {
                p.expert[slot] = empty ? -1 : expert;
                p.count[slot] = count;
            }
            if (tid < count)
                p.pair[slot * kMaxTokens + tid] = sh_pair[tid];
        }
        if (empty)
            return;
    }

    const int c = lane & 15, g = lane >> 4;
    const uint16_t *wrow[2];
#pragma unroll
    for (int v = 0; v < 2; ++v)
        wrow[v] = p.up + (int64_t)expert * p.su + (int64_t)(v * p.I + min(i0 + c, p.I - 1)) * p.ldu + (ODD ? 16 : 8) * g;
    const int64_t plane = (int64_t)p.T * p.top * p.Ip;

    // the products for up to RB rows
    auto body = [&]<int RB>() {
        constexpr int MT = (RB + 15) / 16, D = kUpUnit / 32, PR = kUpUnit / 8;   // pieces of 8 k of a row
        constexpr int NP = RB * PR > 64 * WN ? RB * PR / (64 * WN) : 1;
        const uint16_t *xrow[NP];
        int xdst[NP];
#pragma unroll
        for (int q = 0; q < NP; ++q) {
            const int row = (wn * 64 + lane) / PR + 64 / PR * WN * q, kc = lane % PR;
            const int r = min(row, RB - 1);
            xrow[q] = p.x + (int64_t)(sh_pair[min(r, count - 1)] / p.top) * p.ldx + 8 * kc;
            xdst[q] = place<RB>(r, piece_at<ODD>(kc));
        }
        f32x4 acc[MT][2];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int v = 0; v < 2; ++v)
                acc[i][v] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        static_assert(D == 2, "pieces of a unit that a lane holds");
        struct Pieces {
            u32x4 v[2];
        };
        std::conditional_t<ODD, Odd16, Pieces> w[2][2];
        u32x4 xr[NP];
        auto store_x = [&](int buf) {
#pragma unroll
            for (int q = 0; q < NP; ++q)
                *(u32x4 *)(sh.x[wk][buf] + xdst[q]) = xr[q];
        };
        auto compute = [&](auto (&from)[2], int buf, bool loaded = true) __attribute__((always_inline)) {
            const char *const xs = sh.x[wk][buf];
            if constexpr (ODD)
#pragma unroll
                for (int v = 0; v < 2; ++v)
                    from[v].align(loaded ? (uint32_t)(uintptr_t)wrow[v] & 2u : 0u);
#pragma unroll
            for (int d = 0; d < D; ++d)
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const u32x4 a = *(const u32x4 *)(xs + place<RB>(RB < 16 ? min(c, RB - 1) : 16 * i + c, 4 * d + g));
#pragma unroll
                    for (int v = 0; v < 2; ++v)
                        acc[i][v] = mfma16<DT>(a, from[v].v[d], acc[i][v]);
                }
        };
        // this wave's whole units
        const int units = p.H / kUpUnit;
        const int u0 = wk * (units / WK) + min(wk, units % WK), mine = units / WK + (wk < units % WK);
        auto load_x = [&](int t) {
            const int k = (u0 + min(t, mine - 1)) * kUpUnit;
#pragma unroll
            for (int q = 0; q < NP; ++q)
                xr[q] = load_any<u32x4>(xrow[q] + k);
        };
        auto load_w = [&](auto (&to)[2], int t) {
            const int k = (u0 + min(t, mine - 1)) * kUpUnit;
#pragma unroll
            for (int v = 0; v < 2; ++v)
                if constexpr (ODD)
                    to[v].load(wrow[v] + k);
                else
#pragma unroll
                    for (int d = 0; d < D; ++d)
                        to[v].v[d] = load_any<u32x4>(wrow[v] + k + 32 * d);
        };
        if (mine > 0) {
            load_x(0);
            load_w(w[0], 0);
            load_w(w[1], 1);
            auto step = [&]<int B>(int t) {
                constexpr int buf = BUFS == 1 ? 0 : B;
                store_x(buf);
                load_x(t + 1);
                if (WN > 1)
                    sync_lds();
                compute(w[B], buf);
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
        // what is left of the rows, by the last range (x is zero past H)
        if (units * kUpUnit < p.H && wk == WK - 1) {
            const int64_t k = (int64_t)units * kUpUnit;
#pragma unroll
            for (int q = 0; q < NP; ++q)
                xr[q] = load16_end(xrow[q] - 8 * (lane % PR), 2 * (k + 8 * (lane % PR)), 2 * (int64_t)p.H);
#pragma unroll
            for (int v = 0; v < 2; ++v)
#pragma unroll
                for (int d = 0; d < D; ++d) {
                    const int at = ODD ? 16 * g : 8 * g, step = ODD ? 8 * d : 32 * d;
                    w[0][v].v[d] = load16_end(wrow[v] - at, 2 * (k + at + step), 2 * (int64_t)p.H);
                }
            if (WN > 1)
                sync_lds();   // (the first buffer may still be read)
            store_x(0);
            if (WN > 1)
                sync_lds();
            compute(w[0], 0, false);
        }
        // h of row m (of the slot) and column col from its two sums, the 16
        // columns of a block side by side
        auto finish = [&](int m, int col, float gate, float lift) {
            uint16_t part[PL];
            const int64_t pair = sh_pair[m];
            float v = col < p.I ? gate / (1.0f + expf(-gate)) * lift : 0.0f;
            if constexpr (DT == 1) {
                const int e = row_exponent(v);
                if (c == 0)
                    p.scale[pair * (p.Ip / 16) + (col >> 4)] = (int8_t)e;
                v *= power2(-e);
            }
            split_parts<DT, PL>(v, part);
            uint16_t *const at = p.h + pair * p.Ip + col;
#pragma unroll
            for (int q = 0; q < PL; ++q)
                at[q * plane] = part[q];
        };
        if constexpr (WK == 1) {
            // (columns up to the padded size: 64 a workgroup)
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (16 * i + 4 * g + r < count)
                        finish(16 * i + 4 * g + r, i0 + c, acc[i][0][r], acc[i][1][r]);
        } else {
            sync_lds();   // (x is done with)
            // the waves' blocks, added in ascending order
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int v = 0; v < 2; ++v)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        sh.red[((wave * MT + i) * 2 + v) * 256 + 64 * r + lane] = acc[i][v][r];
            sync_lds();
            for (int o = tid; o < MT * 256; o += THREADS) {
                const int i = o >> 8, r = o >> 6 & 3, l = o & 63;
                const int m = 16 * i + 4 * (l >> 4) + r, col = i0 + (l & 15);
                if (m >= count)
                    continue;
                float sum[2];
#pragma unroll
                for (int v = 0; v < 2; ++v) {
                    sum[v] = sh.red[(i * 2 + v) * 256 + (o & 255)];
#pragma unroll
                    for (int w = 1; w < WK; ++w)
                        sum[v] += sh.red[((w * MT + i) * 2 + v) * 256 + (o & 255)];
                }
                finish(m, col, sum[0], sum[1]);
                // the last workgroup also clears the padding past its columns
                if (blockIdx.x == gridDim.x - 1)
                    for (int past = col + 16; past < p.Ip; past += 16)
                        finish(m, past, 0.0f, 0.0f);
            }
        }
    };
    if constexpr (R < 16) {
        body.template operator()<R>();
    } else {
        if (count <= 4)
            body.template operator()<4>();
        else if (R == 16 || count <= 16)
            body.template operator()<16>();
        else if (R == 32 || (R > 32 && count <= 32))
            body.template operator()<R < 32 ? R : 32>();
        else
            body.template operator()<R>();
    }
    if (one && blockIdx.x == 0)
        ranks(true);
}

// R, PL: as above.  WN waves take 16 columns each of the same range, or (WN ==
// 1) WK waves a range each.  END: 0 for I a multiple of 8, where a piece of a row
// past I is the row's last one again (h is zero there); 1: rows of any alignment
// and a last unit that ends inside, whose lanes load the row's last 16 and move
// them into place; 2: for I below 16.
//
// LDS beyond the declared arrays: down_sum_lds(pairs, slots) bytes.  (Sized by
// the call and not by its limits: 64 tokens and three parts then leave room for
// two workgroups a CU.  2 of 8 experts of 4096 x 14336 590 us, with one 652.)
__host__ __device__ constexpr int down_sum_lds(int pairs, int slots) { return 6 * pairs + 6 * slots + 2; }

template <int DT, int R, int PL, int WN, int WK, int END>
__global__ void __launch_bounds__(64 * WN * WK, R <= 16 ? 4 : R == 32 ? 2 : 1)
down_sum(ExpertsParams p)
{
    static_assert(WN == 1 || WK == 1, "a barrier is the whole workgroup's");
    constexpr int WAVES = WN * WK, THREADS = 64 * WAVES, TOKENS = R;
    constexpr int BUFS = WN == 1 ? 1 : 2;
    constexpr int HB = unit_bytes<R>(kDownUnit);
    __shared__ __attribute__((aligned(16))) char sh_h[WK][BUFS][PL][HB];
    __shared__ __attribute__((aligned(16))) float sh_scale[DT == 1 ? WK : 1][BUFS][DT == 1 ? (R + 15) / 16 * 16 : 4];
    __shared__ __attribute__((aligned(16))) float acc_all[WAVES][TOKENS * 16];
    __shared__ int sh_used, sh_last;
    extern __shared__ __attribute__((aligned(16))) char sh_more[];
    float *const sh_weight = (float *)sh_more;                     // [T * top]
    uint16_t *const sh_pairs = (uint16_t *)(sh_weight + p.T * p.top);   // the pairs,
    uint16_t *const sh_slot = sh_pairs + p.T * p.top;              // the slots in use, in ascending order,
    uint16_t *const sh_expert = sh_slot + p.slots;                 //   their experts,
    uint16_t *const sh_start = sh_expert + p.slots;                //   where their pairs start
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wn = wave % WN, wk = wave / WN;
    const int nw = 16 * WN * blockIdx.x, n0 = nw + 16 * wn;
    const int c = lane & 15, g = lane >> 4;
    float *const mine = acc_all[wave];
    for (int o = lane; o < TOKENS * 16; o += 64)
        mine[o] = 0.0f;

    // the slots in use and where their pairs go, by the first wave
    if (wave == 0) {
        int used = 0, pairs = 0;
        for (int s0 = 0; s0 < p.slots; s0 += 64) {
            const int s = s0 + lane, at = min(s, p.slots - 1);
            const int expert = p.expert[at], listed = p.count[at];
            const bool on = s < p.slots && expert >= 0;
            const int count = on ? listed : 0;
            const uint64_t mask = __ballot(on);
            int before = count;
            for (int d = 1; d < 64; d *= 2) {
                const int v = __shfl_up(before, d, 64);
                before += lane >= d ? v : 0;
            }
            if (on) {
                const int at = used + __popcll(mask & ((1ull << lane) - 1));
                sh_slot[at] = (uint16_t)s;
                sh_expert[at] = (uint16_t)expert;
                sh_start[at] = (uint16_t)(pairs + before - count);
            }
            used += __popcll(mask);
            pairs += __shfl(before, 63, 64);
        }
        if (lane == 0) {
            sh_start[used] = (uint16_t)pairs;
            sh_used = used;
        }
    }
    // the weights, divided by their sum
    for (int o = tid; o < p.T * p.top; o += THREADS) {
        float total = 1.0f;
        if (p.renormalize) {
            total = 0.0f;
            for (int j = 0; j < p.top; ++j)
                total += p.weight[o / p.top * p.top + j];
        }
        sh_weight[o] = total == 0.0f ? 0.0f : p.weight[o] / total;
    }
    sync_lds();
    const int used = __builtin_amdgcn_readfirstlane(sh_used);
    for (int a = wave; a < used; a += WAVES) {
        const int start = sh_start[a], count = sh_start[a + 1] - start;
        if (lane < count)   // (one token's slots are its choices)
            sh_pairs[start + lane] = p.T == 1 && p.slots < p.E ? sh_slot[a] : p.pair[sh_slot[a] * kMaxTokens + lane];
    }
    sync_lds();

    const int chunks = p.Ip / kDownUnit;
    const int64_t units = (int64_t)used * chunks;
    const int ranges = p.parts * WK, range = blockIdx.y * WK + wk;
    int64_t u = units * range / ranges;
    const int64_t u_end = units * (range + 1) / ranges;
    const int64_t plane = (int64_t)p.T * p.top * p.Ip;

    // `len` units of slot `a` from its unit `first`, for up to RB rows
    auto segment = [&]<int RB>(int a, int first, int len) {
        constexpr int MT = (RB + 15) / 16, PIECES = RB * 8 * PL;
        constexpr int NP = (PIECES + 64 * WN - 1) / (64 * WN);
        // (a thread's pieces of one row, or each its own, part included)
        constexpr int NE = NP % PL ? NP : NP / PL;
        static_assert(NE == NP || RB * 8 == NE * 64 * WN, "a thread's pieces of a part");
        const int start = sh_start[a], count = sh_start[a + 1] - start;
        const int expert = __builtin_amdgcn_readfirstlane(sh_expert[a]);
        const uint16_t *const wrow =
            p.down + (int64_t)expert * p.sd + (int64_t)min(n0 + c, p.H - 1) * p.ldd;
        const uint16_t *hrow[NE];
        const int8_t *erow[NE];
        int hdst[NE];
        auto piece_of = [&](int q) { return min(wn * 64 + lane + q * 64 * WN, PIECES - 1); };
#pragma unroll
        for (int q = 0; q < NE; ++q) {
            const int piece = piece_of(q);
            const int kc = piece & 7, row = (piece >> 3) % RB, pl = (piece >> 3) / RB;
            const int64_t pair = sh_pairs[start + min(row, count - 1)];
            hrow[q] = p.h + pl * plane + pair * p.Ip + 8 * kc;
            erow[q] = p.scale + pair * (p.Ip / 16);
            hdst[q] = pl * HB + place<RB>(row, piece_at<END == 1>(kc));
        }
        const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
        f32x4 acc[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i)
            acc[i] = zero;
        struct Pieces {
            u32x4 v[2];
        };
        std::conditional_t<END == 1, Odd16, Pieces> w[2];
        u32x4 hr[NP];
        uint32_t er[NE];   // e of the unit's four blocks
        auto load_h = [&](int t) {
            const int k = (first + min(t, len - 1)) * kDownUnit;
            if constexpr (DT == 1)
#pragma unroll
                for (int q = 0; q < NE; ++q)
                    er[q] = *(const uint32_t *)(erow[q] + k / 16);
#pragma unroll
            for (int q = 0; q < NP; ++q)
                hr[q] = *(const u32x4 *)(hrow[q % NE] + q / NE * plane + k);
        };
        auto load_w = [&](auto &to, int t) {
            const int k = (first + min(t, len - 1)) * kDownUnit;
            if constexpr (END == 1)
                to.load(wrow + min(k + 16 * g, p.I - 16));
            else
#pragma unroll
                for (int d = 0; d < 2; ++d) {
                    const int at = k + 32 * d + 8 * g;
                    if constexpr (END == 2)
                        to.v[d] = load16_end(wrow, 2 * (int64_t)at, 2 * (int64_t)p.I);
                    else
                        to.v[d] = load_any<u32x4>(wrow + min(at, p.I - 8));
                }
        };
        load_h(0);
        load_w(w[0], 0);
        load_w(w[1], 1);
        auto step = [&]<int B>(int t) {
            constexpr int buf = BUFS == 1 ? 0 : B;
            char *const hs = sh_h[wk][buf][0];
            if constexpr (DT == 1)
#pragma unroll
                for (int q = 0; q < NE; ++q) {
                    const int piece = piece_of(q);
                    const int E = max(max((int)(int8_t)er[q], (int)(int8_t)(er[q] >> 8)),
                                      max((int)(int8_t)(er[q] >> 16), (int)er[q] >> 24));
                    const int d = E - (int)(int8_t)(er[q] >> (4 * (piece & 6)));
#pragma unroll
                    for (int i = q; i < NP; i += NE)
                        hr[i] = scale_down(hr[i], d);
                    // (every lane writes its row's: one that did not would be
                    // taken to read what it read before)
                    sh_scale[wk][buf][(piece >> 3) % RB] = power2(E);
                }
#pragma unroll
            for (int q = 0; q < NP; ++q)
                *(u32x4 *)(hs + q / NE * HB + hdst[q % NE]) = hr[q];
            if constexpr (DT == 1 && END == 1)
                __builtin_amdgcn_sched_barrier(0);   // (weights moved into place before this would not fit)
            load_h(t + 1);
            if (WN > 1)
                sync_lds();
            if constexpr (END == 1) {
                const int at = (first + t) * kDownUnit + 16 * g, from = min(at, p.I - 16);
                w[B].align((uint32_t)(uintptr_t)(wrow + from) & 2u);
                if (first + t == chunks - 1)
                    w[B].drop(min(at - from, 16));
            }
            f32x4 part[MT][DT == 1 ? PL : 1];   // the parts' sums over this unit
            // (16 rows or fewer, columns of one range: all of h is read before the
            // first product, or each would wait for its own read.  16 tokens, 6 of
            // 64 of 2048 x 1408: 172 us, 181 without.)
            u32x4 ha[2][MT][PL];
#pragma unroll
            for (int o = 0; o < 2 * MT * PL; ++o) {
                const int d = o / (MT * PL), i = o / PL % MT, q = o % PL;
                ha[d][i][q] =
                    *(const u32x4 *)(hs + q * HB + place<RB>(RB < 16 ? min(c, RB - 1) : 16 * i + c, 4 * d + g));
            }
            if constexpr (MT == 1 && WN > 1)
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int o = 0; o < 2 * MT * PL; ++o) {
                const int d = o / (MT * PL), i = o / PL % MT, q = o % PL;
                if constexpr (DT == 1)
                    part[i][q] = mfma16<DT>(ha[d][i][q], w[B].v[d], d == 0 ? zero : part[i][q]);
                else
                    acc[i] = mfma16<DT>(ha[d][i][q], w[B].v[d], acc[i]);
            }
            if constexpr (DT == 1)
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const f32x4 scale = *(const f32x4 *)&sh_scale[wk][buf][16 * i + 4 * g];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float sum = part[i][PL - 1][r];
#pragma unroll
                        for (int q = PL - 2; q >= 0; --q)
                            sum = fmaf(0x1p-11f, sum, part[i][q][r]);
                        acc[i][r] = fmaf(scale[r], sum, acc[i][r]);
                    }
                }
            load_w(w[B], t + 2);
        };
        for (int t = 0;;) {
            step.template operator()<0>(t);
            if (++t == len)
                break;
            step.template operator()<1>(t);
            if (++t == len)
                break;
        }
        if (WN > 1)
            sync_lds();   // (the next segment starts with the first buffer again)
        // the tokens' weighted sums
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int m = 16 * i + 4 * g + r;
                if (m < count) {
                    const int pair = sh_pairs[start + m], t = pair / p.top;
                    const float v = acc[i][r];
                    // (no weight: nothing of what came out, were it infinite or NaN)
                    const float weight = sh_weight[pair];
                    mine[t * 16 + c] += weight == 0.0f ? 0.0f : weight * v;
                }
            }
    };
    while (u < u_end) {
        const int a = __builtin_amdgcn_readfirstlane((int)(u / chunks));
        const int first = __builtin_amdgcn_readfirstlane((int)(u % chunks));
        const int len = (int)min((int64_t)(chunks - first), u_end - u);
        if constexpr (R < 16) {
            segment.template operator()<R>(a, first, len);
        } else {
            const int count = __builtin_amdgcn_readfirstlane(sh_start[a + 1] - sh_start[a]);
            if (count <= 4)
                segment.template operator()<4>(a, first, len);
            else if (R == 16 || count <= 16)
                segment.template operator()<16>(a, first, len);
            else if (R == 32 || (R > 32 && count <= 32))
                segment.template operator()<R < 32 ? R : 32>(a, first, len);
            else
                segment.template operator()<R>(a, first, len);
        }
        u += len;
    }
    sync_lds();

    // the workgroup's sums, four columns of a token at a time: of its ranges
    // (WK) or of its columns (WN)
    constexpr int G = 4 * WN;
    const int values = p.T * G;
    auto own = [&](int o) {
        const int t = o / G, n = o % G * 4;
        f32x4 v = *(const f32x4 *)&acc_all[n >> 4][t * 16 + (n & 15)];
#pragma unroll
        for (int w = 1; w < WK; ++w)
            v += *(const f32x4 *)&acc_all[w][t * 16 + n];
        return v;
    };
    const bool shared = p.parts > 1;
    const uint32_t hp = (uint32_t)gridDim.x * 16 * WN;   // columns of a row of partial sums
    auto place_of = [&](int q, int o) { return (((uint32_t)(q * p.T + o / G)) * hp + nw + o % G * 4) * 4u; };
    if (shared) {
        // publish them with device-scope stores; once every wave's have
        // completed, count in.  Nobody waits: the last one adds.
        for (int o = tid; o < values; o += THREADS)
            store4_device(p.part, place_of(blockIdx.y, o), own(o));
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        sync_lds();
        if (tid == 0) {
            const int before = __hip_atomic_fetch_add(p.done + blockIdx.x, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            sh_last = before == p.parts - 1;
            if (sh_last)
                __hip_atomic_store(p.done + blockIdx.x, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        sync_lds();
        if (!sh_last)
            return;
    }
    for (int o = tid; o < values; o += THREADS) {
        const int t = o / G, n = nw + o % G * 4;
        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
        if (shared) {
            for (int q0 = 0; q0 < p.parts; q0 += 8) {
                f32x4 x[8];
#pragma unroll
                for (int q = 0; q < 8; ++q)
                    x[q] = load4_device(p.part, place_of(min(q0 + q, p.parts - 1), o));
#pragma unroll
                for (int q = 0; q < 8; ++q)
                    if (q0 + q < p.parts)
                        v += x[q];
            }
        } else {
            v = own(o);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < p.H) {
                if (p.out16)
                    ((uint16_t *)p.y)[(int64_t)t * p.ldy + n + e] = from_float<DT>(v[e]);
                else
                    ((float *)p.y)[(int64_t)t * p.ldy + n + e] = v[e];
            }
    }
}

}  // namespace xexperts_dev
