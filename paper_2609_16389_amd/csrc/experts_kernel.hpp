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
// First launch (route_up): one workgroup a slot and 16 of the inner columns.
// It works out its slot from the scores by itself (a comparison of every
// score with the expert's own, per token, which costs less than a launch),
// then forms 16 gate and 16 up columns for the slot's tokens, the waves
// splitting the hidden dimension, and writes h.  The first workgroup of a
// slot also writes the slot's tokens and weights.
// Second launch (down_sum): one workgroup for 16 columns of y.  Its waves
// share the slots' inner dimensions evenly and keep sums of their own for
// every token in LDS, which are added in the order of the waves: no atomics,
// one order of summation.
//
// The second product needs h on the matrix units, which take 16 bits.  Rounded
// to 16 bits h would lose more than the rounding of y does, so it is written as
// three 16-bit parts that together hold its 24 bits, and multiplied as three
// products (the matrix units are idle most of the time).
//   bfloat16: h = a + b + c, each part the rounding of what the ones before leave.
//   binary16, whose range is short: h = 2^12 (a + 2^-11 (b + 2^-11 c)).  This
//   holds |h| up to 2.6e8 and resolves 2^-34.
#pragma once

#include "decode_device.hpp"

namespace xexperts_dev {

using namespace xdecode_dev;

constexpr int kMaxTokens = 64;    // tokens of a launch
constexpr int kMaxExperts = 1024;
constexpr int kUpThreads = 512, kUpWaves = kUpThreads / 64;
constexpr int kDownThreads = 1024, kDownWaves = kDownThreads / 64;
constexpr int kUnit = 128;        // k per unit of a wave
constexpr int kPad = 128;         // inner columns of h are padded to this

// A chosen expert and the (token, choice) pairs that chose it.
struct Slot {
    int expert;  // -1: empty
    int count;
    uint16_t pair[kMaxTokens];  // token * top + choice
};

struct ExpertsParams {
    const uint16_t *x;
    const float *scores;
    const uint16_t *up, *down;
    void *y;
    int64_t ldx, lds, ldu, su, ldd, sd, ldy;  // elements
    int T, E, top, H, I, Ip;                  // Ip: I rounded up to kPad
    int slots;
    int renormalize, out16;
    Slot *slot;       // [slots]
    float *weight;    // [T * top]: exp(score - largest), over the whole softmax's sum without renormalize
    uint16_t *h;      // [3][T * top][Ip]
};

// A score as a whole number in the same order: NaN above all, the two zeros
// alike.
__device__ __forceinline__ uint32_t order_of(float v)
{
    if (v != v)
        return 0xffffffffu;
    const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.0f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}

// The three parts of h (see above).
template <int DT>
__device__ __forceinline__ void split3(float v, uint16_t (&part)[3])
{
    constexpr float down = DT == 0 ? 1.0f : 0x1p-12f, step = DT == 0 ? 1.0f : 0x1p11f;
    float r = v * down;
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        part[i] = from_float<DT>(r);
        const float got = to_float<DT>(part[i]);
        r = (r - got) * step;
        if (!(__builtin_fabsf(got) < __builtin_inff()))   // nothing is left of what has overflowed
            r = 0.0f;
    }
}

// exp of a score against the largest; a score of -inf has no weight.
__device__ __forceinline__ float score_exp(float v, float largest)
{
    return v == -__builtin_inff() ? 0.0f : expf(v - largest);
}

template <int DT, int MT>
__global__ void __launch_bounds__(kUpThreads)
route_up(ExpertsParams p)
{
    __shared__ union {
        uint32_t key[kMaxExperts];
        float red[kUpWaves * MT * 512];
    } sh;
    __shared__ int sh_expert, sh_count, sh_first;
    __shared__ uint8_t sh_rank[kMaxTokens];
    __shared__ uint16_t sh_pair[kMaxTokens];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int slot = blockIdx.y, i0 = 16 * blockIdx.x;

    // the slot's expert
    const bool by_choice = p.slots < p.E;
    if (by_choice) {
        const int t = slot / p.top, j = slot - t * p.top;
        for (int e = tid; e < p.E; e += kUpThreads)
            sh.key[e] = order_of(p.scores[t * p.lds + e]);
        __syncthreads();
        for (int e = tid; e < p.E; e += kUpThreads) {
            const uint32_t mine = sh.key[e];
            int rank = 0;
            for (int o = 0; o < p.E; ++o)
                rank += sh.key[o] > mine || (sh.key[o] == mine && o < e);
            if (rank == j)
                sh_expert = e;
        }
        __syncthreads();
    }
    const int expert = by_choice ? sh_expert : slot;

    // its rank among each token's scores: `per` lanes a token
    int per = 64;
    while (per > 8 && kUpThreads / per < p.T)
        per /= 2;
    const int tok = tid / per, sub = tid & (per - 1);
    {
        const float *row = p.scores + (int64_t)min(tok, p.T - 1) * p.lds;
        const float own = row[expert];
        const uint32_t mine = order_of(own);
        int rank = 0;
        float largest = -__builtin_inff();
        for (int o = sub; o < p.E; o += per) {
            const uint32_t k = order_of(row[o]);
            rank += k > mine || (k == mine && o < expert);
            largest = fmaxf(largest, row[o]);
        }
        for (int d = per / 2; d >= 1; d /= 2) {
            rank += __shfl_xor(rank, d, 64);
            largest = fmaxf(largest, __shfl_xor(largest, d, 64));
        }
        const bool chosen = rank < p.top && tok < p.T;
        if (tok < kMaxTokens && sub == 0)
            sh_rank[tok] = chosen ? (uint8_t)rank : 255;
        if (blockIdx.x == 0) {
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
    }
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
    const int count = sh_count;
    const bool empty = count == 0 || (by_choice && sh_first != slot / p.top);
    if (blockIdx.x == 0) {
        Slot *const s = p.slot + slot;
        if (tid == 0) {
            s->expert = empty ? -1 : expert;
            s->count = count;
        }
        if (tid < count)
            s->pair[tid] = sh_pair[tid];
    }
    if (empty)
        return;

    const int c = lane & 15, g = lane >> 4;
    const uint16_t *wrow[2];
#pragma unroll
    for (int v = 0; v < 2; ++v)
        wrow[v] = p.up + (int64_t)expert * p.su + (int64_t)(v * p.I + min(i0 + c, p.I - 1)) * p.ldu;
    const uint16_t *xrow[MT];
    bool live[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        live[i] = 16 * i + c < count;
        xrow[i] = p.x + (int64_t)(live[i] ? sh_pair[16 * i + c] / p.top : 0) * p.ldx;
    }
    f32x4 acc[MT][2];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int v = 0; v < 2; ++v)
            acc[i][v] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    for (int k0 = wave * kUnit; k0 < p.H; k0 += kUpWaves * kUnit) {
        const bool whole = k0 + kUnit <= p.H;
        u32x4 w[4][2];
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                const int k = k0 + 32 * d + 8 * g;
                w[d][v] = whole ? load_any<u32x4>(wrow[v] + k) : load16_end(wrow[v], 2 * (int64_t)k, 2 * (int64_t)p.H);
            }
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            const int k = k0 + 32 * d + 8 * g;
#pragma unroll
            for (int i = 0; i < MT; ++i)
                if (16 * i < count) {
                    u32x4 a = {0u, 0u, 0u, 0u};
                    if (live[i])
                        a = whole ? load_any<u32x4>(xrow[i] + k) : load16_end(xrow[i], 2 * (int64_t)k, 2 * (int64_t)p.H);
#pragma unroll
                    for (int v = 0; v < 2; ++v)
                        acc[i][v] = mfma16<DT>(a, w[d][v], acc[i][v]);
                }
        }
    }

    // the waves' blocks, added in ascending order
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int v = 0; v < 2; ++v)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                sh.red[((wave * MT + i) * 2 + v) * 256 + 64 * r + lane] = acc[i][v][r];
    __syncthreads();
    const int64_t plane = (int64_t)p.T * p.top * p.Ip;
    for (int o = tid; o < MT * 256; o += kUpThreads) {
        const int i = o >> 8, r = o >> 6 & 3, l = o & 63;
        const int m = 16 * i + 4 * (l >> 4) + r, col = i0 + (l & 15);
        if (m >= count)
            continue;
        float sum[2];
#pragma unroll
        for (int v = 0; v < 2; ++v) {
            sum[v] = sh.red[(i * 2 + v) * 256 + (o & 255)];
#pragma unroll
            for (int w = 1; w < kUpWaves; ++w)
                sum[v] += sh.red[((w * MT + i) * 2 + v) * 256 + (o & 255)];
        }
        uint16_t part[3] = {0, 0, 0};
        if (col < p.I)
            split3<DT>(sum[0] / (1.0f + expf(-sum[0])) * sum[1], part);
        uint16_t *const at = p.h + (int64_t)sh_pair[m] * p.Ip + col;
#pragma unroll
        for (int q = 0; q < 3; ++q)
            at[q * plane] = part[q];
        // the last workgroup also clears the padding past its columns
        if (blockIdx.x == gridDim.x - 1)
            for (int past = 16; col + past < p.Ip; past += 16)
#pragma unroll
                for (int q = 0; q < 3; ++q)
                    at[q * plane + past] = 0;
    }
}

template <int DT, int MT>
__global__ void __launch_bounds__(kDownThreads)
down_sum(ExpertsParams p)
{
    constexpr int kSums = DT == 0 ? 1 : 3;   // products of the parts that are kept apart
    __shared__ float acc_all[kDownWaves * MT * 256];
    __shared__ float sh_total[16 * MT];
    __shared__ uint16_t sh_active[kMaxExperts];
    __shared__ int sh_wave[kDownWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n0 = 16 * blockIdx.x;
    const int c = lane & 15, g = lane >> 4;

    for (int o = tid; o < kDownWaves * MT * 256; o += kDownThreads)
        acc_all[o] = 0.0f;
    // what a token's weights are divided by
    if (tid < p.T) {
        float total = 1.0f;
        if (p.renormalize) {
            total = 0.0f;
            for (int j = 0; j < p.top; ++j)
                total += p.weight[tid * p.top + j];
        }
        sh_total[tid] = total;
    }
    // the slots in use, in ascending order
    const bool used = tid < p.slots && p.slot[tid].expert >= 0;
    const uint64_t mask = __ballot(used);
    if (lane == 0)
        sh_wave[wave] = __popcll(mask);
    __syncthreads();
    int before = 0, active = 0;
    for (int w = 0; w < kDownWaves; ++w) {
        before += w < wave ? sh_wave[w] : 0;
        active += sh_wave[w];
    }
    if (used)
        sh_active[before + __popcll(mask & ((1ull << lane) - 1))] = (uint16_t)tid;
    __syncthreads();

    const int chunks = p.Ip / kUnit;
    const int64_t units = (int64_t)active * chunks;
    const int64_t u_end = units * (wave + 1) / kDownWaves;
    int64_t u = units * wave / kDownWaves;
    float *const mine = acc_all + wave * MT * 256;
    const int64_t plane = (int64_t)p.T * p.top * p.Ip;
    while (u < u_end) {
        const Slot *const s = p.slot + sh_active[u / chunks];
        const int count = s->count;
        const uint16_t *const wrow = p.down + (int64_t)s->expert * p.sd + (int64_t)min(n0 + c, p.H - 1) * p.ldd;
        const uint16_t *hrow[MT];
        bool live[MT];
        f32x4 acc[MT][kSums];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            live[i] = 16 * i + c < count;
            hrow[i] = p.h + (int64_t)(live[i] ? s->pair[16 * i + c] : 0) * p.Ip;
#pragma unroll
            for (int q = 0; q < kSums; ++q)
                acc[i][q] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
        const int first = (int)(u % chunks);
        const int last = (int)min((int64_t)chunks, first + (u_end - u));
        for (int ch = first; ch < last; ++ch) {
            const int k0 = ch * kUnit;
            const bool whole = k0 + kUnit <= p.I;
            u32x4 w[4];
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                const int k = k0 + 32 * d + 8 * g;
                w[d] = whole ? load_any<u32x4>(wrow + k) : load16_end(wrow, 2 * (int64_t)k, 2 * (int64_t)p.I);
            }
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                const int k = k0 + 32 * d + 8 * g;
#pragma unroll
                for (int i = 0; i < MT; ++i)
                    if (16 * i < count)
#pragma unroll
                        for (int q = 0; q < 3; ++q) {
                            u32x4 a = {0u, 0u, 0u, 0u};
                            if (live[i])
                                a = *(const u32x4 *)(hrow[i] + q * plane + k);
                            constexpr int one = kSums - 1;
                            acc[i][q & (one ? 3 : 0)] = mfma16<DT>(a, w[d], acc[i][q & (one ? 3 : 0)]);
                        }
            }
        }
        // the tokens' weighted sums
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int m = 16 * i + 4 * g + r;
                if (m < count) {
                    const int pair = s->pair[m], t = pair / p.top;
                    const float total = sh_total[t];
                    const float weight = total == 0.0f ? 0.0f : p.weight[pair] / total;
                    float v = acc[i][0][r];
                    if constexpr (kSums == 3)
                        v = 0x1p12f * (v + 0x1p-11f * (acc[i][1][r] + 0x1p-11f * acc[i][2][r]));
                    mine[t * 16 + c] += weight * v;
                }
            }
        u += last - first;
    }
    __syncthreads();
    for (int o = tid; o < p.T * 16; o += kDownThreads) {
        const int t = o >> 4, n = n0 + (o & 15);
        if (n >= p.H)
            continue;
        float v = acc_all[o];
#pragma unroll
        for (int w = 1; w < kDownWaves; ++w)
            v += acc_all[w * MT * 256 + o];
        if (p.out16)
            ((uint16_t *)p.y)[(int64_t)t * p.ldy + n] = from_float<DT>(v);
        else
            ((float *)p.y)[(int64_t)t * p.ldy + n] = v;
    }
}

}  // namespace xexperts_dev
