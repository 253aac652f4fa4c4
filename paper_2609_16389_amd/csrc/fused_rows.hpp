// Products of a few rows (up to 16) with an end (fused_ends.hpp): a token or a small
// batch that decodes.  The weights are read once, and nothing else takes part in
// the time.
//
// Columns go by 16 (16 of either matrix of a gated block), and the waves of a
// workgroup share k: wave w takes the units w, w + W, .. of 256 bytes of a row, four
// matrix instructions each.  The waves' sums are added through LDS in ascending
// order.  rows_stream reads weights whose rows are whole 16-byte chunks through LDS;
// rows_product any others, straight into registers.
#pragma once

#include "fused_ends.hpp"

#include <utility>

namespace xfused_dev {

constexpr int kUnit = 256;          // bytes of k

struct RowsParams {
    const char *x, *w, *w2;   // w2: the second matrix of a gated block
    int64_t ldx, ldw;         // bytes (x to be quantised: values)
    int M, N, K;              // K: bytes of a row of w
};

// Rows at any address: lane l holds bytes 64 j + 16 (l / 16) of the unit of row
// l % 16 for instruction j, of weights and x alike, and the wave's next unit is on
// its way while one is multiplied.  Rows past the last are read as the last and
// their sums dropped; the bytes of the last unit past k are zeros of both operands.
// ODD: rows that begin between dwords.
template <int TYPE, class End, int W, bool ODD>
__global__ void __launch_bounds__(64 * W) rows_product(RowsParams p, typename End::Params e)
{
    constexpr int NM = End::kGated ? 2 : 1;
    typedef typename Sum<TYPE>::type sum_t;
    __shared__ __attribute__((aligned(16))) char smem[W * NM * 1024];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = blockIdx.x * 16, r = lane & 15, g = lane >> 4;
    const int full = p.K / kUnit, rest = p.K % kUnit;
    const int64_t wrow = (int64_t)min(n0 + r, p.N - 1) * p.ldw;
    const char *const wp[2] = {p.w + wrow, NM > 1 ? p.w2 + wrow : nullptr};
    const char *const xp = p.x + (int64_t)min(r, p.M - 1) * p.ldx;

    sum_t acc[NM];
#pragma unroll
    for (int m = 0; m < NM; ++m)
        acc[m] = sum_t{0, 0, 0, 0};
    u32x4 wq[2][NM][4], xq[2][4];
    auto load = [&](int s, int u) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t at = (int64_t)u * kUnit + j * 64 + g * 16;
#pragma unroll
            for (int m = 0; m < NM; ++m)
                wq[s][m][j] = sixteen<ODD>(wp[m] + at);
            xq[s][j] = sixteen<ODD>(xp + at);
        }
    };
    auto multiply = [&](int s) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int m = 0; m < NM; ++m)
                acc[m] = mfma<TYPE>(wq[s][m][j], xq[s][j], acc[m]);
    };

    // this wave's whole units; past the last it is loaded again, so that the
    // loads of the loop are unconditional
    const int mine = full > wave ? (full - wave + W - 1) / W : 0;
    auto unit = [&](int i) { return wave + min(i, mine - 1) * W; };
    if (mine > 0) {
        load(0, unit(0));
        for (int i = 0; i < mine; i += 2) {
            load(1, unit(i + 1));
            multiply(0);
            load(0, unit(i + 2));
            if (i + 1 < mine)
                multiply(1);
        }
    }
    // the unit that k ends in, with zeros past the end
    if (rest > 0 && wave == full % W) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j * 64 < rest) {
                const int64_t at = (int64_t)full * kUnit + j * 64 + g * 16;
                const u32x4 x = load16_end(xp, at, p.K);
#pragma unroll
                for (int m = 0; m < NM; ++m)
                    acc[m] = mfma<TYPE>(load16_end(wp[m], at, p.K), x, acc[m]);
            }
    }
    // lane l: row l % 16, columns 4 (l / 16) .. + 3
    u32x4 *const sums = (u32x4 *)smem;
#pragma unroll
    for (int m = 0; m < NM; ++m)
        sums[(wave * NM + m) * 64 + lane] = __builtin_bit_cast(u32x4, acc[m]);
    __syncthreads();
    if (wave == 0) {
        sum_t s[2] = {sum_t{0, 0, 0, 0}, sum_t{0, 0, 0, 0}};
#pragma unroll
        for (int k = 0; k < W; ++k)
#pragma unroll
            for (int m = 0; m < NM; ++m)
                s[m] += __builtin_bit_cast(sum_t, sums[(k * NM + m) * 64 + lane]);
        const int col = n0 + g * 4;
        if (r < p.M && col < p.N)
            End::quad(e, r, col, p.N, s[0], s[1]);
    }
}

// Rows that are whole 16-byte chunks: four waves, each with a queue of S units of
// its own in LDS, that only its own waits look after.  A load takes 256 bytes of
// four rows, whole lines of memory (fragments loaded straight into registers
// take 64 of 16 rows).  Workgroups stay for several blocks of 16 columns, and
// their queues run on over them: memory never waits for a join.
//
// What bounds it: HBM (gated 1 x 4096 x 14336: 235 MB in 37 us, 6.4 TB/s; fragments
// loaded straight into registers took 49), for small weights the launch and one
// latency (8-bit 4096 x 4096 5.2 us, of which a third is the row's own 8-bit values).
//
// XI: loads of x's part of a unit, 1 for up to 4 rows and 4 for up to 16.  QUANT: x is
// one row of values of that type (kBf16, kFp16, kFp32; at 16-byte addresses, up to
// kQuantBytes), of which each workgroup makes the 8-bit row for itself, in LDS,
// while its first weights are on their way; else -1.
constexpr int kStreamWaves = 4;
constexpr int kQuantBytes = 16384;

template <int TYPE, class End, int XI, int S, int QUANT>
__global__ void __launch_bounds__(64 * kStreamWaves) rows_stream(RowsParams p, typename End::Params e)
{
    constexpr int W = kStreamWaves, NM = End::kGated ? 2 : 1, NX = QUANT >= 0 ? 0 : XI;
    constexpr int LD = 4 * NM + NX, STAGE = LD * 1024;
    static_assert(S * LD < 64, "loads in flight");
    typedef typename Sum<TYPE>::type sum_t;
    constexpr int kSums = W * NM * 1024;   // twice
    __shared__ __attribute__((aligned(16))) char smem[W * S * STAGE + 2 * kSums + (QUANT >= 0 ? 2 * kQuantBytes : 0)];
    __shared__ uint32_t sh_most[W];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4;
    char *const queue = smem + wave * S * STAGE, *const sums = smem + W * S * STAGE, *const qx = sums + 2 * kSums;
    const uint32_t queue_at = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char *)queue;
    const int units = (p.K + kUnit - 1) / kUnit;
    const int each = units > wave ? (units - wave + W - 1) / W : 0;   // of this wave in a block
    const int blocks = (p.N + 15) / 16;
    const int total = each * ((blocks - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x);

    // chunk c of row r of a unit lies in slot c ^ r: the 16 rows of a fragment
    // read cover all banks
    uint32_t off_w[4], off_x[4];
    int chunk[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int row = 4 * j + (lane >> 4);
        chunk[j] = ((lane & 15) ^ row) << 4;
        off_w[j] = (uint32_t)(row * (int)p.ldw + chunk[j]);
        off_x[j] = (uint32_t)(row * (int)p.ldx + chunk[j]);
    }
    int at_block = blockIdx.x, at_i = 0;   // of the next unit to be loaded
    auto load = [&](int stage) {
        const int64_t k = (int64_t)(wave + at_i * W) * kUnit, left = p.K - k;
        const int n0 = at_block * 16, rows = min(p.N - n0, 16);
        const uint32_t to = queue_at + stage * STAGE;
#pragma unroll
        for (int m = 0; m < NM; ++m) {
            const u32x4 d = descriptor((m ? p.w2 : p.w) + (int64_t)n0 * p.ldw + k, (rows - 1) * p.ldw + left);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                load_lds(d, chunk[j] < left ? off_w[j] : kPastEnd, __builtin_amdgcn_readfirstlane(to + (m * 4 + j) * 1024));
        }
        if constexpr (NX > 0) {
            const u32x4 d = descriptor(p.x + k, (p.M - 1) * p.ldx + left);
#pragma unroll
            for (int j = 0; j < NX; ++j)
                load_lds(d, chunk[j] < left ? off_x[j] : kPastEnd,
                         __builtin_amdgcn_readfirstlane(to + (NM * 4 + j) * 1024));
        }
        if (++at_i == each) {
            at_i = 0;
            at_block += gridDim.x;
        }
    };

    constexpr int E = QUANT == kFp32 ? 4 : 2;
    const int first = min(S, total);   // units on their way at the beginning
    // until no more than n units' loads are on their way
    auto wait_units = [](int n) {
        [n]<int... I>(std::integer_sequence<int, I...>) {
            ((n == I ? wait_loads<I * LD>() : (void)0), ...);
        }(std::make_integer_sequence<int, S + 1>());
    };
    if constexpr (QUANT >= 0) {
        // x as it is, 1 KB a load, the waves in turn
        const u32x4 d = descriptor(p.x, (int64_t)p.K * E);
        const uint32_t raw_at = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char *)(qx + kQuantBytes);
        for (int at = wave * 1024; at < p.K * E; at += W * 1024)
            load_lds(d, at + lane * 16, __builtin_amdgcn_readfirstlane(raw_at + at));
    }
#pragma unroll
    for (int s = 0; s < S; ++s)
        if (s < total)
            load(s);
    float row_scale_of_x = 0.0f;
    if constexpr (QUANT >= 0) {
        // (x has landed once no more than the units' loads are left)
        wait_units(first);
        meet();
        const char *const raw = qx + kQuantBytes;
        // (K is a multiple of 16)
        auto here = [&](int k, float (&v)[8]) {
            const u32x4 *const q = (const u32x4 *)(raw + k * E);
            const u32x4 zero = {0, 0, 0, 0}, lo = k < p.K ? q[0] : zero, hi = k < p.K && E == 4 ? q[1] : zero;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if constexpr (QUANT == kFp32)
                    v[j] = __builtin_bit_cast(float, j < 4 ? lo[j] : hi[j - 4]);
                else
                    v[j] = to_float<QUANT>((uint16_t)(lo[j / 2] >> (16 * (j & 1))));
        };
        uint32_t most = 0;
        for (int k = threadIdx.x * 8; k < p.K; k += 64 * W * 8) {
            float v[8];
            here(k, v);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                most = max(most, __builtin_bit_cast(uint32_t, v[j]) & 0x7fffffffu);
        }
        most = most_of(most);
        if (lane == 0)
            sh_most[wave] = most;
        wait_lds();
        meet();
        most = max(max(sh_most[0], sh_most[1]), max(sh_most[2], sh_most[3]));
        row_scale_of_x = row_scale(most);
        for (int k = threadIdx.x * 8; k < units * kUnit; k += 64 * W * 8) {
            float v[8];
            here(k, v);
            *(uint64_t *)(qx + k) = eight_bytes(v, row_scale_of_x);
        }
        wait_lds();
        meet();
    }

    int step = 0, stage = 0;
    for (int block = blockIdx.x, turn = 0; block < blocks; block += gridDim.x, ++turn) {
        sum_t acc[NM];
#pragma unroll
        for (int m = 0; m < NM; ++m)
            acc[m] = sum_t{0, 0, 0, 0};
        for (int i = 0; i < each; ++i, ++step) {
            wait_units(min(total - step, S) - 1);
            asm volatile("" ::: "memory");
            const char *const q = queue + stage * STAGE;
            u32x4 wf[NM][4], xf[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int slot = (((4 * j + g) ^ r) << 4);
#pragma unroll
                for (int m = 0; m < NM; ++m)
                    wf[m][j] = *(const u32x4 *)(q + m * 4096 + r * 256 + slot);
                if constexpr (QUANT >= 0)
                    xf[j] = *(const u32x4 *)(qx + (wave + i * W) * kUnit + j * 64 + g * 16);
                else if constexpr (XI == 1)
                    xf[j] = *(const u32x4 *)(q + NM * 4096 + (r & 3) * 256 + (((4 * j + g) ^ (r & 3)) << 4));
                else
                    xf[j] = *(const u32x4 *)(q + NM * 4096 + r * 256 + slot);
            }
            wait_lds();   // (the stage has been read: it may be loaded again)
            asm volatile("" ::: "memory");
            if (step + S < total)
                load(stage);
            stage = stage == S - 1 ? 0 : stage + 1;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int m = 0; m < NM; ++m)
                    acc[m] = mfma<TYPE>(wf[m][j], xf[j], acc[m]);
        }
        // lane l: row l % 16, columns 4 (l / 16) .. + 3.  Two places for the sums in
        // turn: a wave that is two blocks ahead has met the one that still adds
        u32x4 *const to = (u32x4 *)(sums + (turn & 1) * kSums);
#pragma unroll
        for (int m = 0; m < NM; ++m)
            to[(wave * NM + m) * 64 + lane] = __builtin_bit_cast(u32x4, acc[m]);
        wait_lds();
        meet();
        if (wave == turn % W) {
            sum_t s[2] = {sum_t{0, 0, 0, 0}, sum_t{0, 0, 0, 0}};
#pragma unroll
            for (int k = 0; k < W; ++k)
#pragma unroll
                for (int m = 0; m < NM; ++m)
                    s[m] += __builtin_bit_cast(sum_t, to[(k * NM + m) * 64 + lane]);
            const int col = block * 16 + g * 4;
            if (r < p.M && col < p.N) {
                if constexpr (QUANT >= 0) {
                    typename End::Params q = e;
                    q.row_scale = &row_scale_of_x;
                    End::quad(q, 0, col, p.N, s[0], s[1]);
                } else {
                    End::quad(e, r, col, p.N, s[0], s[1]);
                }
            }
        }
    }
}

}  // namespace xfused_dev
