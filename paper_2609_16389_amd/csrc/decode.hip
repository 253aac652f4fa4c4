// Host side of the operators around a decoding step: argument checks, launch
// selection and launches.  The C ABI is declared in include/xgemm.h.
#include "context.hpp"
#include "experts_kernel.hpp"
#include "logprob_kernel.hpp"
#include "quant_kernel.hpp"

#include <algorithm>
#include <initializer_list>
#include <type_traits>
#include <utility>

using xgemm_host::kMaxDim;

namespace {

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Sizes within the library's limits, a leading dimension that holds a row, and
// offsets that 64 bits address.
bool dims_ok(int64_t rows, int64_t cols, int64_t ld)
{
    return rows >= 0 && cols >= 0 && rows < kMaxDim && cols < kMaxDim && ld >= cols && (double)rows * (double)ld <= 9.0e18;
}

int launch_status(xgemm_ctx *h, const char *what)
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess)
        return XGEMM_OK;
    xgemm_host::set_error(h, what, e);
    return XGEMM_ERR_HIP;
}

// ---------------------------------------------------------------------------
// products with 4-bit weights
// ---------------------------------------------------------------------------

using xquant_dev::QuantParams;

// Waves of a workgroup: 8 ranges of K for 16 columns, or 4 ranges of 64 columns,
// which share x.  One or two rows: 8 ranges up to 512 tiles of 16 columns, 4
// beyond.  (Microseconds of N x K for one row, 8 / 4 ranges: 2048 x 14336 7.4 / 9.0,
// 4096 x 14336 7.8 / 9.2, 4096 x 4096 4.9 / 4.8, 8192 x 14336 15.7 / 15.1, 8192 x
// 4096 6.3 / 5.9, 12288 x 4096 8.1 / 7.0, 14336 x 4096 10.3 / 8.1.)  More rows: the least of (rounds of workgroups that the CUs take) x
// (time of one, in ns a k), with 16 rows a workgroup 1.7 for 16 columns, of which
// two run on a CU, and 2.5 for 64 columns, 3.2 with 32 rows, 5.0 with 64.  A
// workgroup of more rows widens each weight for all of them, but where columns
// leave CUs idle blocks of 16 rows are faster.  Microseconds of N x K, for M
// rows: 32 or 64 rows a workgroup / 16 rows, 64 columns / 16 rows, 16 columns:
//     9216 x 4096    M 16:           9.9 / 11.6
//     6400 x 4096    M 16:          10.4 /  9.1
//     2560 x 1280    M 32:  8.6 /  7.2 /  5.4   M 64: 10.8 /  7.4 /   7.8
//     2560 x 5120    M 32: 19.8 / 15.8 / 11.4   M 64: 21.9 / 12.0 /  13.7
//     4096 x 4096    M 32: 12.7 / 10.2 /  9.1   M 64: 18.0 / 10.7 /  14.9
//     7680 x 7680    M 32: 21.9 / 16.4 / 23.3   M 64: 32.7 / 31.2 /  42.2
//     14336 x 4096   M 32: 14.8 / 20.7 / 24.9   M 64: 21.9 / 39.4 /  45.2
//     16384 x 16384  M 32: 56.0 / 68.7 / 96.7   M 64: 84.1 /  121 /   172
enum QuantKernel { kFewColumns, kRows16, kRows32, kRows64 };
QuantKernel quant_choice(int64_t M, int64_t N, int cu_count)
{
    const int64_t tiles = cdiv(N, 16), shared = cdiv(N, 64), cus = std::max(cu_count, 1);
    const double cost[] = {1.7 * (double)cdiv(tiles * cdiv(M, 16), 2 * cus), 2.5 * (double)cdiv(shared * cdiv(M, 16), cus),
                           3.2 * (double)cdiv(shared * cdiv(M, 32), cus), 5.0 * (double)cdiv(shared * cdiv(M, 64), cus)};
    return (QuantKernel)(std::min_element(cost, cost + 4) - cost);
}

template <int DT, int GS>
void launch_quant(const QuantParams &p, int cu_count, hipStream_t s)
{
    using namespace xquant_dev;
    auto launch = [&](auto kernel, int r, int wn, int wk, int ct) {
        hipLaunchKernelGGL(kernel, dim3(cdiv(p.N, 16 * wn * ct), cdiv(p.M, r)), dim3(64 * wn * wk), 0, s, p);
    };
    // a lane's row of weights starts at most 31 leading dimensions from its wave's first
    if (p.ldq > (int64_t)1 << 27)
        return launch(quant_kernel<DT, 16, 1, 4, 1, 2, GS, int64_t>, 16, 1, 4, 1);
    if (p.M <= 2 && p.N <= 16 * 512)
        return launch(quant_kernel<DT, 2, 1, 8, 1, 2, GS, uint32_t>, 2, 1, 8, 1);
    if (p.M <= 2)
        return launch(quant_kernel<DT, 2, 1, 4, 1, 2, GS, uint32_t>, 2, 1, 4, 1);
    switch (quant_choice(p.M, p.N, cu_count)) {
    case kFewColumns: return launch(quant_kernel<DT, 16, 1, 8, 1, 2, GS, uint32_t>, 16, 1, 8, 1);
    case kRows16: return launch(quant_kernel<DT, 16, 4, 4, 1, 2, GS, uint32_t>, 16, 4, 4, 1);
    case kRows32: return launch(quant_kernel<DT, 32, 2, 4, 2, 1, GS, uint32_t>, 32, 2, 4, 2);
    case kRows64: return launch(quant_kernel<DT, 64, 2, 4, 2, 1, GS, uint32_t>, 64, 2, 4, 2);
    }
}

template <int DT>
void launch_quant(const QuantParams &p, int cu_count, hipStream_t s)
{
    if (p.group == 32)
        launch_quant<DT, 32>(p, cu_count, s);
    else if (p.group == 64)
        launch_quant<DT, 64>(p, cu_count, s);
    else
        launch_quant<DT, 128>(p, cu_count, s);
}

int run_quant(xgemm_ctx *h, int64_t M, int64_t N, int64_t K, const void *x, int64_t ldx, const uint8_t *q, int64_t ldq,
              const void *scales, int64_t lds, const uint8_t *zeros, int64_t ldz, int64_t group, void *y, int64_t ldy,
              int dtype, int out, hipStream_t s)
{
    if (!h || (dtype != XGEMM_BF16 && dtype != XGEMM_FP16) || (out != XGEMM_OUT_FP32 && out != XGEMM_OUT_SAME))
        return XGEMM_ERR_INVALID_ARG;
    if (group != 32 && group != 64 && (group < 128 || group % 128 != 0 || group > kMaxDim))
        return XGEMM_ERR_INVALID_ARG;
    if (!dims_ok(M, K, ldx) || !dims_ok(M, N, ldy) || N < 0 || K < 0)
        return XGEMM_ERR_INVALID_ARG;
    const int64_t G = cdiv(K, group);
    if (!dims_ok(N, cdiv(K, 2), ldq) || !dims_ok(N, G, lds) || (zeros && !dims_ok(N, G, ldz)))
        return XGEMM_ERR_INVALID_ARG;
    h->last_error[0] = '\0';
    if (M == 0 || N == 0)
        return XGEMM_OK;
    if (!y || (K > 0 && (!x || !q || !scales)))
        return XGEMM_ERR_INVALID_ARG;
    QuantParams p;
    p.x = (const uint16_t *)x;
    p.q = q;
    p.s = (const uint16_t *)scales;
    p.z = zeros;
    p.y = y;
    p.ldx = ldx;
    p.ldq = ldq;
    p.lds = lds;
    p.ldz = ldz;
    p.ldy = ldy;
    p.N = (int)N;
    p.K = (int)K;
    p.group = (int)std::min<int64_t>(group, kMaxDim - 128);   // (beyond K every group is the one group)
    p.out16 = out == XGEMM_OUT_SAME;
    // (a grid has at most 65535 rows of workgroups)
    constexpr int64_t kRows = 65535 * 2;
    for (int64_t m = 0; m < M; m += kRows) {
        p.M = (int)std::min(kRows, M - m);
        p.x = (const uint16_t *)x + m * ldx;
        p.y = (char *)y + m * ldy * (p.out16 ? 2 : 4);
        if (dtype == XGEMM_BF16)
            launch_quant<0>(p, h->cu_count, s);
        else
            launch_quant<1>(p, h->cu_count, s);
    }
    return launch_status(h, "quant launch");
}

// ---------------------------------------------------------------------------
// layer of experts
// ---------------------------------------------------------------------------

using xexperts_dev::ExpertsParams;

// R: tokens the launch provides for; UN x UK and WN x WK: waves over columns
// and over k in the two launches.
template <int DT, int R, int PL, int UN, int UK, int WN, int WK>
void launch_experts(const ExpertsParams &p, hipStream_t s)
{
    using namespace xexperts_dev;
    const bool odd = ((int64_t)((uintptr_t)p.up >> 1) | p.ldu | p.su) & 1;   // rows of up at 2 mod 4
    const dim3 up_grid(cdiv(p.I, 16 * UN), p.slots), up_block(64 * UN * UK);
    if (p.slots > 0 && odd)
        hipLaunchKernelGGL((route_up<DT, R, PL, UN, UK, true>), up_grid, up_block, 0, s, p);
    else if (p.slots > 0)
        hipLaunchKernelGGL((route_up<DT, R, PL, UN, UK, false>), up_grid, up_block, 0, s, p);
    const dim3 grid(cdiv(p.H, 16 * WN), p.parts), block(64 * WN * WK);
    const int lds = down_sum_lds(p.T * p.top, p.slots);
    if (p.I % 8 == 0)
        hipLaunchKernelGGL((down_sum<DT, R, PL, WN, WK, 0>), grid, block, lds, s, p);
    else if (p.I > 16)
        hipLaunchKernelGGL((down_sum<DT, R, PL, WN, WK, 1>), grid, block, lds, s, p);
    else if constexpr (R == 64)
        hipLaunchKernelGGL((down_sum<DT, R, PL, WN, WK, 2>), grid, block, lds, s, p);
}

// Whether the waves of a workgroup of the second launch take ranges of their
// own (16 columns, all the tokens' h) or columns of the same range (64).
// Ranges of their own are faster where launches and joins count, columns where
// the bytes do.  Microseconds, own ranges / columns: 7 tokens, 3 of 13 of 1000 x
// 776 23.0 / 28.0; 8 tokens, 4 of 16 of 1024 x 512 20.2 / 25.5; 5 tokens, 6 of 64 of 1024
// x 1024 42.8 / 48.4; 4 tokens, 8 of 64 of 2048 x 768 57.7 / 57.3; 8 tokens, 6 of
// 64 of 2048 x 1408 134 / 128; 12 tokens, 8 of 128 of 2048 x 768 152 / 149.  (The
// number of pairs stands for the bytes: with few of them and large experts, or
// many and small ones, the other side would gain 8 tokens, 2 of 8 of 4096 x
// 14336 462 / 440, and 16 tokens, 4 of 16 of 1024 x 512 21.3 / 26.6.)
bool experts_own_ranges(int64_t T, int64_t top, int64_t I)
{
    return I >= 16 && (T <= 2 || (T <= 16 && T * top <= 32));
}

// Parts that the second launch cuts the slots' inner dimensions into, with a
// counter for the workgroups of each: two workgroups a CU where waves share
// columns, one where they take ranges of their own, and for one or two tokens,
// whose 16 waves already are 16 ranges, half of one where the columns give fewer
// than a quarter.  (6 of 64 experts of 1008 x 1408, 63 workgroups of columns: one
// part 24.7 us, two 22.6, four 21.7; 6 of 64 of 2048 x 1408, 128: 32.6, 31.1, 32.0;
// 2 of 8 of 4096 x 14336, 256: 124, 127, 127.)  A part is at least four units a
// wave: 64 tokens, 2 of 8 of 512 x 512 24.9 us, with two units 30.5, with eight
// 23.5; 5 tokens, 6 of 16 of 512 x 640 19.2, 18.4 and 22.0; one token, 2 of 8 of
// 768 x 4096 19.1, 17.6 and 21.2.
int experts_parts(int64_t T, int64_t top, int64_t H, int64_t I, int64_t slots, int64_t Ip, int cu_count)
{
    using namespace xexperts_dev;
    const bool own = experts_own_ranges(T, top, I);
    const int waves = T <= 2 ? 16 : 8;
    const int64_t blocks = cdiv(H, own ? 16 : 64), units = slots * (Ip / kDownUnit);
    if (blocks > (int64_t)(xgemm_host::kWsPrefix / sizeof(int)))
        return 1;
    const int64_t want = !own ? cdiv(2 * (int64_t)cu_count, blocks)
                       : T > 2 ? cdiv((int64_t)cu_count, blocks)
                               : blocks * 4 < cu_count ? cdiv((int64_t)cu_count / 2, blocks) : 1;
    return (int)std::max<int64_t>(1, std::min({want, units / (own ? 4 * waves : 4), (int64_t)kMaxParts}));
}

template <int DT, int PL>
void launch_experts(const ExpertsParams &p, hipStream_t s)
{
    // (few inner columns are built for 64 tokens only)
    if (p.I < 16)
        launch_experts<DT, 64, PL, 4, 1, 4, 1>(p, s);
    else if (p.T <= 2)
        launch_experts<DT, 2, PL, 1, 8, 1, 16>(p, s);
    else if (experts_own_ranges(p.T, p.top, p.I))
        launch_experts<DT, 16, PL, 1, 4, 1, 8>(p, s);
    else if (p.T <= 16)
        launch_experts<DT, 16, PL, 1, 4, 4, 1>(p, s);
    else if (p.T <= 32)
        launch_experts<DT, 32, PL, 4, 1, 4, 1>(p, s);
    else
        launch_experts<DT, 64, PL, 4, 1, 4, 1>(p, s);
}

int run_experts(xgemm_ctx *h, int64_t T, int64_t E, int64_t top, int64_t H, int64_t I, const void *x, int64_t ldx,
                const float *scores, int64_t lds, const void *up, int64_t ldu, int64_t su, const void *down,
                int64_t ldd, int64_t sd, void *y, int64_t ldy, int renormalize, int dtype, int out, hipStream_t s)
{
    using namespace xexperts_dev;
    if (!h || (dtype != XGEMM_BF16 && dtype != XGEMM_FP16) || (out != XGEMM_OUT_FP32 && out != XGEMM_OUT_SAME) ||
        (renormalize != 0 && renormalize != 1))
        return XGEMM_ERR_INVALID_ARG;
    if (E < 1 || E > XGEMM_EXPERTS_MAX || top < 1 || top > XGEMM_EXPERTS_MAX_TOP || top > E)
        return XGEMM_ERR_INVALID_ARG;
    // (2 I rows of up; the inner dimension padded stays below 2^31)
    if (!dims_ok(T, H, ldx) || !dims_ok(T, E, lds) || !dims_ok(T, H, ldy) || I < 0 || I > kMaxDim / 4 ||
        !dims_ok(2 * I, H, ldu) || !dims_ok(H, I, ldd) || su < 0 || sd < 0 || H > kMaxDim - 16 * kUpUnit)
        return XGEMM_ERR_INVALID_ARG;
    if ((double)E * (double)su > 9.0e18 || (double)E * (double)sd > 9.0e18)
        return XGEMM_ERR_INVALID_ARG;
    h->last_error[0] = '\0';
    if (T == 0 || H == 0)
        return XGEMM_OK;
    if (!x || !scores || !y || (I > 0 && (!up || !down)))
        return XGEMM_ERR_INVALID_ARG;
    ExpertsParams p;
    p.scores = scores;
    p.up = (const uint16_t *)up;
    p.down = (const uint16_t *)down;
    p.ldx = ldx;
    p.lds = lds;
    p.ldu = ldu;
    p.su = su;
    p.ldd = ldd;
    p.sd = sd;
    p.ldy = ldy;
    p.E = (int)E;
    p.top = (int)top;
    p.H = (int)H;
    p.I = (int)I;
    p.Ip = (int)(cdiv(I, kPad) * kPad);
    p.renormalize = renormalize && I > 0;
    p.out16 = out == XGEMM_OUT_SAME;
    const int parts_of_h = dtype == XGEMM_FP16 && p.out16 ? 2 : 3;
    // tokens in chunks of at most kMaxTokens, each in the same workspace
    const int64_t most = std::min<int64_t>(T, kMaxTokens), most_slots = std::min(most * top, E);
    if ((double)most * (double)top * (double)p.Ip * 6.0 > 9.0e15)
        return XGEMM_ERR_INVALID_ARG;
    size_t bytes = 0;
    auto take = [&](size_t n) {
        const size_t at = bytes;
        bytes += cdiv(n, 256) * 256;
        return at;
    };
    const size_t at_expert = take(most_slots * sizeof(int)), at_count = take(most_slots * sizeof(int));
    const size_t at_pair = take(most_slots * kMaxTokens * sizeof(uint16_t));
    const size_t at_weight = take(most * top * sizeof(float));
    const size_t at_h = take((size_t)most * top * p.Ip * 2 * parts_of_h);
    const size_t at_scale = take(dtype == XGEMM_FP16 ? (size_t)most * top * (p.Ip / 16) : 0);
    // partial sums of the chunk that has the most of them: a full one or the last
    auto chunk = [&](int64_t tokens) {
        const int64_t slots = I > 0 ? std::min(tokens * top, E) : 0;   // (without inner columns y is zero)
        return std::pair<int64_t, int64_t>(slots, experts_parts(tokens, top, H, I, slots, p.Ip, h->cu_count));
    };
    size_t sums = 0;
    for (const int64_t tokens : {most, (T - 1) % kMaxTokens + 1})
        if (const int64_t parts = chunk(tokens).second; parts > 1)
            sums = std::max(sums, (size_t)(parts * tokens * cdiv(H, 64) * 64) * sizeof(float));
    const size_t at_part = take(sums);
    const int rc = xgemm_host::acquire_workspace(h, bytes, s);
    if (rc != XGEMM_OK)
        return rc;
    char *const ws = (char *)h->workspace + xgemm_host::kWsPrefix;
    p.expert = (int *)(ws + at_expert);
    p.count = (int *)(ws + at_count);
    p.pair = (uint16_t *)(ws + at_pair);
    p.weight = (float *)(ws + at_weight);
    p.h = (uint16_t *)(ws + at_h);
    p.scale = (int8_t *)(ws + at_scale);
    p.part = (float *)(ws + at_part);
    p.done = (int *)h->workspace;
    for (int64_t t = 0; t < T; t += kMaxTokens) {
        p.T = (int)std::min<int64_t>(kMaxTokens, T - t);
        const auto [slots, parts] = chunk(p.T);
        p.slots = (int)slots;
        p.parts = (int)parts;
        p.x = (const uint16_t *)x + t * ldx;
        p.scores = scores + t * lds;
        p.y = (char *)y + t * ldy * (p.out16 ? 2 : 4);
        if (dtype == XGEMM_BF16)
            launch_experts<0, 3>(p, s);
        else
            parts_of_h == 2 ? launch_experts<1, 2>(p, s) : launch_experts<1, 3>(p, s);
    }
    const int launched = launch_status(h, "experts launch");
    const int released = xgemm_host::release_workspace(h, s);
    return launched != XGEMM_OK ? launched : released;
}

// ---------------------------------------------------------------------------
// log probabilities
// ---------------------------------------------------------------------------

using xlogprob_dev::GradParams;
using xlogprob_dev::LogprobParams;

constexpr int64_t kMaxVocab = (int64_t)1 << 30;
constexpr int64_t kGridRows = 65535;   // rows of workgroups in a grid

bool logits_ok(int64_t R, int64_t V, int64_t ld, int dtype)
{
    return (dtype == XGEMM_BF16 || dtype == XGEMM_FP16 || dtype == XGEMM_FP32) && V >= 1 && V <= kMaxVocab &&
           dims_ok(R, V, ld);
}

template <int DT>
void launch_logprob(const LogprobParams &p, int64_t rows, hipStream_t s)
{
    const dim3 grid(p.parts, (unsigned)rows), block(xlogprob_dev::kThreads);
    if (p.top > 0)
        hipLaunchKernelGGL((xlogprob_dev::logprob_rows<DT, true>), grid, block, 0, s, p);
    else
        hipLaunchKernelGGL((xlogprob_dev::logprob_rows<DT, false>), grid, block, 0, s, p);
}

int run_logprob(xgemm_ctx *h, int64_t R, int64_t V, const void *logits, int64_t ldl, const int64_t *targets, int64_t top,
                float *logprob, float *lse, float *entropy, float *top_logprob, int64_t *top_id, int dtype,
                hipStream_t s)
{
    using namespace xlogprob_dev;
    if (!h || !logits_ok(R, V, ldl, dtype) || top < 0 || top > XGEMM_LOGPROB_MAX_TOP || top > V)
        return XGEMM_ERR_INVALID_ARG;
    h->last_error[0] = '\0';
    if (R == 0)
        return XGEMM_OK;
    if (!logits || (logprob && !targets) || (top > 0 && (!top_logprob || !top_id)))
        return XGEMM_ERR_INVALID_ARG;
    LogprobParams p;
    p.logits = logits;
    p.targets = targets;
    p.logprob = logprob;
    p.lse = lse;
    p.entropy = entropy;
    p.top_logprob = top_logprob;
    p.top_id = top_id;
    p.ld = ldl;
    p.V = (int)V;
    p.top = (int)top;
    // few rows are cut into parts of at least a batch a wave, for two workgroups
    // a CU
    constexpr int64_t kPart = kWaves * kBatch;
    int64_t parts = std::min({2 * (int64_t)h->cu_count / R, cdiv(V, kPart), (int64_t)kMaxParts});
    parts = std::max<int64_t>(parts, 1);
    p.part_len = (int)(cdiv(cdiv(V, parts), kBatch) * kBatch);   // (only the last part ends inside a batch)
    p.parts = (int)cdiv(V, p.part_len);
    p.stat = nullptr;
    p.best = nullptr;
    p.count = nullptr;
    if (p.parts > 1) {
        const size_t stat_bytes = cdiv(R * p.parts * sizeof(Stats), 256) * 256;
        const int rc = xgemm_host::acquire_workspace(h, stat_bytes + R * p.parts * top * sizeof(uint64_t), s);
        if (rc != XGEMM_OK)
            return rc;
        char *const ws = (char *)h->workspace + xgemm_host::kWsPrefix;
        p.count = (int *)h->workspace;   // (parts > 1 only for R up to the number of CUs)
        p.stat = (Stats *)ws;
        p.best = (uint64_t *)(ws + stat_bytes);
    }
    for (int64_t r = 0; r < R; r += kGridRows) {
        p.row0 = r;
        const int64_t rows = std::min(kGridRows, R - r);
        if (dtype == XGEMM_BF16)
            launch_logprob<0>(p, rows, s);
        else if (dtype == XGEMM_FP16)
            launch_logprob<1>(p, rows, s);
        else
            launch_logprob<2>(p, rows, s);
    }
    const int launched = launch_status(h, "logprob launch");
    const int released = p.parts > 1 ? xgemm_host::release_workspace(h, s) : XGEMM_OK;
    return launched != XGEMM_OK ? launched : released;
}

int run_logprob_grad(xgemm_ctx *h, int64_t R, int64_t V, const void *logits, int64_t ldl, const int64_t *targets,
                     const float *lse, const float *entropy, const float *d_logprob, const float *d_entropy,
                     const float *d_lse, void *dlogits, int64_t ldd, int dtype, hipStream_t s)
{
    using namespace xlogprob_dev;
    if (!h || !logits_ok(R, V, ldl, dtype) || !logits_ok(R, V, ldd, dtype))
        return XGEMM_ERR_INVALID_ARG;
    h->last_error[0] = '\0';
    if (R == 0)
        return XGEMM_OK;
    if (!logits || !dlogits || !lse || (d_logprob && !targets) || (d_entropy && !entropy))
        return XGEMM_ERR_INVALID_ARG;
    GradParams p;
    p.logits = logits;
    p.targets = targets;
    p.lse = lse;
    p.entropy = entropy;
    p.d_logprob = d_logprob;
    p.d_entropy = d_entropy;
    p.d_lse = d_lse;
    p.out = dlogits;
    p.ld = ldl;
    p.ldo = ldd;
    p.V = (int)V;
    // (a workgroup that sums its row takes up to 8 spans, as many as leave 4
    // workgroups a CU: one row of 131072 fp32 12 us, in one workgroup 35)
    const int64_t spans = cdiv(V, kGradSpan), shared = R * spans / (4 * std::max(h->cu_count, 1));
    p.group = (int)(dlogits == logits ? spans : std::min<int64_t>(std::max<int64_t>(shared, 1), 8));
    for (int64_t r = 0; r < R; r += kGridRows) {
        p.row0 = r;
        const dim3 grid(spans, (unsigned)std::min(kGridRows, R - r)), block(kGradThreads);
        if (dtype == XGEMM_BF16)
            hipLaunchKernelGGL(logprob_grad<0>, grid, block, 0, s, p);
        else if (dtype == XGEMM_FP16)
            hipLaunchKernelGGL(logprob_grad<1>, grid, block, 0, s, p);
        else
            hipLaunchKernelGGL(logprob_grad<2>, grid, block, 0, s, p);
    }
    return launch_status(h, "logprob gradient launch");
}

}  // namespace

extern "C" {

int xgemm_logprob_run(xgemm_handle_t h, int64_t R, int64_t V, const void *logits, int64_t ldl, const int64_t *targets,
                      int64_t top, float *logprob, float *lse, float *entropy, float *top_logprob, int64_t *top_id,
                      int dtype, void *stream)
{
    return run_logprob(h, R, V, logits, ldl, targets, top, logprob, lse, entropy, top_logprob, top_id, dtype,
                       (hipStream_t)stream);
}

int xgemm_logprob_grad(xgemm_handle_t h, int64_t R, int64_t V, const void *logits, int64_t ldl, const int64_t *targets,
                       const float *lse, const float *entropy, const float *d_logprob, const float *d_entropy,
                       const float *d_lse, void *dlogits, int64_t ldd, int dtype, void *stream)
{
    return run_logprob_grad(h, R, V, logits, ldl, targets, lse, entropy, d_logprob, d_entropy, d_lse, dlogits, ldd,
                            dtype, (hipStream_t)stream);
}

int xgemm_experts_run(xgemm_handle_t h, int64_t T, int64_t E, int64_t top, int64_t H, int64_t I, const void *x,
                      int64_t ldx, const float *scores, int64_t lds, const void *up, int64_t ldu, int64_t stride_up,
                      const void *down, int64_t ldd, int64_t stride_down, void *y, int64_t ldy, int renormalize,
                      int dtype, int out, void *stream)
{
    return run_experts(h, T, E, top, H, I, x, ldx, scores, lds, up, ldu, stride_up, down, ldd, stride_down, y, ldy,
                       renormalize, dtype, out, (hipStream_t)stream);
}

int xgemv_quant_run(xgemm_handle_t h, int64_t M, int64_t N, int64_t K, const void *x, int64_t ldx, const uint8_t *q,
                    int64_t ldq, const void *scales, int64_t lds, const uint8_t *zeros, int64_t ldz, int64_t group,
                    void *y, int64_t ldy, int dtype, int out, void *stream)
{
    return run_quant(h, M, N, K, x, ldx, q, ldq, scales, lds, zeros, ldz, group, y, ldy, dtype, out,
                     (hipStream_t)stream);
}

}  // extern "C"
