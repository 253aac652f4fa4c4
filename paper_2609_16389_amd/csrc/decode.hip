// Host side of the operators around a decoding step: argument checks, launch
// selection and launches.  The C ABI is declared in include/xgemm.h.
#include "context.hpp"
#include "quant_kernel.hpp"

#include <algorithm>
#include <type_traits>

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

template <int DT, int MT, int NT, bool SMALL>
void launch_quant(const QuantParams &p, hipStream_t s)
{
    hipLaunchKernelGGL((xquant_dev::quant_kernel<DT, MT, NT, SMALL>), dim3(cdiv(p.N, 16 * NT), cdiv(p.M, 16 * MT)),
                       dim3(xquant_dev::kThreads), 0, s, p);
}

template <int DT, bool SMALL>
void launch_quant(const QuantParams &p, hipStream_t s)
{
    if (p.M <= 16)
        launch_quant<DT, 1, 1, SMALL>(p, s);
    else if (p.M <= 32)
        launch_quant<DT, 2, 2, SMALL>(p, s);
    else
        launch_quant<DT, 4, 2, SMALL>(p, s);
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
    p.group = (int)std::min<int64_t>(group, kMaxDim - 128);
    p.out16 = out == XGEMM_OUT_SAME;
    // (a grid has at most 65535 rows of workgroups)
    constexpr int64_t kRows = 65535 * 16;
    for (int64_t m = 0; m < M; m += kRows) {
        p.M = (int)std::min(kRows, M - m);
        p.x = (const uint16_t *)x + m * ldx;
        p.y = (char *)y + m * ldy * (p.out16 ? 2 : 4);
        const bool small = group < 128;
        if (dtype == XGEMM_BF16)
            small ? launch_quant<0, true>(p, s) : launch_quant<0, false>(p, s);
        else
            small ? launch_quant<1, true>(p, s) : launch_quant<1, false>(p, s);
    }
    return launch_status(h, "quant launch");
}

}  // namespace

extern "C" {

int xgemv_quant_run(xgemm_handle_t h, int64_t M, int64_t N, int64_t K, const void *x, int64_t ldx, const uint8_t *q,
                    int64_t ldq, const void *scales, int64_t lds, const uint8_t *zeros, int64_t ldz, int64_t group,
                    void *y, int64_t ldy, int dtype, int out, void *stream)
{
    return run_quant(h, M, N, K, x, ldx, q, ldq, scales, lds, zeros, ldz, group, y, ldy, dtype, out,
                     (hipStream_t)stream);
}

}  // extern "C"
