// Host side of the products whose ends are fused: argument checks, layouts,
// launch selection and launches.  The C ABI is declared in include/xgemm.h.
#include "context.hpp"
#include "fused_cut.hpp"
#include "fused_ends.hpp"
#include "fused_rows.hpp"
#include "fused_tile.hpp"

#include <algorithm>

using xgemm_host::kMaxDim;
using namespace xfused_dev;
using namespace xfused_host;

namespace {

bool matrix_ok(int64_t rows, int64_t cols, int64_t ld)
{
    return rows >= 0 && cols >= 0 && rows < kMaxDim && cols < kMaxDim && ld >= cols && (double)rows * (double)ld <= 9.0e18;
}

bool sixteen(int dtype) { return dtype == XGEMM_BF16 || dtype == XGEMM_FP16; }

int launch_status(xgemm_ctx *h, const char *what)
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess)
        return XGEMM_OK;
    xgemm_host::set_error(h, what, e);
    return XGEMM_ERR_HIP;
}

// Places in the workspace, 256 bytes apart.
struct Space {
    size_t bytes = 0;
    size_t take(size_t n)
    {
        const size_t at = bytes;
        bytes += (size_t)cdiv((int64_t)n, 256) * 256;
        return at;
    }
};

// An operand as the tiles read it: in place, or as a copy whose rows are whole
// 16-byte chunks.
struct Matrix {
    const char *p;
    int64_t rows, cols, ld;   // bytes
    bool ragged;              // in place only the staged tiles read it
    bool copied;
    int times;                // the copy holds the rows so many times, one after another
    const HeadRows *part;     // a copy anyhow, in which rows that take no part in this are zeros; null: all do
    size_t at;                // of the copy

    Matrix(const void *data, int64_t r, int64_t c, int64_t leading, int size, int n = 1, const HeadRows *of = nullptr)
        : p((const char *)data), rows(r), cols(c * size), ld(r > 1 ? leading * size : up_to(c * size, 16)), copied(false),
          times(n), part(of), at(0)
    {
        ragged = rows > 0 && cols > 0 && (((uintptr_t)p | ld | cols) % 16 != 0 || ld > kMaxStep);
    }
    // Room for the copy, where there has to be one.
    void reserve(bool staged, Space &ws)
    {
        copied = (ragged && !staged) || ((times > 1 || part) && rows > 0 && cols > 0);
        if (copied)
            at = ws.take((size_t)(rows * times) * up_to(cols, 16));
    }
    // Microseconds that the copy takes: 2.8 TB/s read and written, the launch.
    double cost() const { return ragged ? (double)rows * (double)cols * 2.0 / 2.8e6 : 0.0; }
    // The copies of up to two operands, into the workspace: launched, or, if `later`
    // is given and they are small, left to another launch, which gets as many blocks
    // for them as this returns.
    static int place(Matrix &a, Matrix &b, char *ws, hipStream_t s, CopyParams *later = nullptr)
    {
        CopyParams p{};
        int n = 0;
        for (Matrix *const m : {&a, &b})
            if (m->copied) {
                const int64_t chunks = cdiv(m->cols, 16);
                p.m[n++] = {m->p, ws + m->at, m->ld, m->cols, m->rows, chunks, cdiv(m->rows, 4), m->times, m->part != nullptr};
                if (m->part)
                    p.of = *m->part;
                m->p = ws + m->at;
                m->ld = chunks * 16;
            }
        // (a launch has at most 2^32 threads: what is larger goes in pieces of rows)
        constexpr int64_t most = (int64_t)1 << 22;   // blocks
        const int64_t blocks = p.m[0].blocks + p.m[1].blocks;
        if (blocks <= most) {
            if (later)
                *later = p;
            else if (n > 0)
                hipLaunchKernelGGL(copy_rows, dim3(blocks), dim3(256), 0, s, p);
            return (int)blocks;
        }
        if (later)
            *later = CopyParams{};
        for (int k = 0; k < n; ++k) {
            const auto whole = p.m[k];
            constexpr int64_t some = most * 4;
            for (int t = 0; t < whole.times; ++t)
                for (int64_t r = 0; r < whole.rows; r += some) {
                    CopyParams one{};
                    const int64_t rows = std::min(some, whole.rows - r);
                    one.m[0] = {whole.from + r * whole.ld, whole.to + (t * whole.rows + r) * whole.chunks * 16, whole.ld,
                                whole.bytes, rows, whole.chunks, cdiv(rows, 4), 1, whole.part};
                    one.of = p.of.from(r);
                    hipLaunchKernelGGL(copy_rows, dim3(one.m[0].blocks), dim3(256), 0, s, one);
                }
        }
        return 0;
    }
};

// ---------------------------------------------------------------------------
// products
// ---------------------------------------------------------------------------

// The cut of a product that reads a and b: with copies of what is ragged, or
// through the staged tiles, whichever takes less.
template <class F>
Cut cut_with(const Matrix &a, const Matrix &b, F cut)
{
    const Cut c = cut(false);
    if ((!a.ragged && !b.ragged) || b.cols < 16)   // (the staged tiles read 16 bytes of a row at a time)
        return c;
    const Cut staged = cut(true);
    return takes_less(staged, c, 4.0 + a.cost() + b.cost()) ? staged : c;
}

template <int TYPE, int LA, int LB, class End>
void launch_tiles(TileParams p, const typename End::Params &e, TileKind tile, bool staged, hipStream_t s)
{
    p.tiles_m = (int)cdiv(p.M, kTileRows[tile]);
    p.tiles_n = (int)cdiv(End::kGated ? 2 * (int64_t)p.N : p.N, kTileCols[tile]);
    p.group_m = 8;
    p.grid = p.tiles_m * p.tiles_n * p.split;
    auto launch = [&](auto kernel, int threads) { hipLaunchKernelGGL(kernel, dim3(p.grid), dim3(threads), 0, s, p, e); };
    if (tile == kTile256)
        return launch(tile_product<TYPE, LA, LB, 256, 256, 2, 4, 2, false, End>, 512);
    if constexpr (End::kStages && LA == kAlong && LB == kAlong) {
        if (staged)
            return launch(tile_product<TYPE, LA, LB, 64, 128, 1, 4, 2, true, End>, 256);
    }
    if (tile == kTile128)
        return launch(tile_product<TYPE, LA, LB, 128, 128, 2, 2, 2, false, End>, 256);
    if constexpr (LA == kAlong)
        launch(tile_product<TYPE, LA, LB, 64, 128, 1, 4, 3, false, End>, 256);
}

// One product of rows [.., .. + p.M) of the result, its sums' parts in `part`.
template <int TYPE, int LA, int LB, class End>
void launch_product(TileParams p, const typename End::Params &e, const Cut &c, char *part, hipStream_t s)
{
    p.split = c.split;
    p.chunk = c.chunk;
    if constexpr (End::kJoins) {
        if (c.split * c.halves > 1) {
            typedef PartEnd<TYPE, End::kGated> Part;
            launch_tiles<TYPE, LA, LB, Part>(p, typename Part::Params{part, (int)c.ld}, c.tile, c.staged, s);
            // (the second half's rows follow the first's: a part of their own)
            const int64_t quads = cdiv(p.N, 4), M = p.M / c.halves;
            hipLaunchKernelGGL(join_parts<End>, dim3(cdiv(M * quads, 256)), dim3(256), 0, s, part, c.split * c.halves,
                               (int)M, p.N, (int)c.ld, quads, e);
            return;
        }
    }
    launch_tiles<TYPE, LA, LB, End>(p, e, c.tile, c.staged, s);
}

// Whether rows can be read through LDS: 16-byte chunks, near enough.
bool whole_chunks(const RowsParams &p)
{
    const int64_t x = p.M > 1 ? (int64_t)(uintptr_t)p.x | p.ldx : (int64_t)(uintptr_t)p.x;
    const int64_t w = (int64_t)((uintptr_t)p.w | (uintptr_t)p.w2) | p.ldw;
    return (w | x | p.K) % 16 == 0 && p.ldw <= kMaxStep && (p.M == 1 || p.ldx <= kMaxStep);
}

// Whether the kernels for few rows take a product: through LDS up to 16; rows at any
// address up to 4, while the weights are few.  (Microseconds of one row, 12 rows of
// weights at odd addresses, in these kernels / in tiles: 8-bit 5003 x 2047 9.0, 11.6 /
// 10.7, 11.0; gated 2731 x 1001 9.0 / 10.0; gated 5003 x 2047 25.2, 31.1 / 19.4, 20.5.)
template <int TYPE, class End>
bool few_rows(const RowsParams &p)
{
    return whole_chunks(p) ? p.M <= 16 : p.M <= 4 && (int64_t)p.N * p.K * (End::kGated ? 2 : 1) <= (int64_t)1 << 24;
}

template <int TYPE, class End>
void launch_rows(RowsParams p, const typename End::Params &e, int cu_count, hipStream_t s)
{
    constexpr bool kGated = End::kGated;
    if (p.M == 1)
        p.ldx = 0;
    if (whole_chunks(p)) {
        const dim3 grid(std::min<int64_t>(cdiv(p.N, 16), cu_count)), block(64 * kStreamWaves);
        if (p.M <= 4)
            hipLaunchKernelGGL((rows_stream<TYPE, End, 1, kGated ? 4 : 6, -1>), grid, block, 0, s, p, e);
        else
            hipLaunchKernelGGL((rows_stream<TYPE, End, 4, kGated ? 3 : 4, -1>), grid, block, 0, s, p, e);
        return;
    }
    const bool odd = ((int64_t)((uintptr_t)p.w | (uintptr_t)p.w2 | (uintptr_t)p.x) | p.ldw | p.ldx) & 3;
    const dim3 grid(cdiv(p.N, 16)), block(64 * 4);
    if (odd)
        hipLaunchKernelGGL((rows_product<TYPE, End, 4, true>), grid, block, 0, s, p, e);
    else
        hipLaunchKernelGGL((rows_product<TYPE, End, 4, false>), grid, block, 0, s, p, e);
}

TileParams tile_params(const Matrix &A, const Matrix &B, int64_t M, int64_t N, int64_t K)
{
    TileParams p{};
    p.A = A.p;
    p.B = p.B2 = B.p;
    p.lda = A.ld;
    p.ldb = B.ld;
    p.M = (int)M;
    p.N = (int)N;
    p.K = (int)K;
    return p;
}

// out = a product of 16-bit operands (rows of A and out in launches of
// kRowsLaunch).
template <int LA, int LB>
void product(int dtype, TileParams p, StoreParams e, const Cut &c, char *part, hipStream_t s)
{
    const int64_t M = p.M;
    const char *const A = p.A;
    void *const out = e.out;
    const float *const add = e.add, *const raise = e.raise;
    for (int64_t m = 0; m < M; m += kRowsLaunch) {
        p.M = (int)std::min(kRowsLaunch, M - m);
        p.A = A + m * (LA == kAlong ? p.lda : 2);
        e.out = (char *)out + m * e.ld * (e.kind == kFp32 ? 4 : 2);
        e.add = add ? add + m * e.ld_add : nullptr;
        e.raise = raise ? raise + m : nullptr;
        if (dtype == XGEMM_BF16)
            launch_product<kBf16, LA, LB, StoreEnd>(p, e, c, part, s);
        else   // (rows of slopes are raised)
            launch_product<kFp16, LA, LB, StoreEndOf<LA == kAlong>>(p, e, c, part, s);
    }
}

// ---------------------------------------------------------------------------
// 8-bit products
// ---------------------------------------------------------------------------

bool real(int dtype) { return sixteen(dtype) || dtype == XGEMM_FP32; }

void launch_scale_rows(int dtype, int64_t R, int64_t K, const void *x, int64_t ldx, int8_t *q, int64_t ldq, int64_t padded,
                       float *scales, hipStream_t s)
{
    constexpr int64_t some = (int64_t)1 << 22;
    for (int64_t r = 0; r < R; r += some) {
        const dim3 grid(std::min(some, R - r)), block(256);
        const char *const from = (const char *)x + r * ldx * (dtype == XGEMM_FP32 ? 4 : 2);
        auto launch = [&](auto held, auto any) {
            hipLaunchKernelGGL(padded <= kHeld ? held : any, grid, block, 0, s, from, ldx, K, q + r * ldq, ldq, padded,
                               scales + r);
        };
        if (dtype == XGEMM_BF16)
            launch(scale_rows<kBf16, true>, scale_rows<kBf16, false>);
        else if (dtype == XGEMM_FP16)
            launch(scale_rows<kFp16, true>, scale_rows<kFp16, false>);
        else
            launch(scale_rows<kFp32, true>, scale_rows<kFp32, false>);
    }
}

int run_scaled_rows(xgemm_ctx *h, int64_t R, int64_t K, const void *x, int64_t ldx, int8_t *q, int64_t ldq, float *scales,
                    int dtype, hipStream_t s)
{
    if (!h || !real(dtype) || !matrix_ok(R, K, ldx) || !matrix_ok(R, K, ldq))
        return XGEMM_ERR_INVALID_ARG;
    h->last_error[0] = '\0';
    if (R == 0)
        return XGEMM_OK;
    if (!scales || (K > 0 && (!x || !q)))
        return XGEMM_ERR_INVALID_ARG;
    launch_scale_rows(dtype, R, K, x, ldx, q, ldq, K, scales, s);
    return launch_status(h, "scaled rows launch");
}

int run_scaled(xgemm_ctx *h, int64_t M, int64_t N, int64_t K, const void *x, int64_t ldx, const float *x_scales,
               const int8_t *w, int64_t ldw, const float *w_scales, void *y, int64_t ldy, int x_dtype, int y_dtype,
               hipStream_t s)
{
    if (!h || (x_dtype != XGEMM_INT8 && !real(x_dtype)) || !real(y_dtype))
        return XGEMM_ERR_INVALID_ARG;
    if (!matrix_ok(M, K, ldx) || !matrix_ok(N, K, ldw) || !matrix_ok(M, N, ldy) || M > kMaxRows || N > kMaxSide ||
        K > XGEMM_SCALED_MAX_K)
        return XGEMM_ERR_INVALID_ARG;
    h->last_error[0] = '\0';
    if (M == 0 || N == 0)
        return XGEMM_OK;
    const bool whole = x_dtype == XGEMM_INT8;
    if (!y || !w_scales || (K > 0 && (!x || !w)) || whole != (x_scales != nullptr))
        return XGEMM_ERR_INVALID_ARG;
    const int kind = y_dtype == XGEMM_FP32 ? kFp32 : y_dtype == XGEMM_FP16 ? kFp16 : kBf16;
    RowsParams few{(const char *)x, (const char *)w, nullptr, ldx, ldw, (int)M, (int)N, (int)K};
    if (!whole) {
        few.x = nullptr;   // (its 8-bit rows will lie in the workspace)
        few.ldx = up_to(K, 16);
    }
    if (K > 0 && few_rows<kInt8, ScaledEnd>(few)) {
        ScaledEnd::Params e{x_scales, w_scales, y, ldy, kind};
        // (one row becomes 8-bit within the product)
        const bool here = ((int64_t)(uintptr_t)w | ldw | K | (int64_t)(uintptr_t)x) % 16 == 0 && ldw <= kMaxStep &&
                          K * (x_dtype == XGEMM_FP32 ? 4 : 2) <= kQuantBytes;
        if (!whole && M == 1 && here) {
            few.x = (const char *)x;
            const dim3 grid(std::min<int64_t>(cdiv(N, 16), h->cu_count)), block(64 * kStreamWaves);
            if (x_dtype == XGEMM_BF16)
                hipLaunchKernelGGL((rows_stream<kInt8, ScaledEnd, 1, 6, kBf16>), grid, block, 0, s, few, e);
            else if (x_dtype == XGEMM_FP16)
                hipLaunchKernelGGL((rows_stream<kInt8, ScaledEnd, 1, 6, kFp16>), grid, block, 0, s, few, e);
            else
                hipLaunchKernelGGL((rows_stream<kInt8, ScaledEnd, 1, 6, kFp32>), grid, block, 0, s, few, e);
            return launch_status(h, "scaled product launch");
        }
        if (whole) {
            launch_rows<kInt8, ScaledEnd>(few, e, h->cu_count, s);
            return launch_status(h, "scaled product launch");
        }
        Space ws;
        const int64_t ld = up_to(K, 16);
        const size_t at_q = ws.take((size_t)(M * ld)), at_scales = ws.take((size_t)M * 4);
        const int rc = xgemm_host::acquire_workspace(h, ws.bytes, s);
        if (rc != XGEMM_OK)
            return rc;
        char *const base = (char *)h->workspace + xgemm_host::kWsPrefix;
        e.row_scale = (const float *)(base + at_scales);
        few.x = base + at_q;
        launch_scale_rows(x_dtype, M, K, x, ldx, (int8_t *)(base + at_q), ld, ld, (float *)(base + at_scales), s);
        launch_rows<kInt8, ScaledEnd>(few, e, h->cu_count, s);
        const int launched = launch_status(h, "scaled product launch");
        const int released = xgemm_host::release_workspace(h, s);
        return launched != XGEMM_OK ? launched : released;
    }
    Space ws;
    const int64_t padded = up_to(K, 16);
    const size_t at_q = ws.take(whole ? 0 : (size_t)M * padded), at_scales = ws.take(whole ? 0 : (size_t)M * 4);
    Matrix A(whole ? x : nullptr, whole ? M : 0, K, ldx, 1), B(w, N, K, ldw, 1);
    const Cut c = cut_with(A, B, [&](bool staged) {
        return cut_of(M, N, cdiv(padded, 128), false, false, true, staged, h->cu_count);
    });
    A.reserve(c.staged, ws);
    B.reserve(c.staged, ws);
    const size_t at_part = ws.take(part_bytes(c, M));
    if (ws.bytes > 0) {
        const int rc = xgemm_host::acquire_workspace(h, ws.bytes, s);
        if (rc != XGEMM_OK)
            return rc;
    }
    char *const base = ws.bytes > 0 ? (char *)h->workspace + xgemm_host::kWsPrefix : nullptr;
    Matrix::place(A, B, base, s);
    if (!whole) {
        A.p = base + at_q;
        A.ld = padded;
        launch_scale_rows(x_dtype, M, K, x, ldx, (int8_t *)A.p, padded, padded, (float *)(base + at_scales), s);
        x_scales = (const float *)(base + at_scales);
    }
    TileParams p = tile_params(A, B, M, N, c.staged ? K : padded);
    const Band band = band_of(c, M, N, cdiv(padded, 128), false, h->cu_count);
    for (int64_t m = 0; m < M; m += kRowsLaunch) {
        p.M = (int)std::min(kRowsLaunch, M - m);
        p.A = A.p + m * A.ld;
        ScaledEnd::Params e{x_scales + m, w_scales, (char *)y + m * ldy * (kind == kFp32 ? 4 : 2), ldy, kind};
        p.N = (int)band.body;
        launch_product<kInt8, kAlong, kAlong, ScaledEnd>(p, e, c, base + at_part, s);
        if (band.body < N) {   // (all rows are one launch)
            p.B += band.body * B.ld;
            p.N = (int)(N - band.body);
            e.col_scale += band.body;
            e.out = (char *)e.out + band.body * (kind == kFp32 ? 4 : 2);
            launch_product<kInt8, kAlong, kAlong, ScaledEnd>(p, e, band.rest, nullptr, s);
        }
    }
    const int launched = launch_status(h, "scaled product launch");
    const int released = ws.bytes > 0 ? xgemm_host::release_workspace(h, s) : XGEMM_OK;
    return launched != XGEMM_OK ? launched : released;
}

// ---------------------------------------------------------------------------
// gated feed-forward block
// ---------------------------------------------------------------------------

bool act_ok(int act) { return act == XGEMM_ACT_SILU || act == XGEMM_ACT_GELU || act == XGEMM_ACT_GELU_TANH; }

template <int DT>
void launch_gated(TileParams p, int64_t M, void *out, int64_t ld, int kind, int act, uint16_t *pre, int64_t ldp,
                  const Cut &c, const Band &band, char *part, hipStream_t s)
{
    const char *const A = p.A;
    const int64_t I = p.N;
    for (int64_t m = 0; m < M; m += kRowsLaunch) {
        p.M = (int)std::min(kRowsLaunch, M - m);
        p.A = A + m * p.lda;
        typename GatedEnd<DT>::Params e{(char *)out + m * ld * (kind == kFp32 ? 4 : 2), ld, kind, act,
                                        pre ? pre + m * ldp : nullptr, ldp, I};
        p.N = (int)band.body;
        launch_product<DT, kAlong, kAlong, GatedEnd<DT>>(p, e, c, part, s);
        if (band.body < I) {   // (all rows are one launch)
            p.B += band.body * p.ldb;
            p.B2 += band.body * p.ldb;
            p.N = (int)(I - band.body);
            e.out = (char *)e.out + band.body * (kind == kFp32 ? 4 : 2);
            e.pre = pre ? e.pre + band.body : nullptr;
            launch_product<DT, kAlong, kAlong, GatedEnd<DT>>(p, e, band.rest, nullptr, s);
        }
    }
}

int run_gated(xgemm_ctx *h, int64_t M, int64_t H, int64_t I, const void *x, int64_t ldx, const void *up, int64_t ldu,
              void *y, int64_t ldy, void *pre, int64_t ldp, int act, int dtype, int out, hipStream_t s)
{
    if (!h || !sixteen(dtype) || (out != XGEMM_OUT_FP32 && out != XGEMM_OUT_SAME) || !act_ok(act))
        return XGEMM_ERR_INVALID_ARG;
    if (H < 0 || I < 0 || M > kMaxRows || H > kMaxSide || I > kMaxSide / 2 || !matrix_ok(M, H, ldx) ||
        !matrix_ok(2 * I, H, ldu) || !matrix_ok(M, I, ldy) || (pre && !matrix_ok(M, 2 * I, ldp)))
        return XGEMM_ERR_INVALID_ARG;
    h->last_error[0] = '\0';
    if (M == 0 || I == 0)
        return XGEMM_OK;
    if (!y || (H > 0 && (!x || !up)))
        return XGEMM_ERR_INVALID_ARG;
    const int kind = out == XGEMM_OUT_FP32 ? kFp32 : dtype == XGEMM_BF16 ? kBf16 : kFp16;
    const RowsParams few{(const char *)x, (const char *)up, (const char *)up + I * ldu * 2, ldx * 2, ldu * 2,
                         (int)M, (int)I, (int)H * 2};
    if (H > 0 && few_rows<kBf16, GatedEnd<kBf16>>(few)) {
        if (dtype == XGEMM_BF16)
            launch_rows<kBf16, GatedEnd<kBf16>>(few, {y, ldy, kind, act, (uint16_t *)pre, ldp, I}, h->cu_count, s);
        else
            launch_rows<kFp16, GatedEnd<kFp16>>(few, {y, ldy, kind, act, (uint16_t *)pre, ldp, I}, h->cu_count, s);
        return launch_status(h, "gated launch");
    }
    Space ws;
    Matrix A(x, M, H, ldx, 2), B(up, 2 * I, H, ldu, 2);
    const Cut c = cut_with(A, B, [&](bool staged) {
        return cut_of(M, I, cdiv(H, 64), true, false, true, staged, h->cu_count);
    });
    A.reserve(c.staged, ws);
    B.reserve(c.staged, ws);
    const int64_t K = c.staged ? H : up_to(H, 8);
    const size_t at_part = ws.take(part_bytes(c, M));
    if (ws.bytes > 0) {
        const int rc = xgemm_host::acquire_workspace(h, ws.bytes, s);
        if (rc != XGEMM_OK)
            return rc;
    }
    char *const base = ws.bytes > 0 ? (char *)h->workspace + xgemm_host::kWsPrefix : nullptr;
    Matrix::place(A, B, base, s);
    TileParams p = tile_params(A, B, M, I, K);
    p.B2 = B.p + I * B.ld;
    const Band band = band_of(c, M, I, cdiv(H, 64), true, h->cu_count);
    if (dtype == XGEMM_BF16)
        launch_gated<kBf16>(p, M, y, ldy, kind, act, (uint16_t *)pre, ldp, c, band, base + at_part, s);
    else
        launch_gated<kFp16>(p, M, y, ldy, kind, act, (uint16_t *)pre, ldp, c, band, base + at_part, s);
    const int launched = launch_status(h, "gated launch");
    const int released = ws.bytes > 0 ? xgemm_host::release_workspace(h, s) : XGEMM_OK;
    return launched != XGEMM_OK ? launched : released;
}

int run_gated_grad(xgemm_ctx *h, int64_t M, int64_t H, int64_t I, const void *x, int64_t ldx, const void *up, int64_t ldu,
                   const void *pre, int64_t ldp, const void *d_y, int64_t ldd, void *d_x, int64_t ld_dx, void *d_up,
                   int64_t ld_dup, int act, int dtype, int out, hipStream_t s)
{
    if (!h || !sixteen(dtype) || (out != XGEMM_OUT_FP32 && out != XGEMM_OUT_SAME) || !act_ok(act))
        return XGEMM_ERR_INVALID_ARG;
    if (H < 0 || I < 0 || M > kMaxRows || H > kMaxSide || I > kMaxSide / 2 || (d_up && !matrix_ok(M, H, ldx)) ||
        (d_x && !matrix_ok(2 * I, H, ldu)) || !matrix_ok(M, 2 * I, ldp) || !matrix_ok(M, I, ldd) ||
        (d_x && !matrix_ok(M, H, ld_dx)) || (d_up && !matrix_ok(2 * I, H, ld_dup)))
        return XGEMM_ERR_INVALID_ARG;
    h->last_error[0] = '\0';
    // (d_x is M x H, d_up 2 I x H: empty products are zeros)
    const bool want_x = d_x && M > 0 && H > 0, want_up = d_up && I > 0 && H > 0;
    if (!want_x && !want_up)
        return XGEMM_OK;
    const bool some = M > 0 && I > 0;
    if (some && (!pre || !d_y || (want_x && !up) || (want_up && !x)))
        return XGEMM_ERR_INVALID_ARG;
    const int kind = out == XGEMM_OUT_FP32 ? kFp32 : dtype == XGEMM_BF16 ? kBf16 : kFp16;
    Space ws;
    const bool raised = dtype == XGEMM_FP16 && some;
    const size_t at_word = ws.take((1 + kMostBlocks) * 4);   // the slopes' inverse factor, the blocks' largest
    const int64_t units = M * cdiv(cdiv(I, 8), 64);
    const size_t at_unit = ws.take(raised ? (size_t)units * 4 : 0), at_raise = ws.take(raised ? (size_t)M * 4 : 0);
    const int64_t ld = slope_ld(2 * I);
    const int halves = M <= kTwoParts ? 2 : 1;
    const int64_t rows = M * halves;   // of slopes
    const size_t at_d = ws.take((size_t)rows * ld * 2);
    // (binary16: a copy of x anyhow, lowered as the slopes are raised)
    Matrix X(x, want_up && some && !raised ? M : 0, H, ldx, 2, halves), W(up, want_x && some ? 2 * I : 0, H, ldu, 2);
    X.reserve(false, ws);
    W.reserve(false, ws);
    const int64_t x_chunks = cdiv(H, 8);
    const size_t at_x = ws.take(raised && want_up ? (size_t)(rows * x_chunks) * 16 : 0);
    Cut cx = cut_of(rows, H, cdiv(ld, 64), false, false, true, false, h->cu_count);
    cx.halves = halves;
    const Cut cw = cut_of(2 * I, H, cdiv(rows, 64), false, true, true, false, h->cu_count);
    const size_t at_part = ws.take(std::max(want_x ? part_bytes(cx, rows) : 0, want_up ? part_bytes(cw, 2 * I) : 0));
    const int rc = xgemm_host::acquire_workspace(h, ws.bytes, s);
    if (rc != XGEMM_OK)
        return rc;
    char *const base = (char *)h->workspace + xgemm_host::kWsPrefix;
    CopyParams copies;
    const int copy_blocks = Matrix::place(X, W, base, s, &copies);
    float *const inverse = (float *)(base + at_word);
    GatedSlopeParams g;
    g.ldp = ldp;
    g.ldd = ldd;
    g.ld = ld;
    g.rest = halves > 1 ? M * ld : 0;
    g.I = (int)I;
    g.act = act;
    g.chunks = (int)cdiv(I, 8);
    g.inverse = inverse;
    g.most = (uint32_t *)(inverse + 1);
    g.unit_most = (uint32_t *)(base + at_unit);
    g.raise = (float *)(base + at_raise);
    g.x = RaisedCopy{(const char *)x, base + at_x, ldx * 2, H * 2, want_up ? M : 0, x_chunks, halves};
    g.rows = M;
    g.units = units;
    g.pre = (const uint16_t *)pre;
    g.d = (const uint16_t *)d_y;
    g.out = (uint16_t *)(base + at_d);
    if (some) {
        const int64_t blocks = cdiv(g.units, 4), few = std::min<int64_t>(blocks, kMostBlocks);
        g.blocks = (int)few;
        const int64_t all = std::min<int64_t>(blocks, (int64_t)1 << 22);
        auto launch = [&](auto kernel, int64_t n) {
            hipLaunchKernelGGL(kernel, dim3(g.copies + n), dim3(256), 0, s, g, copies);
            g.copies = 0;   // (with the first launch)
        };
        g.copies = copy_blocks;
        if (dtype == XGEMM_BF16) {
            launch(gated_slope<kBf16, false>, all);
        } else {
            launch(gated_slope<kFp16, true>, few);
            g.copies = (int)std::min<int64_t>(cdiv(g.x.rows, 4), (int64_t)1 << 22);
            // (each block begins with the blocks' largest and its row's: 4096 x 14336 with 14 blocks a CU 140 us,
            // with one for each four units 180)
            launch(gated_slope<kFp16, false>, std::min<int64_t>(all, 14 * (int64_t)std::max(h->cu_count, 1)));
        }
    }
    const float *const scale = raised ? inverse : nullptr, *const raise = raised ? g.raise : nullptr;
    TileParams p{};
    p.A = base + at_d;
    p.lda = ld * 2;
    if (want_x) {
        p.B = p.B2 = W.p;
        p.ldb = W.ld;
        p.M = (int)rows;
        p.N = (int)H;
        p.K = some ? (int)(2 * I) : 0;
        product<kAlong, kAcross>(dtype, p, StoreParams{d_x, ld_dx, kind, scale, nullptr, 0, raise}, cx, base + at_part, s);
    }
    if (want_up) {
        p.B = p.B2 = raised ? g.x.to : X.p;
        p.ldb = raised ? x_chunks * 16 : X.ld;
        p.M = (int)(2 * I);
        p.N = (int)H;
        p.K = some ? (int)rows : 0;
        product<kAcross, kAcross>(dtype, p, StoreParams{d_up, ld_dup, kind, scale, nullptr, 0, nullptr}, cw, base + at_part, s);
    }
    const int launched = launch_status(h, "gated gradient launch");
    const int released = xgemm_host::release_workspace(h, s);
    return launched != XGEMM_OK ? launched : released;
}

// ---------------------------------------------------------------------------
// log probabilities from a head's weights
// ---------------------------------------------------------------------------

constexpr int64_t kHeadRows = 16384;   // rows of statistics at a time

bool head_ok(int64_t T, int64_t V, int64_t H, int64_t ldx, int64_t ldw, int dtype)
{
    return sixteen(dtype) && T <= kMaxRows && V >= 1 && V <= kMaxSide && H <= kMaxSide && matrix_ok(T, H, ldx) &&
           matrix_ok(V, H, ldw);
}

int run_head(xgemm_ctx *h, int64_t T, int64_t V, int64_t H, const void *x, int64_t ldx, const void *head, int64_t ldw,
             const int64_t *targets, float *logprob, float *lse, int dtype, hipStream_t s)
{
    if (!h || !head_ok(T, V, H, ldx, ldw, dtype))
        return XGEMM_ERR_INVALID_ARG;
    h->last_error[0] = '\0';
    if (T == 0)
        return XGEMM_OK;
    if ((H > 0 && (!x || !head)) || (logprob && !targets))
        return XGEMM_ERR_INVALID_ARG;
    if (!logprob && !lse)
        return XGEMM_OK;
    Space ws;
    Matrix X(x, T, H, ldx, 2), W(head, V, H, ldw, 2);
    const int64_t rows = std::min(T, kHeadRows);
    const Cut c = cut_with(X, W, [&](bool staged) {
        return cut_of(rows, V, cdiv(H, 64), false, false, false, staged, h->cu_count);
    });
    X.reserve(c.staged, ws);
    W.reserve(c.staged, ws);
    const int64_t K = c.staged ? H : up_to(H, 8);
    const int64_t tiles = cdiv(V, kTileCols[c.tile]);
    const size_t at_stat = ws.take((size_t)(tiles * rows) * sizeof(float2)), at_logit = ws.take((size_t)rows * 4);
    const int rc = xgemm_host::acquire_workspace(h, ws.bytes, s);
    if (rc != XGEMM_OK)
        return rc;
    char *const base = (char *)h->workspace + xgemm_host::kWsPrefix;
    Matrix::place(X, W, base, s);
    TileParams p = tile_params(X, W, rows, V, K);
    for (int64_t t = 0; t < T; t += kHeadRows) {
        p.M = (int)std::min(kHeadRows, T - t);
        p.A = X.p + t * X.ld;
        const StatsEnd::Params e{logprob ? targets + t : nullptr, (float2 *)(base + at_stat), (float *)(base + at_logit)};
        if (dtype == XGEMM_BF16)
            launch_product<kBf16, kAlong, kAlong, StatsEnd>(p, e, c, nullptr, s);
        else
            launch_product<kFp16, kAlong, kAlong, StatsEnd>(p, e, c, nullptr, s);
        hipLaunchKernelGGL(head_join, dim3(cdiv(p.M, kJoinRows)), dim3(256), 0, s, e.stat, (int)tiles, (int64_t)p.M, e.at,
                           e.targets, V, lse ? lse + t : nullptr, logprob ? logprob + t : nullptr);
    }
    const int launched = launch_status(h, "head launch");
    const int released = xgemm_host::release_workspace(h, s);
    return launched != XGEMM_OK ? launched : released;
}

template <int DT>
void launch_slopes(TileParams p, const typename SlopeEnd<DT>::Params &at, const Cut &c, int64_t T, hipStream_t s)
{
    const char *const A = p.A;
    typename SlopeEnd<DT>::Params e = at;
    for (int64_t t = 0; t < T; t += kRowsLaunch) {
        p.M = (int)std::min(kRowsLaunch, T - t);
        p.A = A + t * p.lda;
        e.of = at.of.from(t);
        e.raise = at.raise ? at.raise + t : nullptr;
        e.out = at.out + t * at.ld;   // (two parts only of fewer rows than a launch's)
        launch_product<DT, kAlong, kAlong, SlopeEnd<DT>>(p, e, c, nullptr, s);
    }
}

int run_head_grad(xgemm_ctx *h, int64_t T, int64_t V, int64_t H, const void *x, int64_t ldx, const void *head, int64_t ldw,
                  const int64_t *targets, const float *lse, const float *d_logprob, const float *d_lse, void *d_x,
                  int64_t ld_dx, void *d_head, int64_t ld_dw, int dtype, int out, hipStream_t s)
{
    if (!h || !head_ok(T, V, H, ldx, ldw, dtype) || (out != XGEMM_OUT_FP32 && out != XGEMM_OUT_SAME) ||
        (d_x && !matrix_ok(T, H, ld_dx)) || (d_head && !matrix_ok(V, H, ld_dw)))
        return XGEMM_ERR_INVALID_ARG;
    h->last_error[0] = '\0';
    const bool want_x = d_x && T > 0 && H > 0, want_w = d_head && H > 0;
    if (!want_x && !want_w)
        return XGEMM_OK;
    if (T > 0 && (!x || !head || !lse || (d_logprob && !targets)))
        return XGEMM_ERR_INVALID_ARG;
    const int kind = out == XGEMM_OUT_FP32 ? kFp32 : dtype == XGEMM_BF16 ? kBf16 : kFp16;
    Space ws;
    const bool raised = dtype == XGEMM_FP16 && T > 0;
    const size_t at_scale = ws.take(8), at_raise = ws.take(raised ? (size_t)T * 4 : 0);
    const int64_t piece = head_piece(T, V), ld = slope_ld(piece);
    const int halves = T <= kTwoParts ? 2 : 1;
    const int64_t rows = T * halves;   // of slopes
    const size_t at_d = ws.take((size_t)rows * ld * 2);
    // (d_head multiplies x by slopes of 0 where a row takes no part: such a row's x, which may hold
    // anything, is left out.  binary16: in a copy that the logits are not made of)
    const HeadRows of{targets, lse, d_logprob, d_lse, V};
    const bool same = want_w && !raised;
    Matrix X(x, T, H, ldx, 2, same ? halves : 1, same ? &of : nullptr), W(head, T > 0 ? V : 0, H, ldw, 2);
    X.reserve(false, ws);
    W.reserve(false, ws);
    const int64_t x_chunks = cdiv(H, 8);
    const size_t at_x = ws.take(raised && want_w ? (size_t)(rows * x_chunks) * 16 : 0);
    const int64_t K = up_to(H, 8), pieces = cdiv(V, piece);
    // d_x over the pieces: in fp32 until the last
    const bool sums = want_x && pieces > 1 && kind != kFp32;
    const size_t at_sum = ws.take(sums ? (size_t)T * up_to(H, 4) * 4 : 0);
    size_t parts = 0;
    auto cut_x = [&](int64_t n) {
        Cut c = cut_of(rows, H, cdiv(n, 64), false, false, true, false, h->cu_count);
        c.halves = halves;
        return c;
    };
    auto cut_w = [&](int64_t n) { return cut_of(n, H, cdiv(rows, 64), false, true, true, false, h->cu_count); };
    for (const int64_t n : {std::min(piece, V), V - (pieces - 1) * piece})
        parts = std::max({parts, part_bytes(cut_x(n), rows), part_bytes(cut_w(n), n)});
    const size_t at_part = ws.take(parts);
    const int rc = xgemm_host::acquire_workspace(h, ws.bytes, s);
    if (rc != XGEMM_OK)
        return rc;
    char *const base = (char *)h->workspace + xgemm_host::kWsPrefix;
    CopyParams copies;
    const int copy_blocks = Matrix::place(X, W, base, s, &copies);
    float *const scales = (float *)(base + at_scale);
    float *const raise = raised ? (float *)(base + at_raise) : nullptr;
    const int raise_blocks = raised ? (int)std::min<int64_t>(cdiv(T, 4), 1024) : 0;
    hipLaunchKernelGGL(slope_scale, dim3(1 + copy_blocks + raise_blocks), dim3(256), 0, s, copies, copy_blocks,
                       RaisedCopy{(const char *)x, raised && want_w ? base + at_x : nullptr, ldx * 2, H * 2, T, x_chunks, halves}, of,
                       T, dtype == XGEMM_FP16 ? 16384.0f : 1.0f, scales, raise);
    uint16_t *const d = (uint16_t *)(base + at_d);
    float *const sum = kind == kFp32 ? (float *)d_x : (float *)(base + at_sum);
    const int64_t ld_sum = kind == kFp32 ? ld_dx : up_to(H, 4);
    for (int64_t v = 0; v < V; v += piece) {
        const int64_t n = std::min(piece, V - v);
        if (T > 0) {
            TileParams p = tile_params(X, W, T, n, K);
            p.B = p.B2 = W.p + v * W.ld;
            const Cut c = cut_of(T, n, cdiv(K, 64), false, false, false, false, h->cu_count);
            uint16_t *const rest = halves > 1 ? d + T * ld : nullptr;
            if (dtype == XGEMM_BF16)
                launch_slopes<kBf16>(p, {of, scales, raise, d, rest, ld, v}, c, T, s);
            else
                launch_slopes<kFp16>(p, {of, scales, raise, d, rest, ld, v}, c, T, s);
        }
        const float *const scale = scales + 1;
        TileParams p{};
        p.A = (const char *)d;
        p.lda = ld * 2;
        if (want_x) {
            const bool last = v + n == V;
            p.B = p.B2 = W.p + v * W.ld;
            p.ldb = W.ld;
            p.M = (int)rows;
            p.N = (int)H;
            p.K = (int)n;
            const StoreParams e{last ? d_x : sum, last ? ld_dx : ld_sum, last ? kind : kFp32, scale, v > 0 ? sum : nullptr, ld_sum,
                                raise};
            product<kAlong, kAcross>(dtype, p, e, cut_x(n), base + at_part, s);
        }
        if (want_w) {
            p.B = p.B2 = raised ? base + at_x : X.p;
            p.ldb = raised ? x_chunks * 16 : X.ld;
            p.M = (int)n;
            p.N = (int)H;
            p.K = (int)rows;
            const StoreParams e{(char *)d_head + v * ld_dw * (kind == kFp32 ? 4 : 2), ld_dw, kind, scale, nullptr, 0, nullptr};
            product<kAcross, kAcross>(dtype, p, e, cut_w(n), base + at_part, s);
        }
    }
    const int launched = launch_status(h, "head gradient launch");
    const int released = xgemm_host::release_workspace(h, s);
    return launched != XGEMM_OK ? launched : released;
}

}  // namespace

extern "C" {

int xgemm_scaled_rows(xgemm_handle_t h, int64_t R, int64_t K, const void *x, int64_t ldx, int8_t *q, int64_t ldq,
                      float *scales, int dtype, void *stream)
{
    return run_scaled_rows(h, R, K, x, ldx, q, ldq, scales, dtype, (hipStream_t)stream);
}

int xgemm_scaled_run(xgemm_handle_t h, int64_t M, int64_t N, int64_t K, const void *x, int64_t ldx, const float *x_scales,
                     const int8_t *w, int64_t ldw, const float *w_scales, void *y, int64_t ldy, int x_dtype, int y_dtype,
                     void *stream)
{
    return run_scaled(h, M, N, K, x, ldx, x_scales, w, ldw, w_scales, y, ldy, x_dtype, y_dtype, (hipStream_t)stream);
}

int xgemm_gated_run(xgemm_handle_t h, int64_t M, int64_t H, int64_t I, const void *x, int64_t ldx, const void *up,
                    int64_t ldu, void *y, int64_t ldy, void *pre, int64_t ldp, int act, int dtype, int out, void *stream)
{
    return run_gated(h, M, H, I, x, ldx, up, ldu, y, ldy, pre, ldp, act, dtype, out, (hipStream_t)stream);
}

int xgemm_gated_grad(xgemm_handle_t h, int64_t M, int64_t H, int64_t I, const void *x, int64_t ldx, const void *up,
                     int64_t ldu, const void *pre, int64_t ldp, const void *d_y, int64_t ldd, void *d_x, int64_t ld_dx,
                     void *d_up, int64_t ld_dup, int act, int dtype, int out, void *stream)
{
    return run_gated_grad(h, M, H, I, x, ldx, up, ldu, pre, ldp, d_y, ldd, d_x, ld_dx, d_up, ld_dup, act, dtype, out,
                          (hipStream_t)stream);
}

int xgemm_head_run(xgemm_handle_t h, int64_t T, int64_t V, int64_t H, const void *x, int64_t ldx, const void *head,
                   int64_t ldw, const int64_t *targets, float *logprob, float *lse, int dtype, void *stream)
{
    return run_head(h, T, V, H, x, ldx, head, ldw, targets, logprob, lse, dtype, (hipStream_t)stream);
}

int xgemm_head_grad(xgemm_handle_t h, int64_t T, int64_t V, int64_t H, const void *x, int64_t ldx, const void *head,
                    int64_t ldw, const int64_t *targets, const float *lse, const float *d_logprob, const float *d_lse,
                    void *d_x, int64_t ld_dx, void *d_head, int64_t ld_dw, int dtype, int out, void *stream)
{
    return run_head_grad(h, T, V, H, x, ldx, head, ldw, targets, lse, d_logprob, d_lse, d_x, ld_dx, d_head, ld_dw, dtype,
                         out, (hipStream_t)stream);
}

}  // extern "C"
