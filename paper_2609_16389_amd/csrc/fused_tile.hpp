// Products of a tile whose end is fused: what becomes of a tile's sums is
// decided by an End (fused_ends.hpp), the rest is shared by the 8-bit products,
// the gated feed-forward block, the log probabilities from a head's weights and
// the products of their gradients.
//
//     sum over k of a(m, k) b(n, k)
//
// An operand is stored with k along its rows (kAlong: rows of m or n) or with
// one row for each k (kAcross: rows hold consecutive m or n), so that
// transposed products read the same matrices in place.
//
// A workgroup computes a BM x BN tile, each wave a TM x TN part of it in 16 x 16
// matrix instructions, in steps of 128 bytes of k for a row of kAlong (64
// values of 16 bits, 128 of 8) that go straight from memory to one of two LDS
// stages.  kAlong rows are read 16 bytes a lane (8 or 16 consecutive k of a
// row); kAcross rows through the transposing read, which hands a lane 4 k of a
// column.  Chunks are permuted within a row of LDS so that the rows of one read
// fall into different banks.
//
// Edges need no code in the loop: the loads go through a buffer descriptor that
// ends with the wave's own part of the matrix, and what lies past it reads as
// zero: rows past M or N, the k rows of kAcross past K.  Chunks of a kAlong row
// past K are sent past the end by their lane.  Rows are whole 16-byte chunks, with
// zeros after k if it ends inside one (the host copies what is not so).
#pragma once

#include "decode_device.hpp"

#include <type_traits>

namespace xfused_dev {

using namespace xdecode_dev;

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short v4i16 __attribute__((ext_vector_type(4)));

constexpr int kNumXcd = 8;

enum { kBf16 = 0, kFp16 = 1, kInt8 = 2 };
enum { kAlong = 0, kAcross = 1 };

struct TileParams {
    const char *A, *B, *B2;   // B2: the second matrix of a gated block
    int64_t lda, ldb;         // bytes
    int M, N, K;              // of the result, and values of k
    int tiles_m, tiles_n, group_m;
    int split, chunk;         // ranges of k, steps in each
    int grid;
};

template <int TYPE>
struct Sum {
    typedef f32x4 type;
};
template <>
struct Sum<kInt8> {
    typedef i32x4 type;
};

template <int TYPE>
__device__ __forceinline__ typename Sum<TYPE>::type mfma(u32x4 a, u32x4 b, typename Sum<TYPE>::type c)
{
    if constexpr (TYPE == kInt8)
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0,
                                                     0);
    else
        return mfma16<TYPE>(a, b, c);
}

// A buffer descriptor of `bytes` from `base` (both the same for all lanes of a
// wave).
__device__ __forceinline__ u32x4 descriptor(const char *base, int64_t bytes)
{
    const uint64_t a = (uint64_t)(uintptr_t)base;
    u32x4 d;
    d[0] = __builtin_amdgcn_readfirstlane((uint32_t)a);
    d[1] = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32) & 0xffffu);
    d[2] = __builtin_amdgcn_readfirstlane((uint32_t)max(bytes, (int64_t)0));
    d[3] = 0x00020000u;
    return d;
}

// 16 bytes a lane at `off` of the descriptor to LDS at `lds` + 16 * lane.  In
// assembly because the compiler would wait for it before every read of LDS; the
// loop places its own waits.
__device__ __forceinline__ void load_lds(u32x4 d, uint32_t off, uint32_t lds)
{
    asm volatile("buffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(off), "s"(d), "{m0}"(lds) : "memory");
}

template <int N>
__device__ __forceinline__ void wait_loads()
{
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
}
__device__ __forceinline__ void wait_lds() { __builtin_amdgcn_s_waitcnt(15 | (3 << 14) | (7 << 4)); }
__device__ __forceinline__ void meet()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

constexpr uint32_t kPastEnd = 0x80000000u;   // past every descriptor (they stay below 2^31 bytes)

// One operand's part of a stage: R rows of m or n, by W waves, each of which
// loads its own share and reads the fragments of `blocks` of 16 rows from `at`.
template <int TYPE, int LAYOUT, int R, int W>
struct Operand {
    static constexpr int E = TYPE == kInt8 ? 1 : 2;
    static constexpr int KS = 128 / E;                 // k in a step
    static constexpr int kRowBytes = LAYOUT == kAlong ? 128 : R * 2;
    static constexpr int kBytes = R * 128;             // LDS of a stage
    static constexpr int kLoads = kBytes / 1024 / W;   // of a wave, for a step
    static constexpr int kRows = (LAYOUT == kAlong ? R : KS) / W;   // LDS rows that a wave loads
    static constexpr int kRowsLoad = 1024 / kRowBytes;
    static_assert(LAYOUT == kAlong || TYPE != kInt8, "8-bit operands have k along their rows");
    static_assert(kLoads * 1024 * W == kBytes && kRows * W * kRowBytes == kBytes, "whole loads");
    static_assert(LAYOUT == kAlong || R == 128 || R == 256, "LDS row");

    const char *base;    // of this wave's rows, at the next step's k
    int64_t bytes;       // from there to the end of what the wave may read
    int64_t advance;     // bytes of a step (kAcross: of its rows)
    uint32_t off[kLoads];
    int last;            // kAcross: bytes of the last row that are there
    int left;            // from this wave's rows on: bytes of k (kAlong), values (kAcross)
    uint32_t lds;        // where this wave's loads land in stage 0
    int chunk;           // kAlong: first byte of k of this lane, in a load of even number

    // slot of 16 (kAlong) or 32 bytes (kAcross) c of a row: c ^ this
    static __device__ __forceinline__ int turn(int row)
    {
        return LAYOUT == kAlong ? (row >> 1) & 7 : ((row & 3) << 1) | ((row >> 3) & 1);
    }

    // `first` row of the matrix `p` (rows of kAlong; columns of kAcross) of the
    // tile, or of this wave's own rows where they are told apart; `rows` of the
    // matrix from there on.  k from k0, up to K.
    __device__ __forceinline__ void start(const char *p, int64_t ld, int64_t first, int64_t rows, int k0, int K, int lane,
                                          int wave, uint32_t lds0)
    {
        lds = lds0 + wave * kRows * kRowBytes;
        if constexpr (LAYOUT == kAlong) {
            base = p + first * ld + (int64_t)k0 * E;
            const int64_t n = min(rows, (int64_t)kRows);
            // (k ends inside a chunk only where the rows hold zeros up to its end)
            left = ((K - k0) * E + 15) / 16 * 16;
            bytes = n > 0 ? (n - 1) * ld + left : 0;
            advance = 128;
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const int r = j * 8 + lane / 8;
                off[j] = (uint32_t)(r * (int)ld + (((lane & 7) ^ turn(r)) << 4));
            }
            chunk = ((lane & 7) ^ turn(lane / 8)) << 4;
        } else {
            const int k = k0 + wave * kRows;
            base = p + (int64_t)k * ld + first * 2;
            last = (int)min((rows + 7) / 8 * 16, (int64_t)kRowBytes);
            left = K - k;
            advance = KS * ld;
            bytes = rows > 0 ? ld : 0;
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const int r = j * kRowsLoad + lane / (kRowBytes / 16);
                const int q = lane % (kRowBytes / 16);
                off[j] = (uint32_t)(r * (int)ld + ((((q >> 1) ^ turn(wave * kRows + r)) << 5) | (q & 1) << 4));
            }
        }
    }
    __device__ __forceinline__ u32x4 view() const
    {
        if constexpr (LAYOUT == kAlong)
            return descriptor(base, bytes);
        else
            return descriptor(base, bytes > 0 && left > 0 ? (int64_t)(min(left, kRows) - 1) * bytes + last : 0);
    }
    __device__ __forceinline__ void load(u32x4 d, int stage, int j) const
    {
        uint32_t o = off[j];
        if constexpr (LAYOUT == kAlong) {
            // (rows 8 further on turn the other way round)
            const int at = j & 1 ? chunk ^ 64 : chunk;
            o = at < left ? o : kPastEnd;
        }
        load_lds(d, o, __builtin_amdgcn_readfirstlane(lds + stage + j * 1024));
    }
    __device__ __forceinline__ void next()
    {
        base += advance;
        left -= LAYOUT == kAlong ? 128 : KS;
        if constexpr (LAYOUT == kAlong)
            bytes -= advance;
    }

    // Fragment of 16 rows from `row0`, sub-step kk (of two) of the step in the
    // stage at `s` (this operand's part of it).
    static __device__ __forceinline__ u32x4 read(const char *s, int row0, int kk, int lane)
    {
        if constexpr (LAYOUT == kAlong) {
            const int r = lane & 15;
            return *(const u32x4 *)(s + (row0 + r) * 128 + (((4 * kk + (lane >> 4)) ^ turn(r)) << 4));
        } else {
            const int k = 8 * (lane >> 4) + ((lane & 15) >> 2);
            const char *q = s + (kk * 32 + k) * kRowBytes + (((row0 >> 4) ^ turn(k)) << 5) + 8 * (lane & 3);
            typedef __attribute__((address_space(3))) v4i16 *lptr;
            const v4i16 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr)q);
            const v4i16 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr)(q + 4 * kRowBytes));
            u32x4 v;
            v.x = __builtin_bit_cast(uint32_t, __builtin_shufflevector(lo, lo, 0, 1));
            v.y = __builtin_bit_cast(uint32_t, __builtin_shufflevector(lo, lo, 2, 3));
            v.z = __builtin_bit_cast(uint32_t, __builtin_shufflevector(hi, hi, 0, 1));
            v.w = __builtin_bit_cast(uint32_t, __builtin_shufflevector(hi, hi, 2, 3));
            return v;
        }
    }
};

// The aligned dwords around an address (in device memory, which a pointer made of a
// masked address would not show).
__device__ __forceinline__ u32x4 dwords_at(uintptr_t q)
{
    typedef u32x4 __attribute__((aligned(4))) some;
    return *(const __attribute__((address_space(1))) some *)(q & ~(uintptr_t)3);
}
__device__ __forceinline__ uint32_t dword_at(uintptr_t q)
{
    return *(const __attribute__((address_space(1))) uint32_t *)(q & ~(uintptr_t)3);
}

// 16 bytes from p.  ODD: from any byte, as the aligned dwords that hold them,
// moved into place (a load of 16 bytes a lane between dwords takes the L1 path
// several times over).
template <bool ODD>
__device__ __forceinline__ u32x4 sixteen(const char *p)
{
    typedef u32x4 __attribute__((aligned(4))) some;
    if constexpr (!ODD)
        return *(const some *)p;
    const uint32_t by = (uint32_t)(uintptr_t)p & 3;
    const u32x4 v = dwords_at((uintptr_t)p);
    const uint32_t last = dword_at((uintptr_t)p + 15);
    u32x4 r;
    r[0] = __builtin_amdgcn_alignbyte(v[1], v[0], by);
    r[1] = __builtin_amdgcn_alignbyte(v[2], v[1], by);
    r[2] = __builtin_amdgcn_alignbyte(v[3], v[2], by);
    r[3] = __builtin_amdgcn_alignbyte(last, v[3], by);
    return r;
}

// A kAlong operand with rows at any address and of any length: the same parts of a
// stage, loaded into registers as aligned dwords, moved into place and written to LDS
// a step later.  The bytes past the end of k are zeros.  Eight neighbouring lanes have
// a row's eight chunks, so that the dword a chunk ends in is the first of the next
// lane's; only the eighth loads it.  A step takes 0.90 us for a workgroup alone on its CU
// (0.94 with that dword loaded by every lane, 1.05 from aligned 16-byte loads with
// the chunks put together from two lanes' dwords, as long with two steps under way;
// 0.5 for whole chunks), which is less than copies and those up to some 10 MB: 8-bit 37 x
// 5003 x 2047 7.3 us, with copies 5.3 and 8.  (Operands with rows across k were twice
// as slow so as with a copy: 44 and 38 us in place of 13 and 15 for the gradients of 333 x
// 1001 x 2731, and 6 for the copies.)
template <int TYPE, int R, int W>
struct StagedOperand : Operand<TYPE, kAlong, R, W> {
    typedef Operand<TYPE, kAlong, R, W> Base;
    static constexpr int kLoads = Base::kLoads;
    const char *row[kLoads];   // this lane's rows
    int at;                    // byte of its chunk in them, in the next step
    int end;                   // bytes of a row up to the end of k
    u32x4 v[kLoads];
    uint32_t last[kLoads];
    char *to[2];               // of this lane's loads of even and odd number, in stage 0
    bool eighth;

    __device__ __forceinline__ void start(const char *p, int64_t ld, int64_t first, int64_t rows, int k0, int K, int lane,
                                          int wave, char *sh)
    {
        // (rows past the last are read as the last, and their sums dropped)
        end = K * Base::E;
        at = k0 * Base::E + (lane & 7) * 16;
        eighth = (lane & 7) == 7;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int r = j * 8 + lane / 8;
            row[j] = p + (first + min((int64_t)r, rows - 1)) * ld;
            if (j < 2)
                to[j] = sh + (wave * Base::kRows + r) * 128 + (((lane & 7) ^ Base::turn(r)) << 4);
        }
    }
    // Past the next step.
    __device__ __forceinline__ void skip() { at += 128; }
    // The loads of the next step, from k (the same for all lanes).  A chunk that goes
    // past the end is read as the row's last 16 bytes (it has as many), and moved
    // down when it is put in place.
    __device__ __forceinline__ void fetch(int k)
    {
        const bool whole = (k + Base::KS) * Base::E <= end;
        const int from = min(at, end - 16);
#pragma unroll
        for (int j = 0; j < kLoads; ++j)
            v[j] = dwords_at((uintptr_t)(row[j] + from));
        if (!whole || eighth)
#pragma unroll
            for (int j = 0; j < kLoads; ++j)
                last[j] = dword_at((uintptr_t)(row[j] + from) + 15);
        skip();
    }
    // What was fetched last, from k.
    __device__ __forceinline__ void put(int stage, int k)
    {
        const bool whole = (k + Base::KS) * Base::E <= end;
        const int c = at - 128, from = min(c, end - 16);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const uint32_t by = (uint32_t)(uintptr_t)(row[j] + from) & 3;
            const uint32_t beside = (uint32_t)__builtin_amdgcn_mov_dpp((int)v[j][0], 0x101, 0xF, 0xF, true);   // of lane + 1
            const uint32_t after = whole && !eighth ? beside : last[j];
            u32x4 r;
            r[0] = __builtin_amdgcn_alignbyte(v[j][1], v[j][0], by);
            r[1] = __builtin_amdgcn_alignbyte(v[j][2], v[j][1], by);
            r[2] = __builtin_amdgcn_alignbyte(v[j][3], v[j][2], by);
            r[3] = __builtin_amdgcn_alignbyte(after, v[j][3], by);
            if (!whole)
                r = shift_down(r, min(c - from, 16));
            *(u32x4 *)(to[j & 1] + stage + j / 2 * 2048) = r;
        }
    }
};

// Workgroup w of the launch -> its tile and range of k.  The hardware hands
// workgroups to the XCDs in turn: consecutive tiles are gathered on one, in
// groups of group_m tile rows, so that what runs there together shares rows of
// A and of B in its L2.
__device__ __forceinline__ void place(const TileParams &p, int w, int &tm, int &tn, int &ks)
{
    const int per = p.grid / kNumXcd;
    int t = w < per * kNumXcd ? w % kNumXcd * per + w / kNumXcd : w;
    const int tiles = p.tiles_m * p.tiles_n;
    ks = t / tiles;
    t -= ks * tiles;
    const int group = p.group_m * p.tiles_n, g = t / group, first = g * p.group_m;
    const int rows = min(p.tiles_m - first, p.group_m), r = t - g * group;
    tm = first + r % rows;
    tn = r / rows;
}

// What bounds it, for tiles of 256 x 256 on random values: LDS and the matrix units
// together (192 KB read and 64 KB written for 2048 cycles of products on each SIMD in a
// step) and the power limit.  A step takes 1.40 us with k along both rows and 1.5 to
// 1.6 with rows across k (K from 1024 to 8192, all CUs at work), as an 8-bit one does,
// and a tile 5 to 13 us more for its beginning, its end and its stores, which
// nothing else on the CU hides.  4096 x 28672 x 4096 with the gated end 752 us (1280
// TFLOP/s; the library's product alone 752), 4096 x 131072 x 4096 with the
// statistics 3120 us (1410), 4096 x 14336 x 4096 8-bit 229 us (2100 TOP/s).  Tiles of 128
// x 128 take 0.82 us a step alone on a CU and 1.1 shared, of 64 x 128 0.43 and 0.67.
// (Measured and left: groups of 2 to 16 tile rows within 3%, 4 and 8 best.)
//
// STAGED: operands at any address, through registers.
template <int TYPE, int LA, int LB, int BM, int BN, int WM, int WN, int S, bool STAGED, class End>
__global__ void __launch_bounds__(WM * WN * 64) tile_product(TileParams p, typename End::Params e)
{
    constexpr int W = WM * WN;
    constexpr int TM = BM / WM, TN = BN / WN, FM = TM / 16, FN = TN / 16;
    typedef std::conditional_t<STAGED, StagedOperand<TYPE, BM, W>, Operand<TYPE, LA, BM, W>> OpA;
    typedef std::conditional_t<STAGED, StagedOperand<TYPE, BN, W>, Operand<TYPE, LB, BN, W>> OpB;
    static_assert(!STAGED || (LA == kAlong && LB == kAlong), "staged operands have k along their rows");
    typedef typename Sum<TYPE>::type sum_t;
    constexpr int STAGE = OpA::kBytes + OpB::kBytes, LD = OpA::kLoads + OpB::kLoads;
    static_assert(!End::kGated || (LB == kAlong && (TN == 64 || TN == 32) && OpB::kRows == 32), "rows of a gated tile");
    static_assert(S >= 2 && (S - 1) * LD < 64, "loads in flight");

    __shared__ __attribute__((aligned(16))) char smem[S * STAGE];
    const int w = blockIdx.x;
    int tm, tn, ks;
    place(p, w, tm, tn, ks);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM;
    const int m0 = tm * BM, n0 = tn * (End::kGated ? BN / 2 : BN);
    const int k0 = ks * p.chunk * OpA::KS, kend = min(p.K, k0 + p.chunk * OpA::KS);
    // (at least S steps, so that the code below is one line; what lies past kend is zero)
    const int nk = max((kend - k0 + OpA::KS - 1) / OpA::KS, S);

    auto place_of = [&](int off) {
        if constexpr (STAGED)
            return smem + off;
        else
            return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char *)smem + off;
    };
    const auto lds0 = place_of(0), lds1 = place_of(OpA::kBytes);
    OpA a;
    OpB b;
    if constexpr (LA == kAlong)
        a.start(p.A, p.lda, m0 + wave * OpA::kRows, (int64_t)p.M - m0 - wave * OpA::kRows, k0, kend, lane, wave, lds0);
    else
        a.start(p.A, p.lda, m0, (int64_t)p.M - m0, k0, kend, lane, wave, lds0);
    if constexpr (End::kGated) {
        // the tile's rows by 32: gate, lift, gate, lift, of which a wave takes as
        // many of either
        const int n = n0 + wave / 2 * 32;
        b.start(wave & 1 ? p.B2 : p.B, p.ldb, n, (int64_t)p.N - n, k0, kend, lane, wave, lds1);
    } else if constexpr (LB == kAlong) {
        b.start(p.B, p.ldb, n0 + wave * OpB::kRows, (int64_t)p.N - n0 - wave * OpB::kRows, k0, kend, lane, wave,
                lds1);
    } else {
        b.start(p.B, p.ldb, n0, (int64_t)p.N - n0, k0, kend, lane, wave, lds1);
    }

    sum_t acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
            acc[i][j] = sum_t{0, 0, 0, 0};

    int kf = k0;   // STAGED: k of the step to be put into LDS next
    auto fetch = [&](int ahead) {
        if constexpr (STAGED) {
            a.fetch(kf + OpA::KS * ahead);
            b.fetch(kf + OpA::KS * ahead);
        }
    };
    auto put = [&](int stage) {
        if constexpr (STAGED) {
            a.put(stage * STAGE, kf);
            b.put(stage * STAGE, kf);
            kf += OpA::KS;
        }
    };
    auto load_step = [&](int stage) {
        if constexpr (!STAGED) {
            const u32x4 da = a.view(), db = b.view();
#pragma unroll
            for (int j = 0; j < OpA::kLoads; ++j)
                a.load(da, stage * STAGE, j);
#pragma unroll
            for (int j = 0; j < OpB::kLoads; ++j)
                b.load(db, stage * STAGE, j);
            a.next();
            b.next();
        }
    };
    auto read_a = [&](int stage, int kk, int i) { return OpA::read(smem + stage * STAGE, wm * TM + i * 16, kk, lane); };
    auto read_b = [&](int stage, int kk, int j) {
        const int row = End::kGated && TN == 32 ? wn / 2 * 64 + wn % 2 * 16 + j * 32 : wn * TN + j * 16;
        return OpB::read(smem + stage * STAGE + OpA::kBytes, row, kk, lane);
    };
    // A step of two sub-steps, whose fragments have registers of their own: those
    // of the next sub-step are read as soon as a row of the current one has issued
    // its products.  One row of the second sub-step runs before the barrier,
    // which gives the last read time; after the barrier, which frees this
    // step's stage, the loads of the step after the next go there, spaced by
    // products, at a raised priority against the other wave of the SIMD.
    constexpr int R = 1;
    constexpr int REST = (FM - R) * FN;               // products after the barrier
    constexpr int APART = REST / LD > 0 ? REST / LD : 1;
    constexpr int BR = (FN + FM - R - 1) / (FM - R);   // fragments of B read with each row after it
    static_assert(FN <= FM && APART * (LD - 1) < REST, "spacing");
    u32x4 ga[2][FM], gb[2][FN];
    // LOAD: the step S further on exists; MORE: so does the next.
    int stage = 0;
    auto step = [&]<bool LOAD, bool MORE>() {
        const int next = S == 2 ? stage ^ 1 : stage == S - 1 ? 0 : stage + 1;
#pragma unroll
        for (int i = 0; i < FM; ++i) {
#pragma unroll
            for (int j = 0; j < FN; ++j)
                acc[i][j] = mfma<TYPE>(gb[0][j], ga[0][i], acc[i][j]);
            ga[1][i] = read_a(stage, 1, i);
            if (i < FN)
                gb[1][i] = read_b(stage, 1, i);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j)
                acc[i][j] = mfma<TYPE>(gb[1][j], ga[1][i], acc[i][j]);
        __builtin_amdgcn_sched_barrier(0);
        // this wave has read all of the stage; its loads of the next step have landed
        wait_lds();
        if constexpr (LOAD && !STAGED)
            wait_loads<(S - 2) * LD>();
        else if constexpr (MORE && !STAGED)
            wait_loads<0>();
        meet();
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
        u32x4 da, db;
        if constexpr (LOAD && STAGED) {
            // (fetched a step ago)
            put(stage);
            fetch(0);
        } else if constexpr (LOAD) {
            da = a.view();
            db = b.view();
        }
        if constexpr (MORE) {
#pragma unroll
            for (int i = 0; i < R; ++i)
                ga[0][i] = read_a(next, 0, i);
        }
#pragma unroll
        for (int i = R; i < FM; ++i) {
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                acc[i][j] = mfma<TYPE>(gb[1][j], ga[1][i], acc[i][j]);
                if constexpr (LOAD && !STAGED) {
                    const int n = (i - R) * FN + j;
                    if (n % APART == 0 && n / APART < LD) {
                        const int l = n / APART;
                        if (l < OpA::kLoads)
                            a.load(da, stage * STAGE, l);
                        else
                            b.load(db, stage * STAGE, l - OpA::kLoads);
                    }
                }
            }
            if constexpr (MORE) {
                ga[0][i] = read_a(next, 0, i);
#pragma unroll
                for (int j = (i - R) * BR; j < (i - R + 1) * BR && j < FN; ++j)
                    gb[0][j] = read_b(next, 0, j);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
        if constexpr (LOAD && !STAGED) {
            a.next();
            b.next();
        }
        stage = next;
    };
    if constexpr (STAGED) {
        static_assert(S == 2, "steps on their way at the beginning");
        OpA a0 = a;
        OpB b0 = b;
        a0.fetch(kf);
        b0.fetch(kf);
        a.skip();
        b.skip();
        fetch(1);
        a0.put(0, kf);
        b0.put(0, kf);
        kf += OpA::KS;
        put(1);
        fetch(0);
        wait_lds();
    } else {
#pragma unroll
        for (int t = 0; t < S; ++t)
            load_step(t);
        wait_loads<(S - 1) * LD>();
    }
    meet();
#pragma unroll
    for (int i = 0; i < FM; ++i)
        ga[0][i] = read_a(0, 0, i);
#pragma unroll
    for (int j = 0; j < FN; ++j)
        gb[0][j] = read_b(0, 0, j);
    for (int t = 0; t < nk - S; ++t)
        step.template operator()<true, true>();
#pragma unroll
    for (int t = 0; t < S - 1; ++t)
        step.template operator()<false, true>();
    step.template operator()<false, false>();
    // lane l holds row l % 16 of each block and columns 4 (l / 16) .. + 3
    End::template finish<BM, BN, TM, TN, FM, FN, WN>(p, e, acc, smem, m0, n0, wm, wn, tn, ks, lane);
}

}  // namespace xfused_dev
