// Rows of logits: log-sum-exp, log probability of a given token, entropy, the
// largest alternatives; and the gradient of the first three in the logits.
//
//     m = max x    S = sum exp(x - m)    U = sum exp(x - m) (x - m)
//     lse = m + log S    logprob = (x[target] - m) - log S    entropy = log S - U / S
//
// One pass over the row: every lane keeps m, S and U of its own values and
// rescales S and U when m grows: with d = m_old - m_new,
//     U' = exp(d) (U + d S)    S' = exp(d) S.
// The same rule joins lanes, waves and, where few rows would leave CUs idle,
// the parts of a row that several workgroups take (the last one to finish
// joins them, in the order of the parts, whichever it is).  (exp is 2^(t log2 e)
// of the difference t: folding the factor into one fused multiply-add, 2^(x log2
// e - r), saves an instruction of eleven a value, but a row of one certain
// token then no longer has an entropy of exactly 0, and the lowest values of
// fp32 and bfloat16, which masks are made of, overflow.)
//
// The alternatives come from the same pass.  A wave sets aside values that may
// be among the row's n largest: with w waves that have whole batches, at least
// n values are as large as the least over them of the ceil(n / w)-th largest of
// a wave's lane maxima so far, so nothing below that bound is kept; the bound is
// renewed after 1, 2, 4, ... batches.  What is kept lies in a buffer of 128 a wave, cut back to the n
// largest when it would run over.  Values are ordered by (value, lower index
// first) as one 64-bit number, so the result does not depend on who found
// what first.
//
// What bounds it: with alternatives vector instructions, ten a value for the
// statistics (a 2^x counts for four) and some nine for choosing; without,
// neither they (59% of the issue slots) nor memory (4.4 TB/s).  With few rows it is the chain of latencies from the
// first load to the last join.  What a call executes once is kept short (code
// that is not in the instruction cache yet costs more to fetch than to run),
// so the paths that are seldom taken are loops and not unrolled.  Measured: 4096
// rows of 50001 bfloat16 with five alternatives 106 us (3.9 TB/s, 1.9 values a
// ns), without 94 us; one row of 131072 fp32 with twenty 13.1 us, without 5.0, of
// which some 3 us are the launch.
//
// Accuracy: the product of x - m with log2 e is rounded to fp32, which leaves a
// relative |x - m| 2^-24 in a term.  A value of 88 below the largest no longer
// counts, so that is at most 2^-17 of a term too small to matter, and 1e-7 in all.
#pragma once

#include "decode_device.hpp"

namespace xlogprob_dev {

using namespace xdecode_dev;

constexpr int kThreads = 512, kWaves = kThreads / 64;
constexpr int kLane = 16;                  // values of a lane in a batch
constexpr int kBatch = 64 * kLane;         // values of a wave in a batch
constexpr int kBuffer = 128;
constexpr int kMaxTop = 32;
constexpr int kMaxParts = 64;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLowest = -1e30f;          // stands in for -inf where it meets a zero factor

struct Stats {
    float m, S, U;
};

struct LogprobParams {
    const void *logits;
    const int64_t *targets;
    float *logprob, *lse, *entropy, *top_logprob;  // each may be null
    int64_t *top_id;
    int64_t ld;       // elements
    int64_t row0;     // first row of the launch
    int V, top;
    int parts, part_len;
    Stats *stat;      // [rows][parts], where parts > 1
    uint64_t *best;   // [rows][parts][top]
    int *count;       // [rows], zero between launches
};

// The largest of the wave's values, and their sum, in all lanes.  Each step
// takes the value of another lane within a row of 16, then of the rows before
// (lanes without one: `none`, which changes nothing).
template <class F>
__device__ __forceinline__ uint32_t wave_reduce(uint32_t v, uint32_t none, F &&f)
{
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, 0x111, 0xf, 0xf, false));  // row_shr 1
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, 0x112, 0xf, 0xf, false));  // row_shr 2
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, 0x114, 0xf, 0xf, false));  // row_shr 4
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, 0x118, 0xf, 0xf, false));  // row_shr 8
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, 0x142, 0xa, 0xf, false));  // row_bcast 15
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, 0x143, 0xc, 0xf, false));  // row_bcast 31
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
    return wave_reduce(v, 0u, [](uint32_t a, uint32_t b) { return max(a, b); });
}
__device__ __forceinline__ float wave_max(float v)
{
    const float none = -__builtin_inff();
    return __builtin_bit_cast(float, wave_reduce(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, none),
                                                 [](uint32_t a, uint32_t b) {
                                                     return __builtin_bit_cast(uint32_t, fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)));
                                                 }));
}
__device__ __forceinline__ float wave_sum(float v)
{
    return __builtin_bit_cast(float, wave_reduce(__builtin_bit_cast(uint32_t, v), 0u, [](uint32_t a, uint32_t b) {
                                  return __builtin_bit_cast(uint32_t, __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b));
                              }));
}

// s with its maximum raised to m (the exponential of -inf and of the NaN of
// equal infinities: 0).
__device__ __forceinline__ Stats raise(Stats s, float m)
{
    const float d = fmaxf(s.m - m, kLowest), f = __builtin_amdgcn_exp2f(d * kLog2e);
    return Stats{m, s.S * f, f * fmaf(s.S, d, s.U)};
}
__device__ __forceinline__ Stats join_wave(Stats s)
{
    s = raise(s, wave_max(s.m));
    return Stats{s.m, wave_sum(s.S), wave_sum(s.U)};
}

// A value as a whole number in the same order, the two zeros alike.
__device__ __forceinline__ uint32_t order_of(float v)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.0f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t k)
{
    return __builtin_bit_cast(float, k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

// (never 0: an index is below 2^31)
__device__ __forceinline__ uint64_t entry_of(uint32_t key, int index)
{
    return (uint64_t)key << 32 | (0xffffffffu - (uint32_t)index);
}

__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Cut a wave's `count` entries (at most kBuffer) back to the `n` largest, in
// descending order.
__device__ __forceinline__ int cut_back(uint64_t *buf, int count, int n, int lane)
{
    wave_sync();
    const uint64_t a = lane < count ? buf[lane] : 0, b = lane + 64 < count ? buf[lane + 64] : 0;
    int ra = 0, rb = 0;
    for (int i = 0; i < count; ++i) {
        const uint64_t v = buf[i];
        ra += v > a;
        rb += v > b;
    }
    wave_sync();
    if (lane < count && ra < n)
        buf[ra] = a;
    if (lane + 64 < count && rb < n)
        buf[rb] = b;
    wave_sync();
    return min(count, n);
}

// VEC values of a row from index v as they are in memory.
template <int DT>
__device__ __forceinline__ u32x4 load_raw(const void *row, int64_t v)
{
    return load_any<u32x4>((const char *)row + v * (DT == 2 ? 4 : 2));
}
template <int DT, int VEC>
__device__ __forceinline__ void convert(u32x4 t, float *x)
{
#pragma unroll
    for (int e = 0; e < VEC; ++e)
        if constexpr (DT == 2)
            x[e] = __builtin_bit_cast(f32x4, t)[e];
        else if constexpr (DT == 0)
            x[e] = __builtin_bit_cast(float, e & 1 ? t[e / 2] & 0xffff0000u : t[e / 2] << 16);
        else
            x[e] = to_float<DT>((uint16_t)(t[e / 2] >> (16 * (e & 1))));
}
template <int DT>
__device__ __forceinline__ float load_value(const void *row, int64_t v)
{
    if constexpr (DT == 2)
        return ((const float *)row)[v];
    else
        return to_float<DT>(((const uint16_t *)row)[v]);
}

template <int DT, bool TOP>
__global__ void __launch_bounds__(kThreads, 4)
logprob_rows(LogprobParams p)
{
    constexpr int VEC = DT == 2 ? 4 : 8, UN = kLane / VEC;
    __shared__ uint64_t buf[TOP ? kWaves : 1][kBuffer];
    __shared__ uint64_t list[TOP ? kMaxParts * kMaxTop : 1];   // candidates of all waves, or of all parts
    __shared__ uint64_t best[kMaxTop];
    __shared__ uint32_t bounds[kWaves];
    __shared__ Stats stats[kWaves];
    __shared__ int sh_listed, sh_last;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t row = p.row0 + blockIdx.y;
    const int part = blockIdx.x;
    const void *const x = (const char *)p.logits + row * p.ld * (DT == 2 ? 4 : 2);
    const int v0 = part * p.part_len, v1 = min(p.V, v0 + p.part_len);
    const int n = p.top;

    // whole batches, and what is left after them, value by value.  (They start
    // with the row wherever it lies, so that a result does not depend on its
    // address.)
    const int batches = (v1 - v0) / kBatch, rest = v0 + batches * kBatch;
    const int bounding = max(min(batches, kWaves), 1);   // waves that set a bound (without whole batches: the first)
    const int every = (n + bounding - 1) / bounding;
    const int mine = batches > wave ? (batches - 1 - wave) / kWaves + 1 : 0;

    Stats s = {-__builtin_inff(), 0.0f, 0.0f};
    float lane_max = -__builtin_inff();
    uint64_t cut = 0;      // nothing at or below it is among this wave's n largest
    int kept = 0;
    if (tid == 0)
        sh_listed = 0;

    auto stat_batch = [&](const float (&v)[kLane]) {
        float most = v[0];
#pragma unroll
        for (int i = 1; i < kLane; ++i)
            most = fmaxf(most, v[i]);
        s = raise(s, fmaxf(s.m, most));
        const float ref = s.m == -__builtin_inff() ? 0.0f : s.m;
#pragma unroll
        for (int i = 0; i < kLane; ++i) {
            const float t = v[i] - ref, e = __builtin_amdgcn_exp2f(t * kLog2e);
            s.S += e;
            s.U = fmaf(e, fmaxf(t, kLowest), s.U);
        }
        lane_max = fmaxf(lane_max, most);
        return most;
    };
    // (waves renew their bounds while others read them, which changes what is set
    // aside on the way but not the result: atomics, in no order)
    auto set_bound = [&](uint32_t v) {
        if (lane == 0)
            __hip_atomic_store(&bounds[wave], v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    };
    // this wave's bound: the `every`-th largest of its lanes' maxima
    auto renew = [&](bool bounds_any) {
        if (!bounds_any) {
            set_bound(0xffffffffu);
            return;
        }
        uint32_t left = order_of(lane_max), most = 0;
#pragma unroll 1
        for (int i = 0; i < every; ++i) {
            most = wave_max(left);
            const uint64_t who = __ballot(left == most);
            if (lane == __builtin_ctzll(who))
                left = 0;
        }
        set_bound(most);
    };
    auto least_bound = [&] {
        uint32_t bound = 0xffffffffu;
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
            bound = min(bound, __hip_atomic_load(&bounds[w], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP));
        return bound;
    };
    // index(i): place of this lane's value i, or -1
    auto keep_batch = [&](const float (&v)[kLane], float most, auto index) {
        uint32_t bound = max(least_bound(), (uint32_t)(cut >> 32));
        if (!__any(order_of(most) >= bound))
            return;
        uint32_t todo = 0;
#pragma unroll
        for (int i = 0; i < kLane; ++i)
            todo |= order_of(v[i]) >= bound && v[i] == v[i] ? 1u << i : 0u;
#pragma unroll 1
        while (__any(todo != 0)) {
            const int i = todo ? __builtin_ctz(todo) : 0;
            float mine = v[0];
#pragma unroll
            for (int j = 1; j < kLane; ++j)
                mine = i == j ? v[j] : mine;
            const int at = index(i);
            const uint64_t entry = entry_of(order_of(mine), at);
            bool on = todo != 0 && at >= 0 && entry > cut;
            todo &= todo - 1;
            uint64_t who = __ballot(on);
            if (kept + __popcll(who) > kBuffer) {
                kept = __builtin_amdgcn_readfirstlane(cut_back(buf[wave], kept, n, lane));
                if (kept == n)
                    cut = buf[wave][n - 1];
                on = on && entry > cut;
                who = __ballot(on);
            }
            if (on)
                buf[wave][kept + __popcll(who & ((1ull << lane) - 1))] = entry;
            kept += __popcll(who);
        }
    };
    // place a wave's candidates (on) in the list
    auto add_to_list = [&](bool on, uint64_t entry) {
        const uint64_t who = __ballot(on);
        int base = 0;
        if (lane == 0 && who)
            base = atomicAdd(&sh_listed, __popcll(who));
        base = __builtin_amdgcn_readfirstlane(base);
        if (on)
            list[base + __popcll(who & ((1ull << lane) - 1))] = entry;
    };
    // the n largest of the list, in descending order
    auto rank_list = [&] {
        const int listed = sh_listed;
        for (int t = tid; t < listed; t += kThreads) {
            const uint64_t entry = list[t];
            int rank = 0;
#pragma unroll 4
            for (int i = 0; i < listed; ++i)
                rank += list[i] > entry;
            if (rank < n)
                best[rank] = entry;
        }
        __syncthreads();
        return min(listed, n);
    };

    // the wave's whole batches, the next one on its way; the first sets the
    // bounds that its own values are held to
    u32x4 raw[UN];
    auto load_batch = [&](int j) {
        const int64_t at = v0 + (int64_t)(wave + kWaves * min(j, mine - 1)) * kBatch;
#pragma unroll
        for (int u = 0; u < UN; ++u)
            raw[u] = load_raw<DT>(x, at + 64 * VEC * u + VEC * lane);
    };
    if (mine > 0)
        load_batch(0);
#pragma unroll 1
    for (int j = 0; j < max(mine, 1); ++j) {
        float v[kLane];
        float most = -__builtin_inff();
        if (mine > 0) {
#pragma unroll
            for (int u = 0; u < UN; ++u)
                convert<DT, VEC>(raw[u], v + VEC * u);
            load_batch(j + 1);
            most = stat_batch(v);
        }
        if constexpr (TOP) {
            if ((j & (j + 1)) == 0)
                renew(mine > 0);
            if (j == 0)
                __syncthreads();
            if (mine > 0) {
                const int at = v0 + (wave + kWaves * j) * kBatch + VEC * lane;
                keep_batch(v, most, [&](int i) { return at + 64 * VEC * (i / VEC) + i % VEC; });
            }
        }
    }
    if (wave == batches % kWaves && rest < v1) {
        const auto index = [&](int i) { return rest + lane + 64 * i < v1 ? rest + lane + 64 * i : -1; };
        float v[kLane];
#pragma unroll
        for (int i = 0; i < kLane; ++i)
            v[i] = load_value<DT>(x, max(index(i), v0));
#pragma unroll
        for (int i = 0; i < kLane; ++i)
            v[i] = index(i) >= 0 ? v[i] : -__builtin_inff();
        const float most = stat_batch(v);
        if constexpr (TOP) {
            if (batches == 0)
                renew(true);
            keep_batch(v, most, index);
        }
    }

    s = join_wave(s);
    if (lane == 0)
        stats[wave] = s;
    int found = 0;
    if constexpr (TOP) {
        renew(wave < bounding);
        __syncthreads();
        const uint32_t bound = least_bound();
        wave_sync();
        for (int i = lane; i < kBuffer; i += 64) {
            const uint64_t entry = i < kept ? buf[wave][i] : 0;
            add_to_list(i < kept && (uint32_t)(entry >> 32) >= bound, entry);
        }
        __syncthreads();
        found = rank_list();
    } else {
        __syncthreads();
    }
    {
        Stats q = lane < kWaves ? stats[lane] : Stats{-__builtin_inff(), 0.0f, 0.0f};
        s = join_wave(q);
    }

    if (p.parts > 1) {
        // publish this part with device-scope stores; once they have
        // completed, count in.  Nobody waits: the last to count in joins.
        const int64_t r = blockIdx.y;
        if (wave == 0) {
            Stats *const to = p.stat + r * p.parts + part;
            if (lane == 0) {
                __hip_atomic_store(&to->m, s.m, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                __hip_atomic_store(&to->S, s.S, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                __hip_atomic_store(&to->U, s.U, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            if (TOP && lane < n)
                __hip_atomic_store(p.best + (r * p.parts + part) * n + lane, lane < found ? best[lane] : 0ull,
                                   __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            if (lane == 0) {
                const int before = __hip_atomic_fetch_add(p.count + r, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                sh_last = before == p.parts - 1;
                if (sh_last)
                    __hip_atomic_store(p.count + r, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                sh_listed = 0;
            }
        }
        __syncthreads();
        if (!sh_last)
            return;
        asm volatile("" ::: "memory");
        Stats q = {-__builtin_inff(), 0.0f, 0.0f};
        uint64_t least = 0;
        if (lane < p.parts) {
            Stats *const from = p.stat + r * p.parts + lane;
            q.m = __hip_atomic_load(&from->m, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            q.S = __hip_atomic_load(&from->S, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            q.U = __hip_atomic_load(&from->U, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if (TOP)
                least = __hip_atomic_load(p.best + (r * p.parts + lane) * n + n - 1, __ATOMIC_RELAXED,
                                          __HIP_MEMORY_SCOPE_AGENT);
        }
        s = join_wave(q);
        if constexpr (TOP) {
            // (a part's n-th is below the row's n-th or it)
            const uint32_t bound = wave_max((uint32_t)(least >> 32));
            for (int q0 = wave; q0 < p.parts; q0 += kWaves) {
                uint64_t e = 0;
                if (lane < n)
                    e = __hip_atomic_load(p.best + (r * p.parts + q0) * n + lane, __ATOMIC_RELAXED,
                                          __HIP_MEMORY_SCOPE_AGENT);
                add_to_list(e != 0 && (uint32_t)(e >> 32) >= bound, e);
            }
            __syncthreads();
            found = rank_list();
        }
    }

    if (wave != 0)
        return;
    const float log_S = logf(s.S);
    const bool empty = s.m == -__builtin_inff() && s.S == 0.0f;   // every logit is -inf
    auto log_of = [&](float v) { return empty ? -__builtin_inff() : (v - s.m) - log_S; };
    if (lane == 0) {
        if (p.lse)
            p.lse[row] = empty ? -__builtin_inff() : s.m + log_S;
        if (p.entropy)
            p.entropy[row] = empty ? 0.0f : log_S - s.U / s.S;
        if (p.logprob) {
            const int64_t t = p.targets[row];
            p.logprob[row] = t < 0 ? 0.0f : t >= p.V ? __builtin_nanf("") : log_of(load_value<DT>(x, t));
        }
    }
    if (TOP && lane < n) {
        const bool is = lane < found;
        const uint64_t e = is ? best[lane] : 0;
        p.top_id[row * n + lane] = is ? (int64_t)(0xffffffffu - (uint32_t)e) : -1;
        p.top_logprob[row * n + lane] = is ? log_of(value_of((uint32_t)(e >> 32))) : __builtin_nanf("");
    }
}

struct GradParams {
    const void *logits;
    const int64_t *targets;
    const float *lse, *entropy;
    const float *d_logprob, *d_entropy, *d_lse;  // each may be null
    void *out;
    int64_t ld, ldo;  // elements
    int64_t row0;
    int V;
    int group;        // spans that one workgroup takes where it sums a row itself
};

// dx = d_logprob (delta - p) - d_entropy p (log p + entropy) + d_lse p, with
// log p = x - lse: a read and a write of every logit, the bytes of which bound
// it (2048 rows of 131072 bfloat16: 173 us, 6.2 TB/s read and written).  A
// workgroup takes a span of kGradSpan values of one row.
//
// A large lse is held too coarsely for this: p is off by a relative |lse| 2^-24,
// and a row of nothing but -1e9 has lse = x and a p of 1.  From coarse_lse() on
// a workgroup forms Z = sum of exp(x - lse) over its row, which is 1 but for the
// rounding of lse, and takes log Z off log p.  (Below, the rounding leaves at
// most 2^-17 in p for fp32 and 2^-15, an eighth of binary16's, for 16 bits.)  One
// workgroup then takes `group` spans, so that a row is read group times less
// often; into the logits themselves one takes the whole row, or it would read what
// others have written.  2048 rows of 131072 bfloat16 at -3000: 371 us, with one span
// a workgroup 1403, a whole row 345.  A Z that rounding does not explain is not this row's sum (a row that is
// part of a longer one), and is left alone.
constexpr int kGradThreads = 256, kGradSpan = kGradThreads * 8 * 2;
template <int DT>
constexpr float coarse_lse()
{
    return DT == 2 ? 256.0f : 1024.0f;
}

template <int DT>
__global__ void __launch_bounds__(kGradThreads, 8)
logprob_grad(GradParams p)
{
    constexpr int VEC = DT == 2 ? 4 : 8, UN = kGradSpan / (kGradThreads * VEC);
    const int64_t row = p.row0 + blockIdx.y;
    const int bytes = DT == 2 ? 4 : 2;
    const void *const x = (const char *)p.logits + row * p.ld * bytes;
    char *const y = (char *)p.out + row * p.ldo * bytes;
    const float lse = p.lse[row];
    const bool empty = lse < -1e37f;   // nothing but -inf or the type's lowest value
    const int64_t target = p.targets ? p.targets[row] : -1;
    float gl = target >= 0 && p.d_logprob ? p.d_logprob[row] : 0.0f;
    if (target >= p.V && p.d_logprob)
        gl = __builtin_nanf("");
    const float c2 = p.d_entropy ? p.d_entropy[row] : 0.0f;
    const float c1 = gl - (p.d_lse ? p.d_lse[row] : 0.0f) + (p.d_entropy ? c2 * p.entropy[row] : 0.0f);

    // VEC values from index `at`
    auto load = [&](int at, float (&v)[VEC], float past) {
        if (at + VEC <= p.V) {
            convert<DT, VEC>(load_raw<DT>(x, at), v);
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                v[e] = at + e < p.V ? load_value<DT>(x, at + e) : past;
        }
    };
    // one span, in two steps; off: log Z, where FINE
    float v[UN][VEC];
    auto fetch = [&](int v0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < UN; ++u)
            load(v0 + (u * kGradThreads + (int)threadIdx.x) * VEC, v[u], 0.0f);
    };
    auto finish = [&]<bool FINE>(int v0, float off) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            const int at = v0 + (u * kGradThreads + (int)threadIdx.x) * VEC;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float t = FINE ? (v[u][e] - lse) - off : v[u][e] - lse;
                const float q = __builtin_amdgcn_exp2f(t * kLog2e);
                float d = -q * fmaf(c2, fmaxf(t, kLowest), c1);
                if (at + e == target)
                    d += gl;
                v[u][e] = empty ? 0.0f : d;
            }
            if (at + VEC <= p.V) {
                if constexpr (DT == 2) {
                    f32x4 o = {v[u][0], v[u][1], v[u][2], v[u][3]};
                    store_any<f32x4>(y + (int64_t)at * 4, o);
                } else {
                    u32x4 o;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[e] = from_float<DT>(v[u][2 * e]) | (uint32_t)from_float<DT>(v[u][2 * e + 1]) << 16;
                    store_any<u32x4>(y + (int64_t)at * 2, o);
                }
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    if (at + e < p.V) {
                        if constexpr (DT == 2)
                            ((float *)y)[at + e] = v[u][e];
                        else
                            ((uint16_t *)y)[at + e] = from_float<DT>(v[u][e]);
                    }
            }
        }
    };

    fetch(blockIdx.x * kGradSpan);   // (before anything waits for lse)
    const float size = __builtin_fabsf(lse);
    if (empty || !(size >= coarse_lse<DT>() && size < __builtin_inff())) {
        finish.template operator()<false>(blockIdx.x * kGradSpan, 0.0f);
        return;
    }
    // (the workgroup of a group that does the work differs from row to row:
    // workgroups go to the XCDs in turn)
    const int first = blockIdx.x - blockIdx.x % p.group, spans = min(p.group, (int)gridDim.x - first);
    if ((int)blockIdx.x - first != (int)(row % spans))
        return;
    float Z = 0.0f;
    auto add = [&](const float (&v)[VEC]) {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            Z += __builtin_amdgcn_exp2f((v[e] - lse) * kLog2e);
    };
    constexpr int kLoads = 4, kPass = kGradThreads * VEC;
    int64_t at = threadIdx.x * VEC;
    for (; at + (kLoads - 1) * kPass + VEC <= p.V; at += kLoads * kPass) {
        u32x4 raw[kLoads];
#pragma unroll
        for (int u = 0; u < kLoads; ++u)
            raw[u] = load_raw<DT>(x, at + u * kPass);
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            float v[VEC];
            convert<DT, VEC>(raw[u], v);
            add(v);
        }
    }
    for (; at < p.V; at += kPass) {
        float v[VEC];
        load((int)at, v, -__builtin_inff());
        add(v);
    }
    __shared__ float sums[kGradThreads / 64];
    Z = wave_sum(Z);
    if ((threadIdx.x & 63) == 0)
        sums[threadIdx.x >> 6] = Z;
    __syncthreads();
    Z = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    float off = logf(Z);
    if (!(__builtin_fabsf(off) <= size * 0x1p-23f))
        off = 0.0f;
#pragma unroll 1
    for (int i = first; i < first + spans; ++i) {
        fetch(i * kGradSpan);
        finish.template operator()<true>(i * kGradSpan, off);
    }
}

}  // namespace xlogprob_dev
