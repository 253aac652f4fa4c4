// Rows of logits: log-sum-exp, log probability of a given token, entropy, the
// largest alternatives; and the gradient of the first three in the logits.
//
//     m = max x    S = sum exp(x - m)    U = sum exp(x - m) (x - m)
//     lse = m + log S    logprob = (x[target] - m) - log S    entropy = log S - U / S
//
// One pass over the row: every lane keeps m, S and U of its own values and
// rescales S and U when m grows:  with d = m_old - m_new,
//     U' = exp(d) (U + d S)    S' = exp(d) S.
// The same rule joins lanes, waves and, where few rows would leave CUs idle,
// the parts of a row that several workgroups take (the last one to finish
// joins them, in the order of the parts, whichever it is).
//
// The alternatives come from the same pass.  A wave sets aside values that may
// be among the row's n largest: at least n values are as large as the least
// over the waves of the ceil(n / 8)-th largest of a wave's lane maxima so far,
// so nothing below that bound is kept; the bound is renewed after 1, 2, 4, ...
// batches.  What is kept lies in a buffer of 128 a wave, cut back to the n
// largest when it would run over.  Values are ordered by (value, lower index
// first) as one 64-bit number, so the result does not depend on who found
// what first.
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
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
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

// exp(d) for d <= 0 (-inf and the NaN of equal infinities: 0).
__device__ __forceinline__ float shrink(float d) { return __builtin_amdgcn_exp2f(fmaxf(d, kLowest) * kLog2e); }

__device__ __forceinline__ Stats join(Stats a, Stats b)
{
    Stats r;
    r.m = fmaxf(a.m, b.m);
    const float da = fmaxf(a.m - r.m, kLowest), db = fmaxf(b.m - r.m, kLowest);
    const float fa = shrink(da), fb = shrink(db);
    r.S = a.S * fa + b.S * fb;
    r.U = fa * fmaf(a.S, da, a.U) + fb * fmaf(b.S, db, b.U);
    return r;
}

__device__ __forceinline__ Stats join_wave(Stats s)
{
    for (int d = 1; d < 64; d *= 2)
        s = join(s, Stats{__shfl_xor(s.m, d, 64), __shfl_xor(s.S, d, 64), __shfl_xor(s.U, d, 64)});
    return s;
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
constexpr uint32_t kOrderNegInf = 0x007fffffu;  // order_of(-inf)

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

// The waves' buffers to the workgroup's n largest entries in descending
// order (all threads take part).
__device__ __forceinline__ int gather(uint64_t (*buf)[kBuffer], int *counts, uint64_t *out, int count, int n, int tid)
{
    const int lane = tid & 63, wave = tid >> 6;
    count = cut_back(buf[wave], count, n, lane);
    if (lane == 0)
        counts[wave] = count;
    __syncthreads();
    int total = 0;
    for (int w = 0; w < kWaves; ++w)
        total += counts[w];
    const int w0 = tid / kMaxTop, i0 = tid % kMaxTop;
    if (w0 < kWaves && i0 < counts[w0]) {
        const uint64_t mine = buf[w0][i0];
        int rank = 0;
        for (int w = 0; w < kWaves; ++w)
            for (int i = 0; i < counts[w]; ++i)
                rank += buf[w][i] > mine;
        if (rank < n)
            out[rank] = mine;
    }
    __syncthreads();
    return min(total, n);
}

// VEC values of a row from index v (those at or past `end`: -inf).
template <int DT, int VEC>
__device__ __forceinline__ void load_values(const void *row, int v, int end, float (&x)[VEC])
{
    if constexpr (DT == 2) {
        const float *const q = (const float *)row + v;
        if (v + VEC <= end) {
            const f32x4 t = load_any<f32x4>(q);
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                x[e] = t[e];
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                x[e] = v + e < end ? q[e] : -__builtin_inff();
        }
    } else {
        const uint16_t *const q = (const uint16_t *)row + v;
        if (v + VEC <= end) {
            const u32x4 t = load_any<u32x4>(q);
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                x[e] = to_float<DT>((uint16_t)(t[e / 2] >> (16 * (e & 1))));
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                x[e] = v + e < end ? to_float<DT>(q[e]) : -__builtin_inff();
        }
    }
}

template <int DT, bool TOP>
__global__ void __launch_bounds__(kThreads)
logprob_rows(LogprobParams p)
{
    constexpr int VEC = DT == 2 ? 4 : 8, UN = kLane / VEC;
    __shared__ uint64_t buf[TOP ? kWaves : 1][kBuffer];
    __shared__ uint64_t best[kMaxTop];
    __shared__ int counts[kWaves];
    __shared__ uint32_t bounds[kWaves];
    __shared__ Stats stats[kWaves];
    __shared__ int sh_last;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row = p.row0 + blockIdx.y;
    const int part = blockIdx.x;
    const void *const x = (const char *)p.logits + row * p.ld * (DT == 2 ? 4 : 2);
    const int v0 = part * p.part_len, v1 = min(p.V, v0 + p.part_len);
    const int n = p.top, every = (n + kWaves - 1) / kWaves;

    Stats s = {-__builtin_inff(), 0.0f, 0.0f};
    float lane_max = -__builtin_inff();
    uint64_t cut = 0;      // nothing at or below it is among this wave's n largest
    int kept = 0;

    auto stat_batch = [&](const float (&v)[UN][VEC]) {
        float most = v[0][0];
#pragma unroll
        for (int i = 1; i < kLane; ++i)
            most = fmaxf(most, v[i / VEC][i % VEC]);
        const float m = fmaxf(s.m, most);
        const float d = fmaxf(s.m - m, kLowest), f = shrink(d);
        s.U = f * fmaf(s.S, d, s.U);
        s.S *= f;
        s.m = m;
        const float ref = m == -__builtin_inff() ? 0.0f : m;
#pragma unroll
        for (int i = 0; i < kLane; ++i) {
            const float t = v[i / VEC][i % VEC] - ref;
            const float e = __builtin_amdgcn_exp2f(t * kLog2e);
            s.S += e;
            s.U = fmaf(e, fmaxf(t, kLowest), s.U);
        }
        lane_max = fmaxf(lane_max, most);
    };
    // this wave's bound: the `every`-th largest of its lanes' maxima
    auto renew = [&] {
        uint32_t mine = order_of(lane_max), most = 0;
        for (int i = 0; i < every; ++i) {
            most = mine;
            for (int d = 1; d < 64; d *= 2)
                most = max(most, (uint32_t)__shfl_xor((int)most, d, 64));
            const uint64_t who = __ballot(mine == most);
            if (lane == __builtin_ctzll(who))
                mine = 0;
        }
        if (lane == 0)
            *(volatile uint32_t *)&bounds[wave] = most;
    };
    auto keep_batch = [&](const float (&v)[UN][VEC], int at) {
        uint32_t bound = 0xffffffffu;
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
            bound = min(bound, *(volatile uint32_t *)&bounds[w]);
        bound = max(bound, (uint32_t)(cut >> 32));
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            float most = v[u][0];
#pragma unroll
            for (int e = 1; e < VEC; ++e)
                most = fmaxf(most, v[u][e]);
            if (!__any(order_of(most) >= bound || bound <= kOrderNegInf))
                continue;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const int index = at + 64 * VEC * u + VEC * lane + e;
                const uint32_t key = order_of(v[u][e]);
                const uint64_t entry = entry_of(key, index);
                bool on = index < v1 && v[u][e] == v[u][e] && key >= bound && entry > cut;
                uint64_t who = __ballot(on);
                if (who == 0)
                    continue;
                if (kept + __popcll(who) > kBuffer) {
                    kept = cut_back(buf[wave], kept, n, lane);
                    if (kept == n) {
                        cut = buf[wave][n - 1];
                        bound = max(bound, (uint32_t)(cut >> 32));
                        on = on && entry > cut;
                        who = __ballot(on);
                    }
                }
                if (on)
                    buf[wave][kept + __popcll(who & ((1ull << lane) - 1))] = entry;
                kept += __popcll(who);
            }
        }
    };
    auto load_batch = [&](float (&v)[UN][VEC], int at) {
#pragma unroll
        for (int u = 0; u < UN; ++u)
            load_values<DT, VEC>(x, at + 64 * VEC * u + VEC * lane, v1, v[u]);
    };

    {
        // the first batch sets the bounds that its own values are held to
        float v[UN][VEC];
        const int at = v0 + wave * kBatch;
        load_batch(v, at);
        stat_batch(v);
        if constexpr (TOP) {
            renew();
            __syncthreads();
            keep_batch(v, at);
        }
    }
    int done = 1;
    for (int at = v0 + (wave + kWaves) * kBatch; at < v1; at += kWaves * kBatch) {
        float v[UN][VEC];
        load_batch(v, at);
        stat_batch(v);
        if constexpr (TOP) {
            ++done;
            if ((done & (done - 1)) == 0)
                renew();
            keep_batch(v, at);
        }
    }

    s = join_wave(s);
    if (lane == 0)
        stats[wave] = s;
    int found = 0;
    if constexpr (TOP)
        found = gather(buf, counts, best, kept, n, tid);
    else
        __syncthreads();
    s = stats[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w)
        s = join(s, stats[w]);

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
            }
        }
        __syncthreads();
        if (!sh_last)
            return;
        asm volatile("" ::: "memory");
        Stats q = {-__builtin_inff(), 0.0f, 0.0f};
        if (lane < p.parts) {
            Stats *const from = p.stat + r * p.parts + lane;
            q.m = __hip_atomic_load(&from->m, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            q.S = __hip_atomic_load(&from->S, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            q.U = __hip_atomic_load(&from->U, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        s = join_wave(q);
        if constexpr (TOP) {
            kept = 0;
            for (int q0 = wave; q0 < p.parts; q0 += kWaves) {
                uint64_t e = 0;
                if (lane < n)
                    e = __hip_atomic_load(p.best + (r * p.parts + q0) * n + lane, __ATOMIC_RELAXED,
                                          __HIP_MEMORY_SCOPE_AGENT);
                const uint64_t who = __ballot(e != 0);   // an entry is never 0: its index is below 2^31
                if (kept + __popcll(who) > kBuffer)
                    kept = cut_back(buf[wave], kept, n, lane);
                if (e != 0)
                    buf[wave][kept + __popcll(who & ((1ull << lane) - 1))] = e;
                kept += __popcll(who);
            }
            found = gather(buf, counts, best, kept, n, tid);
        }
    }

    if (wave != 0)
        return;
    const float log_S = logf(s.S);
    const bool empty = s.m == -__builtin_inff() && s.S == 0.0f;   // every logit is -inf
    if (lane == 0) {
        if (p.lse)
            p.lse[row] = empty ? -__builtin_inff() : s.m + log_S;
        if (p.entropy)
            p.entropy[row] = empty ? 0.0f : log_S - s.U / s.S;
        if (p.logprob) {
            const int64_t t = p.targets[row];
            float v = 0.0f;
            if (t >= p.V)
                v = __builtin_nanf("");
            else if (t >= 0) {
                float xt;
                if constexpr (DT == 2)
                    xt = ((const float *)x)[t];
                else
                    xt = to_float<DT>(((const uint16_t *)x)[t]);
                v = empty ? -__builtin_inff() : (xt - s.m) - log_S;
            }
            p.logprob[row] = v;
        }
    }
    if (TOP && lane < n) {
        const bool is = lane < found;
        const uint64_t e = is ? best[lane] : 0;
        p.top_id[row * n + lane] = is ? (int64_t)(0xffffffffu - (uint32_t)e) : -1;
        p.top_logprob[row * n + lane] = !is ? __builtin_nanf("") : empty ? -__builtin_inff() : (value_of((uint32_t)(e >> 32)) - s.m) - log_S;
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
};

// dx = d_logprob (delta - p) - d_entropy p (log p + entropy) + d_lse p, with
// log p = x - lse: a read and a write of every logit, the bytes of which bound
// it.  A workgroup takes kGradSpan values of one row.
constexpr int kGradThreads = 256, kGradSpan = kGradThreads * 8 * 2;

template <int DT>
__global__ void __launch_bounds__(kGradThreads)
logprob_grad(GradParams p)
{
    constexpr int VEC = DT == 2 ? 4 : 8, UN = kGradSpan / (kGradThreads * VEC);
    const int64_t row = p.row0 + blockIdx.y;
    const int v0 = blockIdx.x * kGradSpan;
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

    float v[UN][VEC];
#pragma unroll
    for (int u = 0; u < UN; ++u)
        load_values<DT, VEC>(x, v0 + (u * kGradThreads + (int)threadIdx.x) * VEC, p.V, v[u]);
#pragma unroll
    for (int u = 0; u < UN; ++u) {
        const int at = v0 + (u * kGradThreads + (int)threadIdx.x) * VEC;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const float t = v[u][e] - lse;
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
}

}  // namespace xlogprob_dev
