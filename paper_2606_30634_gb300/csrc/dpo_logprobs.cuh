// dpo_logprobs.cuh -- a row's distribution: its maximum, sum and entropy in one pass, and its
// most likely ids.
#pragma once

#include "dpo_ends.cuh"
#include "dpo_vec.cuh"

#include <math.h>

namespace dpo {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

// 2^x by the hardware's approximation (relative error about 2^-22); a subnormal result is 0.
__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// What a part of a row comes to: m = max z, s = sum e^(z - m), w = sum e^(z - m) (z - m).
// z = -infinity takes no part, which m = -infinity (nothing yet) must not turn into NaN; a
// NaN or +infinity reaches s.
struct Part {
    float m = -INFINITY, s = 0.0f, w = 0.0f;

    // The same sums from another maximum, >= m.
    __device__ __forceinline__ void raise(float to)
    {
        if (s != 0.0f) {
            const float d = m - to, f = exp2_fast(d * kLog2e);
            w = fmaf(d, s, w) * f;
            s *= f;
            if (f == 0.0f && s == s)
                w = 0.0f;   // d may be -infinity
        }
        m = to;
    }
    __device__ __forceinline__ void join(const Part &o)
    {
        Part p = o;
        const float to = fmaxf(m, p.m);
        raise(to);
        p.raise(to);
        s += p.s;
        w += p.w;
    }
    // over the lanes of the warp, in all of them
    __device__ __forceinline__ void warp_join()
    {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            Part p;
            p.m = __shfl_xor_sync(0xFFFFFFFFu, m, o);
            p.s = __shfl_xor_sync(0xFFFFFFFFu, s, o);
            p.w = __shfl_xor_sync(0xFFFFFFFFu, w, o);
            join(p);
        }
    }
    __device__ __forceinline__ float log_sum() const { return logf(s); }
    __device__ __forceinline__ float entropy() const { return logf(s) - w / s; }
};

// A thread's share of a row, added up in units of 2: t = (l - largest) c, sums of 2^t and 2^t t.
struct Run {
    float m = -INFINITY, s = 0.0f, w = 0.0f;

    // N values whose largest is top; `clamped` are the same, not below -kLow (where the values
    // are products with a scale, that times the scale). From a largest value above `low`, a tenth
    // of it, what is below adds nothing, and then no guard is needed for infinities
    // (scales are from 1e-20 to 1e6); rows that are lower go by `values`.
    static constexpr float kLow = 1e30f;
    template <int N>
    __device__ __forceinline__ void add(const float (&values)[N], const float (&clamped)[N], float top, float c,
                                        float low)
    {
        if (top > m)
            raise(top, c);
        if (m > low) {
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float t = (clamped[j] - m) * c, e = exp2_fast(t);
                s += e;
                w = fmaf(t, e, w);
            }
        } else {
            const float from = m == -INFINITY ? 0.0f : m;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float t = (values[j] - from) * c, e = exp2_fast(t);
                s += e;
                w = fmaf(fmaxf(t, -kLow), e, w);   // no infinity times 0
            }
        }
    }
    __device__ __forceinline__ void raise(float to, float c)
    {
        if (s != 0.0f) {
            const float t = (m - to) * c, f = exp2_fast(t);
            w = fmaf(t, s, w) * f;
            s *= f;
            if (f == 0.0f && s == s)
                w = 0.0f;   // t may be -infinity
        }
        m = to;
    }
    __device__ __forceinline__ Part part(float scale) const
    {
        Part p;
        p.m = __fmul_rn(m, scale);
        p.s = s;
        p.w = w * 0.6931471805599453f;
        if (isinf(p.m) && !isinf(m)) {   // the products are infinite: masked, or no numbers
            p.s = p.m < 0.0f ? 0.0f : NAN;
            p.w = 0.0f;
        }
        return p;
    }
};

// An access's elements in fp32, as they are and not below -Run::kLow (NaN stays), and the
// largest of them, past NaN. Pairs of bf16 are compared as pairs.
__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
template <int V>
__device__ __forceinline__ float open_row(const Vec<__nv_bfloat16, V> &v, float (&l)[V], float (&clamped)[V])
{
    uint32_t top = v.w[0];
#pragma unroll
    for (int i = 1; i < V / 2; ++i)
        top = max_pair(top, v.w[i]);
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        uint32_t c;   // bf16(-1e30) twice
        asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(c) : "r"(v.w[i]), "r"(0xF14AF14Au));
        l[2 * i] = v.get(2 * i);
        l[2 * i + 1] = v.get(2 * i + 1);
        clamped[2 * i] = __uint_as_float(c << 16);
        clamped[2 * i + 1] = __uint_as_float(c & 0xFFFF0000u);
    }
    return fmaxf(__uint_as_float(top << 16), __uint_as_float(top & 0xFFFF0000u));
}
template <int V>
__device__ __forceinline__ float open_row(const Vec<float, V> &v, float (&l)[V], float (&clamped)[V])
{
    float top = v.get(0);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        l[i] = v.get(i);
        top = fmaxf(top, l[i]);
        asm("max.NaN.f32 %0, %1, %2;" : "=f"(clamped[i]) : "f"(l[i]), "f"(-Run::kLow));
    }
    return top;
}

// ---------------------------------------------------------- the largest ----
// 32 (value, id) pairs of a warp, one a lane, the largest first; of equal values the lower id.
struct Pair {
    float v = -INFINITY;
    int id = 0x7FFFFFFF;
    __device__ __forceinline__ bool before(const Pair &o) const { return v > o.v || (v == o.v && id < o.id); }
};
__device__ __forceinline__ Pair shfl(const Pair &p, int lane)
{
    Pair r;
    r.v = __shfl_sync(0xFFFFFFFFu, p.v, lane);
    r.id = __shfl_sync(0xFFFFFFFFu, p.id, lane);
    return r;
}
// One step of a sorting network: the earlier of two lanes' pairs goes to the lower lane, or
// where down is false to the upper one.
__device__ __forceinline__ void exchange(Pair &p, int lane, int stride, bool down)
{
    const Pair o = shfl(p, lane ^ stride);
    if (((lane & stride) == 0) == down ? o.before(p) : p.before(o))
        p = o;
}
__device__ __forceinline__ void sort_pairs(Pair &p, int lane)
{
#pragma unroll
    for (int size = 2; size <= 32; size *= 2)
#pragma unroll
        for (int stride = size / 2; stride > 0; stride /= 2)
            exchange(p, lane, stride, (lane & size) == 0);
}
// The 32 first of two lists; `other` is lane 31 - lane's of the second.
__device__ __forceinline__ void merge_pairs(Pair &p, const Pair &other, int lane)
{
    if (other.before(p))
        p = other;
#pragma unroll
    for (int stride = 16; stride > 0; stride /= 2)
        exchange(p, lane, stride, true);
}

// A warp's list to which values are offered one by one; most are behind `last`, the top-th or a
// bound on it that is known, and cost a vote.
struct TopList {
    Pair p, last;
    int top, lane;

    // One value of each lane; called by the whole warp. NaN counts as -infinity.
    __device__ __forceinline__ void offer(float z, int id)
    {
        Pair c;
        c.v = z == z ? z : -INFINITY;
        c.id = id;
        unsigned who = __ballot_sync(0xFFFFFFFFu, c.before(last));
        while (who != 0u) {
            const Pair q = shfl(c, __ffs(who) - 1);
            who &= who - 1;
            if (!q.before(last))
                continue;   // others came between
            const bool behind = q.before(p);
            const Pair up = shfl(p, lane > 0 ? lane - 1 : 0);
            const bool shift = lane > 0 && q.before(up);
            if (behind)
                p = shift ? up : q;
            const Pair end = shfl(p, top - 1);
            if (end.before(last))
                last = end;
        }
    }
};

}  // namespace
}  // namespace dpo
