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
    template <int N> __device__ __forceinline__ void add(const float (&z)[N])
    {
        float top = z[0];
#pragma unroll
        for (int j = 1; j < N; ++j)
            top = fmaxf(top, z[j]);   // passes over NaN
        if (top > m)
            raise(top);
        const float from = m == -INFINITY ? 0.0f : m;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float d = z[j] - from, e = exp2_fast(d * kLog2e);
            s += e;
            w = fmaf(fmaxf(d, -1e30f), e, w);   // no infinity times 0
        }
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

// The `top` (<= 32) largest values that a warp has seen, with their ids: lane i holds the
// i-th. A value is compared with the last of them and seldom passes it: of n values in any
// order about top (1 + log(n / top)) do.
struct TopList {
    float v = -INFINITY;
    int id = 0x7FFFFFFF;
    float last_v = -INFINITY;   // the last one's, in every lane
    int last_id = 0x7FFFFFFF;
    int top, lane;

    __device__ __forceinline__ TopList(int top_, int lane_) : top(top_), lane(lane_) {}
    static __device__ __forceinline__ bool before(float av, int ai, float bv, int bi)
    {
        return av > bv || (av == bv && ai < bi);
    }
    // One value of each lane; called by the whole warp. NaN counts as -infinity.
    __device__ __forceinline__ void offer(float z, int i)
    {
        z = z == z ? z : -INFINITY;
        unsigned who = __ballot_sync(0xFFFFFFFFu, before(z, i, last_v, last_id));
        while (who != 0u) {
            const int src = __ffs(who) - 1;
            who &= who - 1;
            const float cv = __shfl_sync(0xFFFFFFFFu, z, src);
            const int ci = __shfl_sync(0xFFFFFFFFu, i, src);
            if (!before(cv, ci, last_v, last_id))
                continue;   // others came between
            const bool behind = before(cv, ci, v, id);
            const float uv = __shfl_up_sync(0xFFFFFFFFu, v, 1);
            const int ui = __shfl_up_sync(0xFFFFFFFFu, id, 1);
            const bool shift = __shfl_up_sync(0xFFFFFFFFu, (int)behind, 1) != 0 && lane > 0;
            if (behind) {
                v = shift ? uv : cv;
                id = shift ? ui : ci;
            }
            last_v = __shfl_sync(0xFFFFFFFFu, v, top - 1);
            last_id = __shfl_sync(0xFFFFFFFFu, id, top - 1);
        }
    }
    // Whether any lane's value may have to be offered.
    __device__ __forceinline__ bool wanted(float largest) const
    {
        return __any_sync(0xFFFFFFFFu, !(largest < last_v));
    }
};

}  // namespace
}  // namespace dpo
