// dpo_logprobs.cuh -- a row's distribution: its maximum, sum and entropy in one pass, and its
// most likely ids.
#pragma once

#include "dpo_ends.cuh"
#include "dpo_two.cuh"
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
    // over the lanes of the warp, or every LOW-th of them, in all of these: one exponential, to the
    // largest maximum
    template <int LOW = 1> __device__ __forceinline__ void warp_join()
    {
        float top = m;
#pragma unroll
        for (int o = 16; o >= LOW; o >>= 1)
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        raise(top);
#pragma unroll
        for (int o = 16; o >= LOW; o >>= 1) {
            s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
            w += __shfl_xor_sync(0xFFFFFFFFu, w, o);
        }
    }
    __device__ __forceinline__ float log_sum() const { return logf(s); }
    __device__ __forceinline__ float entropy() const { return logf(s) - w / s; }
};

// A thread's share of a row, added up in units of 2 and as pairs: with the largest logit l so far
// at m and c = scale log2(e), sums of 2^t and 2^t t, t = l c - r by one multiply-add, r = m c rounded.
// t of m itself is then not 0 but `off`, that rounding: what the end takes out again.
struct Run {
    float m = -INFINITY, r = -INFINITY, off = 0.0f;
    Two s = 0, w = 0;

    // For |r| below 2^14 `off` is below 2^-11 (beyond, and for infinities: add_far, at half the
    // speed), and logits below -kLow, which come as that, add nothing: scales are at least 1e-20,
    // so that t is below -1e10. Then nothing needs a guard for infinities.
    static constexpr float kLow = 1e30f;
    __device__ __forceinline__ bool near() const { return fabsf(r) < 16384.0f; }

    __device__ __forceinline__ void raise(float to, float c)
    {
        const float from = m, had = off, sum = of_two(s).x;
        m = to;
        r = to * c;
        off = near() ? fmaf(to, c, -r) : 0.0f;
        if (s != 0) {
            const float t = (from - to) * c + (off - had), f = exp2_fast(t);
            const Two ff = two(f, f);
            w = mul_two(fma_two(two(t, t), s, w), ff);
            s = mul_two(s, ff);
            if (f == 0.0f) {   // t may be -infinity; a NaN stays
                w = 0;
                s = sum == sum && of_two(s).y == of_two(s).y ? 0 : two(NAN, NAN);
            }
        }
    }
    __device__ __forceinline__ void add_near(Two l, Two c, Two minus_r)
    {
        const Two t = fma_two(l, c, minus_r);
        const float2 u = of_two(t);
        const Two e = two(exp2_fast(u.x), exp2_fast(u.y));
        s = add_two(s, e);
        w = fma_two(t, e, w);
    }
    __device__ __forceinline__ void add_far(float l, float c)
    {
        const float t = (l - (m == -INFINITY ? 0.0f : m)) * c, e = exp2_fast(t);
        s = add_two(s, two(e, 0.0f));
        w = add_two(w, two(fmaxf(t, -kLow) * e, 0.0f));   // no infinity times 0
    }
    // One logit.
    __device__ __forceinline__ void add(float l, float c)
    {
        if (l > m)
            raise(l, c);
        if (near()) {
            const float t = fmaf(fmaxf(l, -kLow), c, -r), e = exp2_fast(l == l ? t : l);
            s = add_two(s, two(e, 0.0f));
            w = add_two(w, two(t * e, 0.0f));
        } else {
            add_far(l, c);
        }
    }
    __device__ __forceinline__ Part part(float scale) const
    {
        Part p;
        const float2 ss = of_two(s), ww = of_two(w);
        p.m = __fmul_rn(m, scale);
        p.s = ss.x + ss.y;
        const float f = exp2_fast(-off);
        p.w = fmaf(-off, p.s, ww.x + ww.y) * f * 0.6931471805599453f;
        p.s *= f;
        if (isinf(p.m) && !isinf(m)) {   // the products are infinite: masked, or no numbers
            p.s = p.m < 0.0f ? 0.0f : NAN;
            p.w = 0.0f;
        }
        return p;
    }
};

// An access of -infinity, the largest of its elements, past NaN, and pairs of them in fp32, as they
// are or not below `low` (NaN stays). Pairs of bf16 are compared as pairs.
__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t max_pair_or_nan(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
template <class T> struct RowAccess;
template <> struct RowAccess<__nv_bfloat16> {
    static constexpr int V = 8;
    using Low = uint32_t;      // bf16 twice
    static constexpr Low kLow = 0xF14AF14Au;   // about -Run::kLow
    Vec<__nv_bfloat16, V> v;
    __device__ __forceinline__ void none()
    {
#pragma unroll
        for (int i = 0; i < V / 2; ++i)
            v.w[i] = 0xFF80FF80u;
    }
    __device__ __forceinline__ float largest() const
    {
        const uint32_t top = max_pair(max_pair(v.w[0], v.w[1]), max_pair(v.w[2], v.w[3]));
        return fmaxf(__uint_as_float(top << 16), __uint_as_float(top & 0xFFFF0000u));
    }
    __device__ __forceinline__ Two pair(int i, Low low) const
    {
        const uint32_t q = max_pair_or_nan(v.w[i], low);
        return two(__uint_as_float(q << 16), __uint_as_float(q & 0xFFFF0000u));
    }
};
template <> struct RowAccess<float> {
    static constexpr int V = 4;
    using Low = float;
    static constexpr Low kLow = -Run::kLow;
    Vec<float, V> v;
    __device__ __forceinline__ void none()
    {
#pragma unroll
        for (int i = 0; i < V; ++i)
            v.w[i] = 0xFF800000u;
    }
    __device__ __forceinline__ float largest() const
    {
        return fmaxf(fmaxf(v.get(0), v.get(1)), fmaxf(v.get(2), v.get(3)));
    }
    __device__ __forceinline__ Two pair(int i, Low low) const
    {
        float a, b;
        asm("max.NaN.f32 %0, %1, %2;" : "=f"(a) : "f"(v.get(2 * i)), "f"(low));
        asm("max.NaN.f32 %0, %1, %2;" : "=f"(b) : "f"(v.get(2 * i + 1)), "f"(low));
        return two(a, b);
    }
};

// ---------------------------------------------------------- the largest ----
// A value and its id as one number: the larger value first, of equal ones the lower id; NaN behind
// -infinity, whose first word is 0x007FFFFF. 0 is behind all.
using Key = unsigned long long;
__device__ __forceinline__ Key key_of(float v, int id)
{
    const uint32_t u = __float_as_uint(v + 0.0f);   // -0 is 0
    const uint32_t high = v == v ? u ^ ((uint32_t)((int)u >> 31) | 0x80000000u) : 1u;
    return (Key)high << 32 | (uint32_t)(0x7FFFFFFF - id);
}
__device__ __forceinline__ float value_of(Key k)
{
    const uint32_t u = (uint32_t)(k >> 32);
    return __uint_as_float(u ^ (u >> 31 ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ __forceinline__ int id_of(Key k) { return 0x7FFFFFFF - (int)(uint32_t)k; }

__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float smaller(float a, float b) { return fminf(a, b); }
__device__ __forceinline__ Key larger(Key a, Key b) { return a > b ? a : b; }
__device__ __forceinline__ Key smaller(Key a, Key b) { return a < b ? a : b; }

// One step of a sorting network: the larger of two lanes' numbers goes to the lower lane, or
// where down is false to the upper one.
template <class K> __device__ __forceinline__ void exchange(K &p, int lane, int stride, bool down)
{
    const K o = __shfl_xor_sync(0xFFFFFFFFu, p, stride);
    p = ((lane & stride) == 0) == down ? larger(p, o) : smaller(p, o);
}
// A warp's 32, one a lane, the largest first.
template <class K> __device__ __forceinline__ void sort_lanes(K &p, int lane)
{
#pragma unroll
    for (int size = 2; size <= 32; size *= 2)
#pragma unroll
        for (int stride = size / 2; stride > 0; stride /= 2)
            exchange(p, lane, stride, (lane & size) == 0);
}
// The 32 first of two lists; `other` is lane 31 - lane's of the second.
template <class K> __device__ __forceinline__ void merge_lanes(K &p, K other, int lane)
{
    p = larger(p, other);
#pragma unroll
    for (int stride = 16; stride > 0; stride /= 2)
        exchange(p, lane, stride, true);
}

// A warp's list to which keys are offered one by one; most are behind `last`, the top-th or a
// bound on it that is known, and cost a vote.
struct TopList {
    Key p, last;
    int top, lane;

    // One key of each lane; called by the whole warp.
    __device__ __forceinline__ void offer(Key c)
    {
        unsigned who = __ballot_sync(0xFFFFFFFFu, c > last);
        while (who != 0u) {
            const Key q = __shfl_sync(0xFFFFFFFFu, c, __ffs(who) - 1);
            who &= who - 1;
            if (q <= last)
                continue;   // others came between
            const Key up = __shfl_up_sync(0xFFFFFFFFu, p, 1);
            if (q > p)
                p = lane > 0 && q > up ? up : q;
            last = larger(last, __shfl_sync(0xFFFFFFFFu, p, top - 1));
        }
    }
};

}  // namespace
}  // namespace dpo
