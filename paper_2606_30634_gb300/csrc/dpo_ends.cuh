// dpo_ends.cuh -- what the kernels of the pipeline's ends share: the cluster's shared memory, and checks
// of ids.
#pragma once

#include "dpo_check.h"
#include "dpo_device.cuh"
#include "dpo_ids.cuh"

namespace dpo {
namespace {

__device__ __forceinline__ uint32_t cta_of_cluster()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t ctas_of_cluster()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
// The two halves of the cluster's barrier.
__device__ __forceinline__ void cluster_arrive()
{
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait()
{
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// By all threads of the cluster; orders their accesses to its shared and to global memory.
__device__ __forceinline__ void cluster_barrier()
{
    cluster_arrive();
    cluster_wait();
}
// The address of p, in this CTA's shared memory, in that of another CTA of the cluster.
__device__ __forceinline__ uint32_t in_cta(const void *p, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
                 : "=r"(r)
                 : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ uint32_t ld_cluster(uint32_t addr)
{
    uint32_t v;
    asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void st_cluster(uint32_t addr, uint32_t a)
{
    asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(addr), "r"(a) : "memory");
}
__device__ __forceinline__ void st_cluster(uint32_t addr, uint32_t a, uint32_t b)
{
    asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(addr), "r"(a), "r"(b) : "memory");
}

// n / d for n below 2^31 by a product and a shift: q = floor(n m / 2^(32 + s)) with
// m = ceil(2^(32 + s) / d), 2^s the power of two below d, whose error n / 2^(32 + s) is below 1 / d.
struct Divide {
    uint32_t m, s;
    __device__ __forceinline__ uint32_t operator()(uint32_t n) const { return __umulhi(n, m) >> s; }
};
inline Divide divide_by(uint64_t d)
{
    uint32_t s = 0;
    while (((uint64_t)2 << s) < d)
        ++s;
    return {(uint32_t)((((uint64_t)1 << (32 + s)) + d - 1) / d), s};   // d > 1
}

// Units of work that rows are made of, `per` a row; a division of 64 bits takes as many instructions
// as a short unit's work.
struct Units {
    int64_t per, all;
    Divide by;                 // per, where it is above 1 and all below 2^31
    __device__ __forceinline__ void at(int64_t unit, int64_t &row, int64_t &place) const
    {
        row = per == 1 ? unit : all >> 31 ? unit / per : (int64_t)by((uint32_t)unit);
        place = unit - row * per;
    }
};
inline Units units_of(int64_t rows, int64_t per)
{
    return {per, rows * per, per > 1 ? divide_by((uint64_t)per) : Divide{}};
}

// ---------------------------------------------------------------- host ----

// Of logits.
inline bool good_scale(float s) { return s >= 1e-20f && s <= 1e6f; }

constexpr int64_t kMaxCount = (int64_t)1 << 31;

// Ids as the kernels take them, checked, and their number.
inline int check_ids(const char *what, const dpo_ids &s, Ids *out, int64_t *count)
{
    if (s.rows < 0 || s.cols < 0 || (s.cols > 0 && s.rows >= (kMaxCount + s.cols - 1) / s.cols))
        return call_fail(DPO_EINVAL, "%s: %lld x %lld ids", what, (long long)s.rows, (long long)s.cols);
    *count = s.rows * s.cols;
    if (s.bytes != 4 && s.bytes != 8)
        return call_fail(DPO_EDTYPE, "%s: ids of %d bytes", what, s.bytes);
    if (*count == 0)
        return DPO_OK;
    const int64_t ld = s.rows == 1 ? s.cols : s.ld;
    const int rc = check_matrix(what, "ids", s.p, s.cols, ld, s.bytes);
    *out = ld == s.cols ? Ids{s.p, *count, *count, s.bytes} : Ids{s.p, s.cols, ld, s.bytes};
    return rc;
}
inline void add_ids(Buffers &b, const dpo_ids &s)
{
    b.add("ids", s.p, s.rows, s.cols, s.rows == 1 ? s.cols : s.ld, s.bytes, s.bytes, false);
}

// Elements of an access: `wide`, or 2 or 1 where sizes, pitches or addresses are not multiples.
struct Width {
    int v;
    explicit Width(int wide) : v(wide) {}
    void fit(const void *p, int64_t cols, int64_t ld, int64_t size)
    {
        if (p == nullptr)
            return;
        auto ok = [&](int n) {
            const int64_t bytes = n * size < 16 ? n * size : 16;
            return cols % n == 0 && ld % n == 0 && reinterpret_cast<uintptr_t>(p) % bytes == 0;
        };
        if (v > 2 && !ok(v))
            v = 2;
        if (v == 2 && !ok(2))
            v = 1;
    }
};

}  // namespace
}  // namespace dpo
