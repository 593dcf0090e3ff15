// dpo_check.h -- host helpers of the calls that have no context: checks of types, pointers
// and pitches, and launches with their error.
#pragma once

#include "dpo.h"
#include "dpo_call.h"
#include "dpo_internal.h"

#include <cuda_runtime.h>

namespace dpo {
namespace {

inline int64_t elem_size(int dt) { return dt == DPO_BF16 ? 2 : 4; }
inline bool known(int dt) { return dt == DPO_F32 || dt == DPO_BF16; }

// Whether a matrix can be accessed V elements of `size` bytes at a time.
inline bool whole(const void *p, int64_t ld, int64_t size, int v)
{
    return p == nullptr || (reinterpret_cast<uintptr_t>(p) % (size * v) == 0 && ld % v == 0);
}

inline bool aligned_to(const void *p, int64_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

inline int sm_count()
{
    int device = 0, sms = 0;
    if (cudaGetDevice(&device) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess)
        return 0;
    return sms;
}

template <class... P, class... A>
int launch(const char *what, void (*kernel)(P...), int64_t grid, int threads, size_t smem,
           void *stream, A &&...args)
{
    const cudaError_t e = launch_pdl(kernel, dim3((unsigned)grid), threads, smem,
                                     static_cast<cudaStream_t>(stream), static_cast<A &&>(args)...);
    return e == cudaSuccess ? DPO_OK : call_fail(DPO_ECUDA, "%s: %s", what, cudaGetErrorString(e));
}

// The same in clusters of `cluster` CTAs, which divides grid.
template <class... P, class... A>
int launch_in_clusters(const char *what, void (*kernel)(P...), int64_t grid, int cluster, int threads,
                       size_t smem, void *stream, A &&...args)
{
    cudaLaunchAttribute attr[2] = {};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = static_cast<cudaStream_t>(stream);
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, static_cast<A &&>(args)...);
    const cudaError_t last = cudaGetLastError();
    e = e != cudaSuccess ? e : last;
    return e == cudaSuccess ? DPO_OK : call_fail(DPO_ECUDA, "%s: %s", what, cudaGetErrorString(e));
}

inline int check_matrix(const char *what, const char *name, const void *p, int64_t cols, int64_t ld,
                        int64_t size)
{
    if (p == nullptr)
        return call_fail(DPO_EINVAL, "%s: %s is NULL", what, name);
    if (ld < cols)
        return call_fail(DPO_EINVAL, "%s: pitch %lld of %s is below its %lld columns", what,
                         (long long)ld, name, (long long)cols);
    if (!aligned_to(p, size))
        return call_fail(DPO_EALIGN, "%s: %s is not aligned to its elements", what, name);
    return DPO_OK;
}

// The buffers of a call, for the checks of pointers, pitches and overlaps.
struct Buffers {
    struct Entry {
        const char *name;
        Extent at;
        bool out;
    };
    const char *what;
    Entry e[20];
    int n = 0, rc = DPO_OK;
    explicit Buffers(const char *w) : what(w) {}
    // rows x cols of `size`-byte elements, `align`-byte aligned, its pitch too
    void add(const char *name, const void *p, int64_t rows, int64_t cols, int64_t ld, int64_t size,
             int64_t align, bool out)
    {
        if (rc != DPO_OK)
            return;
        if (p == nullptr)
            rc = call_fail(DPO_EINVAL, "%s: %s is NULL", what, name);
        else if (ld < cols)
            rc = call_fail(DPO_EINVAL, "%s: pitch %lld of %s is below its %lld columns", what,
                           (long long)ld, name, (long long)cols);
        else if (ld > ((int64_t)1 << 36))
            rc = call_fail(DPO_EINVAL, "%s: pitch of %s", what, name);
        else if (reinterpret_cast<uintptr_t>(p) % align != 0 || ld * size % align != 0)
            rc = call_fail(DPO_EALIGN, "%s: %s or its pitch is not %lld-byte aligned", what, name,
                           (long long)align);
        if (rc != DPO_OK)
            return;
        e[n++] = {name, extent_of(p, rows, cols, ld, size), out};
    }
    void packed(const char *name, const dpo_packed8 &p, int64_t rows, int64_t cols, int64_t align,
                bool out)
    {
        add(name, p.codes, rows, cols, p.ld_codes, 1, align, out);
        add("its scales", p.scales, rows, (cols + DPO_PACK8_GROUP - 1) / DPO_PACK8_GROUP, p.ld_scales, 1, 1, out);
    }
    int done()
    {
        for (int i = 0; i < n && rc == DPO_OK; ++i)
            for (int j = 0; j < i && rc == DPO_OK; ++j)
                if ((e[i].out || e[j].out) && overlap(e[i].at, e[j].at))
                    rc = call_fail(DPO_EINVAL, "%s: %s overlaps %s", what, e[i].name, e[j].name);
        return rc;
    }
};

}  // namespace
}  // namespace dpo
