// dpo_ids.cuh -- token ids as they lie in memory.
#pragma once

#include "dpo_device.cuh"

namespace dpo {
namespace {

// Ids of a block of tokens; a vector has cols = ld.
struct Ids {
    const void *p;
    int64_t cols, ld;
    int bytes;
    __device__ __forceinline__ int64_t place(int64_t t) const
    {
        return ld != cols ? t + t / cols * (ld - cols) : t;
    }
    // The id of token t, -1 for one outside 0 .. vocab - 1.
    __device__ __forceinline__ int at(int64_t t, int64_t vocab) const
    {
        t = place(t);
        int64_t id;
        if (bytes == 8) {
            asm volatile("ld.global.b64 %0, [%1];" : "=l"(id) : "l"(static_cast<const int64_t *>(p) + t));
        } else {
            int v;
            asm volatile("ld.global.b32 %0, [%1];" : "=r"(v) : "l"(static_cast<const int *>(p) + t));
            id = v;
        }
        return id >= 0 && id < vocab ? (int)id : -1;
    }
    // Those of tokens t, t + step .., -1 from token `end` on, all requested before the first is
    // looked at (by at(), with its branch, one after the other: 16 of a thread took 6 us).
    template <int N>
    __device__ __forceinline__ void at(int64_t t, int step, int64_t end, int64_t vocab, int (&out)[N]) const
    {
        int64_t id[N];
        if (bytes == 8) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                id[i] = -1;
                if (t + i * step < end)
                    asm volatile("ld.global.b64 %0, [%1];"
                                 : "=l"(id[i])
                                 : "l"(static_cast<const int64_t *>(p) + place(t + i * step)));
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                int v = -1;
                if (t + i * step < end)
                    asm volatile("ld.global.b32 %0, [%1];"
                                 : "=r"(v)
                                 : "l"(static_cast<const int *>(p) + place(t + i * step)));
                id[i] = v;
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            out[i] = id[i] >= 0 && id[i] < vocab ? (int)id[i] : -1;
    }
};

}  // namespace
}  // namespace dpo
