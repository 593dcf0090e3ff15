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
    // The id of token t, -1 for one outside 0 .. vocab - 1.
    __device__ __forceinline__ int at(int64_t t, int64_t vocab) const
    {
        if (ld != cols) {
            const int64_t r = t / cols;
            t += r * (ld - cols);
        }
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
};

}  // namespace
}  // namespace dpo
