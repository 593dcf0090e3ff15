// dpo_vec.cuh -- elements of a row as one access of up to 16 bytes, or two of them, for the kernels
// that move rows.
#pragma once

#include "dpo_device.cuh"

#include <cuda_bf16.h>

namespace dpo {
namespace {

// V elements as one access of at most 16 bytes, or two of them (codes: V bytes).

template <int B> struct Bytes;
template <> struct Bytes<1> {
    static __device__ __forceinline__ void ld(const void *p, uint32_t (&w)[1])
    {
        uint16_t v;
        asm volatile("ld.global.u8 %0, [%1];" : "=h"(v) : "l"(p));
        w[0] = v;
    }
    static __device__ __forceinline__ void st(void *p, const uint32_t (&w)[1])
    {
        *static_cast<uint8_t *>(p) = (uint8_t)w[0];
    }
};
template <> struct Bytes<2> {
    static __device__ __forceinline__ void ld(const void *p, uint32_t (&w)[1])
    {
        uint16_t v;
        asm volatile("ld.global.b16 %0, [%1];" : "=h"(v) : "l"(p));
        w[0] = v;
    }
    static __device__ __forceinline__ void st(void *p, const uint32_t (&w)[1])
    {
        *static_cast<uint16_t *>(p) = (uint16_t)w[0];
    }
};
template <> struct Bytes<4> {
    static __device__ __forceinline__ void ld(const void *p, uint32_t (&w)[1])
    {
        asm volatile("ld.global.b32 %0, [%1];" : "=r"(w[0]) : "l"(p));
    }
    static __device__ __forceinline__ void st(void *p, const uint32_t (&w)[1])
    {
        *static_cast<uint32_t *>(p) = w[0];
    }
};
template <> struct Bytes<8> {
    static __device__ __forceinline__ void ld(const void *p, uint32_t (&w)[2])
    {
        asm volatile("ld.global.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
    }
    static __device__ __forceinline__ void st(void *p, const uint32_t (&w)[2])
    {
        *static_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
    }
};
template <> struct Bytes<16> {
    static __device__ __forceinline__ void ld(const void *p, uint32_t (&w)[4])
    {
        asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                     : "l"(p));
    }
    static __device__ __forceinline__ void st(void *p, const uint32_t (&w)[4])
    {
        *static_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
};

template <> struct Bytes<32> {   // 16-byte aligned
    static __device__ __forceinline__ void ld(const void *p, uint32_t (&w)[8])
    {
        const uint8_t *const q = static_cast<const uint8_t *>(p);
        asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                     : "l"(q));
        asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                     : "l"(q + 16));
    }
    static __device__ __forceinline__ void st(void *p, const uint32_t (&w)[8])
    {
        static_cast<uint4 *>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        static_cast<uint4 *>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
};

__host__ __device__ constexpr int words(int bytes) { return bytes < 4 ? 1 : bytes / 4; }

// V elements of T as loaded.
template <class T, int V> struct Vec;
template <int V> struct Vec<float, V> {
    static constexpr int B = 4 * V;
    uint32_t w[V];
    __device__ __forceinline__ void load(const float *p) { Bytes<B>::ld(p, w); }
    __device__ __forceinline__ float get(int i) const { return __uint_as_float(w[i]); }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < V; ++i)
            w[i] = 0u;
    }
    __device__ __forceinline__ void set(const float (&v)[V])
    {
#pragma unroll
        for (int i = 0; i < V; ++i)
            w[i] = __float_as_uint(v[i]);
    }
    __device__ __forceinline__ void store(float *p) const { Bytes<B>::st(p, w); }
};
template <int V> struct Vec<__nv_bfloat16, V> {
    static constexpr int B = 2 * V;
    uint32_t w[words(B)];
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { Bytes<B>::ld(p, w); }
    __device__ __forceinline__ float get(int i) const
    {
        return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < words(B); ++i)
            w[i] = 0u;
    }
    __device__ __forceinline__ void set(const float (&v)[V])
    {
        if (V == 1) {
            w[0] = pack_bf16x2(v[0], 0.0f);
        } else {
#pragma unroll
            for (int i = 0; i < V / 2; ++i)
                w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
        }
    }
    __device__ __forceinline__ void store(__nv_bfloat16 *p) const { Bytes<B>::st(p, w); }
};

}  // namespace
}  // namespace dpo
