// dpo_rmsnorm.cu -- residual addition with the root-mean-square norm, its
// backward pass, and activations in 8 bits (dpo_rmsnorm, dpo_rmsnorm_backward,
// dpo_pack8, dpo_unpack8 in include/dpo.h).
//
// All four move bytes: a few operations per element against 2 to 9 bytes of it,
// so HBM bounds them, and launch latency where there are few rows.
#include "dpo.h"
#include "dpo_call.h"
#include "dpo_pack8.cuh"

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <math.h>

namespace dpo {
namespace {

// ------------------------------------------------------------- vectors ----
// V elements as one access of at most 16 bytes (codes: V bytes).

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

// V codes.
template <int V> struct Codes {
    uint32_t w[words(V)];
    __device__ __forceinline__ void load(const uint8_t *p) { Bytes<V>::ld(p, w); }
    __device__ __forceinline__ void store(uint8_t *p) const { Bytes<V>::st(p, w); }
    __device__ __forceinline__ void set(const float (&v)[V], float inv)
    {
        if constexpr (V == 1) {
            w[0] = encode2(v[0] * inv, 0.0f) & 0xFFu;
        } else if constexpr (V == 2) {
            w[0] = encode2(v[0] * inv, v[1] * inv);
        } else {
#pragma unroll
            for (int i = 0; i < V / 4; ++i)
                w[i] = encode4(v[4 * i] * inv, v[4 * i + 1] * inv, v[4 * i + 2] * inv,
                               v[4 * i + 3] * inv);
        }
    }
    __device__ __forceinline__ void get(float (&v)[V], float scale) const
    {
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            const float2 f = decode2(w[i / 4] >> (8 * (i & 3)));
            v[i] = f.x * scale;
            if (i + 1 < V)
                v[i + 1] = f.y * scale;
        }
    }
};

__device__ __forceinline__ uint32_t load_byte(const uint8_t *p)
{
    uint32_t v;
    asm volatile("ld.global.u8 %0, [%1];" : "=r"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ float load_scale(const uint8_t *p) { return scale_of(load_byte(p)); }

// Scale byte of a group whose V-element pieces lie in adjacent lanes; infinities become NaN
// in v. The maximum passes over NaN by itself, and infinities, which must not count, are
// looked for only where it found one.
template <int V>
__device__ __forceinline__ uint32_t group_scale(float (&v)[V])
{
    float a = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i)
        a = fmaxf(a, fabsf(v[i]));
#pragma unroll
    for (int off = 1; off < kGroup / V; off <<= 1)
        a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, off));
    if (__any_sync(0xFFFFFFFFu, a > kMaxFinite)) {
        a = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            a = fmaxf(a, finite_abs(v[i]));
            v[i] = inf_to_nan(v[i]);
        }
#pragma unroll
        for (int off = 1; off < kGroup / V; off <<= 1)
            a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, off));
    }
    return scale_byte(a);
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int off = 16; off > 0; off >>= 1)
        v += __shfl_xor_sync(0xFFFFFFFFu, v, off);
    return v;
}

// ---------------------------------------------------------------- norm ----
// A row is held in the registers of W warps, 32 elements a thread, so each
// input is read once. Thread i of the row takes the V-element pieces i, i + 32 W, ...:
// a group of 32 is in 32 / V adjacent lanes.

// Elements of a row per thread: 32, or 8 in the narrow forms (pieces of one or two
// elements, so that a thread's pieces are many and its row's time is their number) up to
// 4096 columns.
constexpr int kRowElems = 32, kNarrowElems = 8;
constexpr int kMinWarps = 4;                  // warps of a CTA, at least
// Threads of a CTA, at most. The bound sets the registers a thread may have.
constexpr int kCta = 512;

struct NormForwardArgs {
    dpo_rmsnorm_args a;
    int warps;                                // per row, a power of two
};

// Sum over the threads of each row of a CTA (every warp calls it); red holds a
// float per warp. The sum order is fixed.
__device__ __forceinline__ float row_sum(float v, int warps, float *red)
{
    v = warp_sum(v);
    if (warps == 1)
        return v;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0)
        red[warp] = v;
    __syncthreads();
    const int first = warp & ~(warps - 1);
    v = warp_sum(lane < warps ? red[first + lane] : 0.0f);
    __syncthreads();
    return v;
}

template <class T, class WT, int V, int E>
__global__ void __launch_bounds__(kCta)
rmsnorm_kernel(const NormForwardArgs args)
{
    constexpr int N = E / V;
    __shared__ float red[32];
    const dpo_rmsnorm_args &a = args.a;
    const int warps = args.warps, tpr = warps * 32;
    const int rows_cta = (int)blockDim.x / tpr;
    const int i0 = threadIdx.x & (tpr - 1);
    const int64_t row = (int64_t)blockIdx.x * rows_cta + threadIdx.x / tpr;
    const bool live = row < a.rows;
    const int cols = (int)a.cols;
    pdl_wait();
    float s[N][V];
    float sum = 0.0f;
    {
        Vec<T, V> x[N], r[N];
        const T *xp = static_cast<const T *>(a.x) + row * a.ld_x;
        const T *rp = static_cast<const T *>(a.residual) + row * a.ld_residual;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int c = (i0 + n * tpr) * V;
            x[n].zero();
            r[n].zero();
            if (live && c < cols) {
                x[n].load(xp + c);
                if (a.residual != nullptr)
                    r[n].load(rp + c);
            }
        }
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                s[n][j] = x[n].get(j) + r[n].get(j);
                sum = fmaf(s[n][j], s[n][j], sum);
            }
    }
    sum = row_sum(sum, warps, red);
    const float rstd = 1.0f / sqrtf(sum / (float)cols + a.eps);
    if (live && i0 == 0)
        a.rstd[row] = rstd;
    T *hp = static_cast<T *>(a.h) + row * a.ld_h;
    T *yp = static_cast<T *>(a.y) + row * a.ld_y;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const int c = (i0 + n * tpr) * V;
        const bool in = live && c < cols;
        Vec<T, V> o;
        if (in && a.h != nullptr) {
            o.set(s[n]);
            o.store(hp + c);
        }
#pragma unroll
        for (int j = 0; j < V; ++j)
            s[n][j] *= rstd;
        if (in && a.y != nullptr) {
            Vec<WT, V> w;
            w.load(static_cast<const WT *>(a.weight) + c);
            float y[V];
#pragma unroll
            for (int j = 0; j < V; ++j)
                y[j] = s[n][j] * w.get(j);
            o.set(y);
            o.store(yp + c);
        }
        if (a.x8.codes != nullptr) {   // uniform: every lane takes part in the shuffles
            const uint32_t b = group_scale<V>(s[n]);
            if (in) {
                Codes<V> q;
                q.set(s[n], inv_scale_of(b));
                q.store(a.x8.codes + row * a.x8.ld_codes + c);
                if (c % kGroup == 0)
                    a.x8.scales[row * a.x8.ld_scales + c / kGroup] = (uint8_t)b;
            }
        }
    }
}

// Backward: a persistent grid of CTAs walks the rows; a thread keeps the sums of
// dy n of its columns in registers, so dweight costs one partial row per CTA,
// which the second kernel adds up. A row is its inputs' loads, a sum over the row's
// threads and the stores; what bounds it is how many rows' inputs are on their way at
// once, since HBM answers after about 2 us under load and a row is 12 to 24 bytes a
// column. With 16-byte pieces (RING) each thread copies its own pieces of the next three
// rows to shared memory with cp.async, in places that only it reads, so no barrier
// guards them. GB300, 8192 x 4096 from 8-bit rows: one row ahead in registers 65 us, the
// ring 45.6 with the sum of the partial rows (5.2 TB/s of the 236 MB; this kernel alone
// 42.7). Slower: dy and the normalised row taken from the ring once more instead of kept
// (48.9), and with the 80 registers that this leaves three CTAs an SM (55.3).
struct NormBackArgs {
    dpo_rmsnorm_backward_args a;
    int warps;
    float *partials;                          // one row of cols per CTA
};

// E elements of a row per thread: 16, or 32 where that would take more than 512 threads
// (cols above 8192). 32 are from registers, row by row, and more than they hold: 128 to 560
// bytes spilled in the 16-byte forms (4096 x 16384 bf16 from h 140 us, 79 at the copy rate), up
// to 1.7 KB in those of one element.
constexpr int kBackElems = 16, kBackThreads = 512, kBackMinWarps = 8;
constexpr int kDepth = 4;                     // rows of the ring

// B bytes from global to shared memory, or zeros.
template <int B>
__device__ __forceinline__ void copy_async(uint32_t dst, const void *src, bool in)
{
    const int n = in ? B : 0;
    if (B == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n)
                     : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(B),
                     "r"(n)
                     : "memory");
}

// A row's inputs as one thread holds them: dy, dh, and h or the codes and scales.
template <class T, int V, int E, bool X8> struct RowRegs {
    static constexpr int N = E / V;
    Vec<T, V> dy_[N], dh_[N];
    Vec<T, X8 ? 1 : V> h[X8 ? 1 : N];
    Codes<V> q[X8 ? N : 1];
    float scale[X8 ? N : 1];
    float rstd;

    __device__ __forceinline__ void load(const dpo_rmsnorm_backward_args &a, int64_t row, int i0,
                                         int tpr)
    {
        const bool live = row < a.rows;
        rstd = live ? ld1(a.rstd + row) : 0.0f;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int c = (i0 + n * tpr) * V;
            const bool in = live && c < (int)a.cols;
            dy_[n].zero();
            dh_[n].zero();
            if (in) {
                dy_[n].load(static_cast<const T *>(a.dy) + row * a.ld_dy + c);
                if (a.dh != nullptr)
                    dh_[n].load(static_cast<const T *>(a.dh) + row * a.ld_dh + c);
            }
            if constexpr (X8) {
#pragma unroll
                for (int j = 0; j < words(V); ++j)
                    q[n].w[j] = 0u;
                scale[n] = 0.0f;
                if (in) {
                    q[n].load(a.x8.codes + row * a.x8.ld_codes + c);
                    scale[n] = load_scale(a.x8.scales + row * a.x8.ld_scales + c / kGroup);
                }
            } else {
                h[n].zero();
                if (in)
                    h[n].load(static_cast<const T *>(a.h) + row * a.ld_h + c);
            }
        }
    }
    __device__ __forceinline__ Vec<T, V> dy(int n) const { return dy_[n]; }
    __device__ __forceinline__ Vec<T, V> dh(int n) const { return dh_[n]; }
    __device__ __forceinline__ void normalised(int n, float (&v)[V]) const
    {
        if constexpr (X8) {
            q[n].get(v, scale[n]);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j)
                v[j] = h[n].get(j) * rstd;
        }
    }
};

// The same from a slot of the ring: pieces of dy, dh, and h or the codes, each [n][thread].
// rstd and the scales, single bytes, wait in registers.
// TH threads a CTA, so that a place in the ring is a constant behind the thread's own.
template <class T, int V, int E, bool X8, int TH> struct RowSlot {
    static constexpr int N = E / V, B = V * (int)sizeof(T), BH = X8 ? V : B;
    static constexpr int bytes = N * (2 * B + BH) * TH;
    uint8_t *slot;
    float rstd;
    uint32_t scale[X8 ? N : 1];   // as loaded: converting it here would wait for it

    __device__ __forceinline__ const uint8_t *piece(int kind, int n) const
    {
        const uint8_t *base = slot + (int)threadIdx.x * (kind == 2 ? BH : B);
        return base + TH * ((kind == 2 ? 2 * N * B + n * BH : (kind * N + n) * B));
    }
    __device__ __forceinline__ void load(const dpo_rmsnorm_backward_args &a, int64_t row, int i0,
                                         int tpr)
    {
        const bool live = row < a.rows;
        rstd = live ? ld1(a.rstd + row) : 0.0f;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int c = (i0 + n * tpr) * V;
            const bool in = live && c < (int)a.cols;
            auto to = [&](int kind) { return (uint32_t)__cvta_generic_to_shared(piece(kind, n)); };
            // nothing is read for a piece that is not there: its address is the matrix's
            const int64_t r = in ? row : 0;
            const int at = in ? c : 0;
            copy_async<B>(to(0), static_cast<const T *>(a.dy) + r * a.ld_dy + at, in);
            if (a.dh != nullptr)
                copy_async<B>(to(1), static_cast<const T *>(a.dh) + r * a.ld_dh + at, in);
            if constexpr (X8) {
                copy_async<BH>(to(2), a.x8.codes + r * a.x8.ld_codes + at, in);
                scale[n] = 0;
                if (in)
                    scale[n] = load_byte(a.x8.scales + row * a.x8.ld_scales + c / kGroup);
            } else {
                copy_async<BH>(to(2), static_cast<const T *>(a.h) + r * a.ld_h + at, in);
            }
        }
    }
    template <class P> __device__ __forceinline__ P get(int kind, int n) const
    {
        return *reinterpret_cast<const P *>(piece(kind, n));
    }
    struct alignas(B) Raw { uint32_t w[words(B)]; };
    struct alignas(BH) RawH { uint32_t w[words(BH)]; };
    __device__ __forceinline__ Vec<T, V> dy(int n) const
    {
        const Raw r = get<Raw>(0, n);
        Vec<T, V> v;
#pragma unroll
        for (int i = 0; i < words(B); ++i)
            v.w[i] = r.w[i];
        return v;
    }
    __device__ __forceinline__ Vec<T, V> dh(int n) const
    {
        const Raw r = get<Raw>(1, n);
        Vec<T, V> v;
#pragma unroll
        for (int i = 0; i < words(B); ++i)
            v.w[i] = r.w[i];
        return v;
    }
    __device__ __forceinline__ void normalised(int n, float (&v)[V]) const
    {
        const RawH r = get<RawH>(2, n);
        if constexpr (X8) {
            Codes<V> q;
#pragma unroll
            for (int i = 0; i < words(BH); ++i)
                q.w[i] = r.w[i];
            q.get(v, scale_of(scale[n]));
        } else {
            Vec<T, V> h;
#pragma unroll
            for (int i = 0; i < words(BH); ++i)
                h.w[i] = r.w[i];
#pragma unroll
            for (int j = 0; j < V; ++j)
                v[j] = h.get(j) * rstd;
        }
    }
};

// RING: the CTA's threads where rows come through the ring, or 0
template <class T, class WT, int V, int E, bool X8, int RING>
__global__ void __launch_bounds__(RING ? RING : kBackThreads)
rmsnorm_backward_kernel(const NormBackArgs args)
{
    constexpr int N = E / V;
    __shared__ float red[2][32];              // by the row's parity: one barrier a row
    extern __shared__ __align__(16) uint8_t smem[];   // the ring; at the end, cols floats
    const dpo_rmsnorm_backward_args &a = args.a;
    const int warps = args.warps, tpr = warps * 32;
    const int rows_cta = (int)blockDim.x / tpr;
    const int i0 = threadIdx.x & (tpr - 1), r0 = threadIdx.x / tpr;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int cols = (int)a.cols;
    const int64_t stride = (int64_t)gridDim.x * rows_cta;
    pdl_wait();
    Vec<WT, V> w[N];
    float dw[N][V];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const int c = (i0 + n * tpr) * V;
        w[n].zero();
        if (c < cols)
            w[n].load(static_cast<const WT *>(a.weight) + c);
#pragma unroll
        for (int j = 0; j < V; ++j)
            dw[n][j] = 0.0f;
    }
    int parity = 0;
    auto one_row = [&](const auto &in, int64_t row) {
        float sum = 0.0f, gk[N][V], vk[N][V];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const Vec<T, V> dyv = in.dy(n);
            in.normalised(n, vk[n]);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float dy = dyv.get(j);
                gk[n][j] = dy * w[n].get(j);
                sum = fmaf(gk[n][j], vk[n][j], sum);
                dw[n][j] = fmaf(dy, vk[n][j], dw[n][j]);
            }
        }
        sum = warp_sum(sum);
        if (warps > 1) {
            if (lane == 0)
                red[parity][warp] = sum;
            __syncthreads();
            sum = warp_sum(lane < warps ? red[parity][(warp & ~(warps - 1)) + lane] : 0.0f);
            parity ^= 1;
        }
        sum /= (float)cols;
        if (a.dx == nullptr || row >= a.rows)
            return;
        T *dxp = static_cast<T *>(a.dx) + row * a.ld_dx;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int c = (i0 + n * tpr) * V;
            if (c < cols) {
                float v[V];
                if (a.dh != nullptr) {
                    const Vec<T, V> dhv = in.dh(n);
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        v[j] = fmaf(in.rstd, fmaf(-vk[n][j], sum, gk[n][j]), dhv.get(j));
                } else {
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        v[j] = in.rstd * fmaf(-vk[n][j], sum, gk[n][j]);
                }
                Vec<T, V> o;
                o.set(v);
                o.store(dxp + c);
            }
        }
    };
    int64_t base = (int64_t)blockIdx.x * rows_cta;
    if constexpr (RING != 0) {
        using Slot = RowSlot<T, V, E, X8, RING>;
        Slot ring[kDepth];
        auto fetch = [&](Slot &s, int64_t b) {
            if (b < a.rows)
                s.load(a, b + r0, i0, tpr);
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
#pragma unroll
        for (int d = 0; d < kDepth; ++d) {
            ring[d].slot = smem + d * Slot::bytes;
            if (d < kDepth - 1)
                fetch(ring[d], base + d * stride);
        }
        while (base < a.rows) {
#pragma unroll
            for (int d = 0; d < kDepth; ++d) {
                if (base >= a.rows)
                    break;
                fetch(ring[(d + kDepth - 1) % kDepth], base + (kDepth - 1) * stride);
                asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 1) : "memory");
                one_row(ring[d], base + r0);
                base += stride;
            }
        }
    } else {
        for (; base < a.rows; base += stride) {
            RowRegs<T, V, E, X8> in;
            in.load(a, base + r0, i0, tpr);
            one_row(in, base + r0);
        }
    }
    if (a.dweight == nullptr)
        return;
    float *out = args.partials + (int64_t)blockIdx.x * cols;
    if (rows_cta > 1) {   // the CTA's rows, in order
        float *dw_cta = reinterpret_cast<float *>(smem);
        __syncthreads();   // nobody reads the ring any more
        for (int r = 0; r < rows_cta; ++r) {
            if (r0 == r)
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    const int c = (i0 + n * tpr) * V;
                    if (c < cols)
#pragma unroll
                        for (int j = 0; j < V; ++j) {
                            if (r > 0)
                                dw[n][j] = dw_cta[c + j] + dw[n][j];
                            dw_cta[c + j] = dw[n][j];
                        }
                }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < cols; c += blockDim.x)
            out[c] = dw_cta[c];
        return;
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const int c = (i0 + n * tpr) * V;
        if (c < cols)
#pragma unroll
            for (int j = 0; j < V; ++j)
                out[c + j] = dw[n][j];
    }
}

// dweight[c] = the sum of the n partial rows, in a fixed order. A CTA takes 8 columns, a
// sector of each row: 64 shares of the rows, four to a warp, ten loads of each in flight,
// added up in order; more columns to a CTA are fewer CTAs and a longer chain of loads.
constexpr int kSumCols = 8, kSumWarps = 16, kSumLoads = 10, kSumShares = kSumWarps * 4;
template <class GT>
__global__ void __launch_bounds__(32 * kSumWarps)
rmsnorm_dweight_kernel(const float *partials, int n, int cols, GT *dweight, int accumulate)
{
    __shared__ float share[kSumWarps][kSumCols];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = blockIdx.x * kSumCols + (lane & 7);
    pdl_wait();
    float sum = 0.0f;
    if (c < cols)
        for (int i = warp * 4 + (lane >> 3); i < n; i += kSumShares * kSumLoads) {
            float v[kSumLoads];
#pragma unroll
            for (int u = 0; u < kSumLoads; ++u) {
                const int at = i + u * kSumShares;
                v[u] = at < n ? ld1(partials + (int64_t)at * cols + c) : 0.0f;
            }
#pragma unroll
            for (int u = 0; u < kSumLoads; ++u)
                sum += v[u];
        }
    sum += __shfl_down_sync(0xFFFFFFFFu, sum, 16);
    sum += __shfl_down_sync(0xFFFFFFFFu, sum, 8);
    if (lane < kSumCols)
        share[warp][lane] = sum;
    __syncthreads();
    if (warp != 0 || lane >= kSumCols || c >= cols)
        return;
    sum = share[0][lane];
#pragma unroll
    for (int i = 1; i < kSumWarps; ++i)
        sum += share[i][lane];
    if (accumulate)
        sum += ld1(dweight + c);
    st1(dweight + c, sum);
}

// ---------------------------------------------------------------- pack ----
// A warp takes spans of span_of_pieces(V) elements of a row, V a lane at a time: 1024, or in
// the narrow forms eight pieces a lane, whose number is then the time of a small matrix.

constexpr int kPackThreads = 256;
__host__ __device__ constexpr int span_of_pieces(int v) { return v >= 4 ? 1024 : 8 * 32 * v; }

struct PackArgs {
    const void *x;                            // pack: in; unpack: out
    uint8_t *codes, *scales;
    int64_t ld_x, ld_codes, ld_scales;
    int64_t rows;
    int cols, spans;                          // spans per row
    int64_t step_rows;                        // from a warp's span to its next one
    int step_spans;
    int beside;                               // see unpack8_beside
};

template <class T, int V, bool Unpack>
__global__ void __launch_bounds__(kPackThreads)
pack8_kernel(const PackArgs a)
{
    constexpr int kSpan = span_of_pieces(V), N = kSpan / 32 / V;
    const int lane = threadIdx.x & 31;
    const int64_t first = (int64_t)blockIdx.x * (kPackThreads / 32) + (threadIdx.x >> 5);
    int64_t row = first / a.spans;
    int span = (int)(first - row * a.spans);
    if (a.beside)
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    else
        pdl_wait();
    for (; row < a.rows; row += a.step_rows) {
        const int c0 = span * kSpan;
        T *const xp = const_cast<T *>(static_cast<const T *>(a.x)) + row * a.ld_x;
        uint8_t *const qp = a.codes + row * a.ld_codes;
        uint8_t *const sp = a.scales + row * a.ld_scales;
        if (Unpack) {
            Codes<V> q[N];
            uint32_t sc[N];
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int c = c0 + (lane + n * 32) * V;
                if (c < a.cols) {
                    q[n].load(qp + c);
                    sc[n] = load_byte(sp + c / kGroup);
                }
            }
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int c = c0 + (lane + n * 32) * V;
                if (c < a.cols) {
                    float v[V];
                    q[n].get(v, scale_of(sc[n]));
                    Vec<T, V> o;
                    o.set(v);
                    o.store(xp + c);
                }
            }
        } else {
            Vec<T, V> x[N];
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int c = c0 + (lane + n * 32) * V;
                x[n].zero();
                if (c < a.cols)
                    x[n].load(xp + c);
            }
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int c = c0 + (lane + n * 32) * V;
                float v[V];
#pragma unroll
                for (int j = 0; j < V; ++j)
                    v[j] = x[n].get(j);
                const uint32_t b = group_scale<V>(v);
                if (c < a.cols) {
                    Codes<V> q;
                    q.set(v, inv_scale_of(b));
                    q.store(qp + c);
                    if (c % kGroup == 0)
                        sp[c / kGroup] = (uint8_t)b;
                }
            }
        }
        span += a.step_spans;
        if (span >= a.spans) {
            span -= a.spans;
            ++row;
        }
    }
    if (a.beside)
        pdl_wait();
}

// ---------------------------------------------------------------- host ----

int64_t elem_size(int dt) { return dt == DPO_BF16 ? 2 : 4; }
bool known(int dt) { return dt == DPO_F32 || dt == DPO_BF16; }

// Whether a matrix can be accessed V elements of `size` bytes at a time.
bool whole(const void *p, int64_t ld, int64_t size, int v)
{
    return p == nullptr || (reinterpret_cast<uintptr_t>(p) % (size * v) == 0 && ld % v == 0);
}

bool aligned_to(const void *p, int64_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

int sm_count()
{
    int device = 0, sms = 0;
    if (cudaGetDevice(&device) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess)
        return 0;
    return sms;
}

// Warps of a row with so many elements a thread.
int row_warps(int64_t cols, int elems)
{
    int w = 1;
    while ((int64_t)w * 32 * elems < cols)
        w *= 2;
    return w;
}

// The backward's shape: elements of a row per thread, warps of a row and of a CTA, CTAs.
struct BackShape {
    int elems, warps, cta;
    int64_t grid;
};
BackShape back_shape(int64_t rows, int64_t cols, int sms)
{
    BackShape b;
    b.elems = cols <= (int64_t)kBackThreads * kBackElems ? kBackElems : kRowElems;
    b.warps = row_warps(cols, b.elems);
    b.cta = b.warps > kBackMinWarps ? b.warps : kBackMinWarps;
    const int64_t want = (rows + b.cta / b.warps - 1) / (b.cta / b.warps);
    // 16 warps an SM, as many as are resident by registers. Of an fp32 ring's CTAs (8 warps,
    // 192 KB, from 8-bit rows 144 KB) one is, and the grid runs in two waves: 4096 x 4096 from
    // h 47.5 us (39.6 at the copy rate), from 8-bit rows 49.3 (32.2).
    const int64_t most = (int64_t)sms * (16 / b.cta);
    b.grid = want < most ? want : most;
    return b;
}

template <class... P, class... A>
int launch(const char *what, void (*kernel)(P...), int64_t grid, int threads, size_t smem,
           void *stream, A &&...args)
{
    const cudaError_t e = launch_pdl(kernel, dim3((unsigned)grid), threads, smem,
                                     static_cast<cudaStream_t>(stream), static_cast<A &&>(args)...);
    return e == cudaSuccess ? DPO_OK : call_fail(DPO_ECUDA, "%s: %s", what, cudaGetErrorString(e));
}

int check_packed(const char *what, const dpo_packed8 &p, int64_t cols)
{
    if (p.codes == nullptr || p.scales == nullptr)
        return call_fail(DPO_EINVAL, "%s: codes and scales are needed", what);
    if (p.ld_codes < cols || p.ld_scales < groups_of(cols))
        return call_fail(DPO_EINVAL, "%s: a pitch of the 8-bit matrix is below its row", what);
    return DPO_OK;
}

constexpr int64_t kMaxRows = (int64_t)1 << 31;
constexpr int kMaxSmem = 226 * 1024;   // dynamic, beside the kernel's own 256 bytes

int check_matrix(const char *what, const char *name, const void *p, int64_t cols, int64_t ld,
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

template <class T, bool Unpack>
auto pack_kernel(int v) -> void (*)(PackArgs)
{
    if (sizeof(T) == 2 && v == 8)
        return pack8_kernel<T, sizeof(T) == 2 ? 8 : 4, Unpack>;
    if (sizeof(T) == 4 && v >= 4)
        return pack8_kernel<T, 4, Unpack>;
    if (sizeof(T) == 2 && v == 2)
        return pack8_kernel<T, sizeof(T) == 2 ? 2 : 1, Unpack>;
    return pack8_kernel<T, 1, Unpack>;
}

int pack_or_unpack(const char *what, const void *x, dpo_dtype dtype, int64_t rows, int64_t cols,
                   int64_t ld_x, const dpo_packed8 *p, bool unpack, void *stream, bool beside = false)
{
    if (!known(dtype))
        return call_fail(DPO_EDTYPE, "%s: dtype %d", what, (int)dtype);
    if (rows < 0 || cols < 0 || rows >= kMaxRows || cols >= kMaxRows / 2)
        return call_fail(DPO_EINVAL, "%s: %lld x %lld", what, (long long)rows, (long long)cols);
    if (p == nullptr)
        return call_fail(DPO_EINVAL, "%s: no 8-bit matrix", what);
    if (rows == 0 || cols == 0)
        return DPO_OK;
    const int64_t size = elem_size(dtype);
    int rc = check_matrix(what, unpack ? "out" : "x", x, cols, ld_x, size);
    if (rc == DPO_OK)
        rc = check_packed(what, *p, cols);
    if (rc != DPO_OK)
        return rc;
    const Extent sx = extent_of(x, rows, cols, ld_x, size),
               sc = extent_of(p->codes, rows, cols, p->ld_codes, 1),
               ss = extent_of(p->scales, rows, groups_of(cols), p->ld_scales, 1);
    if (overlap(sx, sc) || overlap(sx, ss) || (!unpack && overlap(sc, ss)))
        return call_fail(DPO_EINVAL, "%s: buffers overlap", what);
    const int sms = sm_count();
    if (sms == 0)
        return call_fail(DPO_ECUDA, "%s: no device", what);
    int v = dtype == DPO_BF16 ? 8 : 4;
    while (v > 1 && !(cols % v == 0 && whole(x, ld_x, size, v) && whole(p->codes, p->ld_codes, 1, v)))
        v = v == 8 ? 2 : 1;
    PackArgs a = {x, p->codes, p->scales, ld_x, p->ld_codes, p->ld_scales, rows, (int)cols, 0, 0, 0, beside};
    a.spans = (int)((cols + span_of_pieces(v) - 1) / span_of_pieces(v));
    constexpr int kWarps = kPackThreads / 32;
    // packing keeps its CTAs, all resident; widening, with little to compute, starts them as
    // they end (8192 x 11008 bf16: 4 an SM 47.8 / 40.9 us, 8 48.0 / 42.7, 64 50.0 / 37.6)
    const int64_t want = (rows * a.spans + kWarps - 1) / kWarps, most = (int64_t)sms * (unpack ? 64 : 4);
    const int64_t grid = want < most ? want : most;
    a.step_rows = grid * kWarps / a.spans;
    a.step_spans = (int)(grid * kWarps % a.spans);
    void (*k)(PackArgs);
    if (dtype == DPO_BF16)
        k = unpack ? pack_kernel<__nv_bfloat16, true>(v) : pack_kernel<__nv_bfloat16, false>(v);
    else
        k = unpack ? pack_kernel<float, true>(v) : pack_kernel<float, false>(v);
    return launch(what, k, grid, kPackThreads, 0, stream, a);
}

// The kernels by types, elements an access and elements a thread.
using FwdFn = void (*)(NormForwardArgs);
using BackFn = void (*)(NormBackArgs);
using B16 = __nv_bfloat16;

template <int E> FwdFn forward_narrow(int dtype, int wdtype, int v)
{
    if (dtype == DPO_F32)
        return rmsnorm_kernel<float, float, 1, E>;
    if (wdtype == DPO_F32)
        return v == 2 ? rmsnorm_kernel<B16, float, 2, E> : rmsnorm_kernel<B16, float, 1, E>;
    return v == 2 ? rmsnorm_kernel<B16, B16, 2, E> : rmsnorm_kernel<B16, B16, 1, E>;
}
FwdFn forward_of(int dtype, int wdtype, int v, int elems)
{
    if (v <= 2)
        return elems == kNarrowElems ? forward_narrow<kNarrowElems>(dtype, wdtype, v)
                                     : forward_narrow<kRowElems>(dtype, wdtype, v);
    if (dtype == DPO_F32)
        return rmsnorm_kernel<float, float, 4, kRowElems>;
    return wdtype == DPO_F32 ? rmsnorm_kernel<B16, float, 4, kRowElems>
                             : rmsnorm_kernel<B16, B16, 8, kRowElems>;
}

template <class T, class WT, int V, int E> BackFn back_regs(bool x8)
{
    return x8 ? rmsnorm_backward_kernel<T, WT, V, E, true, 0>
              : rmsnorm_backward_kernel<T, WT, V, E, false, 0>;
}
template <int E> BackFn back_narrow(int dtype, int wdtype, int v, bool x8)
{
    if (dtype == DPO_F32)
        return back_regs<float, float, 1, E>(x8);
    if (wdtype == DPO_F32)
        return v == 2 ? back_regs<B16, float, 2, E>(x8) : back_regs<B16, float, 1, E>(x8);
    return v == 2 ? back_regs<B16, B16, 2, E>(x8) : back_regs<B16, B16, 1, E>(x8);
}
// ... with the ring, and its shared memory for CTAs of so many threads
template <class T, class WT, int V, bool X8, int TH> BackFn back_ring(int *smem)
{
    *smem = kDepth * RowSlot<T, V, kBackElems, X8, TH>::bytes;
    if constexpr (kDepth * RowSlot<T, V, kBackElems, X8, TH>::bytes <= kMaxSmem)
        return rmsnorm_backward_kernel<T, WT, V, kBackElems, X8, TH>;
    return nullptr;
}
template <class T, class WT, int V> BackFn back_ring(bool x8, int threads, int *smem)
{
    static_assert(kBackThreads == 64 * kBackMinWarps, "two sizes of CTAs");
    constexpr int TH = kBackThreads;   // or half of them
    if (threads == TH)
        return x8 ? back_ring<T, WT, V, true, TH>(smem) : back_ring<T, WT, V, false, TH>(smem);
    return x8 ? back_ring<T, WT, V, true, TH / 2>(smem) : back_ring<T, WT, V, false, TH / 2>(smem);
}
// The ring where the pieces are the widest ones and it fits: for bf16 always, for fp32 with
// CTAs of 256 threads.
BackFn back_of(int dtype, int wdtype, int v, int elems, bool x8, int threads, int *smem)
{
    *smem = 0;
    if (v <= 2)
        return elems == kBackElems ? back_narrow<kBackElems>(dtype, wdtype, v, x8)
                                   : back_narrow<kRowElems>(dtype, wdtype, v, x8);
    if (elems == kBackElems) {
        const BackFn fn = dtype == DPO_F32    ? back_ring<float, float, 4>(x8, threads, smem)
                          : wdtype == DPO_F32 ? back_ring<B16, float, 4>(x8, threads, smem)
                                              : back_ring<B16, B16, 8>(x8, threads, smem);
        if (fn != nullptr)
            return fn;
        *smem = 0;
        return back_regs<float, float, 4, kBackElems>(x8);
    }
    if (dtype == DPO_F32)
        return back_regs<float, float, 4, kRowElems>(x8);
    return wdtype == DPO_F32 ? back_regs<B16, float, 4, kRowElems>(x8)
                             : back_regs<B16, B16, 8, kRowElems>(x8);
}
// bf16: pieces of 16 bytes, or 8 beside fp32 weights; at most 48 bytes of inputs per
// 16-byte piece of dy, 16 elements a thread
static_assert(kDepth * (kBackElems / 8) * 48 * kBackThreads <= kMaxSmem, "the ring fits for bf16");

int check_norm(const char *what, int64_t rows, int64_t cols, int dtype, int wdtype,
               const void *weight)
{
    if (!known(dtype) || (wdtype != dtype && wdtype != DPO_F32))
        return call_fail(DPO_EDTYPE, "%s: dtype %d, weight dtype %d", what, dtype, wdtype);
    if (rows < 0 || rows >= kMaxRows || cols < 1 || cols > DPO_RMSNORM_MAX_COLS)
        return call_fail(DPO_EINVAL, "%s: %lld x %lld", what, (long long)rows, (long long)cols);
    return check_matrix(what, "weight", weight, cols, cols, elem_size(wdtype));
}

}  // namespace

int unpack8_beside(const dpo_packed8 &in, int64_t rows, int64_t cols, void *out, void *cuda_stream)
{
    return pack_or_unpack("dpo_ffn_backward", out, DPO_BF16, rows, cols, cols, &in, true, cuda_stream,
                          true);
}

}  // namespace dpo

using namespace dpo;

extern "C" int dpo_pack8(const void *x, dpo_dtype dtype, int64_t rows, int64_t cols, int64_t ld_x,
                         const dpo_packed8 *out, void *cuda_stream)
{
    return pack_or_unpack("dpo_pack8", x, dtype, rows, cols, ld_x, out, false, cuda_stream);
}

extern "C" int dpo_unpack8(const dpo_packed8 *in, int64_t rows, int64_t cols, void *out,
                           dpo_dtype dtype, int64_t ld_out, void *cuda_stream)
{
    return pack_or_unpack("dpo_unpack8", out, dtype, rows, cols, ld_out, in, true, cuda_stream);
}

extern "C" int dpo_rmsnorm(const dpo_rmsnorm_args *args, void *cuda_stream)
{
    const char *what = "dpo_rmsnorm";
    if (args == nullptr)
        return call_fail(DPO_EINVAL, "%s: no arguments", what);
    const dpo_rmsnorm_args &a = *args;
    int rc = check_norm(what, a.rows, a.cols, a.dtype, a.weight_dtype, a.weight);
    if (rc != DPO_OK)
        return rc;
    if (!(a.eps >= 0.0f) || !isfinite(a.eps))
        return call_fail(DPO_EINVAL, "%s: eps", what);
    if (a.rows == 0)
        return DPO_OK;
    const int64_t size = elem_size(a.dtype);
    const struct { const char *name; const void *p; int64_t ld; bool needed; } mats[] = {
        {"x", a.x, a.ld_x, true}, {"residual", a.residual, a.ld_residual, false},
        {"h", a.h, a.ld_h, false}, {"y", a.y, a.ld_y, false}};
    for (const auto &m : mats)
        if ((m.needed || m.p != nullptr) &&
            (rc = check_matrix(what, m.name, m.p, a.cols, m.ld, size)) != DPO_OK)
            return rc;
    if ((rc = check_matrix(what, "rstd", a.rstd, 1, 1, 4)) != DPO_OK)
        return rc;
    if (a.x8.codes != nullptr && (rc = check_packed(what, a.x8, a.cols)) != DPO_OK)
        return rc;
    const int64_t ng = groups_of(a.cols);
    const Extent in[] = {extent_of(a.x, a.rows, a.cols, a.ld_x, size),
                       extent_of(a.residual, a.rows, a.cols, a.ld_residual, size),
                       extent_of(a.weight, 1, a.cols, a.cols, elem_size(a.weight_dtype))};
    const Extent out[] = {extent_of(a.h, a.rows, a.cols, a.ld_h, size),
                        extent_of(a.y, a.rows, a.cols, a.ld_y, size),
                        extent_of(a.rstd, 1, a.rows, a.rows, 4),
                        extent_of(a.x8.codes, a.rows, a.cols, a.x8.ld_codes, 1),
                        extent_of(a.x8.codes ? a.x8.scales : nullptr, a.rows, ng, a.x8.ld_scales, 1)};
    for (int i = 0; i < 5; ++i) {
        for (const Extent &s : in)
            if (overlap(out[i], s))
                return call_fail(DPO_EINVAL, "%s: an output overlaps an input", what);
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j]))
                return call_fail(DPO_EINVAL, "%s: outputs overlap", what);
    }
    int v = a.dtype == DPO_BF16 ? 8 : 4;
    while (v > 1 &&
           !(a.cols % v == 0 && whole(a.x, a.ld_x, size, v) && whole(a.residual, a.ld_residual, size, v) &&
             whole(a.h, a.ld_h, size, v) && whole(a.y, a.ld_y, size, v) &&
             aligned_to(a.weight, a.weight_dtype == DPO_F32 ? (v == 2 ? 8 : 16) : 2 * v) &&
             whole(a.x8.codes, a.x8.ld_codes, 1, v)))
        v = v == 8 ? 2 : 1;
    const bool narrow = v <= 2 && a.cols <= (int64_t)kCta * kNarrowElems;
    const NormForwardArgs k = {a, row_warps(a.cols, narrow ? kNarrowElems : kRowElems)};
    const int cta = k.warps > kMinWarps ? k.warps : kMinWarps;
    const int64_t grid = (a.rows + cta / k.warps - 1) / (cta / k.warps);
    return launch(what, forward_of(a.dtype, a.weight_dtype, v, narrow ? kNarrowElems : kRowElems), grid,
                  cta * 32, 0, cuda_stream, k);
}

extern "C" int dpo_rmsnorm_workspace(int64_t rows, int64_t cols, int64_t *bytes)
{
    const char *what = "dpo_rmsnorm_workspace";
    if (bytes == nullptr || rows < 0 || rows >= kMaxRows || cols < 1 || cols > DPO_RMSNORM_MAX_COLS)
        return call_fail(DPO_EINVAL, "%s: %lld x %lld", what, (long long)rows, (long long)cols);
    const int sms = sm_count();
    if (sms == 0)
        return call_fail(DPO_ECUDA, "%s: no device", what);
    *bytes = back_shape(rows, cols, sms).grid * cols * 4;
    return DPO_OK;
}

extern "C" int dpo_rmsnorm_backward(const dpo_rmsnorm_backward_args *args, void *cuda_stream)
{
    const char *what = "dpo_rmsnorm_backward";
    if (args == nullptr)
        return call_fail(DPO_EINVAL, "%s: no arguments", what);
    const dpo_rmsnorm_backward_args &a = *args;
    int rc = check_norm(what, a.rows, a.cols, a.dtype, a.weight_dtype, a.weight);
    if (rc != DPO_OK)
        return rc;
    if (a.dweight != nullptr) {
        if (!known(a.dweight_dtype))
            return call_fail(DPO_EDTYPE, "%s: dweight dtype %d", what, a.dweight_dtype);
        if (!aligned_to(a.dweight, elem_size(a.dweight_dtype)))
            return call_fail(DPO_EALIGN, "%s: dweight", what);
    }
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (a.rows == 0) {
        if (a.dweight == nullptr || a.accumulate)
            return DPO_OK;
        const cudaError_t e =
            cudaMemsetAsync(a.dweight, 0, (size_t)(a.cols * elem_size(a.dweight_dtype)), stream);
        return e == cudaSuccess ? DPO_OK : call_fail(DPO_ECUDA, "%s: %s", what, cudaGetErrorString(e));
    }
    if (a.dx == nullptr && a.dweight == nullptr)
        return DPO_OK;
    const int64_t size = elem_size(a.dtype);
    const struct { const char *name; const void *p; int64_t ld; bool needed; } mats[] = {
        {"dy", a.dy, a.ld_dy, true}, {"h", a.h, a.ld_h, false},
        {"dh", a.dh, a.ld_dh, false}, {"dx", a.dx, a.ld_dx, false}};
    for (const auto &m : mats)
        if ((m.needed || m.p != nullptr) &&
            (rc = check_matrix(what, m.name, m.p, a.cols, m.ld, size)) != DPO_OK)
            return rc;
    if ((rc = check_matrix(what, "rstd", a.rstd, 1, 1, 4)) != DPO_OK)
        return rc;
    if (a.h == nullptr && (rc = check_packed(what, a.x8, a.cols)) != DPO_OK)
        return rc;
    const int sms = sm_count();
    if (sms == 0)
        return call_fail(DPO_ECUDA, "%s: no device", what);
    const BackShape shape = back_shape(a.rows, a.cols, sms);
    const int64_t grid = shape.grid;
    if (a.dweight != nullptr) {
        if (a.workspace == nullptr || a.workspace_bytes < grid * a.cols * 4)
            return call_fail(DPO_EINVAL, "%s: workspace of %lld bytes, %lld needed", what,
                             (long long)a.workspace_bytes, (long long)(grid * a.cols * 4));
        if (!aligned_to(a.workspace, 16))
            return call_fail(DPO_EALIGN, "%s: workspace", what);
    }
    const uint8_t *codes = a.h == nullptr ? a.x8.codes : nullptr;
    const Extent in[] = {extent_of(a.dy, a.rows, a.cols, a.ld_dy, size),
                       extent_of(a.h, a.rows, a.cols, a.ld_h, size),
                       extent_of(a.dh, a.rows, a.cols, a.ld_dh, size),
                       extent_of(a.rstd, 1, a.rows, a.rows, 4),
                       extent_of(a.weight, 1, a.cols, a.cols, elem_size(a.weight_dtype)),
                       extent_of(codes, a.rows, a.cols, a.x8.ld_codes, 1),
                       extent_of(codes ? a.x8.scales : nullptr, a.rows, groups_of(a.cols),
                               a.x8.ld_scales, 1)};
    const Extent out[] = {extent_of(a.dx, a.rows, a.cols, a.ld_dx, size),
                        extent_of(a.dweight, 1, a.cols, a.cols, elem_size(a.dweight_dtype)),
                        extent_of(a.dweight ? a.workspace : nullptr, 1, grid * a.cols, grid * a.cols, 4)};
    for (int i = 0; i < 3; ++i) {
        for (const Extent &s : in)
            if (overlap(out[i], s))
                return call_fail(DPO_EINVAL, "%s: an output overlaps an input", what);
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j]))
                return call_fail(DPO_EINVAL, "%s: outputs overlap", what);
    }
    int v = a.dtype == DPO_BF16 ? 8 : 4;
    while (v > 1 &&
           !(a.cols % v == 0 && whole(a.dy, a.ld_dy, size, v) && whole(a.h, a.ld_h, size, v) &&
             whole(a.dh, a.ld_dh, size, v) && whole(a.dx, a.ld_dx, size, v) &&
             aligned_to(a.weight, a.weight_dtype == DPO_F32 ? (v == 2 ? 8 : 16) : 2 * v) &&
             whole(codes, a.x8.ld_codes, 1, v)))
        v = v == 8 ? 2 : 1;
    const NormBackArgs k = {a, shape.warps, static_cast<float *>(a.workspace)};
    int smem = 0;
    const BackFn fn = back_of(a.dtype, a.weight_dtype, v, shape.elems, a.h == nullptr, shape.cta * 32, &smem);
    if (smem > 0) {
        const cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void *>(fn),
                                                   cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem);
        if (e != cudaSuccess)
            return call_fail(DPO_ECUDA, "%s: %s", what, cudaGetErrorString(e));
    }
    const int sums = shape.cta > shape.warps ? (int)a.cols * 4 : 0;   // of the CTA's rows
    smem = smem > sums ? smem : sums;
    rc = launch(what, fn, grid, shape.cta * 32, (size_t)smem, cuda_stream, k);
    if (rc != DPO_OK || a.dweight == nullptr)
        return rc;
    const int64_t sum_grid = (a.cols + kSumCols - 1) / kSumCols;
    if (a.dweight_dtype == DPO_F32)
        return launch(what, rmsnorm_dweight_kernel<float>, sum_grid, 32 * kSumWarps, 0, cuda_stream,
                      static_cast<const float *>(k.partials), (int)grid, (int)a.cols,
                      static_cast<float *>(a.dweight), a.accumulate);
    return launch(what, rmsnorm_dweight_kernel<__nv_bfloat16>, sum_grid, 32 * kSumWarps, 0,
                  cuda_stream, static_cast<const float *>(k.partials), (int)grid, (int)a.cols,
                  static_cast<__nv_bfloat16 *>(a.dweight), a.accumulate);
}
