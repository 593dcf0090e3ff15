// dpo_dropout.cu -- residual + dropout(x) with a mask that is drawn and not stored
// (dpo_dropout in include/dpo.h).
//
// The mask's bits are a function of the element's place, so the backward pass draws the same
// ones and nothing is kept. One draw of the generator is 128 bits, 16 for each of eight
// elements: with 32 bits an element the draw's instructions, some 40 multiplications and
// exclusive-ors, would be twice as many. HBM bounds it, two or three streams: 8192 x 4096 bf16 with
// a residual 30 us, 6.7 TB/s, 0.99 of the measured copy; 8192 x 4095 38.
#include "dpo_ends.cuh"
#include "dpo_vec.cuh"

#include <math.h>

namespace dpo {
namespace {

// Philox4x32-10: ten rounds on a 128-bit counter under a 64-bit key (Salmon, Moraes, Dror and
// Shaw, "Parallel Random Numbers: As Easy as 1, 2, 3", SC'11).
__device__ __forceinline__ uint4 philox(uint4 c, uint32_t k0, uint32_t k1)
{
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p = (uint64_t)0xD2511F53u * c.x, q = (uint64_t)0xCD9E8D57u * c.z;
        c = make_uint4((uint32_t)(q >> 32) ^ c.y ^ k0, (uint32_t)q, (uint32_t)(p >> 32) ^ c.w ^ k1,
                       (uint32_t)p);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return c;
}

constexpr int kDraw = 8;          // elements of a draw
constexpr int kThreads = 256;

struct DropArgs {
    const void *x, *residual;
    void *y;
    int64_t rows, cols, ld_x, ld_residual, ld_y;
    Units units;                  // draws, or spans of a warp
    uint64_t seed;
    const uint64_t *seed_source;
    uint32_t site, cut;
    float scale;
};

__device__ __forceinline__ uint64_t seed_of(const DropArgs &a)
{
    uint64_t seed = a.seed;
    if (a.seed_source != nullptr)
        asm volatile("ld.global.b64 %0, [%1];" : "=l"(seed) : "l"(a.seed_source));
    // known to be the same in all lanes: the rounds' keys then take no instructions of theirs
    return (uint64_t)(uint32_t)__shfl_sync(0xFFFFFFFFu, (int)(seed >> 32), 0) << 32 |
           (uint32_t)__shfl_sync(0xFFFFFFFFu, (int)seed, 0);
}

// A thread takes one draw's eight elements, in one access. (30 instructions an element, with a
// division, products and sums apart and keys of its own for every thread, were what bounded
// 8192 x 4096 bf16 with a residual: 35.8 us.)
template <class T, bool RES>
__global__ void __launch_bounds__(kThreads) dropout_kernel(const DropArgs a)
{
    constexpr int V = 16 / (int)sizeof(T), N = kDraw / V;
    const int64_t unit = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    pdl_wait();
    int64_t row, g;
    a.units.at(min(unit, a.units.all - 1), row, g);
    const int64_t c0 = g * kDraw;
    const uint64_t seed = seed_of(a);
    if (unit >= a.units.all)
        return;
    const T *const x = static_cast<const T *>(a.x) + row * a.ld_x + c0;
    const T *const r = static_cast<const T *>(a.residual) + row * a.ld_residual + c0;
    T *const y = static_cast<T *>(a.y) + row * a.ld_y + c0;
    Vec<T, V> vx[N], vr[N];
#pragma unroll
    for (int n = 0; n < N; ++n)
        if (n == 0 || c0 + n * V < a.cols) {   // rows are whole accesses
            vx[n].load(x + n * V);
            if (RES)
                vr[n].load(r + n * V);
        }
    const uint4 w = philox(make_uint4((uint32_t)g, (uint32_t)row, (uint32_t)(row >> 32), a.site),
                           (uint32_t)seed, (uint32_t)(seed >> 32));
    const uint32_t word[4] = {w.x, w.y, w.z, w.w}, high = a.cut << 16;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        if (n > 0 && c0 + n * V >= a.cols)
            break;
        float o[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int e = n * V + j;
            const bool kept = e & 1 ? word[e / 2] >= high : (word[e / 2] & 0xFFFFu) >= a.cut;
            o[j] = RES ? vr[n].get(j) : 0.0f;
            if (kept)
                o[j] = RES ? fmaf(vx[n].get(j), a.scale, o[j]) : vx[n].get(j) * a.scale;
        }
        Vec<T, V> out;
        out.set(o);
        out.store(y + n * V);
    }
}

// Rows of other sizes, pitches or addresses: a warp takes 32 draws' elements in a row, 32 V at a
// time, one access of V a lane; the draws' bits pass through shared memory. (By threads with a
// draw each, whose accesses then lie 8 elements apart: 8192 x 4095 bf16 81 us.)
template <class T, bool RES, int V>
__global__ void __launch_bounds__(kThreads) dropout_odd_kernel(const DropArgs a)
{
    constexpr int N = kDraw / V;
    __shared__ uint4 bits_[kThreads];
    const int lane = threadIdx.x & 31;
    const int64_t unit = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    pdl_wait();
    if (unit >= a.units.all)
        return;
    int64_t row, g;
    a.units.at(unit, row, g);
    const uint64_t seed = seed_of(a);
    const int64_t c0 = g * 32 * kDraw + lane * V;
    const T *const x = static_cast<const T *>(a.x) + row * a.ld_x + c0;
    const T *const r = static_cast<const T *>(a.residual) + row * a.ld_residual + c0;
    T *const y = static_cast<T *>(a.y) + row * a.ld_y + c0;
    const int left = (int)min(a.cols - c0, (int64_t)32 * kDraw);   // of this lane's accesses
    Vec<T, V> vx[N], vr[N];
#pragma unroll
    for (int n = 0; n < N; ++n)
        if (n * 32 * V < left) {
            vx[n].load(x + n * 32 * V);
            if (RES)
                vr[n].load(r + n * 32 * V);
        }
    uint4 *const bits = bits_ + (threadIdx.x & ~31);
    bits[lane] = philox(make_uint4((uint32_t)(g * 32 + lane), (uint32_t)row, (uint32_t)(row >> 32), a.site),
                        (uint32_t)seed, (uint32_t)(seed >> 32));
    __syncwarp();
    const uint16_t *const half = reinterpret_cast<const uint16_t *>(bits) + lane * V;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        if (n * 32 * V >= left)
            break;
        float o[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            o[j] = RES ? vr[n].get(j) : 0.0f;
            if (half[n * 32 * V + j] >= a.cut)
                o[j] = RES ? fmaf(vx[n].get(j), a.scale, o[j]) : vx[n].get(j) * a.scale;
        }
        Vec<T, V> out;
        out.set(o);
        out.store(y + n * 32 * V);
    }
}

template <class T, bool RES> void (*dropout_fn(int v))(DropArgs)
{
    return v > 2 ? dropout_kernel<T, RES> : v == 2 ? dropout_odd_kernel<T, RES, 2> : dropout_odd_kernel<T, RES, 1>;
}
template <class T> void (*dropout_fn(bool residual, int v))(DropArgs)
{
    return residual ? dropout_fn<T, true>(v) : dropout_fn<T, false>(v);
}

}  // namespace
}  // namespace dpo

using namespace dpo;

extern "C" int dpo_dropout(const dpo_dropout_args *args, void *cuda_stream)
{
    const char *what = "dpo_dropout";
    if (args == nullptr)
        return call_fail(DPO_EINVAL, "%s: no arguments", what);
    const dpo_dropout_args &a = *args;
    if (!known(a.dtype))
        return call_fail(DPO_EDTYPE, "%s: dtype %d", what, a.dtype);
    if (a.rows < 0 || a.cols < 0 || a.rows >= kMaxCount || a.cols >= kMaxCount)
        return call_fail(DPO_EINVAL, "%s: %lld x %lld", what, (long long)a.rows, (long long)a.cols);
    const double cut = a.p >= 0.0 ? floor(65536.0 * a.p + 0.5) : -1.0;
    if (!(a.p >= 0.0) || !(cut < 65536.0))
        return call_fail(DPO_EINVAL, "%s: p = %g (0 <= p < 1 - 2^-17)", what, a.p);
    if (a.rows == 0 || a.cols == 0)
        return DPO_OK;
    const int64_t size = elem_size(a.dtype);
    Buffers b(what);
    // y in the place of x or of the residual is fine: a thread reads what it then writes
    const bool in_x = a.y == a.x && a.ld_y == a.ld_x;
    const bool in_r = a.y == a.residual && a.ld_y == a.ld_residual;
    b.add("x", a.x, a.rows, a.cols, a.ld_x, size, size, in_x);
    if (a.residual != nullptr)
        b.add("residual", a.residual, a.rows, a.cols, a.ld_residual, size, size, in_r && !in_x);
    if (!in_x && !in_r)
        b.add("y", a.y, a.rows, a.cols, a.ld_y, size, size, true);
    if (a.seed_source != nullptr)
        b.add("seed_source", a.seed_source, 1, 1, 1, 8, 8, false);
    int rc = b.done();
    if (rc != DPO_OK)
        return rc;
    Width w(a.dtype == DPO_F32 ? 4 : 8);
    w.fit(a.x, a.cols, a.ld_x, size);
    w.fit(a.residual, a.cols, a.ld_residual, size);
    w.fit(a.y, a.cols, a.ld_y, size);
    DropArgs k{};
    k.x = a.x;
    k.residual = a.residual;
    k.y = a.y;
    k.rows = a.rows;
    k.cols = a.cols;
    k.ld_x = a.ld_x;
    k.ld_residual = a.ld_residual;
    k.ld_y = a.ld_y;
    // an access's elements are a draw's, or a warp's span is 32 draws'
    const int64_t span = w.v > 2 ? kDraw : 32 * kDraw, of_cta = w.v > 2 ? kThreads : kThreads / 32;
    k.units = units_of(a.rows, (a.cols + span - 1) / span);
    k.seed = a.seed;
    k.seed_source = a.seed_source;
    k.site = a.site;
    k.cut = (uint32_t)cut;
    k.scale = (float)(65536.0 / (65536.0 - cut));
    const int64_t grid = (k.units.all + of_cta - 1) / of_cta;
    if (grid >= kMaxCount)
        return call_fail(DPO_EINVAL, "%s: %lld x %lld is too large", what, (long long)a.rows, (long long)a.cols);
    const bool res = a.residual != nullptr;
    return launch(what, a.dtype == DPO_F32 ? dropout_fn<float>(res, w.v) : dropout_fn<__nv_bfloat16>(res, w.v),
                  grid, kThreads, 0, cuda_stream, k);
}
