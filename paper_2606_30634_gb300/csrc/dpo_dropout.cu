// dpo_dropout.cu -- residual + dropout(x) with a mask that is drawn and not stored
// (dpo_dropout in include/dpo_ends.h).
//
// The mask's bits are a function of the element's place, so the backward pass draws the same
// ones and nothing is kept. One draw of the generator is 128 bits, 16 for each of eight
// elements: with 32 bits an element the draw's instructions, some 40 multiplications and
// exclusive-ors, would be twice as many. HBM bounds it: two or three streams.
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
    int64_t draws, units;         // of a row, in all
    uint64_t seed;
    const uint64_t *seed_source;
    uint32_t site, cut;
    float scale;
};

// A thread takes one draw's eight elements, in accesses of V.
template <class T, int V>
__global__ void __launch_bounds__(kThreads) dropout_kernel(const DropArgs a)
{
    constexpr int N = kDraw / V;
    const int64_t unit = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    pdl_wait();
    if (unit >= a.units)
        return;
    const int64_t row = a.units >> 32 ? unit / a.draws : (uint32_t)unit / (uint32_t)a.draws;
    const int64_t g = unit - row * a.draws;
    const int64_t c0 = g * kDraw;
    uint64_t seed = a.seed;
    if (a.seed_source != nullptr)
        asm volatile("ld.global.b64 %0, [%1];" : "=l"(seed) : "l"(a.seed_source));
    const T *const x = static_cast<const T *>(a.x) + row * a.ld_x + c0;
    const T *const r = static_cast<const T *>(a.residual) + row * a.ld_residual + c0;
    T *const y = static_cast<T *>(a.y) + row * a.ld_y + c0;
    Vec<T, V> vx[N], vr[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        vx[n].zero();
        vr[n].zero();
        if (c0 + n * V < a.cols) {
            vx[n].load(x + n * V);
            if (a.residual != nullptr)
                vr[n].load(r + n * V);
        }
    }
    const uint4 w = philox(make_uint4((uint32_t)g, (uint32_t)row, (uint32_t)(row >> 32), a.site),
                           (uint32_t)seed, (uint32_t)(seed >> 32));
    const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int n = 0; n < N; ++n) {
        float o[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int e = n * V + j;
            const uint32_t bits = e & 1 ? word[e / 2] >> 16 : word[e / 2] & 0xFFFFu;
            const float kept = bits >= a.cut ? __fmul_rn(vx[n].get(j), a.scale) : 0.0f;
            o[j] = a.residual != nullptr ? vr[n].get(j) + kept : kept;
        }
        Vec<T, V> out;
        out.set(o);
        if (c0 + n * V < a.cols)
            out.store(y + n * V);
    }
}

template <class T> void (*dropout_fn(int v))(DropArgs)
{
    constexpr int W = sizeof(T) == 4 ? 4 : 8;
    return v > 2 ? dropout_kernel<T, W> : v == 2 ? dropout_kernel<T, 2> : dropout_kernel<T, 1>;
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
    k.draws = (a.cols + kDraw - 1) / kDraw;
    k.units = a.rows * k.draws;
    k.seed = a.seed;
    k.seed_source = a.seed_source;
    k.site = a.site;
    k.cut = (uint32_t)cut;
    k.scale = (float)(65536.0 / (65536.0 - cut));
    const int64_t grid = (k.units + kThreads - 1) / kThreads;
    if (grid >= kMaxCount)
        return call_fail(DPO_EINVAL, "%s: %lld x %lld is too large", what, (long long)a.rows, (long long)a.cols);
    return launch(what, a.dtype == DPO_F32 ? dropout_fn<float>(w.v) : dropout_fn<__nv_bfloat16>(w.v), grid,
                  kThreads, 0, cuda_stream, k);
}
