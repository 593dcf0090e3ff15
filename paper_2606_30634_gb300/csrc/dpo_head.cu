// dpo_head.cu -- the head: log probabilities from the stream and the head's weights, and the
// gradients of both (dpo_head, dpo_head_backward in include/dpo.h).
//
// Forward, two launches: the product x w^T, whose epilogue reduces 128 columns of a row to
// (maximum m, sum of e^(z - m), entropy sum), so that no logits are written; and the join of a
// row's parts. For `top` the logits are written and read once more (dpo_logprobs.cu).
// Kept for the backward: e^(z - m) in fp16, and m. Forming the logits again would cost a third
// of the backward's two products; reading this costs 2 bytes a logit, and holding it as many.
// Backward, two launches: G from what was kept; dx = G w and dw = G^T x, one list of tiles. Where few
// tokens leave dx a few tiles of the whole vocabulary's K, these are shared out among more tiles of
// the list, and a third launch adds the shares up (1001 x 768 x 50257: 205 -> 147 us, the products 82
// at the burst rate).
// 8192 x 4096 x 32000, both: 3.6 to 4.1 ms by box and power, 0.9 to 1.0 of the sustained rate; its
// products 1.07 and 2.24, G 0.17 (6.1 TB/s), the join 0.01.
#include "dpo_logprobs.cuh"
#include "dpo_products.h"

#include <cuda_fp16.h>

namespace dpo {
namespace {

// ---------------------------------------------------------------- join ----
// A CTA joins kJoinRows rows, a lane one part of one of them, several at a time; then a warp has a
// row, with its warps' sums in the lanes.
constexpr int kJoinMaxWarps = 32, kJoinRows = 8, kJoinLanes = 32 / kJoinRows, kJoinAhead = 4;

struct JoinArgs {
    const float *maxima, *target;
    const float2 *sums;
    Ids ids;
    float *logp, *entropy, *stats;
    int64_t rows, vocab;
    int parts;
};

__global__ void __launch_bounds__(32 * kJoinMaxWarps) head_join_kernel(const JoinArgs a)
{
    __shared__ Part part_[kJoinMaxWarps][kJoinRows + 1];
    const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t row0 = (int64_t)blockIdx.x * kJoinRows, r = min(row0 + lane % kJoinRows, a.rows - 1);
    const int step = warps * kJoinLanes;
    pdl_wait();
    Part part;
    for (int i = warp * kJoinLanes + lane / kJoinRows; i < a.parts; i += step * kJoinAhead) {
        Part p[kJoinAhead];
        float top = part.m;
#pragma unroll
        for (int u = 0; u < kJoinAhead; ++u)
            if (i + u * step < a.parts) {
                const int64_t at = (int64_t)(i + u * step) * a.rows + r;
                const float2 sw = a.sums[at];
                p[u].m = a.maxima[at];
                p[u].s = sw.x;
                p[u].w = sw.y;
            }
#pragma unroll
        for (int u = 0; u < kJoinAhead; ++u)
            top = fmaxf(top, p[u].m);
        part.raise(top);
#pragma unroll
        for (int u = 0; u < kJoinAhead; ++u) {
            p[u].raise(top);
            part.s += p[u].s;
            part.w += p[u].w;
        }
    }
    part.warp_join<kJoinRows>();
    if (lane < kJoinRows)
        part_[warp][lane] = part;
    __syncthreads();
    for (int i = warp; i < kJoinRows; i += warps) {
        const int64_t row = row0 + i;
        if (row >= a.rows)
            break;
        Part p;
        if (lane < warps)
            p = part_[lane][i];
        p.warp_join();
        if (lane != 0)
            continue;
        const float logs = p.log_sum();
        a.stats[2 * row] = p.m;
        a.stats[2 * row + 1] = logs;
        a.entropy[row] = p.entropy();
        if (a.logp != nullptr)
            a.logp[row] = a.ids.at(row, a.vocab) < 0 ? 0.0f : a.target[row] - p.m - logs;
    }
}

// ------------------------------------------------------------- dlogits ----
// G in bf16 from the kept values x = 2^15 e^(z - m_part): with q = m_part - m - log S,
//   g = -scale p (a + b (log p + h)),   p = x 2^-15 e^q,   log2 p = log2 x + q log2(e) - 15,
// so g = x (k0 + k1 log2 x) with two factors of 128 columns of a row. The id's own element is
// a (1 - p) from the log probability itself: a kept p near 1 would leave little of it.
// bf16 because one MMA takes both operands in one type and w and x have that: dx and dw are 0.0023 off in
// the norm for it, where their own rounding to bf16 is 0.0017 and fp32's nothing; G as two terms would
// double both products' MMAs. What the tensor cores truncate with the vocabulary or the tokens as K in one
// chain is less: dx and dw shrink by 1e-5 to 1.3e-4, for 1003 to 128256 of K, so these chains are not
// cut as the forward's is.
// rows of a CTA; accesses of 8 columns a lane (by 4, 8 and 16 rows a backward of 1001 x 768 x 50257 is
// 147, 151 and 154 us)
constexpr int kGradWarps = 4, kGradPieces = 4;
constexpr int kGradCols = 32 * 8;        // of one access of a warp, whole parts
static_assert(kGradCols % kHeadStatCols == 0, "parts of an access");
constexpr float kUnitLog2 = 15.0f;       // of kHeadUnit
static_assert(kHeadUnit == 32768.0f, "its logarithm");

struct GradArgs {
    const __half *kept;
    const float *maxima;
    Ids ids;
    const float *logp, *entropy, *stats, *dlogp, *dentropy;
    __nv_bfloat16 *g;
    int64_t rows, vocab, ld, kept_rows;
    int spans, batches;          // of a row; of kGradPieces accesses in a span
    float scale;
};

// log2 by the hardware's approximation (2^-22); of 0 a number too, so that 0 times it is 0.
__device__ __forceinline__ float log2_fast(float x)
{
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return fmaxf(y, -100.0f);
}

__global__ void __launch_bounds__(32 * kGradWarps) head_gradient_kernel(const GradArgs a)
{
    const int lane = threadIdx.x & 31;
    const uint32_t group = blockIdx.x / (uint32_t)a.spans, span = blockIdx.x - group * (uint32_t)a.spans;
    const int64_t row = (int64_t)group * kGradWarps + (threadIdx.x >> 5);
    pdl_wait();
    if (row >= a.rows)
        return;
    const int id = a.ids.at(row, a.vocab);
    const float ga = id >= 0 ? ld1(a.dlogp + row) : 0.0f;
    const float gb = a.dentropy != nullptr ? ld1(a.dentropy + row) : 0.0f;
    const float m = ld1(a.stats + 2 * row), logs = ld1(a.stats + 2 * row + 1);
    const float h = gb != 0.0f ? ld1(a.entropy + row) : 0.0f;
    const bool none = ga == 0.0f && gb == 0.0f;
    const float k0 = -a.scale * fmaf(gb, h, ga), k1 = -a.scale * gb * 0.6931471805599453f;
    __nv_bfloat16 *const g = a.g + row * a.ld;
    const int vocab = (int)a.vocab;
    int c0 = (int)span * a.batches * kGradPieces * kGradCols + lane * 8;
    // this lane's columns in their part, and how far the next ones' are
    const __half *e = a.kept + ((int64_t)(c0 / kHeadStatCols) * a.kept_rows + row) * kHeadStatCols + c0 % kHeadStatCols;
    const float *largest = a.maxima + (int64_t)(c0 / kHeadStatCols) * a.rows + row;
    const int64_t next_e = kGradCols * a.kept_rows, next_largest = kGradCols / kHeadStatCols * a.rows;
    for (int n = 0; n < a.batches && c0 < vocab; ++n, c0 += kGradPieces * kGradCols) {
        uint4 q[kGradPieces];
        float top[kGradPieces];
#pragma unroll
        for (int u = 0; u < kGradPieces; ++u) {
            const int c = c0 + u * kGradCols;
            q[u] = make_uint4(0u, 0u, 0u, 0u);
            top[u] = 0.0f;
            if (c < vocab && !none) {
                asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];"
                             : "=r"(q[u].x), "=r"(q[u].y), "=r"(q[u].z), "=r"(q[u].w)
                             : "l"(e));
                top[u] = ld1(largest);
            }
            e += next_e;
            largest += next_largest;
        }
#pragma unroll
        for (int u = 0; u < kGradPieces; ++u) {
            const int c = c0 + u * kGradCols;
            if (c >= vocab)
                break;
            const float t = (top[u] - m - logs) * kLog2e, part = exp2_fast(t) * (1.0f / kHeadUnit);
            const float f0 = part * fmaf(k1, fmaxf(t, -1000.0f) - kUnitLog2, k0), f1 = part * k1;
            const Two f00 = two(f0, f0), f11 = two(f1, f1);
            const uint32_t w[4] = {q[u].x, q[u].y, q[u].z, q[u].w};
            uint32_t o[4];
            if (none) {
                o[0] = o[1] = o[2] = o[3] = 0u;
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 v = __half22float2(*reinterpret_cast<const __half2 *>(w + j));
                    Two f = f00;
                    if (gb != 0.0f)
                        f = fma_two(f11, two(log2_fast(v.x), log2_fast(v.y)), f00);
                    const float2 y = of_two(mul_two(two(v.x, v.y), f));
                    o[j] = pack_bf16x2(y.x, y.y);
                }
                const int at = id - c;
                if (at >= 0 && at < 8) {
                    const float lp = ld1(a.logp + row), p = expf(lp);
                    float y = -ga * expm1f(lp);
                    if (gb != 0.0f && p != 0.0f)
                        y = fmaf(-gb * p, lp + h, y);
                    const uint32_t own = pack_bf16x2(y * a.scale, y * a.scale);
                    const uint32_t mask = at & 1 ? 0xFFFF0000u : 0x0000FFFFu;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        o[j] = at / 2 == j ? (o[j] & ~mask) | (own & mask) : o[j];
                }
            }
            // columns past the vocabulary, up to the pitch, are not read by the products
            *reinterpret_cast<uint4 *>(g + c) = make_uint4(o[0], o[1], o[2], o[3]);
        }
    }
}

// ---------------------------------------------------------------- host ----

int64_t align_up(int64_t v) { return (v + 255) / 256 * 256; }
int64_t pitch_of(int64_t vocab) { return (vocab + 7) / 8 * 8; }

int check_head(const char *what, int64_t tokens, int64_t dim, int64_t vocab, float scale)
{
    constexpr int64_t kMaxSide = (int64_t)1 << 26;
    if (tokens < 0 || tokens > kMaxSide || dim < 8 || dim % 8 != 0 || dim > kMaxSide || vocab < 1 ||
        vocab > kMaxSide)
        return call_fail(DPO_EINVAL, "%s: tokens %lld, dim %lld (a multiple of 8), vocab %lld", what,
                         (long long)tokens, (long long)dim, (long long)vocab);
    if ((tokens + 127) / 128 * ((vocab + 127) / 128) >= ((int64_t)1 << 28) ||
        (dim + 127) / 128 * ((vocab + 127) / 128) >= ((int64_t)1 << 28))
        return call_fail(DPO_EINVAL, "%s: %lld x %lld x %lld is too large", what, (long long)tokens,
                         (long long)dim, (long long)vocab);
    if (!good_scale(scale))
        return call_fail(DPO_EINVAL, "%s: scale %g (1e-20 to 1e6)", what, (double)scale);
    return DPO_OK;
}

// What is kept, and the workspaces: where each part begins.
struct Sizes {
    int64_t ld, parts, kept_rows;
    int64_t kept, maxima;              // kept: the values, their maxima
    int64_t target, sums, own, logits; // forward: without kept its maxima, for `top` logits
    int64_t shares;                    // backward: G, the shares of dx
    int64_t forward, backward;
};
Sizes sizes_of(int64_t tokens, int64_t dim, int64_t vocab, bool keep, int top)
{
    Sizes s;
    s.ld = pitch_of(vocab);
    s.parts = (vocab + kHeadStatCols - 1) / kHeadStatCols;
    s.kept_rows = (tokens + 31) / 32 * 32;
    s.maxima = align_up(s.parts * s.kept_rows * kHeadStatCols * 2);
    s.kept = s.maxima + align_up(s.parts * tokens * 4);
    s.target = 0;
    s.sums = align_up(tokens * 4);
    s.own = s.sums + align_up(s.parts * tokens * 8);
    s.logits = s.own + (keep ? 0 : align_up(s.parts * tokens * 4));
    if (top > 0 && !keep)
        s.logits = 0;
    s.forward = s.logits + (top > 0 ? align_up(tokens * s.ld * 4) : 0);
    s.shares = align_up(tokens * s.ld * 2);
    s.backward = s.shares + align_up(product_share_bytes(tokens, dim, vocab));
    return s;
}

int check_workspace(const char *what, Buffers &b, const void *p, int64_t bytes, int64_t need)
{
    if (need == 0)
        return DPO_OK;
    if (p != nullptr && bytes < need)
        return call_fail(DPO_EINVAL, "%s: workspace of %lld bytes, %lld needed", what, (long long)bytes,
                         (long long)need);
    b.add("workspace", p, 1, need, need, 1, 256, true);
    return DPO_OK;
}

int check_token_ids(const char *what, const dpo_ids &ids, int64_t tokens, Ids *out)
{
    int64_t n = 0;
    const int rc = check_ids(what, ids, out, &n);
    if (rc == DPO_OK && n != tokens)
        return call_fail(DPO_EINVAL, "%s: %lld ids for %lld tokens", what, (long long)n, (long long)tokens);
    return rc;
}

}  // namespace
}  // namespace dpo

using namespace dpo;

extern "C" int dpo_head_workspace(int64_t tokens, int64_t dim, int64_t vocab, int keep, int top,
                                  int64_t *forward_bytes, int64_t *kept_bytes, int64_t *backward_bytes)
{
    const char *what = "dpo_head_workspace";
    const int rc = check_head(what, tokens, dim, vocab, 1.0f);
    if (rc != DPO_OK)
        return rc;
    if (top < 0 || top > DPO_MAX_TOP || top > vocab)
        return call_fail(DPO_EINVAL, "%s: top %d of %lld", what, top, (long long)vocab);
    const Sizes s = sizes_of(tokens, dim, vocab, keep != 0, top);
    if (forward_bytes != nullptr)
        *forward_bytes = s.forward;
    if (kept_bytes != nullptr)
        *kept_bytes = s.kept;
    if (backward_bytes != nullptr)
        *backward_bytes = s.backward;
    return DPO_OK;
}

extern "C" int dpo_head(const dpo_head_args *args, void *cuda_stream)
{
    const char *what = "dpo_head";
    if (args == nullptr)
        return call_fail(DPO_EINVAL, "%s: no arguments", what);
    const dpo_head_args &a = *args;
    int rc = check_head(what, a.tokens, a.dim, a.vocab, a.scale);
    if (rc != DPO_OK)
        return rc;
    if (a.top < 0 || a.top > DPO_MAX_TOP || a.top > a.vocab)
        return call_fail(DPO_EINVAL, "%s: top %d of %lld", what, a.top, (long long)a.vocab);
    Ids ids{};
    if (a.ids.p != nullptr && (rc = check_token_ids(what, a.ids, a.tokens, &ids)) != DPO_OK)
        return rc;
    if (a.tokens == 0)
        return DPO_OK;
    const int64_t T = a.tokens;
    const Sizes s = sizes_of(T, a.dim, a.vocab, a.kept != nullptr, a.top);
    Buffers b(what);
    b.add("x", a.x, T, a.dim, a.ld_x, 2, 16, false);
    b.add("w", a.w, a.vocab, a.dim, a.dim, 2, 16, false);
    if (a.ids.p != nullptr) {
        add_ids(b, a.ids);
        b.add("logp", a.logp, 1, T, T, 4, 4, true);
    }
    b.add("entropy", a.entropy, 1, T, T, 4, 4, true);
    b.add("stats", a.stats, 1, 2 * T, 2 * T, 4, 4, true);
    if (a.top > 0) {
        b.add("top_logp", a.top_logp, 1, T * a.top, T * a.top, 4, 4, true);
        b.add("top_ids", a.top_ids, 1, T * a.top, T * a.top, 8, 8, true);
    }
    if (a.kept != nullptr)
        b.add("kept", a.kept, 1, s.kept, s.kept, 1, 256, true);
    if ((rc = check_workspace(what, b, a.workspace, a.workspace_bytes, s.forward)) != DPO_OK ||
        (rc = b.done()) != DPO_OK)
        return rc;
    uint8_t *const ws = static_cast<uint8_t *>(a.workspace), *const kept = static_cast<uint8_t *>(a.kept);
    HeadProduct p{};
    p.x = a.x;
    p.w = a.w;
    p.tokens = T;
    p.dim = a.dim;
    p.vocab = a.vocab;
    p.ld_x = a.ld_x;
    p.ids = ids;
    p.scale = a.scale;
    p.ld = s.ld;
    p.kept_rows = s.kept_rows;
    if (a.top == 0 || kept != nullptr) {
        p.target = reinterpret_cast<float *>(ws + s.target);
        p.sums = reinterpret_cast<float2 *>(ws + s.sums);
        p.maxima = reinterpret_cast<float *>(kept != nullptr ? kept + s.maxima : ws + s.own);
        p.kept = kept;
    }
    if (a.top > 0)
        p.logits = ws + s.logits;
    if ((rc = head_product(what, p, cuda_stream)) != DPO_OK)
        return rc;
    if (a.top == 0) {
        JoinArgs j{p.maxima, p.target, p.sums, ids, a.ids.p != nullptr ? a.logp : nullptr, a.entropy, a.stats,
                   T, a.vocab, (int)s.parts};
        int warps = 4;
        while (warps < kJoinMaxWarps && warps * kJoinLanes * kJoinAhead < s.parts)
            warps *= 2;
        return launch(what, head_join_kernel, (T + kJoinRows - 1) / kJoinRows, 32 * warps, 0, cuda_stream, j);
    }
    dpo_logprobs_args l{};
    l.logits = p.logits;
    l.ids = a.ids;
    l.logp = a.logp;
    l.entropy = a.entropy;
    l.stats = a.stats;
    l.top_logp = a.top_logp;
    l.top_ids = a.top_ids;
    l.rows = T;
    l.vocab = a.vocab;
    l.ld_logits = s.ld;
    l.scale = a.scale;
    l.dtype = DPO_F32;
    l.top = a.top;
    return dpo_logprobs(&l, cuda_stream);
}

extern "C" int dpo_head_backward(const dpo_head_backward_args *args, void *cuda_stream)
{
    const char *what = "dpo_head_backward";
    if (args == nullptr)
        return call_fail(DPO_EINVAL, "%s: no arguments", what);
    const dpo_head_backward_args &a = *args;
    int rc = check_head(what, a.tokens, a.dim, a.vocab, a.scale);
    if (rc != DPO_OK)
        return rc;
    if (!known(a.grad_dtype))
        return call_fail(DPO_EDTYPE, "%s: grad dtype %d", what, a.grad_dtype);
    Ids ids{};
    if ((rc = check_token_ids(what, a.ids, a.tokens, &ids)) != DPO_OK)
        return rc;
    const int64_t T = a.tokens, D = a.dim, V = a.vocab, gsize = elem_size(a.grad_dtype);
    Buffers b(what);
    b.add("dw", a.dw, V, D, D, gsize, 16, true);
    if (T == 0) {
        if ((rc = b.done()) != DPO_OK || a.accumulate)
            return rc;
        const cudaError_t e =
            cudaMemsetAsync(a.dw, 0, (size_t)(V * D * gsize), static_cast<cudaStream_t>(cuda_stream));
        return e == cudaSuccess ? DPO_OK : call_fail(DPO_ECUDA, "%s: %s", what, cudaGetErrorString(e));
    }
    const Sizes s = sizes_of(T, D, V, true, 0);
    b.add("x", a.x, T, D, a.ld_x, 2, 16, false);
    b.add("w", a.w, V, D, D, 2, 16, false);
    add_ids(b, a.ids);
    b.add("kept", a.kept, 1, s.kept, s.kept, 1, 256, false);
    b.add("logp", a.logp, 1, T, T, 4, 4, false);
    b.add("entropy", a.entropy, 1, T, T, 4, 4, false);
    b.add("stats", a.stats, 1, 2 * T, 2 * T, 4, 4, false);
    b.add("dlogp", a.dlogp, 1, T, T, 4, 4, false);
    if (a.dentropy != nullptr)
        b.add("dentropy", a.dentropy, 1, T, T, 4, 4, false);
    if (a.dx != nullptr)
        b.add("dx", a.dx, T, D, a.ld_dx, 2, 16, true);
    if ((rc = check_workspace(what, b, a.workspace, a.workspace_bytes, s.backward)) != DPO_OK ||
        (rc = b.done()) != DPO_OK)
        return rc;
    const uint8_t *const kept = static_cast<const uint8_t *>(a.kept);
    void *const G = a.workspace;
    GradArgs g{};
    g.kept = reinterpret_cast<const __half *>(kept);
    g.maxima = reinterpret_cast<const float *>(kept + s.maxima);
    g.ids = ids;
    g.logp = a.logp;
    g.entropy = a.entropy;
    g.stats = a.stats;
    g.dlogp = a.dlogp;
    g.dentropy = a.dentropy;
    g.g = static_cast<__nv_bfloat16 *>(G);
    g.rows = T;
    g.vocab = V;
    g.ld = s.ld;
    g.kept_rows = s.kept_rows;
    g.scale = a.scale;
    // up to four batches a span, where that leaves CTAs enough for all SMs
    const int64_t groups = (T + kGradWarps - 1) / kGradWarps, batches = (V + kGradPieces * kGradCols - 1) / (kGradPieces * kGradCols);
    g.batches = groups * batches >= 4 * 2048 ? 4 : 1;
    g.spans = (int)((batches + g.batches - 1) / g.batches);
    const int64_t grid = groups * g.spans;
    if (grid >= kMaxCount)
        return call_fail(DPO_EINVAL, "%s: %lld x %lld is too large", what, (long long)T, (long long)V);
    if ((rc = launch(what, head_gradient_kernel, grid, 32 * kGradWarps, 0, cuda_stream, g)) != DPO_OK)
        return rc;
    StoreProduct p[2];
    int n = 0;
    if (a.dx != nullptr)
        p[n++] = {G, a.w, a.dx, T, D, V, s.ld, D, a.ld_dx, 0, 1, 0, 0,
                  s.backward > s.shares ? static_cast<uint8_t *>(G) + s.shares : nullptr};
    p[n++] = {G, a.x, a.dw, V, D, T, s.ld, a.ld_x, D, 1, 1, a.grad_dtype == DPO_F32, a.accumulate != 0, nullptr};
    return store_products(what, p, n, cuda_stream);
}
