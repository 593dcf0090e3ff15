// dpo_logprobs.cu -- log probabilities of given tokens, entropy and most likely ids from logits,
// and their gradient (dpo_logprobs, dpo_logprobs_backward in include/dpo_ends.h).
//
// Forward: every logit is read once; a thread keeps the running maximum m, sum S and entropy
// sum W of its own, and the threads' are joined. Backward: every logit once more, dlogits
// written. Both are bound by HBM; few rows by latency, where a cluster shares a row.
#include "dpo_logprobs.cuh"

namespace dpo {
namespace {

constexpr int kMaxThreads = 512, kMaxWarps = kMaxThreads / 32, kMaxCtas = 8;

struct LogArgs {
    const void *logits;
    Ids ids;
    float *logp, *entropy, *stats, *top_logp;
    int64_t *top_ids;
    int64_t rows, vocab, ld;
    float scale;
    int top;
};

// Elements before the first 16-byte boundary, at most n.
template <class T> __device__ __forceinline__ int64_t to_boundary(const T *p, int64_t n)
{
    const int64_t k = (int64_t)((16u - (uint32_t)(reinterpret_cast<uintptr_t>(p) & 15u)) & 15u) / (int)sizeof(T);
    return k < n ? k : n;
}

// A cluster's CTAs share a row, in equal spans; accesses of 16 bytes from the span's first
// boundary on, so rows of odd pitches cost two short ends.
template <class T, bool TOP>
__global__ void __launch_bounds__(kMaxThreads) logprobs_kernel(const LogArgs a)
{
    constexpr int V = 16 / (int)sizeof(T), U = 4;
    __shared__ Part parts[kMaxWarps];
    __shared__ float tops_v[TOP ? kMaxWarps * 32 : 1];
    __shared__ int tops_id[TOP ? kMaxWarps * 32 : 1];
    const int nt = blockDim.x, warps = nt >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cta_of_cluster(), ranks = ctas_of_cluster();
    const int64_t row = blockIdx.x / ranks;
    const int64_t share = (a.vocab + ranks - 1) / ranks, begin = min(share * rank, a.vocab);
    const int64_t n = min(share, a.vocab - begin);
    pdl_wait();
    const T *const p = static_cast<const T *>(a.logits) + row * a.ld + begin;
    Part part;
    TopList list(TOP ? a.top : 1, lane);

    const int64_t head = to_boundary(p, n), body = (n - head) / V, tail = head + body * V;
    auto one = [&](int64_t i, bool in) {   // one element a lane, by whole warps
        float z[1] = {-INFINITY};
        if (in) {
            z[0] = __fmul_rn(ld1(p + i), a.scale);
            part.add(z);
        }
        if (TOP && list.wanted(in ? z[0] : -INFINITY))
            list.offer(z[0], in ? (int)(begin + i) : 0x7FFFFFFF);
    };
    if (warp == 0)
        one(lane, lane < head);
    if (warp == warps - 1)
        one(tail + lane, tail + lane < n);
    for (int64_t i0 = (int64_t)warp * 32; i0 < body; i0 += (int64_t)nt * U) {
        Vec<T, V> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i0 + lane + (int64_t)u * nt < body)
                v[u].load(p + head + (i0 + lane + (int64_t)u * nt) * V);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t i = i0 + lane + (int64_t)u * nt;
            const bool in = i < body;
            float z[V];
#pragma unroll
            for (int j = 0; j < V; ++j)
                z[j] = in ? __fmul_rn(v[u].get(j), a.scale) : -INFINITY;
            if (in)
                part.add(z);
            if (TOP) {
                float largest = z[0];
#pragma unroll
                for (int j = 1; j < V; ++j)
                    largest = fmaxf(largest, z[j]);
                if (list.wanted(in ? largest : -INFINITY))
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        list.offer(z[j], in ? (int)(begin + head + i * V + j) : 0x7FFFFFFF);
            }
        }
    }

    part.warp_join();
    if (lane == 0)
        parts[warp] = part;
    if (TOP) {
        tops_v[warp * 32 + lane] = list.v;
        tops_id[warp * 32 + lane] = list.id;
    }
    __syncthreads();
    if (warp == 0) {
        for (int w = 1; w < warps; ++w) {
            part.join(parts[w]);
            if (TOP && list.wanted(tops_v[w * 32]))
                list.offer(lane < a.top ? tops_v[w * 32 + lane] : -INFINITY,
                           lane < a.top ? tops_id[w * 32 + lane] : 0x7FFFFFFF);
        }
    }
    if (ranks > 1) {
        if (warp == 0) {
            if (lane == 0)
                parts[0] = part;
            if (TOP) {
                tops_v[lane] = list.v;
                tops_id[lane] = list.id;
            }
        }
        cluster_barrier();
        if (rank == 0 && warp == 0) {
            for (uint32_t r = 1; r < ranks; ++r) {
                Part o;
                const uint32_t at = in_cta(&parts[0], r);
                o.m = ld_cluster_f32(at);
                o.s = ld_cluster_f32(at + 4);
                o.w = ld_cluster_f32(at + 8);
                part.join(o);
                if (TOP)
                    list.offer(lane < a.top ? ld_cluster_f32(in_cta(tops_v + lane, r)) : -INFINITY,
                               lane < a.top ? (int)ld_cluster(in_cta(tops_id + lane, r)) : 0x7FFFFFFF);
            }
        }
        cluster_barrier();   // no CTA leaves while the first may read its part
    }
    if (rank != 0 || warp != 0)
        return;
    const float logs = part.log_sum();
    if (lane == 0) {
        a.stats[2 * row] = part.m;
        a.stats[2 * row + 1] = logs;
        if (a.entropy != nullptr)
            a.entropy[row] = part.entropy();
        if (a.logp != nullptr) {
            const int id = a.ids.at(row, a.vocab);
            float logp = 0.0f;
            if (id >= 0)
                logp = __fmul_rn(ld1(static_cast<const T *>(a.logits) + row * a.ld + id), a.scale) - part.m - logs;
            a.logp[row] = logp;
        }
    }
    if (TOP && lane < a.top) {
        a.top_logp[row * a.top + lane] = list.v - part.m - logs;
        a.top_ids[row * a.top + lane] = list.id;
    }
}

// ------------------------------------------------------------ backward ----
constexpr int kBackThreads = 256, kBackPieces = 4;

struct LogBackArgs {
    const void *logits;
    Ids ids;
    const float *stats, *entropy, *dlogp, *dentropy;
    void *dlogits;
    int64_t rows, vocab, ld, ld_d;
    int64_t spans;               // of a row
    float scale;
};

// A row's scalars and its gradient's elements. p = e^(z - m - log S) by the accurate
// exponential where fp32 is stored, by the approximation (2^-20 here) where bf16 is.
template <bool ACCURATE> struct RowGradient {
    float m, logs, h, a, b, scale;
    int id;
    __device__ __forceinline__ float operator()(float logit, int64_t col) const
    {
        const float lp = __fmul_rn(logit, scale) - m - logs;
        const float p = ACCURATE ? expf(lp) : exp2_fast(lp * kLog2e);
        float g = col == id ? a * -expm1f(lp) : -a * p;
        if (b != 0.0f && p != 0.0f)
            g = fmaf(-b * p, lp + h, g);
        return g * scale;
    }
};

// CTAs of a row take spans of kBackThreads * kBackPieces accesses; V elements an access, the
// same alignment on both sides, or 1.
template <class T, int V>
__global__ void __launch_bounds__(kBackThreads) logprobs_backward_kernel(const LogBackArgs a)
{
    const int64_t row = blockIdx.x / a.spans, span = blockIdx.x - row * a.spans;
    pdl_wait();
    const T *const p = static_cast<const T *>(a.logits) + row * a.ld;
    T *const d = static_cast<T *>(a.dlogits) + row * a.ld_d;
    RowGradient<sizeof(T) == 4> f;
    f.id = a.ids.at(row, a.vocab);
    f.a = f.id >= 0 ? ld1(a.dlogp + row) : 0.0f;
    f.b = a.dentropy != nullptr ? ld1(a.dentropy + row) : 0.0f;
    f.h = a.dentropy != nullptr ? ld1(a.entropy + row) : 0.0f;
    f.m = ld1(a.stats + 2 * row);
    f.logs = ld1(a.stats + 2 * row + 1);
    f.scale = a.scale;
    const bool none = f.a == 0.0f && f.b == 0.0f;
    const int64_t head = V == 1 ? 0 : to_boundary(p, a.vocab), body = (a.vocab - head) / V;
    auto one = [&](int64_t i) { st1(d + i, none ? 0.0f : f(ld1(p + i), i)); };
    if (span == 0) {
        if ((int64_t)threadIdx.x < head)
            one(threadIdx.x);
        const int64_t i = head + body * V + threadIdx.x;
        if (i < a.vocab)
            one(i);
    }
    const int64_t i0 = span * (kBackThreads * kBackPieces) + threadIdx.x;
    Vec<T, V> v[kBackPieces];
#pragma unroll
    for (int u = 0; u < kBackPieces; ++u)
        if (!none && i0 + u * kBackThreads < body)
            v[u].load(p + head + (i0 + u * kBackThreads) * V);
#pragma unroll
    for (int u = 0; u < kBackPieces; ++u) {
        const int64_t i = head + (i0 + u * kBackThreads) * V;
        float g[V];
#pragma unroll
        for (int j = 0; j < V; ++j)
            g[j] = none ? 0.0f : f(v[u].get(j), i + j);
        Vec<T, V> o;
        o.set(g);
        if (i0 + u * kBackThreads < body)
            o.store(d + i);
    }
}

// ---------------------------------------------------------------- host ----

int check_rows(const char *what, int64_t rows, int64_t vocab, int dtype, float scale)
{
    if (!known(dtype))
        return call_fail(DPO_EDTYPE, "%s: dtype %d", what, dtype);
    if (rows < 0 || rows >= kMaxCount / kMaxCtas || vocab < 1 || vocab >= kMaxCount - 1)
        return call_fail(DPO_EINVAL, "%s: %lld rows of %lld", what, (long long)rows, (long long)vocab);
    if (!isfinite(scale) || !(scale > 0.0f))
        return call_fail(DPO_EINVAL, "%s: scale %g", what, (double)scale);
    return DPO_OK;
}

int check_row_ids(const char *what, const dpo_ids &ids, int64_t rows, Ids *out)
{
    int64_t n = 0;
    const int rc = check_ids(what, ids, out, &n);
    if (rc == DPO_OK && n != rows)
        return call_fail(DPO_EINVAL, "%s: %lld ids for %lld rows", what, (long long)n, (long long)rows);
    return rc;
}

template <class T> auto back_fn(bool wide) -> void (*)(LogBackArgs)
{
    return wide ? logprobs_backward_kernel<T, 16 / (int)sizeof(T)> : logprobs_backward_kernel<T, 1>;
}

}  // namespace
}  // namespace dpo

using namespace dpo;

extern "C" int dpo_logprobs(const dpo_logprobs_args *args, void *cuda_stream)
{
    const char *what = "dpo_logprobs";
    if (args == nullptr)
        return call_fail(DPO_EINVAL, "%s: no arguments", what);
    const dpo_logprobs_args &a = *args;
    int rc = check_rows(what, a.rows, a.vocab, a.dtype, a.scale);
    if (rc != DPO_OK)
        return rc;
    if (a.top < 0 || a.top > DPO_MAX_TOP || a.top > a.vocab)
        return call_fail(DPO_EINVAL, "%s: top %d of %lld", what, a.top, (long long)a.vocab);
    LogArgs k{};
    if (a.ids.p != nullptr && (rc = check_row_ids(what, a.ids, a.rows, &k.ids)) != DPO_OK)
        return rc;
    if (a.rows == 0)
        return DPO_OK;
    const int64_t size = elem_size(a.dtype);
    Buffers b(what);
    b.add("logits", a.logits, a.rows, a.vocab, a.ld_logits, size, size, false);
    if (a.ids.p != nullptr) {
        add_ids(b, a.ids);
        b.add("logp", a.logp, 1, a.rows, a.rows, 4, 4, true);
        k.logp = a.logp;
    }
    if (a.entropy != nullptr)
        b.add("entropy", a.entropy, 1, a.rows, a.rows, 4, 4, true);
    b.add("stats", a.stats, 1, 2 * a.rows, 2 * a.rows, 4, 4, true);
    if (a.top > 0) {
        b.add("top_logp", a.top_logp, 1, a.rows * a.top, a.rows * a.top, 4, 4, true);
        b.add("top_ids", a.top_ids, 1, a.rows * a.top, a.rows * a.top, 8, 8, true);
    }
    if ((rc = b.done()) != DPO_OK)
        return rc;
    const int sms = sm_count();
    if (sms == 0)
        return call_fail(DPO_ECUDA, "%s: no device", what);
    k.logits = a.logits;
    k.entropy = a.entropy;
    k.stats = a.stats;
    k.top_logp = a.top_logp;
    k.top_ids = a.top_ids;
    k.rows = a.rows;
    k.vocab = a.vocab;
    k.ld = a.ld_logits;
    k.scale = a.scale;
    k.top = a.top;
    // a thread has some 16 elements at least; CTAs share a row while there are few rows
    int threads = 32, ctas = 1;
    while (threads < kMaxThreads && (int64_t)threads * 32 < a.vocab)
        threads *= 2;
    while (ctas < kMaxCtas && a.rows * ctas * 2 <= sms && (int64_t)ctas * threads * 32 < a.vocab)
        ctas *= 2;
    void (*fn)(LogArgs);
    if (a.dtype == DPO_F32)
        fn = a.top > 0 ? logprobs_kernel<float, true> : logprobs_kernel<float, false>;
    else
        fn = a.top > 0 ? logprobs_kernel<__nv_bfloat16, true> : logprobs_kernel<__nv_bfloat16, false>;
    return launch_in_clusters(what, fn, a.rows * ctas, ctas, threads, 0, cuda_stream, k);
}

extern "C" int dpo_logprobs_backward(const dpo_logprobs_backward_args *args, void *cuda_stream)
{
    const char *what = "dpo_logprobs_backward";
    if (args == nullptr)
        return call_fail(DPO_EINVAL, "%s: no arguments", what);
    const dpo_logprobs_backward_args &a = *args;
    int rc = check_rows(what, a.rows, a.vocab, a.dtype, a.scale);
    LogBackArgs k{};
    if (rc != DPO_OK || (rc = check_row_ids(what, a.ids, a.rows, &k.ids)) != DPO_OK || a.rows == 0)
        return rc;
    const int64_t size = elem_size(a.dtype);
    const bool in_place = a.dlogits == a.logits && a.ld_dlogits == a.ld_logits;
    Buffers b(what);
    b.add("logits", a.logits, a.rows, a.vocab, a.ld_logits, size, size, in_place);
    if (!in_place)
        b.add("dlogits", a.dlogits, a.rows, a.vocab, a.ld_dlogits, size, size, true);
    add_ids(b, a.ids);
    b.add("stats", a.stats, 1, 2 * a.rows, 2 * a.rows, 4, 4, false);
    b.add("dlogp", a.dlogp, 1, a.rows, a.rows, 4, 4, false);
    if (a.dentropy != nullptr) {
        b.add("dentropy", a.dentropy, 1, a.rows, a.rows, 4, 4, false);
        b.add("entropy", a.entropy, 1, a.rows, a.rows, 4, 4, false);
    }
    if ((rc = b.done()) != DPO_OK)
        return rc;
    const int64_t wide = 16 / size;
    const bool aligned = (reinterpret_cast<uintptr_t>(a.logits) - reinterpret_cast<uintptr_t>(a.dlogits)) % 16 == 0 &&
                         (a.ld_logits - a.ld_dlogits) % wide == 0;
    k.logits = a.logits;
    k.stats = a.stats;
    k.entropy = a.entropy;
    k.dlogp = a.dlogp;
    k.dentropy = a.dentropy;
    k.dlogits = a.dlogits;
    k.rows = a.rows;
    k.vocab = a.vocab;
    k.ld = a.ld_logits;
    k.ld_d = a.ld_dlogits;
    k.scale = a.scale;
    const int64_t span = (int64_t)kBackThreads * kBackPieces * (aligned ? wide : 1);
    k.spans = (a.vocab + span - 1) / span;
    if (k.spans * a.rows >= kMaxCount)
        return call_fail(DPO_EINVAL, "%s: %lld rows of %lld are too many", what, (long long)a.rows,
                         (long long)a.vocab);
    return launch(what, a.dtype == DPO_F32 ? back_fn<float>(aligned) : back_fn<__nv_bfloat16>(aligned),
                  k.spans * a.rows, kBackThreads, 0, cuda_stream, k);
}
