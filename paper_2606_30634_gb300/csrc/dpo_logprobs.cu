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

// The warps' lists, in shared memory, merged into the first one's p.
__device__ __forceinline__ void merge_warps(Pair &p, Pair (*lists)[32], int warps, int warp, int lane)
{
    lists[warp][lane] = p;
    for (int step = 1; step < warps; step *= 2) {
        __syncthreads();
        if (warp % (2 * step) == 0) {   // the number of warps is a power of two
            merge_pairs(p, lists[warp + step][31 - lane], lane);
            lists[warp][lane] = p;
        }
    }
    __syncthreads();
}

// A cluster's CTAs share a row, in equal spans; accesses of 16 bytes from the span's first
// boundary on, so rows of odd pitches cost two short ends.
// The `top` largest: each thread knows the largest of its own values, and the top-th of these
// bounds the top-th of all from below. So only the threads that hold one of the first `top`
// of them, `top` threads at most, can hold others, and their values alone are read again.
template <class T, bool TOP>
__global__ void __launch_bounds__(kMaxThreads) logprobs_kernel(const LogArgs a)
{
    constexpr int V = 16 / (int)sizeof(T), U = 4;
    __shared__ Part parts[kMaxWarps];
    __shared__ Pair lists[TOP ? kMaxWarps : 1][32];
    const int nt = blockDim.x, warps = nt >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cta_of_cluster(), ranks = ctas_of_cluster();
    const int64_t row = blockIdx.x / ranks;
    const int64_t share = (a.vocab + ranks - 1) / ranks, begin = min(share * rank, a.vocab);
    const int64_t n = min(share, a.vocab - begin);
    pdl_wait();
    const T *const p = static_cast<const T *>(a.logits) + row * a.ld + begin;
    const int head = (int)to_boundary(p, n);
    const int64_t body = (n - head) / V, tail = head + body * V;
    const T *const vectors = p + head;
    // where ids are wanted the values are the products z, else the logits themselves
    const float pre = TOP ? a.scale : 1.0f, c = TOP ? kLog2e : a.scale * kLog2e;
    const float low = -Run::kLow / 10 * pre;
    Run run;
    int64_t best = threadIdx.x;   // the access with this thread's largest value
    for (int64_t i0 = threadIdx.x; i0 < body; i0 += (int64_t)nt * U) {
        Vec<T, V> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i0 + (int64_t)u * nt < body)
                v[u].load(vectors + (i0 + (int64_t)u * nt) * V);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i0 + (int64_t)u * nt >= body)
                break;
            float l[V], k[V];
            float top = open_row(v[u], l, k);
            if (TOP) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    l[j] = __fmul_rn(l[j], pre);
                    k[j] = __fmul_rn(k[j], pre);
                }
                top = __fmul_rn(top, pre);
                if (top > run.m)
                    best = i0 + (int64_t)u * nt;
            }
            run.add(l, k, top, c, low);
        }
    }
    Pair mine;
    if (TOP && threadIdx.x < body) {
        Vec<T, V> v;
        v.load(vectors + best * V);
        mine.v = run.m;
#pragma unroll
        for (int j = V - 1; j >= 0; --j) {
            const float z = __fmul_rn(v.get(j), pre);
            if ((z == z ? z : -INFINITY) == run.m)
                mine.id = (int)(begin + head + best * V + j);
        }
    }
    // the short ends: the first warp's lanes, one element each (V <= 8 of either)
    const int64_t end = lane < 16 ? (lane < head ? lane : -1) : tail + lane - 16 < n ? tail + lane - 16 : -1;
    float end_z = -INFINITY;
    if (warp == 0 && end >= 0) {
        const float l[1] = {__fmul_rn(ld1(p + end), pre)};
        const float k[1] = {l[0] == l[0] ? fmaxf(l[0], -Run::kLow * pre) : l[0]};
        end_z = l[0];
        run.add(l, k, l[0], c, low);
    }

    Part part = run.part(TOP ? 1.0f : a.scale);
    part.warp_join();
    if (lane == 0)
        parts[warp] = part;
    if (TOP) {
        sort_pairs(mine, lane);
        merge_warps(mine, lists, warps, warp, lane);
        TopList more;   // what the others left out
        more.top = a.top;
        more.lane = lane;
        more.last = lists[0][a.top - 1];
        for (int i = warp; i < a.top; i += warps) {
            const int id = lists[0][i].id;
            if (id == 0x7FFFFFFF)
                break;
            const int64_t own = (id - begin - head) / V % nt;
            for (int64_t q0 = own; q0 < body; q0 += 32 * (int64_t)nt) {
                const int64_t q = q0 + lane * (int64_t)nt;
                Vec<T, V> v;
                v.zero();
                if (q < body)
                    v.load(vectors + q * V);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const int at = (int)(begin + head + q * V + j);
                    const bool in = q < body && at != id;
                    more.offer(in ? __fmul_rn(v.get(j), pre) : -INFINITY, in ? at : 0x7FFFFFFF);
                }
            }
        }
        if (warp == 0)
            more.offer(end_z, end >= 0 ? (int)(begin + end) : 0x7FFFFFFF);
        if (__syncthreads_or(more.p.id != 0x7FFFFFFF)) {
            Pair base = mine;   // the first warp's
            merge_warps(more.p, lists, warps, warp, lane);
            if (warp == 0) {
                merge_pairs(base, shfl(more.p, 31 - lane), lane);
                mine = base;
            }
        }
    } else {
        __syncthreads();
    }
    if (warp == 0)
        for (int w = 1; w < warps; ++w)
            part.join(parts[w]);
    if (ranks > 1) {
        if (warp == 0) {
            if (lane == 0)
                parts[0] = part;
            if (TOP)
                lists[0][lane] = mine;
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
                if (TOP) {
                    const uint32_t q = in_cta(&lists[0][31 - lane], r);
                    Pair other;
                    other.v = ld_cluster_f32(q);
                    other.id = (int)ld_cluster(q + 4);
                    merge_pairs(mine, other, lane);
                }
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
        a.top_logp[row * a.top + lane] = mine.v - part.m - logs;
        a.top_ids[row * a.top + lane] = mine.id;
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

// A row's scalars and its gradient's elements,
//   dlogit = -scale p (a + b (log p + h)) = p (k0 + k1 log p),
// the id's own apart. fp32 results: log p = (z - m) - log S and the accurate exponential. bf16
// results: t = log2 p by two multiply-adds and the approximation, 2^-20 with t's rounding.
template <class T> struct RowGradient {
    static constexpr bool kAccurate = sizeof(T) == 4;
    float m, logs, h, a, b, scale, k0, k1, t0;
    int id;
    bool none;
    __device__ __forceinline__ RowGradient(const LogBackArgs &s, int64_t row)
    {
        id = s.ids.at(row, s.vocab);
        a = id >= 0 ? ld1(s.dlogp + row) : 0.0f;
        b = s.dentropy != nullptr ? ld1(s.dentropy + row) : 0.0f;
        h = s.dentropy != nullptr ? ld1(s.entropy + row) : 0.0f;
        m = ld1(s.stats + 2 * row);
        logs = ld1(s.stats + 2 * row + 1);
        scale = s.scale;
        none = a == 0.0f && b == 0.0f;
        if (b == 0.0f)
            h = 0.0f;
        k0 = -scale * fmaf(b, h, a);
        k1 = -scale * b * (kAccurate ? 1.0f : 0.6931471805599453f);
        t0 = -logs * kLog2e;
    }
    __device__ __forceinline__ float other(float logit) const
    {
        const float t = kAccurate ? __fmul_rn(logit, scale) - m - logs
                                  : fmaf(fmaf(logit, scale, -m), kLog2e, t0);
        const float p = kAccurate ? expf(t) : exp2_fast(t);
        return p * fmaf(k1, fmaxf(t, -1e30f), k0);   // no infinity times 0
    }
    __device__ __forceinline__ float own(float logit) const   // col == id
    {
        const float lp = __fmul_rn(logit, scale) - m - logs, p = expf(lp);
        float g = a * -expm1f(lp);
        if (b != 0.0f && p != 0.0f)
            g = fmaf(-b * p, lp + h, g);
        return g * scale;
    }
    __device__ __forceinline__ float operator()(float logit, int64_t col) const
    {
        return none ? 0.0f : col == id ? own(logit) : other(logit);
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
    const int64_t head = V == 1 ? 0 : to_boundary(p, a.vocab), body = (a.vocab - head) / V;
    const int64_t i0 = span * (kBackThreads * kBackPieces) + threadIdx.x;
    Vec<T, V> v[kBackPieces];
#pragma unroll
    for (int u = 0; u < kBackPieces; ++u)
        if (i0 + u * kBackThreads < body)
            v[u].load(p + head + (i0 + u * kBackThreads) * V);
    const RowGradient<T> f(a, row);
    if (V > 1 && span == 0) {
        const int64_t end = threadIdx.x < 16 ? (threadIdx.x < head ? threadIdx.x : a.vocab)
                                             : head + body * V + threadIdx.x - 16;
        if (end < a.vocab)
            st1(d + end, f(ld1(p + end), end));
    }
#pragma unroll
    for (int u = 0; u < kBackPieces; ++u) {
        if (i0 + u * kBackThreads >= body)
            break;
        const int64_t i = head + (i0 + u * kBackThreads) * V;
        float g[V];
#pragma unroll
        for (int j = 0; j < V; ++j)
            g[j] = f.none ? 0.0f : f.other(v[u].get(j));
        const int64_t at = f.id - i;
        if (at >= 0 && at < V && !f.none)
#pragma unroll
            for (int j = 0; j < V; ++j)
                g[j] = at == j ? f.own(v[u].get(j)) : g[j];
        Vec<T, V> o;
        o.set(g);
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
    if (!good_scale(scale))
        return call_fail(DPO_EINVAL, "%s: scale %g (1e-20 to 1e6)", what, (double)scale);
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
