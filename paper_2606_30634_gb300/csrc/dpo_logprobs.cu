// dpo_logprobs.cu -- log probabilities of given tokens, entropy and most likely ids from logits,
// and their gradient (dpo_logprobs, dpo_logprobs_backward in include/dpo.h).
//
// Forward: every logit is read once; a thread keeps the running maximum m, sum S and entropy
// sum W of its own, and the threads' are joined. Backward: every logit once more, dlogits
// written. Both are bound by HBM (4096 x 50257 bf16: 66 and 132 us, 6.2 TB/s both); few rows
// by latency, where a cluster shares a row. What instructions they take is seen: with 15 an
// element instead of 6 the forward took 107 us, with 20 instead of 7 the backward 180.
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
    int warps;                   // of a row: all of the CTA's, or one
};

// Elements before the first 16-byte boundary, at most n.
template <class T> __device__ __forceinline__ int64_t to_boundary(const T *p, int64_t n)
{
    const int64_t k = (int64_t)((16u - (uint32_t)(reinterpret_cast<uintptr_t>(p) & 15u)) & 15u) / (int)sizeof(T);
    return k < n ? k : n;
}

// By all threads that have a row.
__device__ __forceinline__ void row_sync(int warps)
{
    if (warps == 1)
        __syncwarp();
    else
        __syncthreads();
}

// The warps' sorted lists, in shared memory, merged into the first one's p.
template <class K>
__device__ __forceinline__ void merge_warps(K &p, K (*lists)[32], int warps, int warp, int lane)
{
    lists[warp][lane] = p;
    for (int step = 1; step < warps; step *= 2) {
        __syncthreads();
        if (warp % (2 * step) == 0) {   // the number of warps is a power of two
            merge_lanes(p, lists[warp + step][31 - lane], lane);
            lists[warp][lane] = p;
        }
    }
    row_sync(warps);
}

// A warp, a CTA or a cluster has a row, a cluster's CTAs in equal spans; accesses of 16 bytes from
// the span's first boundary on, so rows of odd pitches cost two short ends. A thread takes kAhead
// accesses at a time, their largest first (4096 x 50257 bf16: 71 us by four, 66 by eight).
// The `top` largest: each thread knows the largest of its own values, and the top-th of these
// bounds the top-th of all from below. So only the threads whose largest reaches the bound, `top`
// and what is equal, can hold one of them; their values are read again, and what reaches the
// bound is sorted, or offered to lists where it is much (equal values, masked rows): more than 32
// values a warp, or 128 (7 rows of 199 bf16 with 20: 31 us by lists, for more than 32).
// us by the threads of a row, 32 / 128 / 512: 4096 rows of 50257 bf16 by four accesses 71 / 77 / 104,
// 300 of 32000 fp32 - / 12.4 / 9.4; with 5 of 1000 rows of 32000 fp32 64 / 128 / 256: 25.7 / 25.6 / 27.2, 4000
// rows 117 / 92 / 92 (a bound from few threads lets more values be read again). 4000 rows of
// 32000 fp32: 76 us, 6.7 TB/s, 0.99 of the measured copy.
constexpr int kAhead = 8, kBatch = 32, kSmThreads = 800, kTopThreads = 128;

template <class T, bool TOP>
__global__ void __launch_bounds__(kMaxThreads, 2) logprobs_kernel(const LogArgs a)
{
    using Access = RowAccess<T>;
    constexpr int V = Access::V, U = kAhead;
    __shared__ Part parts[kMaxWarps], from_cta[kMaxCtas];
    constexpr int kLists = TOP ? kMaxWarps : 1;
    __shared__ Key lists_[kLists][32], list_from[TOP ? kMaxCtas : 1][32];
    __shared__ float largest_[kLists][32];
    __shared__ uint16_t chosen_[TOP ? kMaxThreads : 1];
    __shared__ int counts_[kLists][2];
    const int warps = a.warps, nt = 32 * warps, lane = threadIdx.x & 31;
    const int first_warp = warps == 1 ? (int)threadIdx.x >> 5 : 0;   // of this row
    const int warp = ((int)threadIdx.x >> 5) - first_warp, thread = 32 * warp + lane;
    const uint32_t rank = cta_of_cluster(), ranks = ctas_of_cluster();
    const int64_t its = ranks > 1 ? blockIdx.x / ranks : (int64_t)blockIdx.x * (blockDim.x / nt) + first_warp;
    const int64_t row = min(its, a.rows - 1);
    constexpr int kRowLists = 4;   // of a row, at least; a CTA has four rows at most
    Key (*const lists)[32] = lists_ + (TOP ? kRowLists * first_warp : 0);
    const int room = 32 * max(warps, kRowLists);
    const int vocab = (int)a.vocab, share = (int)((a.vocab + ranks - 1) / ranks);
    const int begin = (int)min((int64_t)share * rank, a.vocab), n = min(share, vocab - begin);
    if (ranks > 1)
        cluster_arrive();   // its shared memory may be written from now on
    pdl_wait();
    const bool last = rank == 0 && warp == 0 && its < a.rows;   // the warp that ends the row
    int id = -1;
    if (last && a.logp != nullptr)
        id = a.ids.at(row, a.vocab);
    const T *const p = static_cast<const T *>(a.logits) + row * a.ld + begin;
    const int head = (int)to_boundary(p, n);
    const int body = (n - head) / V, tail = head + body * V;
    const T *const vectors = p + head;
    const float c = a.scale * kLog2e;
    const Two cc = two(c, c);
    Run run;
    for (int i0 = thread; i0 < body; i0 += nt * U) {
        Access v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i0 + u * nt < body)
                v[u].v.load(vectors + (int64_t)(i0 + u * nt) * V);
            else
                v[u].none();
        }
        float top = v[0].largest();
#pragma unroll
        for (int u = 1; u < U; ++u)
            top = fmaxf(top, v[u].largest());
        if (top > run.m)
            run.raise(top, c);
        if (run.near()) {
            const Two minus_r = two(-run.r, -run.r);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (i0 + u * nt >= body)
                    break;
#pragma unroll
                for (int j = 0; j < V / 2; ++j)
                    run.add_near(v[u].pair(j, Access::kLow), cc, minus_r);
            }
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int j = 0; j < V; ++j)
                    run.add_far(v[u].v.get(j), c);
        }
    }
    float bound = TOP ? __fmul_rn(run.m, a.scale) : 0.0f;
    // the short ends: a row's first warp's lanes, one element each (V <= 8 of either)
    const int at_end = lane < 16 ? lane : tail + lane - 16;
    const int end = warp == 0 && at_end < (lane < 16 ? head : n) ? at_end : -1;
    float end_z = -INFINITY, own = 0.0f;
    if (end >= 0) {
        const float l = ld1(p + end);
        end_z = __fmul_rn(l, a.scale);
        run.add(l, c);
    }
    if (id >= 0)
        own = ld1(static_cast<const T *>(a.logits) + row * a.ld + id);

    Part part = run.part(a.scale);
    part.warp_join();
    if (lane == 0 && warps > 1)
        parts[warp] = part;
    Key mine = 0;
    if (TOP) {
        uint16_t *const chosen = chosen_ + 32 * first_warp;
        int *const counts = counts_[first_warp];   // of threads, of values
        const float own_largest = bound;
        if (thread < 2)
            counts[thread] = 0;
        sort_lanes(bound, lane);
        merge_warps(bound, largest_ + first_warp, warps, warp, lane);
        bound = largest_[first_warp][a.top - 1];
        if (thread < body && own_largest >= bound)
            chosen[atomicAdd(counts, 1)] = (uint16_t)thread;
        row_sync(warps);
        // 32 of a thread's accesses are a block; the warps take the blocks in turn
        const int blocks = (body + 32 * nt - 1) / (32 * nt), all = counts[0] * blocks;
        auto scan = [&](auto &&use) {   // by whole warps
            constexpr int kBoth = 2;
            for (int k0 = warp; k0 < all; k0 += warps * kBoth) {
                Access v[kBoth];
                int q[kBoth];
#pragma unroll
                for (int u = 0; u < kBoth; ++u) {
                    const int k = k0 + u * warps, i = k / blocks;
                    v[u].none();
                    q[u] = k < all ? chosen[i] + ((k - i * blocks) * 32 + lane) * nt : body;
                    if (q[u] < body)
                        v[u].v.load(vectors + (int64_t)q[u] * V);
                }
#pragma unroll
                for (int u = 0; u < kBoth; ++u) {
                    const bool in = q[u] < body && !(__fmul_rn(v[u].largest(), a.scale) < bound);
                    if (__any_sync(0xFFFFFFFFu, in))
#pragma unroll
                        for (int j = 0; j < V; ++j)
                            use(in, __fmul_rn(v[u].v.get(j), a.scale), begin + head + q[u] * V + j);
                }
            }
            if (warp == 0)
                use(end >= 0, end_z, begin + end);
        };
        scan([&](bool in, float z, int at) {
            if (in && !(z < bound) && (z == z || bound == -INFINITY)) {
                const int slot = atomicAdd(counts + 1, 1);
                if (slot < room)
                    lists[0][slot] = key_of(z, at);
            }
        });
        row_sync(warps);
        const int found = counts[1];
        if (found <= room) {
            for (int l = warp; 32 * l < found; l += warps) {
                Key more = 32 * l + lane < found ? lists[l][lane] : 0;
                sort_lanes(more, lane);
                if (l == warp)
                    mine = more;
                else
                    merge_lanes(mine, __shfl_sync(0xFFFFFFFFu, more, 31 - lane), lane);
            }
            if (found > 32 && warps > 1) {
                row_sync(warps);
                merge_warps(mine, lists, warps, warp, lane);
            }
        } else {
            TopList list{0, bound == -INFINITY ? 0 : key_of(bound, 0x7FFFFFFF), a.top, lane};   // 0: NaN too
            row_sync(warps);
            scan([&](bool in, float z, int at) { list.offer(in ? key_of(z, at) : 0); });
            mine = list.p;
            merge_warps(mine, lists, warps, warp, lane);
        }
    } else if (warps > 1) {
        __syncthreads();
    }
    if (warp == 0 && warps > 1) {
        part = lane < warps ? parts[lane] : Part();
        part.warp_join();
    }
    if (ranks > 1) {   // the first CTA gets the others' parts; all of its warps are there (ranks <= warps)
        cluster_wait();
        if (warp == 0 && rank > 0) {
            if (lane == 0) {
                const uint32_t at = in_cta(&from_cta[rank], 0);
                st_cluster(at, __float_as_uint(part.m));
                st_cluster(at + 4, __float_as_uint(part.s));
                st_cluster(at + 8, __float_as_uint(part.w));
            }
            if (TOP)
                st_cluster(in_cta(&list_from[rank][lane], 0), (uint32_t)mine, (uint32_t)(mine >> 32));
        }
        cluster_barrier();
        if (rank != 0)
            return;
        if (TOP) {
            if (warp > 0)
                mine = warp < (int)ranks ? list_from[warp][lane] : 0;
            merge_warps(mine, lists, (int)ranks, warp, lane);
        }
        if (warp == 0) {
            const Part o = lane > 0 && lane < (int)ranks ? from_cta[lane] : Part();
            part = lane == 0 ? part : o;
            part.warp_join();
        }
    }
    if (!last)
        return;
    const float logs = part.log_sum();
    if (lane == 0) {
        a.stats[2 * row] = part.m;
        a.stats[2 * row + 1] = logs;
        if (a.entropy != nullptr)
            a.entropy[row] = part.entropy();
        if (a.logp != nullptr)
            a.logp[row] = id >= 0 ? __fmul_rn(own, a.scale) - part.m - logs : 0.0f;
    }
    if (TOP && lane < a.top) {
        a.top_logp[row * a.top + lane] = value_of(mine) - part.m - logs;
        a.top_ids[row * a.top + lane] = id_of(mine);
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
    float scale, inverse;        // 1 / scale
};

// A row's scalars and its gradient's elements,
//   dlogit = -scale p (a + b (log p + h)) = p (k0 + k1 log p),
// the id's own apart. fp32 results: log p = (z - m) - log S and the accurate exponential. bf16
// results: log p from the differences to the largest logit l0, which a bf16 number is and m, its
// rounded product, gives back: t = l c - r by one multiply-add, c = scale log2(e), r = l0 c + log2 S
// rounded. What t of l0 itself is off by then is the same for the whole row and comes out of k0 and
// k1; left are 2^-22 of the exponential and 2^-22 of log p, wherever the row lies (with m c rounded in
// r: 2^-13 of p for logits of 1000). Logits so low that p is 0 come as one of these, so that t times 0 is 0.
// Rows whose r is far out take the differences themselves.
template <class T> struct RowGradient {
    static constexpr bool kAccurate = sizeof(T) == 4;
    float m, logs, h, a, b, scale, k0, k1, c, r;
    float top, logs2;            // bf16: l0, log2 S
    typename RowAccess<T>::Low low;
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
        c = scale * kLog2e;
        if constexpr (!kAccurate) {
            const float q = m * s.inverse;   // l0 but for 2^-22, less than half a step of bf16
            top = __bfloat162float(__float2bfloat16_rn(q));
            if (__fmul_rn(top, scale) != m)
                top = q;                     // a maximum from elsewhere
            logs2 = logs * kLog2e;
            r = fmaf(top, c, logs2);
            if (near()) {
                const float off = fmaf(top, c, -r) + logs2, f = exp2_fast(-off);
                k0 = fmaf(-k1, off, k0) * f;
                k1 *= f;
            }
        }
        set_low(&low);
    }
    __device__ __forceinline__ void set_low(float *v) const { *v = -INFINITY; }
    __device__ __forceinline__ void set_low(uint32_t *v) const   // t at most -1000, about
    {
        const __nv_bfloat162 q = __float2bfloat162_rn(fmaxf((r - 1000.0f) / c, -1e30f));
        *v = *reinterpret_cast<const uint32_t *>(&q);
    }
    __device__ __forceinline__ bool near() const { return fabsf(r) < 16384.0f; }
    __device__ __forceinline__ float other(float logit) const   // row_gradient's, one at a time
    {
        float t;
        if constexpr (kAccurate)
            t = __fmul_rn(logit, scale) - m - logs;
        else if (near())
            t = fmaf(logit == logit ? fmaxf(logit, __uint_as_float(low << 16)) : logit, c, -r);
        else
            t = fmaf(logit - top, c, -logs2);
        const float p = kAccurate ? expf(t) : exp2_fast(t);
        return p * fmaf(k1, fmaxf(t, -1e30f), k0);   // no infinity times 0
    }
    __device__ __forceinline__ float own(float logit) const   // col == id
    {
        const float lp = kAccurate ? __fmul_rn(logit, scale) - m - logs : fmaf(logit - top, scale, -logs);
        const float p = expf(lp);
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

template <class T, int V>
__device__ __forceinline__ void row_gradient(const RowGradient<T> &f, const Vec<T, V> &v, float (&g)[V])
{
    if (sizeof(T) == 4 || V == 1 || !f.near()) {
#pragma unroll
        for (int j = 0; j < V; ++j)
            g[j] = f.other(v.get(j));
    } else if constexpr (sizeof(T) == 2 && V > 1) {
        RowAccess<T> x;
        x.v = v;
        const Two cc = two(f.c, f.c), rr = two(-f.r, -f.r), k0 = two(f.k0, f.k0), k1 = two(f.k1, f.k1);
#pragma unroll
        for (int j = 0; j < V / 2; ++j) {
            const Two t = fma_two(x.pair(j, f.low), cc, rr);
            const float2 u = of_two(t);
            const float2 y = of_two(mul_two(two(exp2_fast(u.x), exp2_fast(u.y)), fma_two(k1, t, k0)));
            g[2 * j] = y.x;
            g[2 * j + 1] = y.y;
        }
    }
}

// CTAs of a row take spans of kBackThreads * kBackPieces accesses; V elements an access, the
// same alignment on both sides, or 1.
template <class T, int V>
__global__ void __launch_bounds__(kBackThreads) logprobs_backward_kernel(const LogBackArgs a)
{
    const int64_t row = blockIdx.x / (unsigned)a.spans, span = blockIdx.x - row * a.spans;
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
        const int64_t end = threadIdx.x < 16 ? ((int)threadIdx.x < head ? threadIdx.x : a.vocab)
                                             : head + body * V + threadIdx.x - 16;
        if (end < a.vocab)
            st1(d + end, f(ld1(p + end), end));
    }
#pragma unroll
    for (int u = 0; u < kBackPieces; ++u) {
        if (i0 + u * kBackThreads >= body)
            break;
        const int64_t i = head + (i0 + u * kBackThreads) * V;
        Vec<T, V> o;
        o.zero();
        if (!f.none) {
            float g[V];
            row_gradient<T, V>(f, v[u], g);
            const int64_t at = f.id - i;
            if (at >= 0 && at < V)
#pragma unroll
                for (int j = 0; j < V; ++j)
                    g[j] = at == j ? f.own(v[u].get(j)) : g[j];
            o.set(g);
        }
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
    // As few threads of a row as give every SM kSmThreads, so that little is joined; where there
    // are too few rows for that, as many as find kBatch logits each, and then the CTAs of a cluster.
    int threads = 32, ctas = 1;
    while (threads < kMaxThreads && (int64_t)threads * kBatch < a.vocab &&
           (a.rows * threads < (int64_t)sms * kSmThreads || (a.top > 0 && threads < kTopThreads)))
        threads *= 2;
    // The bound by few of many threads, where a first access each leaves some to others: 500 rows of
    // 300 fp32 with 32: 41 us by 32 threads, 9 by 128; but 5000 of 900 bf16 with 20: 31 and 38.
    while (threads < kTopThreads && threads * (16 / size) < a.vocab &&
           (a.top > 24 || (2 * a.top > threads && a.rows * threads < (int64_t)sms * kSmThreads)))
        threads *= 2;
    k.warps = threads / 32;
    const int per = k.warps == 1 ? 4 : 1;   // rows of a CTA
    while (threads == kMaxThreads && ctas < kMaxCtas && a.rows * ctas * 2 <= sms &&
           (int64_t)ctas * threads * 32 < a.vocab)
        ctas *= 2;
    void (*fn)(LogArgs);
    if (a.dtype == DPO_F32)
        fn = a.top > 0 ? logprobs_kernel<float, true> : logprobs_kernel<float, false>;
    else
        fn = a.top > 0 ? logprobs_kernel<__nv_bfloat16, true> : logprobs_kernel<__nv_bfloat16, false>;
    return launch_in_clusters(what, fn, (a.rows + per - 1) / per * ctas, ctas, threads * per, 0, cuda_stream, k);
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
    k.inverse = 1.0f / a.scale;
    const int64_t span = (int64_t)kBackThreads * kBackPieces * (aligned ? wide : 1);
    k.spans = (a.vocab + span - 1) / span;
    if (k.spans * a.rows >= kMaxCount)
        return call_fail(DPO_EINVAL, "%s: %lld rows of %lld are too many", what, (long long)a.rows,
                         (long long)a.vocab);
    return launch(what, a.dtype == DPO_F32 ? back_fn<float>(aligned) : back_fn<__nv_bfloat16>(aligned),
                  k.spans * a.rows, kBackThreads, 0, cuda_stream, k);
}
