// dpo_embed.cu -- the embedding of token ids and its gradient (dpo_embed, dpo_embed_backward in
// include/dpo.h).
//
// Forward: out[t] = scale table[id_t]; one pass, the rows' bytes in and out.
// Backward: dtable[v] = scale sum over the t with id_t = v of dy[t]. The tokens are sorted by id
// (each id's tokens in order), and the sorted list is cut into chunks of equal length; a CTA adds
// up the rows of a chunk, id by id, in fp32. An id's run within one chunk is finished there; of
// one that crosses chunks every chunk leaves a partial sum, and the chunks' sums are added in a
// fixed order. So the work is even whatever the ids are, and its order depends on the ids, their
// number and the rows' width alone.
// (Joined by the last CTA to leave a sum, behind a fence and a counter, instead of a third launch:
// 1.3 us more.)
// A gradient that is written is first cleared as a whole by CTAs beside the sort's, which leaves
// HBM idle; the rows that ids have are written twice. 8192 tokens of a 32000 x 4096 bf16 buffer:
// sort and clearing 41 us, 6.3 TB/s; sums 17; joins 6. 5003 of 50257 x 777 fp32, added: 8, 10 and 5, by
// latency.
#include "dpo_ends.cuh"
#include "dpo_vec.cuh"

#include <math.h>

namespace dpo {
namespace {

// ------------------------------------------------------------- forward ----
// A warp takes four accesses a lane of one row: 2 KB of a bf16 row of 16-byte accesses, so
// that a single token's row is shared by several warps and its latency is one access's. Of accesses
// of one or two elements eight, where the row has so many (us by 4 / 8 of them: 8192 tokens of
// 4094 bf16, two an access, 27 / 21; of 4095 47 / 41; 60000 of 77 8.3 / 11).
__host__ __device__ constexpr int pieces(int v, bool many) { return v <= 2 && many ? 8 : 4; }
constexpr int kEmbedWarps = 8;

struct EmbedArgs {
    Ids ids;
    const void *table;
    void *out;
    int64_t vocab, dim, ld_table, ld_out;
    Units units;               // spans of a warp
    float scale;
};

template <class TT, class OT, int V, bool MANY>
__global__ void __launch_bounds__(32 * kEmbedWarps) embed_kernel(const EmbedArgs a)
{
    const int lane = threadIdx.x & 31;
    const int64_t unit = (int64_t)blockIdx.x * kEmbedWarps + (threadIdx.x >> 5);
    pdl_wait();
    if (unit >= a.units.all)
        return;
    int64_t t, span;
    a.units.at(unit, t, span);
    const int64_t c0 = span * (32 * pieces(V, MANY) * V) + lane * V;
    const int id = a.ids.at(t, a.vocab);
    const TT *const row = static_cast<const TT *>(a.table) + (int64_t)max(id, 0) * a.ld_table;
    OT *const out = static_cast<OT *>(a.out) + t * a.ld_out;
    Vec<TT, V> v[pieces(V, MANY)];
#pragma unroll
    for (int n = 0; n < pieces(V, MANY); ++n) {
        v[n].zero();
        if (id >= 0 && c0 + n * 32 * V < a.dim)
            v[n].load(row + c0 + n * 32 * V);
    }
#pragma unroll
    for (int n = 0; n < pieces(V, MANY); ++n) {
        float x[V];
#pragma unroll
        for (int j = 0; j < V; ++j)
            x[j] = v[n].get(j) * (id >= 0 ? a.scale : 0.0f);
        Vec<OT, V> o;
        o.set(x);
        if (c0 + n * 32 * V < a.dim)
            o.store(out + c0 + n * 32 * V);
    }
}

// ------------------------------------------------------------- clearing ----
// dtable's rows as bytes, set to zero 4 KB a warp; contiguous rows are one.
struct ClearArgs {
    uint8_t *p;                // nullptr: nothing to clear
    int64_t rows, bytes, pitch;
    int size;                  // of an element, to whose multiple p is aligned
};
constexpr int kClearBytes = 4096;

// By the CTAs from number `first` of the grid on.
__device__ __forceinline__ void clear_rows(const ClearArgs &a, int first)
{
    const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
    const int64_t pieces = (a.bytes + kClearBytes - 1) / kClearBytes, all = a.rows * pieces;
    const int64_t step = (int64_t)((int)gridDim.x - first) * warps;
    for (int64_t u = (int64_t)((int)blockIdx.x - first) * warps + (threadIdx.x >> 5); u < all; u += step) {
        const int64_t row = u / pieces, at = (u - row * pieces) * kClearBytes;
        const int n = (int)min((int64_t)kClearBytes, a.bytes - at);
        uint8_t *const p = a.p + row * a.pitch + at;
        const int head = min((int)((16u - (uint32_t)(reinterpret_cast<uintptr_t>(p) & 15u)) & 15u), n);
        const int body = (n - head) / 16 * 16;
        auto ends = [&](uint8_t *q, int bytes) {   // less than 16 bytes
            if (lane * a.size < bytes) {
                if (a.size == 4)
                    *reinterpret_cast<uint32_t *>(q + lane * 4) = 0u;
                else
                    *reinterpret_cast<uint16_t *>(q + lane * 2) = 0u;
            }
        };
        ends(p, head);
        for (int i = lane * 16; i < body; i += 512)
            *reinterpret_cast<uint4 *>(p + head + i) = make_uint4(0u, 0u, 0u, 0u);
        ends(p + head + body, n - head - body);
    }
}

// ---------------------------------------------------------------- sort ----
// (id, token) pairs by id, and then by token, padding behind the last id.
struct SortArgs {
    Ids ids;
    int64_t first, count;      // tokens of this span
    int64_t vocab;
    int passes, bits;          // of a pass
    uint2 *sorted;             // (id, token of the span)
    int *n_valid;              // how many are no padding
    int ctas;                  // that sort; the others clear
    ClearArgs clear;
};

// Up to 8192 tokens: a pair's place is the number of pairs before it, counted by comparing it
// with all of them. 67 million comparisons of two instructions each are 4 us on all SMs, with
// no step that waits for another (5003 tokens: 8 us; the cluster's sort below, two passes: 12).
constexpr int kRankTokens = 8192, kRankBits = 13, kRankWarps = 16, kRankKeys = 4;   // keys of a warp
constexpr uint32_t kRankNone = 0x7FFFFFFFu;
constexpr int64_t kRankVocab = (int64_t)1 << (31 - kRankBits);

__global__ void __launch_bounds__(32 * kRankWarps) rank_ids_kernel(const SortArgs a)
{
    __shared__ uint4 keys_[kRankTokens / 4];
    pdl_wait();
    if ((int)blockIdx.x >= a.ctas) {
        clear_rows(a.clear, a.ctas);
        return;
    }
    uint32_t *const keys = reinterpret_cast<uint32_t *>(keys_);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = (int)a.count;
    const int padded = (n + 127) / 128 * 128;
    int id[kRankTokens / (32 * kRankWarps)], some = 0;
    a.ids.at(a.first + threadIdx.x, 32 * kRankWarps, a.first + n, a.vocab, id);
#pragma unroll
    for (int u = 0; u < kRankTokens / (32 * kRankWarps); ++u) {
        const int i = u * 32 * kRankWarps + (int)threadIdx.x;
        some += id[u] >= 0;
        if (i < padded)
            keys[i] = id[u] >= 0 ? (uint32_t)id[u] << kRankBits | (uint32_t)i : kRankNone;
    }
    __shared__ int counts[kRankWarps];
    some = __reduce_add_sync(0xFFFFFFFFu, some);
    if (lane == 0)
        counts[warp] = some;
    __syncthreads();
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        int sum = 0;
        for (int w = 0; w < kRankWarps; ++w)
            sum += counts[w];
        *a.n_valid = sum;
    }
    const int t0 = ((int)blockIdx.x * kRankWarps + warp) * kRankKeys;
    if (t0 >= n)
        return;
    uint32_t mine[kRankKeys], before[kRankKeys];
#pragma unroll
    for (int j = 0; j < kRankKeys; ++j) {
        mine[j] = t0 + j < n ? keys[t0 + j] : kRankNone;
        before[j] = 0u;
    }
#pragma unroll 2
    for (int i = lane; i < padded / 4; i += 32) {
        const uint4 q = keys_[i];
#pragma unroll
        for (int j = 0; j < kRankKeys; ++j)
            for (const uint32_t other : {q.x, q.y, q.z, q.w})
                before[j] += (other - mine[j]) >> 31;   // keys are below 2^31: a sign, shifted and added in one
    }
#pragma unroll
    for (int j = 0; j < kRankKeys; ++j) {
        const uint32_t place = __reduce_add_sync(0xFFFFFFFFu, before[j]);
        if (lane == j && mine[j] != kRankNone)
            a.sorted[place] = make_uint2(mine[j] >> kRankBits, (uint32_t)(t0 + j));
    }
}

// Others, up to DPO_EMBED_SPAN: least significant digit first, in the shared memory of one
// cluster. In a pass every warp ranks its own 256 pairs, in their order, among those with the
// same digit (match.any), the counts are added up over warps and CTAs, and the pairs are sent
// to their places, wherever in the cluster these are.
constexpr int kSortItems = 8, kSortThreads = 512, kSortMinThreads = 128, kSortCtas = 16;
constexpr int kDigitBits = 9;   // of a pass, at most
static_assert(kSortItems * kSortThreads * kSortCtas == DPO_EMBED_SPAN, "a span is a cluster's");

__host__ __device__ constexpr int sort_smem(int threads, int bits)
{
    return threads * kSortItems * 8 + (threads / 32 + kSortCtas + 1) * (1 << bits) * 4;
}

__global__ void __launch_bounds__(kSortThreads) sort_ids_kernel(const SortArgs a)
{
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ uint32_t warp_sums[32];
    const int nt = blockDim.x, warps = nt >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cta_of_cluster(), ranks = ctas_of_cluster();
    const int per = nt * kSortItems, digits = 1 << a.bits;
    uint2 *const items = reinterpret_cast<uint2 *>(smem);
    uint32_t *const count = reinterpret_cast<uint32_t *>(items + per);   // [warp][digit]
    uint32_t *const total = count + warps * digits;                      // [CTA][digit]
    uint32_t *const base = total + kSortCtas * digits;                   // first place, in all
    uint32_t *const mine = count + warp * digits;
    const uint32_t pad = (uint32_t)a.vocab;
    const int at0 = warp * 32 * kSortItems + lane;
    pdl_wait();
    if ((int)blockIdx.x >= a.ctas) {   // whole clusters
        clear_rows(a.clear, a.ctas);
        return;
    }
    cluster_barrier();   // the others' shared memory is written before the next one
    uint32_t key[kSortItems], pos[kSortItems], place[kSortItems];
    int id[kSortItems];
    a.ids.at(a.first + (int64_t)rank * per + at0, 32, a.first + a.count, a.vocab, id);
#pragma unroll
    for (int i = 0; i < kSortItems; ++i) {
        key[i] = id[i] < 0 ? pad : (uint32_t)id[i];
        pos[i] = rank * (uint32_t)per + (uint32_t)(at0 + i * 32);
    }
    for (int p = 0; p < a.passes; ++p) {
        const int shift = p * a.bits;
        auto digit = [&](int i) { return key[i] >> shift & (uint32_t)(digits - 1); };
        for (int d = lane; d < digits; d += 32)
            mine[d] = 0u;
        __syncwarp();
#pragma unroll
        for (int i = 0; i < kSortItems; ++i) {
            const uint32_t d = digit(i), peers = __match_any_sync(0xFFFFFFFFu, d);
            const uint32_t before = __popc(peers & ((1u << lane) - 1u)), old = mine[d];
            __syncwarp();
            if (before == 0)
                mine[d] = old + __popc(peers);
            __syncwarp();
            place[i] = old + before;
        }
        __syncthreads();
        for (int d = threadIdx.x; d < digits; d += nt) {   // counts of earlier warps
            uint32_t sum = 0;
#pragma unroll 4
            for (int w = 0; w < warps; ++w) {
                const uint32_t c = count[w * digits + d];
                count[w * digits + d] = sum;
                sum += c;
            }
            // to every CTA: a store is not waited for, and what was fetched from eight others
            // one after the other took 4 of a pass's 8 us
            for (uint32_t r = 0; r < ranks; ++r)
                st_cluster(in_cta(total + rank * digits + d, r), sum);
        }
        cluster_barrier();
        // first places: digits below, then the same digit in earlier CTAs
        const int each = digits > nt ? digits / nt : 1;   // consecutive digits of a thread
        uint32_t sum = 0;
        for (int j = 0; j < each; ++j) {
            const int d = threadIdx.x * each + j;
            if (d < digits) {
                uint32_t all = 0, earlier = 0;
#pragma unroll
                for (uint32_t r = 0; r < kSortCtas; ++r) {
                    const uint32_t c = r < ranks ? total[r * digits + d] : 0u;
                    earlier += r < rank ? c : 0u;
                    all += c;
                }
                base[d] = sum + earlier;
                sum += all;
            }
        }
        uint32_t scan = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, scan, o);
            scan += lane >= o ? v : 0u;
        }
        if (lane == 31)
            warp_sums[warp] = scan;
        __syncthreads();
        uint32_t below = scan - sum;
        for (int w = 0; w < warp; ++w)
            below += warp_sums[w];
        for (int j = 0; j < each; ++j) {
            const int d = threadIdx.x * each + j;
            if (d < digits)
                base[d] += below;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kSortItems; ++i) {
            const uint32_t d = digit(i), to = base[d] + mine[d] + place[i];
            st_cluster(in_cta(items + to % (uint32_t)per, to / (uint32_t)per), key[i], pos[i]);
        }
        cluster_barrier();
#pragma unroll
        for (int i = 0; i < kSortItems; ++i) {
            key[i] = items[at0 + i * 32].x;
            pos[i] = items[at0 + i * 32].y;
        }
    }
#pragma unroll
    for (int i = 0; i < kSortItems; ++i) {
        const int at = at0 + i * 32;
        const int64_t g = (int64_t)rank * per + at;
        const uint32_t prev = at > 0     ? items[at - 1].x
                              : rank > 0 ? ld_cluster(in_cta(items + per - 1, rank - 1))
                                         : ~0u;
        if (key[i] != pad) {
            a.sorted[g] = make_uint2(key[i], pos[i]);
            if (g + 1 == (int64_t)ranks * per)
                *a.n_valid = (int)(g + 1);
        } else if (prev != pad) {
            *a.n_valid = (int)g;   // the first of the padding
        }
    }
    cluster_barrier();   // no CTA leaves while its neighbour may read its last pair
}

// ------------------------------------------------------------ backward ----
constexpr int kSumThreads = 128;
constexpr int kSpan = 32;                        // pairs of a chunk, at least
constexpr int kMaxChunk = DPO_EMBED_SPAN / 256;

struct SumArgs {
    const void *dy;
    void *dtable;
    const uint2 *sorted;
    const int *n_valid;
    float *partial;            // [chunk][begun here, not here][dim]
    int64_t dim, ld_dy, ld_dtable;
    int chunk, segs;
    float scale;
    int accumulate;
};

__device__ __forceinline__ uint2 ld_pair(const uint2 *p)
{
    uint2 q;
    asm volatile("ld.global.v2.b32 {%0, %1}, [%2];" : "=r"(q.x), "=r"(q.y) : "l"(p));
    return q;
}
__device__ __forceinline__ int ld_int(const int *p)
{
    int v;
    asm volatile("ld.global.b32 %0, [%1];" : "=r"(v) : "l"(p));
    return v;
}

// dtable[id, c ..] (+)= scale sum; one rounding of the product and the sum.
template <class GT, int V>
__device__ __forceinline__ void finish(const SumArgs &a, uint32_t id, int64_t c, const float (&sum)[V])
{
    GT *const p = static_cast<GT *>(a.dtable) + (int64_t)id * a.ld_dtable + c;
    float y[V];
    Vec<GT, V> o;
    o.zero();
    if (a.accumulate)
        o.load(p);
#pragma unroll
    for (int j = 0; j < V; ++j)
        y[j] = a.accumulate ? fmaf(sum[j], a.scale, o.get(j)) : sum[j] * a.scale;
    o.set(y);
    o.store(p);
}

// A CTA: a chunk of the sorted pairs and 128 N V columns, a thread N accesses of V of them. (With
// one access of one bf16 a row's bookkeeping is most of the instructions: 60000 tokens of 777 72 us, with
// four 54.)
template <class T, class GT, int V, int N, bool ADD>
__global__ void __launch_bounds__(kSumThreads) embed_sum_kernel(const SumArgs a)
{
    __shared__ uint2 pair_[kMaxChunk + 2];
    uint2 *const pair = pair_ + 1;
    pdl_wait();
    const int chunk = (int)blockIdx.x / a.segs, seg = (int)blockIdx.x - chunk * a.segs;
    const int n = ld_int(a.n_valid), i0 = chunk * a.chunk;
    const int len = min(a.chunk, n - i0);
    if (len <= 0)
        return;
    for (int i = threadIdx.x - 1; i <= len; i += kSumThreads)
        pair[i] = i0 + i < 0 || i0 + i >= n ? make_uint2(~0u, 0u) : ld_pair(a.sorted + i0 + i);
    __syncthreads();
    constexpr int kStep = kSumThreads * V;   // from one access to the next
    const int64_t c = (int64_t)seg * kStep * N + threadIdx.x * V;
    if (c >= a.dim)
        return;
    const int own = N == 1 ? 1 : (int)min((int64_t)N, (a.dim - c + kStep - 1) / kStep);   // accesses
    const T *const dy = static_cast<const T *>(a.dy) + c;
    const uint32_t begun = pair[-1].x;   // this id's run began before this chunk
    // the last of its run, which is all in this chunk: what dtable's row takes
    auto whole = [&](int i) { return pair[i + 1].x != pair[i].x && pair[i].x != begun; };
    GT *const table = static_cast<GT *>(a.dtable) + c;
    constexpr int kSumRows = N * V == 1 ? 16 : 8;   // requested at a time
    float sum[N][V] = {};
    for (int i = 0; i < len; i += kSumRows) {
        Vec<T, V> v[kSumRows][N];
        Vec<GT, V> old[ADD ? kSumRows : 1][N];
#pragma unroll
        for (int u = 0; u < kSumRows; ++u)
            if (i + u < len)
#pragma unroll
                for (int q = 0; q < N; ++q)
                    if (q < own)
                        v[u][q].load(dy + (int64_t)pair[i + u].y * a.ld_dy + q * kStep);
        if constexpr (ADD)   // with them, not one after the other at the ends of the runs
#pragma unroll
            for (int u = 0; u < kSumRows; ++u)
                if (i + u < len && whole(i + u))
#pragma unroll
                    for (int q = 0; q < N; ++q)
                        if (q < own)
                            old[u][q].load(table + (int64_t)pair[i + u].x * a.ld_dtable + q * kStep);
#pragma unroll
        for (int u = 0; u < kSumRows; ++u) {
            if (i + u >= len)
                break;
#pragma unroll
            for (int q = 0; q < N; ++q)
#pragma unroll
                for (int j = 0; j < V; ++j)
                    sum[q][j] += v[u][q].get(j);
            if (whole(i + u)) {
#pragma unroll
                for (int q = 0; q < N; ++q) {
                    float y[V];
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        y[j] = ADD ? fmaf(sum[q][j], a.scale, old[ADD ? u : 0][q].get(j)) : sum[q][j] * a.scale;
                    Vec<GT, V> o;
                    o.set(y);
                    if (q < own)
                        o.store(table + (int64_t)pair[i + u].x * a.ld_dtable + q * kStep);
                }
            } else if (i + u + 1 == len || pair[i + u + 1].x != pair[i + u].x) {
                float *const p = a.partial + ((int64_t)chunk * 2 + (pair[i + u].x == begun)) * a.dim + c;
#pragma unroll
                for (int q = 0; q < N; ++q)
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        if (q < own)
                            p[q * kStep + j] = sum[q][j];
            } else {
                continue;
            }
#pragma unroll
            for (int q = 0; q < N; ++q)
#pragma unroll
                for (int j = 0; j < V; ++j)
                    sum[q][j] = 0.0f;
        }
    }
}

// The runs that cross chunks: the CTA of the chunk where one begins adds its chunks' sums, its four
// warps every fourth of them, 32 N V columns a CTA.
constexpr int kJoinWarps = kSumThreads / 32;

template <class GT, int V, int N>
__global__ void __launch_bounds__(kSumThreads) embed_join_kernel(const SumArgs a)
{
    constexpr int kCols = 32 * N * V;
    __shared__ float sums[kJoinWarps - 1][kCols];
    pdl_wait();
    const int segs = (int)((a.dim + kCols - 1) / kCols);
    const int chunk = (int)blockIdx.x / segs, seg = (int)blockIdx.x - chunk * segs;
    const int i0 = chunk * a.chunk, i1 = i0 + a.chunk, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // all at once: the list has room for the pair after this chunk, which is not the last one
    const uint32_t id = ld_pair(a.sorted + i1 - 1).x, after = ld_pair(a.sorted + i1).x,
                   before = i0 > 0 ? ld_pair(a.sorted + i0 - 1).x : ~id;
    const int n = ld_int(a.n_valid);
    if (i1 >= n || after != id || before == id)
        return;   // ends here, or was begun before this chunk
    int last = chunk + 1;   // the chunk where it ends: the next one does not begin with it
    for (;; last += 32) {
        const int64_t next = (int64_t)(last + lane + 1) * a.chunk;
        const uint32_t key = ld_pair(a.sorted + (next < n ? next : i1)).x;
        const unsigned ends = __ballot_sync(0xFFFFFFFFu, next >= n || key != id);
        if (ends != 0u) {
            last += __ffs(ends) - 1;
            break;
        }
    }
    const int64_t c = (int64_t)seg * kCols + lane * V;
    float sum[N][V] = {};
    // the chunk's own sum, then those of runs that did not begin where they lie
#pragma unroll 4
    for (int k = chunk + warp; k <= last; k += kJoinWarps) {
        const float *const p = a.partial + ((int64_t)k * 2 + (k != chunk)) * a.dim + c;
#pragma unroll
        for (int q = 0; q < N; ++q)
            if (c + q * 32 * V < a.dim)
#pragma unroll
                for (int j = 0; j < V; ++j)
                    sum[q][j] += p[q * 32 * V + j];
    }
    if (warp > 0)
#pragma unroll
        for (int q = 0; q < N; ++q)
#pragma unroll
            for (int j = 0; j < V; ++j)
                sums[warp - 1][(q * 32 + lane) * V + j] = sum[q][j];
    __syncthreads();
    if (warp > 0)
        return;
#pragma unroll
    for (int q = 0; q < N; ++q) {
        if (c + q * 32 * V >= a.dim)
            break;
#pragma unroll
        for (int w = 0; w < kJoinWarps - 1; ++w)
#pragma unroll
            for (int j = 0; j < V; ++j)
                sum[q][j] += sums[w][(q * 32 + lane) * V + j];
        finish<GT, V>(a, id, c + q * 32 * V, sum[q]);
    }
}

// ---------------------------------------------------------------- host ----

using EmbedFn = void (*)(EmbedArgs);
using SumFn = void (*)(SumArgs);
using B16 = __nv_bfloat16;

template <class A, class B> constexpr int wide() { return sizeof(A) == 4 && sizeof(B) == 4 ? 4 : 8; }
int wide_of(int a, int b) { return a == DPO_F32 && b == DPO_F32 ? 4 : 8; }

template <class TT, class OT> EmbedFn embed_fn(int v, bool many)
{
    if (v > 2)
        return embed_kernel<TT, OT, wide<TT, OT>(), false>;
    if (v == 2)
        return many ? embed_kernel<TT, OT, 2, true> : embed_kernel<TT, OT, 2, false>;
    return many ? embed_kernel<TT, OT, 1, true> : embed_kernel<TT, OT, 1, false>;
}
EmbedFn embed_fn(int tt, int ot, int v, bool many)
{
    if (tt == DPO_F32)
        return ot == DPO_F32 ? embed_fn<float, float>(v, many) : embed_fn<float, B16>(v, many);
    return ot == DPO_F32 ? embed_fn<B16, float>(v, many) : embed_fn<B16, B16>(v, many);
}
// The accesses of a thread: several of few elements, where that leaves each SM so many CTAs.
int accesses(int v, int64_t chunks, int64_t dim, int threads, int64_t ctas)
{
    const int n = v == 1 ? 4 : v == 2 ? 2 : 1;
    const int64_t cols = (int64_t)n * threads * v;
    return chunks * ((dim + cols - 1) / cols) >= ctas ? n : 1;
}
template <class T, class GT, bool ADD> SumFn sum_fn(int v, int n)
{
    if (v > 2)
        return embed_sum_kernel<T, GT, wide<T, GT>(), 1, ADD>;
    if (v == 2)
        return n > 1 ? embed_sum_kernel<T, GT, 2, 2, ADD> : embed_sum_kernel<T, GT, 2, 1, ADD>;
    return n > 1 ? embed_sum_kernel<T, GT, 1, 4, ADD> : embed_sum_kernel<T, GT, 1, 1, ADD>;
}
template <class T, class GT> SumFn sum_fn(int v, int n, bool add)
{
    return add ? sum_fn<T, GT, true>(v, n) : sum_fn<T, GT, false>(v, n);
}
SumFn sum_fn(int t, int gt, int v, int n, bool add)
{
    if (t == DPO_F32)
        return gt == DPO_F32 ? sum_fn<float, float>(v, n, add) : sum_fn<float, B16>(v, n, add);
    return gt == DPO_F32 ? sum_fn<B16, float>(v, n, add) : sum_fn<B16, B16>(v, n, add);
}
template <class GT, int W> SumFn join_fn(int v, int n)
{
    if (v > 2)
        return embed_join_kernel<GT, W, 1>;
    if (v == 2)
        return n > 1 ? embed_join_kernel<GT, 2, 2> : embed_join_kernel<GT, 2, 1>;
    return n > 1 ? embed_join_kernel<GT, 1, 4> : embed_join_kernel<GT, 1, 1>;
}
SumFn join_fn(int t, int gt, int v, int n)
{
    if (gt == DPO_F32)
        return t == DPO_F32 ? join_fn<float, 4>(v, n) : join_fn<float, 8>(v, n);
    return join_fn<B16, 8>(v, n);
}

int check_table(const char *what, int64_t vocab, int64_t dim, float scale)
{
    if (vocab < 1 || dim < 1 || vocab >= kMaxCount - 1 || dim >= kMaxCount)
        return call_fail(DPO_EINVAL, "%s: vocab %lld, dim %lld", what, (long long)vocab, (long long)dim);
    if (!isfinite(scale))
        return call_fail(DPO_EINVAL, "%s: scale", what);
    return DPO_OK;
}

// The workspace of a span, and how its sorted pairs are cut.
struct Plan {
    int chunk, chunks;
    int64_t sorted, partial, bytes;   // where each begins; n_valid is at 0
};
Plan plan_of(int64_t tokens, int64_t dim)
{
    auto up = [](int64_t v) { return (v + 255) / 256 * 256; };
    const int64_t n = tokens < DPO_EMBED_SPAN ? tokens : DPO_EMBED_SPAN;
    Plan p;
    p.chunk = kSpan;
    // at most 256 chunks of wide rows, more of those that few CTAs share
    const int64_t segs = (dim + 8 * kSumThreads - 1) / (8 * kSumThreads), most = 1024 / segs;
    while ((int64_t)p.chunk * (most > 256 ? most : 256) < n)
        p.chunk *= 2;
    p.chunks = (int)((n + p.chunk - 1) / p.chunk);
    p.sorted = 256;
    p.partial = p.sorted + up(n * 8);
    p.bytes = p.partial + (p.chunks > 1 ? up((int64_t)p.chunks * 2 * dim * 4) : 0);
    return p;
}

}  // namespace
}  // namespace dpo

using namespace dpo;

extern "C" int dpo_embed(const dpo_embed_args *args, void *cuda_stream)
{
    const char *what = "dpo_embed";
    if (args == nullptr)
        return call_fail(DPO_EINVAL, "%s: no arguments", what);
    const dpo_embed_args &a = *args;
    if (!known(a.table_dtype) || !known(a.out_dtype))
        return call_fail(DPO_EDTYPE, "%s: table dtype %d, out dtype %d", what, a.table_dtype, a.out_dtype);
    EmbedArgs k{};
    int64_t tokens = 0;
    int rc = check_table(what, a.vocab, a.dim, a.scale);
    if (rc != DPO_OK || (rc = check_ids(what, a.ids, &k.ids, &tokens)) != DPO_OK || tokens == 0)
        return rc;
    const int64_t ts = elem_size(a.table_dtype), os = elem_size(a.out_dtype);
    Buffers b(what);
    add_ids(b, a.ids);
    b.add("table", a.table, a.vocab, a.dim, a.ld_table, ts, ts, false);
    b.add("out", a.out, tokens, a.dim, a.ld_out, os, os, true);
    if ((rc = b.done()) != DPO_OK)
        return rc;
    Width w(wide_of(a.table_dtype, a.out_dtype));
    w.fit(a.table, a.dim, a.ld_table, ts);
    w.fit(a.out, a.dim, a.ld_out, os);
    k.table = a.table;
    k.out = a.out;
    k.vocab = a.vocab;
    k.dim = a.dim;
    k.ld_table = a.ld_table;
    k.ld_out = a.ld_out;
    k.scale = a.scale;
    const bool many = a.dim > 32 * 4 * w.v;
    const int64_t seg = 32 * pieces(w.v, many) * w.v;
    k.units = units_of(tokens, (a.dim + seg - 1) / seg);
    const int64_t grid = (k.units.all + kEmbedWarps - 1) / kEmbedWarps;
    if (grid >= kMaxCount)
        return call_fail(DPO_EINVAL, "%s: %lld tokens of %lld are too many", what, (long long)tokens,
                         (long long)a.dim);
    return launch(what, embed_fn(a.table_dtype, a.out_dtype, w.v, many), grid, 32 * kEmbedWarps, 0, cuda_stream, k);
}

extern "C" int dpo_embed_workspace(int64_t tokens, int64_t vocab, int64_t dim, int64_t *bytes)
{
    const char *what = "dpo_embed_workspace";
    const int rc = check_table(what, vocab, dim, 1.0f);
    if (rc != DPO_OK)
        return rc;
    if (bytes == nullptr || tokens < 0 || tokens >= kMaxCount)
        return call_fail(DPO_EINVAL, "%s: %lld tokens", what, (long long)tokens);
    *bytes = plan_of(tokens, dim).bytes;
    return DPO_OK;
}

extern "C" int dpo_embed_backward(const dpo_embed_backward_args *args, void *cuda_stream)
{
    const char *what = "dpo_embed_backward";
    if (args == nullptr)
        return call_fail(DPO_EINVAL, "%s: no arguments", what);
    const dpo_embed_backward_args &a = *args;
    if (!known(a.dtype) || !known(a.grad_dtype))
        return call_fail(DPO_EDTYPE, "%s: dtype %d, grad dtype %d", what, a.dtype, a.grad_dtype);
    SortArgs so{};
    int64_t tokens = 0;
    int rc = check_table(what, a.vocab, a.dim, a.scale);
    if (rc != DPO_OK || (rc = check_ids(what, a.ids, &so.ids, &tokens)) != DPO_OK)
        return rc;
    const int64_t size = elem_size(a.dtype), gsize = elem_size(a.grad_dtype);
    const Plan plan = plan_of(tokens, a.dim);
    Buffers b(what);
    b.add("dtable", a.dtable, a.vocab, a.dim, a.ld_dtable, gsize, gsize, true);
    if (tokens == 0) {
        if ((rc = b.done()) != DPO_OK || a.accumulate)
            return rc;
        const cudaError_t e =
            cudaMemset2DAsync(a.dtable, (size_t)(a.ld_dtable * gsize), 0, (size_t)(a.dim * gsize),
                              (size_t)a.vocab, static_cast<cudaStream_t>(cuda_stream));
        return e == cudaSuccess ? DPO_OK : call_fail(DPO_ECUDA, "%s: %s", what, cudaGetErrorString(e));
    }
    if (a.workspace != nullptr && a.workspace_bytes < plan.bytes)
        return call_fail(DPO_EINVAL, "%s: workspace of %lld bytes, %lld needed", what,
                         (long long)a.workspace_bytes, (long long)plan.bytes);
    add_ids(b, a.ids);
    b.add("dy", a.dy, tokens, a.dim, a.ld_dy, size, size, false);
    b.add("workspace", a.workspace, 1, plan.bytes, plan.bytes, 1, 256, true);
    if ((rc = b.done()) != DPO_OK)
        return rc;
    Width w(wide_of(a.dtype, a.grad_dtype));
    w.fit(a.dy, a.dim, a.ld_dy, size);
    w.fit(a.dtable, a.dim, a.ld_dtable, gsize);

    uint8_t *const ws = static_cast<uint8_t *>(a.workspace);
    SumArgs su{};
    su.dtable = a.dtable;
    su.n_valid = so.n_valid = reinterpret_cast<int *>(ws);
    su.sorted = so.sorted = reinterpret_cast<uint2 *>(ws + plan.sorted);
    su.partial = reinterpret_cast<float *>(ws + plan.partial);
    so.vocab = a.vocab;
    su.dim = a.dim;
    su.ld_dy = a.ld_dy;
    su.ld_dtable = a.ld_dtable;
    su.scale = a.scale;
    su.chunk = plan.chunk;
    const int sms = sm_count();
    if (sms == 0)
        return call_fail(DPO_ECUDA, "%s: no device", what);
    const int each = accesses(w.v, plan.chunks, a.dim, kSumThreads, (int64_t)8 * sms);
    const int join_each = accesses(w.v, plan.chunks, a.dim, 32, (int64_t)16 * sms);
    const int64_t seg = (int64_t)kSumThreads * w.v * each;
    su.segs = (int)((a.dim + seg - 1) / seg);
    int bits = 1;   // of the ids and of the padding's key
    while ((a.vocab >> bits) != 0)
        ++bits;
    so.passes = (bits + kDigitBits - 1) / kDigitBits;
    so.bits = (bits + so.passes - 1) / so.passes;
    const int64_t joins = (a.dim + 32 * join_each * w.v - 1) / (32 * join_each * w.v);
    if ((int64_t)plan.chunks * joins >= kMaxCount)
        return call_fail(DPO_EINVAL, "%s: %lld columns are too many", what, (long long)a.dim);
    const void *const sort = reinterpret_cast<const void *>(sort_ids_kernel);
    cudaError_t e = cudaFuncSetAttribute(sort, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         sort_smem(kSortThreads, kDigitBits));
    if (e == cudaSuccess)
        e = cudaFuncSetAttribute(sort, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return call_fail(DPO_ECUDA, "%s: %s", what, cudaGetErrorString(e));
    }
    for (int64_t first = 0; first < tokens; first += DPO_EMBED_SPAN) {
        so.first = first;
        so.count = tokens - first < DPO_EMBED_SPAN ? tokens - first : DPO_EMBED_SPAN;
        int64_t clears = 0;
        so.clear = {};
        if (!a.accumulate && first == 0) {
            const bool whole = a.ld_dtable == a.dim;
            so.clear = {static_cast<uint8_t *>(a.dtable), whole ? 1 : a.vocab,
                        (whole ? a.vocab : 1) * a.dim * gsize, a.ld_dtable * gsize, (int)gsize};
            clears = (so.clear.rows * ((so.clear.bytes + kClearBytes - 1) / kClearBytes) + 31) / 32;
            clears = clears < (int64_t)sms * 4 ? clears : (int64_t)sms * 4;
        }
        if (so.count <= kRankTokens && a.vocab < kRankVocab) {
            so.ctas = (int)((so.count + kRankWarps * kRankKeys - 1) / (kRankWarps * kRankKeys));
            rc = launch(what, rank_ids_kernel, so.ctas + clears, 32 * kRankWarps, 0, cuda_stream, so);
        } else {   // small CTAs first: the ranking's votes and the counts' sums on as many SMs
            int threads = kSortMinThreads, ctas = 1;
            while (ctas < kSortCtas && (int64_t)ctas * threads * kSortItems < so.count)
                ctas *= 2;
            while ((int64_t)ctas * threads * kSortItems < so.count)
                threads *= 2;
            so.ctas = ctas;
            rc = launch_in_clusters(what, sort_ids_kernel, ctas + (clears + ctas - 1) / ctas * ctas, ctas,
                                    threads, (size_t)sort_smem(threads, so.bits), cuda_stream, so);
        }
        if (rc != DPO_OK)
            return rc;
        su.dy = static_cast<const uint8_t *>(a.dy) + first * a.ld_dy * size;
        su.accumulate = a.accumulate || first > 0;
        const int chunks = (int)((so.count + su.chunk - 1) / su.chunk);
        rc = launch(what, sum_fn(a.dtype, a.grad_dtype, w.v, each, su.accumulate), (int64_t)chunks * su.segs, kSumThreads, 0,
                    cuda_stream, su);
        if (rc == DPO_OK && chunks > 1)
            rc = launch(what, join_fn(a.dtype, a.grad_dtype, w.v, join_each), (chunks - 1) * joins, kSumThreads, 0,
                        cuda_stream, su);
        if (rc != DPO_OK)
            return rc;
    }
    return DPO_OK;
}
