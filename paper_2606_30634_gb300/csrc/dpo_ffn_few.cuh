// dpo_ffn_few.cuh -- the feed-forward block's forward products for few tokens.
//
//   C[t, r] = sum_k X[t, k] W[r, k]        (W row-major, K contiguous; fp32 sums)
//
// Every weight is read once and used for a handful of multiplications, so the time is
// the weights' way from HBM and what matters is that all SMs pull on it at once. The
// tiles of dpo_ffn_gemm.cuh are too coarse for that: a 7B layer's down projection has 32
// tiles of 128 columns for 152 SMs. Here 16 weight rows are the M side of
// mma.sync.m16n8k16 and the tokens its N side; a CTA's eight warps, and
// the CTAs of a cluster, split K among them and add their sums up in a fixed order, the
// warps through shared memory, the CTAs through the cluster's.
// The weights go from global memory straight to the fragments' registers: the order of
// k inside an MMA is free as long as both operands agree, so a lane takes 16 bytes of a
// row at once (8 consecutive k, the four lanes of a row 32 of them), which is two MMAs'
// worth, and the tokens' fragments come the same way, from L1.
// GB300, whole forward, this against the split tiles: 7B widths, 1 token 48.5 / 59.5 us,
// 8 tokens 52.5 / 59.6 (floor 39.9); 1B 20.5 / 27.5, 22.5 / 27.5 (14.8); 768 x 2048 8.2 / 11.0.
#pragma once

#include "dpo_ffn_gemm.cuh"

namespace dpo {
namespace ffn {

constexpr int kFewThreads = 256, kFewWarps = kFewThreads / 32;
constexpr int kFewTokens = 8;      // at most: N of the MMA
constexpr int kFewRows = 16;       // weight rows of a unit
constexpr int kFewChunk = 4;       // blocks of 32 k a warp takes at a time
constexpr int kFewCtas = 4;        // resident on an SM

// The start of the second product's weight rows, read into L2 by the first one's last CTAs
// once their own loads are done, so that HBM is not idle from there until the second
// product's CTAs, most of which wait for places, have theirs under way.
struct Ahead {
    const uint8_t *base;
    int64_t pitch;
    int rows, bytes;               // of each; a multiple of 16, as are base and pitch
    int ctas;                      // that share the rows
};

struct FewArgs {
    const __nv_bfloat16 *x;        // tokens x k
    const __nv_bfloat16 *w0, *w1;  // rows x k; kGate: w_gate, w_up
    __nv_bfloat16 *out;            // tokens x rows
    __nv_bfloat16 *keep0, *keep1;  // kGate with kKeep16: G, U
    int64_t ld_x, ld_out;
    int tokens, rows, k;           // kGate: rows of one projection
    int act;
    Ahead ahead;                   // kGate
};

__device__ __forceinline__ uint4 ld_weights(const __nv_bfloat16 *p)
{
    uint4 q;
    asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w)
                 : "l"(p));
    return q;
}

__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                          uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
        "{%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ float ld_cluster(uint32_t addr)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}

// A unit is 16 weight rows: kGate: the first eight are
// w_gate's and the others the same rows of w_up, so one lane holds G and U of one
// element; kStore: sixteen rows of w0. One unit per CTA, or per cluster: walking several
// from CTAs that stay, the next one's weights requested before the sums of the last,
// takes longer (7B layer, one token: 9.7 us, with 80 registers instead of 64).
template <int EPI>
__global__ void __launch_bounds__(kFewThreads) few_kernel(const FewArgs a)
{
    constexpr int U = kFewChunk, kTok = kFewTokens, kSums = kFewRows * kTok;
    constexpr int kOut = EPI == kGate ? 8 : 16;    // output columns of a unit
    __shared__ float sums[kFewWarps * kSums];      // [warp][row][token], then [row][token]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    uint32_t rank, ranks;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
    const int col0 = (int)(blockIdx.x / ranks) * kOut;
    if (EPI == kGate) {
        pdl_wait();
        // The second product's CTAs may take the places that this one's leave: they start
        // once all of these are here, behind all earlier work of the stream.
        launch_dependents();
    }

    // this lane's rows g and g + 8 and its token; past the end they read the last ones
    const __nv_bfloat16 *w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
        w[h] = (EPI == kGate && h ? a.w1 : a.w0) +
               (int64_t)min(col0 + (EPI == kGate ? 0 : h * 8) + g, a.rows - 1) * a.k;
    const __nv_bfloat16 *const x = a.x + (int64_t)min(g, a.tokens - 1) * a.ld_x;
    float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};

    // chunks of U blocks of 32 k, dealt to the cluster's warps in turn; k is a multiple
    // of 8, so a lane's 8 are all there or none
    const int step = (int)ranks * kFewWarps * U * 32;
    int k0 = ((int)rank * kFewWarps + warp) * U * 32 + t * 8;
    uint4 wq[2][U];
    auto load_w = [&](int k) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                wq[h][u] = make_uint4(0u, 0u, 0u, 0u);
                if (k + u * 32 < a.k)
                    wq[h][u] = ld_weights(w[h] + k + u * 32);
            }
    };
    load_w(k0);
    // The second product follows the first one in the same call, which has waited for all
    // that came before it and writes no weights: its first weights are read ahead.
    if (EPI != kGate)
        pdl_wait();
    for (; k0 - t * 8 < a.k; k0 += step) {
        uint4 cur[2][U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            cur[0][u] = wq[0][u];
            cur[1][u] = wq[1][u];
        }
        load_w(k0 + step);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = k0 + u * 32;
            uint4 xq = make_uint4(0u, 0u, 0u, 0u);
            if (k < a.k)
                xq = gemm::load_c(x + k);
            const uint4 p = cur[0][u], q = cur[1][u];
            mma_16816(acc, p.x, q.x, p.y, q.y, xq.x, xq.y);
            mma_16816(acc, p.z, q.z, p.w, q.w, xq.z, xq.w);
        }
    }

    if (EPI == kGate && threadIdx.x == 0) {
        const int first = (int)gridDim.x - a.ahead.ctas;
        for (int r = (int)blockIdx.x - first; r >= 0 && r < a.ahead.rows; r += a.ahead.ctas)
            asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;"
                         ::"l"(a.ahead.base + r * a.ahead.pitch), "r"(a.ahead.bytes) : "memory");
    }

    float *s = sums + warp * kSums + g * kTok + t * 2;
    *reinterpret_cast<float2 *>(s) = make_float2(acc[0], acc[1]);
    *reinterpret_cast<float2 *>(s + 8 * kTok) = make_float2(acc[2], acc[3]);
    __syncthreads();
    for (int i = threadIdx.x; i < kSums; i += kFewThreads) {
        float v = sums[i];
#pragma unroll
        for (int q = 1; q < kFewWarps; ++q)
            v += sums[q * kSums + i];
        sums[i] = v;   // only this thread reads element i of warp 0's block
    }
    if (ranks > 1)
        gemm::group_sync<2>();   // the cluster's barrier: every CTA's sums are written
    else
        __syncthreads();
    if (rank == 0) {
        const uint32_t here = (uint32_t)__cvta_generic_to_shared(sums);
        auto total = [&](int i) {
            float v = sums[i];
            for (uint32_t q = 1; q < ranks; ++q)
                v += ld_cluster(map_to_rank(here + 4u * (uint32_t)i, q));
            return v;
        };
        for (int i = threadIdx.x; i < kOut * a.tokens; i += kFewThreads) {
            const int tok = i / kOut, r = i - tok * kOut, col = col0 + r;
            if (col >= a.rows)
                continue;
            if (EPI == kGate) {
                const float gv = total(r * kTok + tok), uv = total((r + 8) * kTok + tok);
                if (a.keep0 != nullptr) {
                    a.keep0[(int64_t)tok * a.rows + col] = __float2bfloat16_rn(gv);
                    a.keep1[(int64_t)tok * a.rows + col] = __float2bfloat16_rn(uv);
                }
                float dq;
                const float s = a.act == kGelu ? logistic<kGelu>(gv, dq) : logistic<kSilu>(gv, dq);
                a.out[tok * a.ld_out + col] = __float2bfloat16_rn(uv * (gv * s));
            } else {
                a.out[tok * a.ld_out + col] = __float2bfloat16_rn(total(r * kTok + tok));
            }
        }
    }
    if (ranks > 1)
        gemm::group_sync<2>();   // no CTA leaves while rank 0 may read its sums
}

}  // namespace ffn
}  // namespace dpo
