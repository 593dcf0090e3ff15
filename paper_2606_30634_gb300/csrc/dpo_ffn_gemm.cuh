// dpo_ffn_gemm.cuh -- the products of the gated feed-forward block on the
// sm_103a tensor cores (tcgen05, TMA, TMEM), with the block's element-wise work
// in their epilogues.
//
//   D = sum over segments s of A_s B_s      (M x N, fp32 accumulation)
//
// Operands are bf16 and taken as they lie in memory: A_s is M x K row-major
// (K contiguous) or K x M row-major (M contiguous), B_s is N x K or K x N
// likewise, so no transposed copy of a weight, an activation or a gradient is
// ever made. A product has one or two segments of K (dx = dG w_gate + dU w_up).
// Boxes past the edge of a matrix read as zeros and stores past it are
// clipped by TMA, so no size needs padding.
//
// Roles, rings and barriers are those of the Newton-Schulz GEMM (dpo_gemm.cuh,
// whose primitives this kernel uses): a persistent grid of CTA pairs on 256 x 256
// tiles with the 2-SM MMA (CG = 2), or of single CTAs on 128 x 128 tiles (CG = 1)
// where there are few; warp 0 loads, warp 1 issues the MMAs, eight warps drain
// one accumulator while the MMAs fill the other. Every wait is bounded.
// A product of few tiles has them split along K (SPLIT): the CTAs of a cluster take
// a share of one tile's K blocks each and exchange their fp32 sums through the
// cluster's shared memory, each finishing its share of the rows.
//
// Epilogues:
//   kGate      the tile's columns are T / 2 of G beside the same T / 2 of U (the B
//              operand is half w_gate rows, half w_up rows), so act(G) U is formed
//              where both are in registers; writes A and what is kept of G and U
//   kGateBack8, kGateBack16  the tile is of dA; reads what was kept of G and U (8 bits, or
//              bf16), writes dG, dU and A
//   kStore     writes D in bf16 or fp32, with factors along the columns and the old
//              contents added where asked for
#pragma once

#include "dpo_gemm.cuh"
#include "dpo_pack8.cuh"

namespace dpo {
namespace ffn {

using gemm::BH;
using gemm::BM;
using gemm::group_sync;
using gemm::kBoxK;
using gemm::kChunkBytes;
using gemm::kErrDrain;
using gemm::kErrWaitDone;
using gemm::kErrWaitEmpty;
using gemm::kErrWaitFull;
using gemm::kTile;
using gemm::map_to_rank;
using gemm::mbar_arrive;
using gemm::mbar_arrive_expect_tx;
using gemm::mbar_init;
using gemm::mbar_wait;
using gemm::mma_bf16;
using gemm::mma_commit;
using gemm::smem_desc;
using gemm::swz64;
using gemm::tmem_ld32;

enum Epilogue { kGate = 0, kGateBack8 = 1, kGateBack16 = 2, kStore = 3 };
__host__ __device__ constexpr bool gate_back(int epi)
{
    return epi == kGateBack8 || epi == kGateBack16;
}
enum Keep { kKeepNone = 0, kKeep8 = 1, kKeep16 = 2 };
enum Act { kSilu = 0, kGelu = 1 };

constexpr int kEpiWarps = 8;
constexpr int kThreads = 64 + 32 * kEpiWarps;
// The ring of operand stages and the epilogue warps' staging behind it. Three stages of
// 128 of K (six of 64 are slower, see dpo_gemm.cuh). Where K is split, a CTA has few blocks
// and waits for the first ones to arrive, so the bytes in flight count: stages of 64 of K,
// which leave room for more of them, and of A only the 32, 64 or 128 rows that a product of
// so few tokens has (so too single CTAs without a split: boxes of 128 rows for 17 to 24
// tokens of a 1B layer 38 us, of 32 rows 31). The MMA reads 128 rows all the same; what lies
// behind a short box ends up in accumulator rows that nothing reads.
constexpr int kRowBytes = kBoxK * 2;                          // of a box: the swizzle span
constexpr int kMaxStages = 16;
constexpr int kMaxSmem = 232448 - 1024;   // of a CTA, beside its static variables
template <bool SPLIT> struct Ring {
    static constexpr int BK = SPLIT ? 64 : 128;
    static constexpr int box = BM * kRowBytes;                // of one box of 128 rows
    static constexpr int mn_box = BK * kRowBytes;             // of a box of 64 columns, BK of K
    static constexpr int staging = SPLIT ? 8192 : 2 * kChunkBytes;   // per epilogue warp
    // of a stage: `rows` of A, `cols` of B
    static __host__ __device__ constexpr int bytes(int n) { return n * BK * 2; }
    // epilogue warps of tiles with so many rows
    static __host__ __device__ constexpr int warps(int rows) { return kEpiWarps * rows / BM; }
    static __host__ __device__ constexpr int stages(int rows, int cols)
    {
        const int fit = (kMaxSmem - 1024 - warps(rows) * staging) / (bytes(rows) + bytes(cols));
        return fit < kMaxStages ? fit : kMaxStages;
    }
    static __host__ __device__ constexpr int smem(int rows, int cols)
    {
        return stages(rows, cols) * (bytes(rows) + bytes(cols)) + 1024 + warps(rows) * staging;
    }
};
static_assert(Ring<false>::stages(BM, BH) == 3, "stages");

constexpr int kMaxProducts = 4;
constexpr int kBandRows = 16;   // block rows per band, as in dpo_gemm.cuh

// One product of a launch.
struct Product {
    CUtensorMap a[2], b[2];       // operands per segment (kGate: b[0] w_gate, b[1] w_up)
    CUtensorMap d0, d1, d2;       // stores: kGate A, G, U; kGateBack dG, dU, A; kStore D
    int m, n;                     // kGate: n is one projection's columns
    int k_blocks[2];              // K blocks of each segment (second 0: one segment)
    int a_mn, b_mn;               // the operand is M- or N-contiguous
    int m_tiles, n_tiles, first;  // tiles, and the launch's number of the first
    // kStore
    int f32, accumulate;
    const void *old;              // accumulate: D itself
    int64_t ld_old;
    const void *gain;             // N factors, or nullptr
    int gain_f32;
    // kGate, kGateBack
    uint8_t *scale_g, *scale_u;   // kKeep8
    int64_t ld_scale;
    const void *kept_g, *kept_u;  // kGateBack: codes or bf16
    int64_t ld_kept;
    int keep, act;                // Keep, Act
    int wide;                     // kGate: scale rows 2-byte aligned; kGateBack: kept values
                                  // in whole, 32-byte aligned chunks
    // split K: the same outputs as pointers (kStore: bf16, nothing added)
    __nv_bfloat16 *o0, *o1, *o2;
    int64_t ld_o;
    uint8_t *codes_g, *codes_u;
    int64_t ld_codes_g, ld_codes_u;
};

struct Launch {
    Product p[kMaxProducts];
    int n_products, n_tiles;
    int a_rows;                   // rows of A that a stage loads, BM where A is M-contiguous
    int cols;                     // single CTAs: the tile's columns, kTile(1), or half of them
                                  // where K is split
    int early;                    // another launch of this kernel follows in the same call
    unsigned int *err;
};

// A value that every lane of the warp has, known to be so by the compiler: what the copies
// and MMAs take from uniform registers then comes without a move to them each time.
__device__ __forceinline__ int uniform(int v) { return __shfl_sync(0xFFFFFFFFu, v, 0); }

// True in one lane of the (whole) warp.
__device__ __forceinline__ bool elect()
{
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0u;
}

// By the whole warp: false when the wait gave up in any lane, or another role did (*aborted,
// set here too); looked at only where the phase is not there yet.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int *aborted)
{
    if (__all_sync(0xFFFFFFFFu, gemm::mbar_try(bar, parity)))
        return true;
    const unsigned long long t0 = gemm::globaltimer();
    for (;;) {
        const bool there = gemm::mbar_try(bar, parity);
        if (__all_sync(0xFFFFFFFFu, there))
            return true;
        if (__any_sync(0xFFFFFFFFu, *aborted || gemm::globaltimer() - t0 > gemm::kWaitNs)) {
            *aborted = 1;
            return false;
        }
    }
}

// Between the launches of one feed-forward call: the kernels here, the streaming one and the
// widening of 8-bit rows (dpo_call.h) let their successor start early. What dpo_device.cuh says of
// "no kernel" is of the optimizers', whose figures it gives.
__device__ __forceinline__ void launch_dependents()
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// 2-D TMA load and store (see the 3-D ones in dpo_gemm.cuh).
template <int CG>
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap *map, int x, int y,
                                         uint32_t bar)
{
    if (CG == 2)
        asm volatile(
            "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes"
            " [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
            "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes"
            " [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
            "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar)
            : "memory");
}

__device__ __forceinline__ void tma_store(const CUtensorMap *map, uint32_t src, int x, int y)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(
                     reinterpret_cast<uint64_t>(map)),
                 "r"(src), "r"(x), "r"(y)
                 : "memory");
}

// kind::f16 with fp32 accumulation and bf16 operands, M = kTile(cg), operands
// K-major, or MN-major with bits 15 (A) and 16 (B).
__device__ __forceinline__ uint32_t idesc_of(int cg, int n, int a_mn, int b_mn)
{
    return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) |
           ((uint32_t)(kTile(cg) >> 4) << 24) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16);
}

// The descriptors of an operand stage's steps of 16 of K: 32 bytes apart in a K-major box
// of 64, 16 rows apart where the operand is M- or N-contiguous. The address is the low
// word's, in 16 bytes, so a step is one addition.
struct Steps {
    uint32_t lo, hi, step, four;
    __device__ __forceinline__ Steps stage(int bytes) const
    {
        return {lo + ((uint32_t)bytes >> 4), hi, step, four};
    }
    __device__ __forceinline__ uint64_t at(int k) const
    {
        return (uint64_t)hi << 32 | (lo + (uint32_t)(k % 4) * step + (uint32_t)(k / 4) * four);
    }
};
template <int BK> __device__ __forceinline__ Steps steps_of(uint32_t addr, bool mn)
{
    // M- or N-contiguous: smem_desc_mn of dpo_gemm.cuh but for the distance between boxes of
    // 64 columns (there 8 KiB, here BK rows): bits 16 to 29, in 16 bytes
    const uint64_t d = mn ? gemm::smem_desc_mn(addr) ^
                                ((uint64_t)((8192 >> 4) ^ (BK * kRowBytes >> 4)) << 16)
                          : smem_desc(addr);
    const uint32_t step = mn ? 16 * kRowBytes : 32, four = mn ? 64 * kRowBytes : BM * kRowBytes;
    return {(uint32_t)d, (uint32_t)(d >> 32), step >> 4, four >> 4};
}

// K blocks of shares 0 .. share of `split` (share -1: none); with split <= all, none is
// empty.
__device__ __forceinline__ int share_end(int all, uint32_t share, uint32_t split)
{
    return (int)((uint32_t)all * (share + 1u) / split);
}

// Product and position of tile t: bands of kBandRows block rows, column by column.
struct Tile {
    int p, m, n;   // product, block row, block column
};
__device__ __forceinline__ Tile tile_at(const Launch &L, int t)
{
    int p = 0;
    while (p + 1 < L.n_products && t >= L.p[p + 1].first)
        ++p;
    const Product &P = L.p[p];
    const int i = t - P.first, band = kBandRows * P.n_tiles;
    const int b = i / band, r = i - b * band;
    const int rows = min(kBandRows, P.m_tiles - b * kBandRows);
    const int n = r / rows;
    return {p, b * kBandRows + r - n * rows, n};
}

// Tile of round r: back and forth, so that whoever has one of a list's first tiles, the
// longest, is the last one to get another (1001 tokens of 520 x 1560 widths, the gradients'
// launch: 40 CTAs had a tile of dx, 25 K blocks, and one of 8).
__device__ __forceinline__ int turn_of(int r, int pair, int n)
{
    return r * n + (r & 1 ? n - 1 - pair : pair);
}

// 2^x and 1 / x by the hardware's approximations (relative errors of about 2^-22 and 2^-23),
// without the steps that keep subnormal results: 1 + 2^x does not see them, and its
// reciprocal, of a number from 1 to infinity, is 0 where it would be one. The epilogues are
// bound by their instructions: with __expf and __fdividef 36 a value for the gate.
__device__ __forceinline__ float exp2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// act(z) = z s(q(z)) with s the logistic function: SiLU with q = z, GELU's tanh form
// with q = 2 sqrt(2/pi) (z + 0.044715 z^3), since (1 + tanh(q / 2)) / 2 = s(q).
// act' = s + z q' s (1 - s), taken as ((1 - s) q') (z s) + s: past |z| = 10^19 q' would be
// infinite, where 1 - s or z s is 0, so dq ends at the largest finite number.
template <int ACT>
__device__ __forceinline__ float logistic(float z, float &dq)
{
    float q = z;
    dq = 1.0f;
    if (ACT == kGelu) {
        const float c = 1.5957691216057308f, k = 0.044715f * c, z2 = z * z;
        q = z * fmaf(k, z2, c);
        dq = fminf(fmaf(3.0f * k, z2, c), kMaxFinite);
    }
    return rcp(1.0f + exp2(-1.4426950408889634f * q));
}

// Scale byte of 32 values that one lane holds; infinities become NaN (rare:
// looked for only where the maximum, which passes over NaN, found one).
__device__ __forceinline__ uint32_t row_scale(float (&v)[32])
{
    float a = 0.0f;
#pragma unroll
    for (int j = 0; j < 32; ++j)
        a = fmaxf(a, fabsf(v[j]));
    if (a > kMaxFinite) {
        a = 0.0f;
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            a = fmaxf(a, finite_abs(v[j]));
            v[j] = inf_to_nan(v[j]);
        }
    }
    return scale_byte(a);
}

// What one epilogue warp stages and stores: 32 x 32 chunks through two buffers in
// turn. Each chunk is a bulk async-group of its own, so a buffer is free once all
// groups but the last one have been read.
struct Stager {
    uint32_t buf;
    int lane, turn;
    __device__ __forceinline__ uint32_t begin()
    {
        if (lane == 0) {
            if (turn == 0)   // the chunk before may have been fp32, in both buffers
                asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            else
                asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
        }
        __syncwarp();
        const uint32_t b = buf + (uint32_t)((turn & 1) * kChunkBytes);
        ++turn;
        return b;
    }
    __device__ __forceinline__ void end(const CUtensorMap *map, uint32_t b, int x, int y)
    {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
            tma_store(map, b, x, y);
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
    }
    __device__ __forceinline__ void bf16(const CUtensorMap *map, const float (&v)[32], int x, int y)
    {
        uint32_t w[16];
#pragma unroll
        for (int i = 0; i < 16; ++i)
            w[i] = gemm::pack_bf16(v[2 * i], v[2 * i + 1]);
        bf16(map, w, x, y);
    }
    __device__ __forceinline__ void bf16(const CUtensorMap *map, const uint32_t (&w)[16], int x,
                                         int y)
    {
        const uint32_t b = begin();
#pragma unroll
        for (int g = 0; g < 4; ++g)
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(b + swz64(lane, g)),
                         "r"(w[4 * g]), "r"(w[4 * g + 1]), "r"(w[4 * g + 2]), "r"(w[4 * g + 3])
                         : "memory");
        end(map, b, x, y);
    }
    // one 4 KiB chunk in the 128-byte swizzle (granule index XOR row mod 8), in both
    // buffers
    __device__ __forceinline__ void f32(const CUtensorMap *map, const float (&v)[32], int x, int y)
    {
        if (lane == 0)
            asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        __syncwarp();
#pragma unroll
        for (int g = 0; g < 8; ++g)
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(
                             buf + (uint32_t)(lane * 128 + ((g ^ (lane & 7)) << 4))),
                         "r"(__float_as_uint(v[g * 4])), "r"(__float_as_uint(v[g * 4 + 1])),
                         "r"(__float_as_uint(v[g * 4 + 2])), "r"(__float_as_uint(v[g * 4 + 3]))
                         : "memory");
        end(map, buf, x, y);
        turn = 0;
    }
    // 32 rows of 32 codes; returns this row's scale byte. v is taken over.
    __device__ __forceinline__ uint32_t codes(const CUtensorMap *map, float (&v)[32], int x, int y)
    {
        const uint32_t s = row_scale(v);
        const float inv = inv_scale_of(s);
        const uint32_t b = begin();
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int i = g * 16 + 4 * j;
                w[j] = encode4(v[i] * inv, v[i + 1] * inv, v[i + 2] * inv, v[i + 3] * inv);
            }
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(
                             b + (uint32_t)(lane * 32 + g * 16)),
                         "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3])
                         : "memory");
        }
        end(map, b, x, y);
        return s;
    }
};

__device__ __forceinline__ void load_acc(uint32_t acc, float (&v)[32])
{
    uint32_t r[32];
    tmem_ld32(acc, r);
#pragma unroll
    for (int j = 0; j < 32; ++j)
        v[j] = __uint_as_float(r[j]);
}

// u := act(g) u
template <int ACT> __device__ __forceinline__ void gate(const float (&g)[32], float (&u)[32])
{
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        float dq;
        u[j] *= g[j] * logistic<ACT>(g[j], dq);
    }
}

// dG, dU, A in bf16 pairs of the gate's g and u and dA = da.
template <int ACT>
__device__ __forceinline__ void back_pair(float2 g, float2 u, float2 da, uint32_t &dg, uint32_t &du,
                                          uint32_t &a)
{
    float q0, q1;
    const float s0 = logistic<ACT>(g.x, q0), s1 = logistic<ACT>(g.y, q1);
    const float a0 = g.x * s0, a1 = g.y * s1;
    a = gemm::pack_bf16(a0 * u.x, a1 * u.y);
    du = gemm::pack_bf16(da.x * a0, da.y * a1);
    dg = gemm::pack_bf16(da.x * u.x * fmaf((1.0f - s0) * q0, a0, s0),
                         da.y * u.y * fmaf((1.0f - s1) * q1, a1, s1));
}

// 32 columns of one row of what was kept of G and U, as loaded: codes with their scale
// bytes (CODES), or bf16, zeros past the matrix. A lane holds a row, so every load of the
// warp touches 32 lines whatever its width, and their number is what the loads cost (1B
// layer, the whole launch, each chunk's loads just before their use: 8-byte pieces 142 us,
// 16-byte ones 125, none at all 112; loaded a chunk ahead they are hidden):
// Product::wide says that all rows are 32-byte aligned and whole chunks of 128 columns, so
// a row's chunk of codes is one load (past L1: 134 -> 124 us) and four chunks' scales
// another. Otherwise rows and pitches are 8-byte (codes) or 16-byte (bf16) aligned and hidden
// is a multiple of 8: pieces of 8 elements. Rows past the end read the last one.
template <bool CODES> struct Kept {
    static constexpr int W = CODES ? 2 : 4;   // words of 8 elements
    uint32_t g[4 * W], u[4 * W];
    uint32_t sg, su;                          // scale bytes; wide: of four chunks

    __device__ __forceinline__ void load(const Product &P, int row, int col0, bool first)
    {
        const int n = P.n - col0;
        const int64_t at = (row * P.ld_kept + col0) * (CODES ? 1 : 2);
        const uint8_t *gp = static_cast<const uint8_t *>(P.kept_g) + at;
        const uint8_t *up = static_cast<const uint8_t *>(P.kept_u) + at;
        const int64_t sat = row * P.ld_scale + col0 / kGroup;
        if (P.wide) {
            if (CODES && first) {   // col0 is a multiple of 64: bytes 0 or 2 of the four
                asm volatile("ld.global.b32 %0, [%1];" : "=r"(sg) : "l"(P.scale_g + (sat & ~3ll)));
                asm volatile("ld.global.b32 %0, [%1];" : "=r"(su) : "l"(P.scale_u + (sat & ~3ll)));
            }
#pragma unroll
            for (int i = 0; i < W / 2; ++i) {
                load32(gp + 32 * i, g + 8 * i);
                load32(up + 32 * i, u + 8 * i);
            }
            return;
        }
        if (CODES) {
            asm volatile("ld.global.u8 %0, [%1];" : "=r"(sg) : "l"(P.scale_g + sat));
            asm volatile("ld.global.u8 %0, [%1];" : "=r"(su) : "l"(P.scale_u + sat));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int j = 0; j < W; ++j)
                g[i * W + j] = u[i * W + j] = 0u;
            if (i * 8 < n) {
                piece(gp + i * 4 * W, g + i * W);
                piece(up + i * 4 * W, u + i * W);
            }
        }
    }
    static __device__ __forceinline__ void load32(const uint8_t *p, uint32_t *w)
    {
        asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]),
                       "=r"(w[6]), "=r"(w[7])
                     : "l"(p));
    }
    static __device__ __forceinline__ void piece(const uint8_t *p, uint32_t *w)
    {
        if constexpr (CODES)
            asm volatile("ld.global.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
        else
            asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                         : "l"(p));
    }
    static __device__ __forceinline__ float2 pair(const uint32_t *w, int i, float scale)
    {
        if constexpr (CODES) {
            const float2 v = decode2(w[i / 2] >> (16 * (i & 1)));
            return make_float2(v.x * scale, v.y * scale);
        } else {
            return make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
        }
    }
    // dG, dU, A of the chunk from its dA
    template <int ACT>
    __device__ __forceinline__ void back(const float (&da)[32], int shift, uint32_t (&dg)[16],
                                         uint32_t (&du)[16], uint32_t (&a)[16]) const
    {
        const float fg = scale_of(sg >> shift & 0xFFu), fu = scale_of(su >> shift & 0xFFu);
#pragma unroll
        for (int i = 0; i < 16; ++i)
            back_pair<ACT>(pair(g, i, fg), pair(u, i, fu), make_float2(da[2 * i], da[2 * i + 1]),
                           dg[i], du[i], a[i]);
    }
    __device__ __forceinline__ void back(const Product &P, const float (&da)[32], int col0,
                                         uint32_t (&dg)[16], uint32_t (&du)[16],
                                         uint32_t (&a)[16]) const
    {
        const int shift = P.wide ? col0 / kGroup % 4 * 8 : 0;
        if (P.act == kGelu)
            back<kGelu>(da, shift, dg, du, a);
        else
            back<kSilu>(da, shift, dg, du, a);
    }
};

// One 32 x 32 chunk of the tile: accumulator columns from acc (kGate: of G, U's
// half_cols further), output rows from row0 and columns from col0. Called by the
// whole warp with the same arguments; tcgen05.ld and the stores are the warp's.
template <int EPI>
__device__ __forceinline__ void drain(const Product &P, Stager &st, Kept<EPI == kGateBack8> &kept,
                                      uint32_t acc, int half_cols, int row0, int col0, bool first)
{
    if (row0 >= P.m || col0 >= P.n)
        return;
    const int row = min(row0 + st.lane, P.m - 1);   // rows past the end: the stores clip them
    if constexpr (EPI == kGate) {
        float g[32], u[32];
        load_acc(acc, g);
        load_acc(acc + (uint32_t)half_cols, u);
        if (P.keep == kKeep16) {
            st.bf16(&P.d1, g, col0, row0);
            st.bf16(&P.d2, u, col0, row0);
        } else if (P.keep == kKeep8) {
            float q[32];
#pragma unroll
            for (int j = 0; j < 32; ++j)
                q[j] = g[j];
            const uint32_t sg = st.codes(&P.d1, q, col0, row0);
#pragma unroll
            for (int j = 0; j < 32; ++j)
                q[j] = u[j];
            const uint32_t su = st.codes(&P.d2, q, col0, row0);
            // scale bytes, two chunks' in one store where a pair's warp has both: single
            // bytes were a third of the launch's writes to L2
            const int64_t at = row * P.ld_scale + col0 / kGroup;
            const bool in = row0 + st.lane < P.m, two = half_cols == 128 && P.wide;
            if (two && first && col0 + 32 < P.n) {
                kept.sg = sg;
                kept.su = su;
            } else if (two && !first) {
                if (in) {
                    *reinterpret_cast<uint16_t *>(P.scale_g + at - 1) = (uint16_t)(kept.sg | sg << 8);
                    *reinterpret_cast<uint16_t *>(P.scale_u + at - 1) = (uint16_t)(kept.su | su << 8);
                }
            } else if (in) {
                P.scale_g[at] = (uint8_t)sg;
                P.scale_u[at] = (uint8_t)su;
            }
        }
        if (P.act == kGelu)
            gate<kGelu>(g, u);
        else
            gate<kSilu>(g, u);
        st.bf16(&P.d0, u, col0, row0);
    } else if constexpr (gate_back(EPI)) {
        float d[32];
        uint32_t dg[16], du[16], a[16];
        load_acc(acc, d);
        kept.back(P, d, col0, dg, du, a);
        st.bf16(&P.d0, dg, col0, row0);
        st.bf16(&P.d1, du, col0, row0);
        st.bf16(&P.d2, a, col0, row0);
    } else {
        float v[32];
        load_acc(acc, v);
        if (P.gain != nullptr) {
            const int c = min(col0 + st.lane, P.n - 1);
            const float f = P.gain_f32 ? ld1(static_cast<const float *>(P.gain) + c)
                                       : ld1(static_cast<const __nv_bfloat16 *>(P.gain) + c);
#pragma unroll
            for (int j = 0; j < 32; ++j)
                v[j] *= __shfl_sync(0xFFFFFFFFu, f, j);
        }
        if (P.accumulate) {   // in 16-byte pieces: rows are 16-byte aligned, n is a multiple of 8
            const int size = P.f32 ? 4 : 2, left = P.n - col0;
            const uint8_t *old = static_cast<const uint8_t *>(P.old) + (row * P.ld_old + col0) * size;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if ((P.f32 ? 4 : 8) * i < min(left, 32)) {
                    const uint4 q = gemm::load_c(reinterpret_cast<const __nv_bfloat16 *>(old + 16 * i));
                    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
                    if (P.f32) {
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            v[4 * i + j] += __uint_as_float(w[j]);
                    } else if (i < 4) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            v[(8 * i + 2 * j) & 31] += __uint_as_float(w[j] << 16);
                            v[(8 * i + 2 * j + 1) & 31] += __uint_as_float(w[j] & 0xFFFF0000u);
                        }
                    }
                }
        }
        if (P.f32)
            st.f32(&P.d0, v, col0, row0);
        else
            st.bf16(&P.d0, v, col0, row0);
    }
}

// ---- split K ----
// Warp w of each of the S CTAs holds its K share's sums of the same 32 rows, in two
// chunks of 32 columns. Rank j finishes rows 32/S j .. of them: each lane sends its row
// of a chunk (128 bytes, granules XOR-ed with the row) to the buffer of the rank that
// owns it, in the place of the rank it comes from, and the owner adds the S rows up in
// rank order, so the result does not depend on timing. The stores are asynchronous ones
// that complete on the owner's mbarrier, both chunks in one phase.
//   xfull[w]   all S ranks' bytes have landed in this warp's buffer
//   xempty[w]  all S ranks have read what this warp sent before
__device__ __forceinline__ bool mbar_wait_cluster(uint32_t bar, uint32_t parity)
{
    unsigned long long t0 = 0;
    for (;;) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(bar), "r"(parity)
            : "memory");
        if (ok)
            return true;
        const unsigned long long now = gemm::globaltimer();
        if (t0 == 0)
            t0 = now;
        if (now - t0 > gemm::kWaitNs)
            return false;
    }
}

constexpr int kSendBytes = 32 * 32 * 4;   // one chunk

struct Exchange {
    uint32_t buf, xfull, xempty;   // this CTA's, of this warp
    uint32_t rank, ranks;
    int lane, turn;
    unsigned int *err;

    __device__ __forceinline__ bool give_up(bool ok) const
    {
        if (__all_sync(0xFFFFFFFFu, ok))
            return false;
        if (lane == 0)
            atomicOr(err, kErrWaitDone);
        return true;
    }
    // Before a tile's `chunks` sends; false when the wait gave up.
    __device__ __forceinline__ bool begin(int chunks)
    {
        if (give_up(mbar_wait_cluster(xempty, ((uint32_t)turn & 1u) ^ 1u)))
            return false;
        if (lane == 0)
            mbar_arrive_expect_tx(xfull, (uint32_t)(chunks * kSendBytes));
        return true;
    }
    __device__ __forceinline__ void send(int chunk, const float (&v)[32]) const
    {
        const int rows = 32 / (int)ranks;
        const uint32_t owner = (uint32_t)(lane / rows);
        const uint32_t to =
            map_to_rank(buf + (uint32_t)(chunk * kSendBytes + ((int)rank * rows + lane % rows) * 128),
                        owner);
        const uint32_t bar = map_to_rank(xfull, owner);
#pragma unroll
        for (int g = 0; g < 8; ++g)
            asm volatile(
                "st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], "
                "{%1, %2, %3, %4}, [%5];" ::"r"(to + (uint32_t)((g ^ (lane & 7)) << 4)),
                "f"(v[4 * g]), "f"(v[4 * g + 1]), "f"(v[4 * g + 2]), "f"(v[4 * g + 3]), "r"(bar)
                : "memory");
    }
    // All ranks' sends have landed; false when the wait gave up.
    __device__ __forceinline__ bool landed() const
    {
        return !give_up(mbar_wait_cluster(xfull, (uint32_t)turn & 1u));
    }
    // Once landed, the warp's 32 / ranks rows are dealt to its lanes in pieces of 4 columns:
    // `ranks` lanes to a row, pieces() of each chunk to a lane. Eight lanes read 128
    // consecutive bytes of the buffer's banks at a time. A lane's values are few, so the code
    // is short: run once in a launch, it costs its way to the instruction cache.
    __device__ __forceinline__ int pieces() const { return 8 / (int)ranks; }
    __device__ __forceinline__ int my_row() const   // of the 32
    {
        return (int)rank * (32 / (int)ranks) + lane / (int)ranks;
    }
    __device__ __forceinline__ int granule(int i) const   // where the buffer has piece i
    {
        return lane % (int)ranks + (int)ranks * ((i + lane / (int)ranks) & (pieces() - 1));
    }
    __device__ __forceinline__ int column(int i) const   // first of its four
    {
        return 4 * (granule(i) ^ (my_row() & 7));
    }
    __device__ __forceinline__ void total(int chunk, int i, float (&v)[4]) const
    {
        const int rows = 32 / (int)ranks;
        uint32_t from = buf + (uint32_t)(chunk * kSendBytes + lane / (int)ranks * 128 + granule(i) * 16);
        v[0] = v[1] = v[2] = v[3] = 0.0f;
        for (int r = 0; r < (int)ranks; ++r, from += (uint32_t)rows * 128) {
            float4 f;
            asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                         : "=f"(f.x), "=f"(f.y), "=f"(f.z), "=f"(f.w)
                         : "r"(from)
                         : "memory");
            v[0] += f.x;
            v[1] += f.y;
            v[2] += f.z;
            v[3] += f.w;
        }
    }
    // Over the lanes of a row.
    __device__ __forceinline__ float row_max(float v) const
    {
        for (int o = 1; o < (int)ranks; o <<= 1)
            v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
        return v;
    }
    // The buffer has been read: tell every rank.
    __device__ __forceinline__ void end()
    {
        __syncwarp();
        if (lane < (int)ranks)
            asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(
                             map_to_rank(xempty, (uint32_t)lane))
                         : "memory");
        ++turn;
    }
};

__device__ __forceinline__ void store4(__nv_bfloat16 *p, const float (&v)[4])
{
    *reinterpret_cast<uint2 *>(p) = make_uint2(gemm::pack_bf16(v[0], v[1]), gemm::pack_bf16(v[2], v[3]));
}
__device__ __forceinline__ void store4(uint8_t *p, const float (&v)[4], float inv)
{
    *reinterpret_cast<uint32_t *>(p) =
        encode4(inf_to_nan(v[0]) * inv, inf_to_nan(v[1]) * inv, inf_to_nan(v[2]) * inv,
                inf_to_nan(v[3]) * inv);
}
__device__ __forceinline__ float finite_max(const float (&v)[4])
{
    return fmaxf(fmaxf(finite_abs(v[0]), finite_abs(v[1])),
                 fmaxf(finite_abs(v[2]), finite_abs(v[3])));
}

// Four kept values, 4- (codes) or 8-byte (bf16) aligned.
template <bool CODES> struct Kept4 {
    uint32_t w[CODES ? 1 : 2];
    __device__ __forceinline__ void load(const void *base, int64_t at)
    {
        if constexpr (CODES)
            asm volatile("ld.global.b32 %0, [%1];"
                         : "=r"(w[0])
                         : "l"(static_cast<const uint8_t *>(base) + at));
        else
            asm volatile("ld.global.v2.b32 {%0, %1}, [%2];"
                         : "=r"(w[0]), "=r"(w[1])
                         : "l"(static_cast<const __nv_bfloat16 *>(base) + at));
    }
    __device__ __forceinline__ float2 pair(int i, float scale) const
    {
        return Kept<CODES>::pair(w, i, scale);
    }
};

// What a lane needs of one chunk's kept values, all loads under way at once.
template <bool CODES> struct KeptPieces {
    Kept4<CODES> g[8], u[8];
    uint32_t sg, su;
    __device__ __forceinline__ void load(const Product &P, const Exchange &ex, int row, int col0)
    {
        row = min(row, P.m - 1);
        if (CODES) {
            const int64_t sat = row * P.ld_scale + col0 / kGroup;
            asm volatile("ld.global.u8 %0, [%1];" : "=r"(sg) : "l"(P.scale_g + sat));
            asm volatile("ld.global.u8 %0, [%1];" : "=r"(su) : "l"(P.scale_u + sat));
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < ex.pieces() && col0 + ex.column(i) < P.n) {
                const int64_t at = row * P.ld_kept + col0 + ex.column(i);
                g[i].load(P.kept_g, at);
                u[i].load(P.kept_u, at);
            }
    }
};

// A warp's part of a tile split along K: 32 rows of kGate: 32 columns of G and of U,
// otherwise of up to 64 columns, from row0 and col0 on, in `chunks` chunks (0: none are in
// the matrix, the same on every rank). bf16 outputs o0, o1, o2 (as d0, d1, d2).
// acc_empty is arrived on as soon as the accumulator is read. False when a wait gave up.
template <int EPI>
__device__ __forceinline__ bool drain_split(const Product &P, Exchange &ex, uint32_t acc,
                                            int half_cols, int row0, int col0, int chunks,
                                            uint32_t acc_empty)
{
    const int row = row0 + ex.my_row();
    KeptPieces<EPI == kGateBack8> kept;
    if (gate_back(EPI) && chunks > 0)
        kept.load(P, ex, row, col0);
    if (chunks > 0 && !ex.begin(chunks))
        return false;
#pragma unroll 1
    for (int c = 0; c < chunks; ++c) {
        float v[32];
        load_acc(acc + (uint32_t)(c * (EPI == kGate ? half_cols : 32)), v);
        ex.send(c, v);
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncwarp();
    if (ex.lane == 0)
        mbar_arrive<1>(acc_empty);
    if (chunks == 0)
        return true;
    if (!ex.landed())
        return false;
    const bool in = row < P.m;
    if constexpr (EPI == kGate) {
        float inv_g = 0.0f, inv_u = 0.0f;
        if (P.keep == kKeep8) {
            float ag = 0.0f, au = 0.0f;
#pragma unroll 1
            for (int i = 0; i < ex.pieces(); ++i) {
                float g[4], u[4];
                ex.total(0, i, g);
                ex.total(1, i, u);
                if (col0 + ex.column(i) < P.n) {
                    ag = fmaxf(ag, finite_max(g));
                    au = fmaxf(au, finite_max(u));
                }
            }
            const uint32_t sg = scale_byte(ex.row_max(ag)), su = scale_byte(ex.row_max(au));
            inv_g = inv_scale_of(sg);
            inv_u = inv_scale_of(su);
            if (in && ex.lane % (int)ex.ranks == 0) {
                const int64_t sat = row * P.ld_scale + col0 / kGroup;
                P.scale_g[sat] = (uint8_t)sg;
                P.scale_u[sat] = (uint8_t)su;
            }
        }
#pragma unroll 1
        for (int i = 0; i < ex.pieces(); ++i) {
            const int col = col0 + ex.column(i);
            float g[4], u[4];
            ex.total(0, i, g);
            ex.total(1, i, u);
            if (!in || col >= P.n)
                continue;
            const int64_t at = row * P.ld_o + col;
            if (P.keep == kKeep16) {
                store4(P.o1 + at, g);
                store4(P.o2 + at, u);
            } else if (P.keep == kKeep8) {
                store4(P.codes_g + row * P.ld_codes_g + col, g, inv_g);
                store4(P.codes_u + row * P.ld_codes_u + col, u, inv_u);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float dq;
                u[j] *= g[j] * (P.act == kGelu ? logistic<kGelu>(g[j], dq) : logistic<kSilu>(g[j], dq));
            }
            store4(P.o0 + at, u);
        }
        ex.end();
    } else if constexpr (gate_back(EPI)) {
#pragma unroll 1
        for (int c = 0; c < chunks; ++c, col0 += 32) {
            if (c > 0)
                kept.load(P, ex, row, col0);
            const float fg = scale_of(kept.sg), fu = scale_of(kept.su);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (i >= ex.pieces())
                    break;
                const int col = col0 + ex.column(i);
                float v[4];
                ex.total(c, i, v);
                if (!in || col >= P.n)
                    continue;
                uint32_t dg[2], du[2], a[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float2 g = kept.g[i].pair(j, fg), u = kept.u[i].pair(j, fu);
                    const float2 da = make_float2(v[2 * j], v[2 * j + 1]);
                    if (P.act == kGelu)
                        back_pair<kGelu>(g, u, da, dg[j], du[j], a[j]);
                    else
                        back_pair<kSilu>(g, u, da, dg[j], du[j], a[j]);
                }
                const int64_t at = row * P.ld_o + col;
                *reinterpret_cast<uint2 *>(P.o0 + at) = make_uint2(dg[0], dg[1]);
                *reinterpret_cast<uint2 *>(P.o1 + at) = make_uint2(du[0], du[1]);
                *reinterpret_cast<uint2 *>(P.o2 + at) = make_uint2(a[0], a[1]);
            }
        }
        ex.end();
    } else {
#pragma unroll 1
        for (int c = 0; c < chunks; ++c, col0 += 32)
#pragma unroll 1
            for (int i = 0; i < ex.pieces(); ++i) {
                const int col = col0 + ex.column(i);
                float v[4];
                ex.total(c, i, v);
                if (in && col < P.n)
                    store4(P.o0 + row * P.ld_o + col, v);
            }
        ex.end();
    }
    return true;
}

//   full[s]      (leader) both ranks' TMA bytes of stage s have landed
//   empty[s]     (each)   the leader's MMAs have finished reading stage s
//   acc_full[a]  (each)   accumulator a holds a finished tile
//   acc_empty[a] (leader) all epilogue warps of the pair have read it
// CG CTAs share a tile (a pair's 2-SM MMA); SPLIT (CG = 1): the CTAs of a cluster
// share a tile's K blocks. The cluster's size comes with the launch.
template <int CG, int EPI, bool SPLIT>
__global__ void __launch_bounds__(kThreads, 1) ffn_gemm_kernel(const __grid_constant__ Launch L)
{
    static_assert(CG == 1 || !SPLIT, "pairs do not split K");
    using R = Ring<SPLIT>;
    constexpr int T = kTile(CG), BK = R::BK;
    const int a_rows = CG == 1 ? L.a_rows : BM, cols = SPLIT ? L.cols : T;
    // of a stage; where K is not split its layout is that of whole boxes
    const int a_bytes = R::bytes(SPLIT ? a_rows : BM), b_bytes = R::bytes(SPLIT ? cols : BH);
    const int n_stages = SPLIT ? R::stages(a_rows, cols) : R::stages(BM, BH);
    extern __shared__ uint8_t smem_raw[];
    constexpr int kStages = SPLIT ? kMaxStages : R::stages(BM, BH);   // barriers laid out for
    __shared__ uint64_t bars[2 * kStages + 4 + (SPLIT ? 2 * kEpiWarps : 0)];
    __shared__ uint32_t tmem_slot;
    __shared__ int aborted;

    const int warp = uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31;
    const uint32_t rank = CG == 2 ? (uint32_t)uniform((int)gemm::cluster_rank()) : 0u;
    const bool leader = rank == 0;
    uint32_t split = 1, share = 0;   // CTAs on a tile's K blocks, and which this is
    if (SPLIT) {
        asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(split));
        split = (uint32_t)uniform((int)split);
        share = (uint32_t)uniform((int)gemm::cluster_rank());
    }
    const int group = SPLIT ? (int)split : CG;
    const int pair = blockIdx.x / group, n_pairs = gridDim.x / group;
    const uint32_t raw = (uint32_t)__cvta_generic_to_shared(smem_raw);
    const uint32_t ring = (raw + 1023u) & ~1023u;
    const uint32_t sa = ring, sb = ring + (uint32_t)(n_stages * a_bytes);
    const uint32_t bar0 = (uint32_t)__cvta_generic_to_shared(bars);
    auto full = [&](int s) { return bar0 + 8u * (uint32_t)s; };
    auto empty = [&](int s) { return bar0 + 8u * (uint32_t)(kStages + s); };
    auto acc_full = [&](int a) { return bar0 + 8u * (uint32_t)(2 * kStages + a); };
    auto acc_empty = [&](int a) { return bar0 + 8u * (uint32_t)(2 * kStages + 2 + a); };

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(acc_full(a), 1);
            mbar_init(acc_empty(a), CG * kEpiWarps);
        }
        if (SPLIT)
            for (int w = 0; w < kEpiWarps; ++w) {
                mbar_init(bar0 + 8u * (uint32_t)(2 * kStages + 4 + 2 * w), 1);
                mbar_init(bar0 + 8u * (uint32_t)(2 * kStages + 5 + 2 * w), split);
            }
        aborted = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1)
        gemm::tmem_alloc<CG>((uint32_t)__cvta_generic_to_shared(&tmem_slot));
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    group_sync<SPLIT ? 2 : CG>();   // barriers of every CTA initialised before remote use
    if (SPLIT)
        __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = (uint32_t)uniform((int)tmem_slot);
    const int n_tiles = L.n_tiles;
    if (warp == 0 && lane < L.n_products) {   // the maps are parameters: read before the wait
        for (int i = 0; i < 2; ++i) {
            asm volatile("prefetch.tensormap [%0];"
                         ::"l"(reinterpret_cast<uint64_t>(&L.p[lane].a[i])) : "memory");
            asm volatile("prefetch.tensormap [%0];"
                         ::"l"(reinterpret_cast<uint64_t>(&L.p[lane].b[i])) : "memory");
        }
    }
    pdl_wait();
    // The next launch's CTAs, one to an SM like these, may set themselves up wherever one
    // of these has ended; they wait at the same place until all of them have. Only where
    // the next launch is this kernel's: others spread unevenly (dpo_device.cuh). Forward of
    // 768 x 2048 widths, 17 to 200 tokens: 16.4 -> 15.1 us.
    if (L.early)
        launch_dependents();

    // Loading and MMA warps run as a whole, with one lane for the copies, the MMAs and the
    // error bits: in a branch of one lane the compiler takes no operand for uniform and moves
    // each to where the instruction wants it (7B step 4.13 -> 3.93 ms, 1B 0.83 -> 0.79; a
    // 64-K stage of single CTAs took 570 clocks of issue for MMAs of 256).
    if (warp == 0) {
        const bool one = elect();
        int it = 0, s = 0;   // K blocks issued by this CTA, the ring's next stage
        uint32_t ph = 1;     // parity of the stage's release
        const uint32_t bytes = (uint32_t)(CG * (R::bytes(a_rows) + b_bytes));
        bool ok = true;
        for (int t, r = 0; ok && (t = turn_of(r, pair, n_pairs)) < n_tiles; ++r) {
            const Tile tile = tile_at(L, t);
            const Product &P = L.p[tile.p];
            const bool a_mn = P.a_mn, b_mn = P.b_mn;
            const int ma = tile.m * T + (int)rank * BM;
            // B rows of this CTA: T / CG of the tile's columns; kGate: a pair's CTAs
            // hold one projection each, a single CTA half a box of either
            const int nb = EPI == kGate ? tile.n * (cols / 2) : tile.n * cols + (int)rank * BH;
            const int kb0 = P.k_blocks[0], kb_all = kb0 + P.k_blocks[1];
            const int kb_n = SPLIT ? share_end(kb_all, share, split) : kb_all;
            for (int kb = SPLIT ? share_end(kb_all, share - 1, split) : 0; kb < kb_n; ++kb, ++it) {
                ok = warp_wait(empty(s), ph, &aborted);
                if (!ok) {
                    if (one)
                        atomicOr(L.err, kErrWaitEmpty);
                    break;
                }
                if (one) {
                    const uint32_t fbar = CG == 2 ? map_to_rank(full(s), 0) : full(s);
                    if (leader)
                        mbar_arrive_expect_tx(full(s), bytes);
                    const int seg = kb >= kb0, k = (kb - (seg ? kb0 : 0)) * BK;
                    const CUtensorMap *ta = &P.a[seg];
                    const CUtensorMap *tb = EPI == kGate ? &P.b[CG == 2 ? rank : 0] : &P.b[seg];
                    const uint32_t as = sa + (uint32_t)(s * a_bytes);
                    const uint32_t bs = sb + (uint32_t)(s * b_bytes);
                    if (!SPLIT && a_mn) {
                        tma_load<CG>(as, ta, ma, k, fbar);
                        tma_load<CG>(as + R::mn_box, ta, ma + 64, k, fbar);
                    } else {
#pragma unroll
                        for (int h = 0; h < BK / kBoxK; ++h)
                            tma_load<CG>(as + (uint32_t)(h * R::box), ta, k + h * kBoxK, ma, fbar);
                    }
                    if (EPI != kGate && b_mn) {
                        tma_load<CG>(bs, tb, nb, k, fbar);
                        if (cols > 64)
                            tma_load<CG>(bs + R::mn_box, tb, nb + 64, k, fbar);
                    } else {
#pragma unroll
                        for (int h = 0; h < BK / kBoxK; ++h) {
                            const uint32_t bh = bs + (uint32_t)(h * R::box);
                            tma_load<CG>(bh, tb, k + h * kBoxK, nb, fbar);
                            if (EPI == kGate && CG == 1)   // half the rows of each projection
                                tma_load<CG>(bh + (uint32_t)(cols / 2 * kRowBytes), &P.b[1],
                                             k + h * kBoxK, nb, fbar);
                        }
                    }
                }
                __syncwarp();
                if (++s == n_stages) {
                    s = 0;
                    ph ^= 1u;
                }
            }
        }
        if (leader && one)   // no CTA leaves before the loads in flight have landed
            for (int q = it - n_stages < 0 ? 0 : it - n_stages; q < it; ++q)
                if (!mbar_wait(full(q % n_stages), (uint32_t)(q / n_stages) & 1u))
                    atomicOr(L.err, kErrDrain);
        __syncwarp();
    } else if (warp == 1) {
        if (leader) {
            const bool one = elect();
            int lt = 0, s = 0;
            uint32_t ph = 0;
            bool ok = true;
            for (int t; ok && (t = turn_of(lt, pair, n_pairs)) < n_tiles; ++lt) {
                const Product &P = L.p[tile_at(L, t).p];
                const int kb_all = P.k_blocks[0] + P.k_blocks[1];
                const int kb_n = SPLIT ? share_end(kb_all, share, split) -
                                             share_end(kb_all, share - 1, split)
                                       : kb_all;
                const bool a_mn = P.a_mn, b_mn = P.b_mn;
                const uint32_t idesc = idesc_of(CG, cols, a_mn, b_mn);
                const Steps a0 = steps_of<BK>(sa, a_mn), b0 = steps_of<BK>(sb, b_mn);
                const int a = lt & 1;
                const uint32_t aph = (uint32_t)(lt >> 1) & 1u;
                ok = warp_wait(acc_empty(a), aph ^ 1u, &aborted);
                if (!ok) {
                    if (one)
                        atomicOr(L.err, kErrWaitDone);
                    break;
                }
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t d = tmem + (uint32_t)(a * T);
                for (int kb = 0; kb < kb_n; ++kb) {
                    ok = warp_wait(full(s), ph, &aborted);
                    if (!ok) {
                        if (one)
                            atomicOr(L.err, kErrWaitFull);
                        break;
                    }
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    if (one) {
                        const Steps da = a0.stage(s * a_bytes), db = b0.stage(s * b_bytes);
#pragma unroll
                        for (int k = 0; k < BK / 16; ++k)
                            mma_bf16<CG>(d, da.at(k), db.at(k), idesc, (kb | k) != 0 ? 1u : 0u);
                        mma_commit<CG>(empty(s));
                    }
                    __syncwarp();
                    if (++s == n_stages) {
                        s = 0;
                        ph ^= 1u;
                    }
                }
                if (one)
                    mma_commit<CG>(acc_full(a));
                __syncwarp();
                if (!ok && !mbar_wait(acc_full(a), aph) && one)
                    atomicOr(L.err, kErrDrain);
            }
        }
    } else {
        // Warp w reads TMEM lanes 32 (w % 4) .. +31, rows BM rank + 32 (w % 4) + lane of
        // the tile, and the half of its columns that (w - 2) / 4 names.
        const int q = warp & 3, half = (warp - 2) >> 2;
        // staging of the warps that have rows
        const int slot = SPLIT ? half * (a_rows / 32) + q : warp - 2;
        Stager st = {ring + (uint32_t)(n_stages * (a_bytes + b_bytes) + slot * R::staging), lane, 0};
        const uint32_t xbar = bar0 + 8u * (uint32_t)(2 * kStages + 4 + (warp - 2) * 2);
        Exchange ex = {st.buf, xbar, xbar + 8u, share, split, lane, 0, L.err};
        // Output columns of a tile, and where its second half of the warps begins; 32 columns
        // of kGate (a scale's group) are the first half's alone.
        const int out_cols = EPI == kGate ? cols / 2 : cols;
        const int half0 = half * (SPLIT && EPI == kGate ? 32 : out_cols / 2);
        int lt = 0;
        for (int t; (t = turn_of(lt, pair, n_pairs)) < n_tiles; ++lt) {
            const Tile tile = tile_at(L, t);
            const Product &P = L.p[tile.p];
            const int a = lt & 1;
            const int row0 = tile.m * T + (int)rank * BM + q * 32;
            const int col_0 = tile.n * out_cols + half0;
            Kept<EPI == kGateBack8> kept;
            auto load_kept = [&](int ch) {   // a chunk ahead of its use
                const int col0 = col_0 + ch * 32;
                if (row0 < P.m && col0 < P.n)
                    kept.load(P, min(row0 + lane, P.m - 1), col0, ch == 0);
            };
            if constexpr (gate_back(EPI) && !SPLIT)
                load_kept(0);
            bool seen = mbar_wait(acc_full(a), (uint32_t)(lt >> 1) & 1u);
            if (!seen)
                atomicOr(L.err, kErrWaitDone);
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            seen = __all_sync(0xFFFFFFFFu, seen && !*(volatile int *)&aborted);
            if (!seen)
                break;
            const uint32_t acc =
                tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(a * T + half0);
#pragma unroll 1
            for (int ch = 0; ch < (SPLIT ? 1 : out_cols / 64); ++ch) {
                const uint32_t at = acc + (uint32_t)(ch * 32);
                const int col0 = col_0 + ch * 32;
                if constexpr (SPLIT) {
                    const bool any = row0 < P.m && col0 < P.n && half0 < out_cols;
                    const bool two = EPI == kGate || (cols > 64 && col0 + 32 < P.n);
                    seen = drain_split<EPI>(P, ex, at, out_cols, row0, col0, any ? 1 + two : 0,
                                            acc_empty(a));
                } else if constexpr (gate_back(EPI)) {
                    Kept<EPI == kGateBack8> now = kept;
                    if (ch + 1 < out_cols / 64)
                        load_kept(ch + 1);
                    drain<EPI>(P, st, now, at, out_cols, row0, col0, ch == 0);
                } else {
                    drain<EPI>(P, st, kept, at, out_cols, row0, col0, ch == 0);
                }
            }
            if (SPLIT) {
                if (seen)
                    continue;
                aborted = 1;
                break;
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0)
                mbar_arrive<CG>(acc_empty(a));
        }
        if (lane == 0)
            asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        __syncwarp();
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }
    __syncthreads();
    if (CG == 2 || SPLIT)
        group_sync<2>();   // no CTA leaves while a peer may use its shared memory
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        gemm::tmem_free<CG>(tmem);
    }
}

}  // namespace ffn
}  // namespace dpo
