// dpo_products.h -- products on the tensor cores (dpo_ffn_gemm.cuh) for other calls than the
// feed-forward block's.
#pragma once

#include "dpo_ids.cuh"

#include <stdint.h>

namespace dpo {

// out = A B (m x n), or out += A B: bf16 operands, fp32 accumulation. A is m x k row-major, or
// with a_mn k x m; B is n x k, or with b_mn k x n. Pointers 16-byte aligned, pitches of whole 16
// bytes, an added out with n a multiple of 8.
struct StoreProduct {
    const void *a, *b;
    void *out;
    int64_t m, n, k;
    int64_t ld_a, ld_b, ld_out;
    int a_mn, b_mn;
    int f32, accumulate;
    void *shares;                 // the first of a list, bf16: product_share_bytes, or nullptr
};

constexpr int kMaxStoreProducts = 4;

// How far the K of the first of two products whose list is out = G w (m x n, k) and G^T x (k x n, m) is
// divided so that no tile takes longer than some eight tenths of the list, by 76 pairs' shares of
// it, and the bytes that the shares' sums take (0: not divided).
int product_ways(int64_t m, int64_t n, int64_t k);
int64_t product_share_bytes(int64_t m, int64_t n, int64_t k);

// Up to four of them, in one launch in whose order their tiles are begun (longest first), or the
// first one before the others where its K is better split.
int store_products(const char *what, const StoreProduct *p, int n, void *stream);

// A head's logits x w^T: what their distributions need, by kHeadStatCols columns, or the logits
// themselves, or both. What is kept of e^(z - maximum), in fp16, comes times kHeadUnit, so that values
// down to 2^-29 keep 11 bits.
constexpr int kHeadStatCols = 128;
constexpr float kHeadUnit = 32768.0f;
struct HeadProduct {
    const void *x, *w;            // bf16, tokens x dim at pitch ld_x, vocab x dim
    int64_t tokens, dim, vocab, ld_x;
    Ids ids;                      // p nullptr: none
    float scale;
    float *target;                // z of each token's id
    float *maxima;                // [columns / kHeadStatCols][token], or nullptr: no statistics
    float2 *sums;                 // likewise
    void *kept;                   // fp16 e^(z - maximum) kHeadUnit, or nullptr (with statistics):
    int64_t kept_rows;            // [columns / kHeadStatCols][kept_rows][kHeadStatCols], kept_rows the
                                  // tokens to a multiple of 32
    void *logits;                 // fp32, before the scale, or nullptr
    int64_t ld;                   // its pitch
};
int head_product(const char *what, const HeadProduct &h, void *stream);

}  // namespace dpo
