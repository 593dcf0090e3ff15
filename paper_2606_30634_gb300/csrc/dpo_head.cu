// dpo_head.cu -- the head: log probabilities from the stream and the head's weights, and the
// gradients of both (dpo_head, dpo_head_backward in include/dpo_ends.h).
//
// Forward, two launches: logits = x w^T in fp32; the rows' distributions (dpo_logprobs.cu).
// Backward, two launches: G from the kept logits; dx = G w and dw = G^T x, one list of tiles.
#include "dpo_logprobs.cuh"
#include "dpo_products.h"

namespace dpo {
namespace {

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
    if (!isfinite(scale) || !(scale > 0.0f))
        return call_fail(DPO_EINVAL, "%s: scale %g", what, (double)scale);
    return DPO_OK;
}

struct Sizes {
    int64_t ld, forward, kept, backward;
};
Sizes sizes_of(int64_t tokens, int64_t vocab, bool keep)
{
    Sizes s;
    s.ld = pitch_of(vocab);
    const int64_t logits = align_up(tokens * s.ld * 4);
    s.forward = keep ? 0 : logits;
    s.kept = logits;
    s.backward = align_up(tokens * s.ld * 2);
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
    const Sizes s = sizes_of(tokens, vocab, keep != 0);
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
    const Sizes s = sizes_of(T, a.vocab, a.kept != nullptr);
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
    void *const logits = a.kept != nullptr ? a.kept : a.workspace;
    const StoreProduct p = {a.x, a.w, logits, T, a.vocab, a.dim, a.ld_x, a.dim, s.ld, 0, 0, 1, 0};
    if ((rc = store_products(what, &p, 1, cuda_stream)) != DPO_OK)
        return rc;
    dpo_logprobs_args l{};
    l.logits = logits;
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
    const Sizes s = sizes_of(T, V, true);
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
    void *const G = a.workspace;
    dpo_logprobs_backward_args l{};
    l.logits = a.kept;
    l.ids = a.ids;
    l.stats = a.stats;
    l.entropy = a.entropy;
    l.dlogp = a.dlogp;
    l.dentropy = a.dentropy;
    l.dlogits = G;
    l.rows = T;
    l.vocab = V;
    l.ld_logits = l.ld_dlogits = s.ld;
    l.scale = a.scale;
    l.dtype = DPO_F32;
    if ((rc = logits_gradient(what, l, cuda_stream)) != DPO_OK)
        return rc;
    StoreProduct p[2];
    int n = 0;
    if (a.dx != nullptr)
        p[n++] = {G, a.w, a.dx, T, D, V, s.ld, D, a.ld_dx, 0, 1, 0, 0};
    p[n++] = {G, a.x, a.dw, V, D, T, s.ld, a.ld_x, D, 1, 1, a.grad_dtype == DPO_F32, a.accumulate != 0};
    return store_products(what, p, n, cuda_stream);
}
