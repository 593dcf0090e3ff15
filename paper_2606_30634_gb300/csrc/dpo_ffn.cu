// dpo_ffn.cu -- the gated feed-forward block, forward and backward
// (dpo_ffn_forward, dpo_ffn_backward in include/dpo.h): argument checks and the
// launches of the tensor-core kernel of dpo_ffn_gemm.cuh.
//
// Forward, two launches:   A = act(x w_gate^T) (x w_up^T), both projections in one;
//                          out = A w_down^T
// Backward, two launches:  dG, dU, A from dA = dout w_down and what was kept;
//                          dx, dw_gate, dw_up, dw_down, one list of tiles
// (and one more to widen the 8-bit rows when the block's input was kept so).
#include "dpo.h"
#include "dpo_call.h"
#include "dpo_ffn_gemm.cuh"

#include <cuda_runtime.h>

#include <mutex>

namespace {

using namespace dpo;
using namespace dpo::ffn;

static_assert(kSilu == DPO_ACT_SILU && kGelu == DPO_ACT_GELU, "activations");
static_assert(kKeepNone == DPO_KEEP_NONE && kKeep8 == DPO_KEEP_8BIT && kKeep16 == DPO_KEEP_BF16,
              "what is kept");
static_assert(kGroup == DPO_PACK8_GROUP, "group");

// Error bits of this library's feed-forward kernels on a device (sticky).
__device__ unsigned int g_ffn_err;

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *,
                                 const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                 const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

using KernelFn = void (*)(const Launch);
constexpr int kForms = 3;   // epilogues

// What the launches need to know of a device, found by its first call.
struct Device {
    bool ready = false;
    unsigned int *err = nullptr;
    int slots[2][kForms] = {};   // resident CTAs (0) and CTA pairs (1) of each kernel
};
constexpr int kMaxDevices = 64;
std::mutex g_mu;
Device g_devices[kMaxDevices];
EncodeTiled g_encode = nullptr;

KernelFn kernel_of(int cg, int epi)
{
    if (cg == 1)
        return epi == kGate ? ffn_gemm_kernel<1, kGate>
                            : epi == kGateBack ? ffn_gemm_kernel<1, kGateBack>
                                               : ffn_gemm_kernel<1, kStore>;
    return epi == kGate ? ffn_gemm_kernel<2, kGate>
                        : epi == kGateBack ? ffn_gemm_kernel<2, kGateBack>
                                           : ffn_gemm_kernel<2, kStore>;
}

cudaError_t prepare(Device &d)
{
    if (g_encode == nullptr) {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000,
                                                               cudaEnableDefault, &q);
        if (e != cudaSuccess)
            return e;
        if (q != cudaDriverEntryPointSuccess)
            return cudaErrorNotSupported;
        g_encode = reinterpret_cast<EncodeTiled>(p);
    }
    for (int cg = 1; cg <= 2; ++cg)
        for (int epi = 0; epi < kForms; ++epi) {
            const KernelFn k = kernel_of(cg, epi);
            cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void *>(k),
                                                 cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                 kSmemBytes);
            if (e != cudaSuccess)
                return e;
            cudaLaunchAttribute attr{};
            attr.id = cudaLaunchAttributeClusterDimension;
            attr.val.clusterDim.x = (unsigned)cg;
            attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
            cudaLaunchConfig_t cfg{};
            cfg.gridDim = dim3(1024);
            cfg.blockDim = dim3(kThreads);
            cfg.dynamicSmemBytes = kSmemBytes;
            cfg.attrs = &attr;
            cfg.numAttrs = 1;
            e = cudaOccupancyMaxActiveClusters(&d.slots[cg - 1][epi],
                                               reinterpret_cast<const void *>(k), &cfg);
            if (e != cudaSuccess)
                return e;
            if (d.slots[cg - 1][epi] < 1)
                return cudaErrorInvalidConfiguration;
        }
    void *p = nullptr;
    const cudaError_t e = cudaGetSymbolAddress(&p, g_ffn_err);
    if (e != cudaSuccess)
        return e;
    d.err = static_cast<unsigned int *>(p);
    d.ready = true;
    return cudaSuccess;
}

int device_info(const char *what, const Device **out)
{
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e == cudaSuccess && (device < 0 || device >= kMaxDevices))
        e = cudaErrorInvalidDevice;
    if (e == cudaSuccess) {
        std::lock_guard<std::mutex> lock(g_mu);
        Device &d = g_devices[device];
        if (!d.ready)
            e = prepare(d);
        *out = &d;
    }
    if (e != cudaSuccess) {
        cudaGetLastError();
        return call_fail(DPO_ECUDA, "%s: %s", what, cudaGetErrorString(e));
    }
    return DPO_OK;
}

// 2-D map of a row-major matrix.
struct Maps {
    bool ok = true;
    void make(CUtensorMap *m, CUtensorMapDataType type, int size, const void *base, int64_t rows,
              int64_t cols, int64_t ld, int box_rows, int box_cols, CUtensorMapSwizzle swizzle,
              CUtensorMapL2promotion l2)
    {
        const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
        const cuuint64_t strides[1] = {(cuuint64_t)(ld * size)};
        const cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows};
        const cuuint32_t es[2] = {1, 1};
        ok = ok && g_encode(m, type, 2, const_cast<void *>(base), dims, strides, box, es,
                            CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, l2,
                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    }
    // operand boxes of 64 columns, 128-byte swizzle
    void operand(CUtensorMap *m, const void *base, int64_t rows, int64_t cols, int64_t ld,
                 int box_rows)
    {
        make(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, rows, cols, ld, box_rows, kBoxK,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
    }
    // stores of 32 x 32 chunks
    void bf16(CUtensorMap *m, void *base, int64_t rows, int64_t cols, int64_t ld)
    {
        make(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, rows, cols, ld, 32, 32,
             CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE);
    }
    void f32(CUtensorMap *m, void *base, int64_t rows, int64_t cols, int64_t ld)
    {
        make(m, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, base, rows, cols, ld, 32, 32,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE);
    }
    void codes(CUtensorMap *m, void *base, int64_t rows, int64_t cols, int64_t ld)
    {
        make(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, base, rows, cols, ld, 32, 32,
             CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_NONE);
    }
};

int blocks_of(int64_t k) { return (int)((k + BK - 1) / BK); }

// A product's sizes, before its operands.
struct Shape {
    int64_t m, n, k;    // kGate: n of one projection
    int segments;
};

int64_t tiles_of(const Shape &s, int cg, int epi)
{
    const int64_t t = kTile(cg), tn = epi == kGate ? t / 2 : t;
    return (s.m + t - 1) / t * ((s.n + tn - 1) / tn);
}

// CTA pairs or single CTAs: the clocks the launch takes either way, its tiles dealt
// round-robin (the estimate of the Newton-Schulz launches, launch_clocks in
// dpo_muon.cu). More than four rounds of single CTAs go to the pairs unweighed.
int form_of(const Device &d, const Shape *s, int n, int epi)
{
    int64_t clocks[2];
    for (int cg = 1; cg <= 2; ++cg) {
        const int64_t block = cg == 1 ? 700 : 1100, epilogue = cg == 1 ? 2600 : 5000;
        const int64_t slots = d.slots[cg - 1][epi];
        int64_t tiles = 0;
        for (int i = 0; i < n; ++i)
            tiles += tiles_of(s[i], cg, epi);
        if (cg == 1 && tiles > 4 * slots)
            return 2;
        int64_t work = 0, longest = 0;
        for (int i = 0; i < n; ++i) {
            const int64_t c = blocks_of(s[i].k) * s[i].segments * block;
            const int64_t each = c > epilogue ? c : epilogue;
            work += tiles_of(s[i], cg, epi) * each;
            longest = longest > each ? longest : each;
        }
        // whole rounds of equal tiles, or the longest one's end
        const int64_t even = (work + slots - 1) / slots;
        const int64_t rounds = n == 1 ? (tiles + slots - 1) / slots * longest : even;
        clocks[cg - 1] = (rounds > longest ? rounds : longest) + epilogue;
    }
    return clocks[0] < clocks[1] ? 1 : 2;
}

int run(const char *what, const Device &d, Launch &L, const Shape *s, int n, int epi, int cg,
        bool maps_ok, void *stream)
{
    if (!maps_ok)
        return call_fail(DPO_ECUDA, "%s: a tensor map was refused", what);
    int64_t total = 0;
    for (int i = 0; i < n; ++i) {
        const int64_t t = kTile(cg), tn = epi == kGate ? t / 2 : t;
        Product &P = L.p[i];
        P.m = (int)s[i].m;
        P.n = (int)s[i].n;
        P.k_blocks[0] = blocks_of(s[i].k);
        P.k_blocks[1] = s[i].segments == 2 ? P.k_blocks[0] : 0;
        P.m_tiles = (int)((s[i].m + t - 1) / t);
        P.n_tiles = (int)((s[i].n + tn - 1) / tn);
        P.first = (int)total;
        total += tiles_of(s[i], cg, epi);
    }
    L.n_products = n;
    L.n_tiles = (int)total;
    L.err = d.err;
    const int64_t slots = d.slots[cg - 1][epi];
    const int64_t ctas = (total < slots ? total : slots) * cg;
    const cudaError_t e = launch_pdl(kernel_of(cg, epi), dim3((unsigned)ctas), kThreads, kSmemBytes,
                                     static_cast<cudaStream_t>(stream), L);
    return e == cudaSuccess ? DPO_OK : call_fail(DPO_ECUDA, "%s: %s", what, cudaGetErrorString(e));
}

int64_t align_up(int64_t v) { return (v + 255) / 256 * 256; }
int64_t hidden_bytes(int64_t tokens, int64_t hidden) { return align_up(tokens * hidden * 2); }

// ---- checks ----

constexpr int64_t kMaxSide = (int64_t)1 << 26;

int check_sizes(const char *what, int64_t tokens, int64_t dim, int64_t hidden)
{
    if (tokens < 0 || dim < 8 || hidden < 8 || dim % 8 != 0 || hidden % 8 != 0)
        return call_fail(DPO_EINVAL, "%s: tokens %lld, dim %lld, hidden %lld (multiples of 8)", what,
                         (long long)tokens, (long long)dim, (long long)hidden);
    const Shape s[] = {{tokens, hidden, dim, 1}, {tokens, dim, hidden, 1}, {hidden, dim, tokens, 1}};
    bool fits = tokens <= kMaxSide && dim <= kMaxSide && hidden <= kMaxSide;
    for (const Shape &q : s)
        fits = fits && tiles_of(q, 2, kGate) < ((int64_t)1 << 28);
    if (!fits)
        return call_fail(DPO_EINVAL, "%s: %lld x %lld x %lld is too large", what, (long long)tokens,
                         (long long)dim, (long long)hidden);
    return DPO_OK;
}

// The buffers of a call, for the checks of pointers, pitches and overlaps.
struct Buffers {
    struct Entry {
        const char *name;
        uintptr_t lo, hi;
        bool out;
    };
    const char *what;
    Entry e[20];
    int n = 0, rc = DPO_OK;
    explicit Buffers(const char *w) : what(w) {}
    // rows x cols of `size`-byte elements, `align`-byte aligned, its pitch too
    void add(const char *name, const void *p, int64_t rows, int64_t cols, int64_t ld, int64_t size,
             int64_t align, bool out)
    {
        if (rc != DPO_OK)
            return;
        if (p == nullptr)
            rc = call_fail(DPO_EINVAL, "%s: %s is NULL", what, name);
        else if (ld < cols)
            rc = call_fail(DPO_EINVAL, "%s: pitch %lld of %s is below its %lld columns", what,
                           (long long)ld, name, (long long)cols);
        else if (ld > ((int64_t)1 << 36))
            rc = call_fail(DPO_EINVAL, "%s: pitch of %s", what, name);
        else if (reinterpret_cast<uintptr_t>(p) % align != 0 || ld * size % align != 0)
            rc = call_fail(DPO_EALIGN, "%s: %s or its pitch is not %lld-byte aligned", what, name,
                           (long long)align);
        if (rc != DPO_OK)
            return;
        const uintptr_t b = reinterpret_cast<uintptr_t>(p);
        e[n++] = {name, b, b + (uintptr_t)(((rows - 1) * ld + cols) * size), out};
    }
    void packed(const char *name, const dpo_packed8 &p, int64_t rows, int64_t cols, int64_t align,
                bool out)
    {
        add(name, p.codes, rows, cols, p.ld_codes, 1, align, out);
        add("its scales", p.scales, rows, (cols + kGroup - 1) / kGroup, p.ld_scales, 1, 1, out);
    }
    int done()
    {
        for (int i = 0; i < n && rc == DPO_OK; ++i)
            for (int j = 0; j < i && rc == DPO_OK; ++j)
                if ((e[i].out || e[j].out) && e[i].lo < e[j].hi && e[j].lo < e[i].hi)
                    rc = call_fail(DPO_EINVAL, "%s: %s overlaps %s", what, e[i].name, e[j].name);
        return rc;
    }
};

}  // namespace

extern "C" int dpo_ffn_workspace(int64_t tokens, int64_t dim, int64_t hidden, int from_x8,
                                 int64_t *forward_bytes, int64_t *backward_bytes)
{
    const char *what = "dpo_ffn_workspace";
    const int rc = check_sizes(what, tokens, dim, hidden);
    if (rc != DPO_OK)
        return rc;
    if (forward_bytes != nullptr)
        *forward_bytes = hidden_bytes(tokens, hidden);
    if (backward_bytes != nullptr)
        *backward_bytes =
            3 * hidden_bytes(tokens, hidden) + (from_x8 ? align_up(tokens * dim * 2) : 0);
    return DPO_OK;
}

extern "C" int dpo_ffn_forward(const dpo_ffn_args *args, void *cuda_stream)
{
    const char *what = "dpo_ffn_forward";
    if (args == nullptr)
        return call_fail(DPO_EINVAL, "%s: no arguments", what);
    const dpo_ffn_args &a = *args;
    int rc = check_sizes(what, a.tokens, a.dim, a.hidden);
    if (rc != DPO_OK)
        return rc;
    if ((a.act != DPO_ACT_SILU && a.act != DPO_ACT_GELU) ||
        (a.keep != DPO_KEEP_NONE && a.keep != DPO_KEEP_8BIT && a.keep != DPO_KEEP_BF16))
        return call_fail(DPO_EINVAL, "%s: act %d, keep %d", what, a.act, a.keep);
    const int64_t T = a.tokens, D = a.dim, F = a.hidden;
    if (T == 0)
        return DPO_OK;
    const int64_t need = hidden_bytes(T, F);
    if (a.workspace != nullptr && a.workspace_bytes < need)
        return call_fail(DPO_EINVAL, "%s: workspace of %lld bytes, %lld needed", what,
                         (long long)a.workspace_bytes, (long long)need);
    Buffers b(what);
    b.add("x", a.x, T, D, a.ld_x, 2, 16, false);
    b.add("w_gate", a.w_gate, F, D, D, 2, 16, false);
    b.add("w_up", a.w_up, F, D, D, 2, 16, false);
    b.add("w_down", a.w_down, D, F, F, 2, 16, false);
    b.add("out", a.out, T, D, a.ld_out, 2, 16, true);
    b.add("workspace", a.workspace, 1, need, need, 1, 256, true);
    if (a.keep == DPO_KEEP_8BIT) {
        b.packed("gate8", a.gate8, T, F, 16, true);
        b.packed("up8", a.up8, T, F, 16, true);
        if (b.rc == DPO_OK && a.gate8.ld_scales != a.up8.ld_scales)
            b.rc = call_fail(DPO_EINVAL, "%s: gate8 and up8 have different scale pitches", what);
    } else if (a.keep == DPO_KEEP_BF16) {
        b.add("gate", a.gate, T, F, F, 2, 16, true);
        b.add("up", a.up, T, F, F, 2, 16, true);
    }
    if ((rc = b.done()) != DPO_OK)
        return rc;
    const Device *d = nullptr;
    if ((rc = device_info(what, &d)) != DPO_OK)
        return rc;

    {
        const Shape s = {T, F, D, 1};
        const int cg = form_of(*d, &s, 1, kGate);
        Launch L{};
        Maps m;
        Product &P = L.p[0];
        m.operand(&P.a[0], a.x, T, D, a.ld_x, BM);
        m.operand(&P.b[0], a.w_gate, F, D, D, cg == 2 ? BH : BH / 2);
        m.operand(&P.b[1], a.w_up, F, D, D, cg == 2 ? BH : BH / 2);
        m.bf16(&P.d0, a.workspace, T, F, F);
        if (a.keep == DPO_KEEP_8BIT) {
            m.codes(&P.d1, a.gate8.codes, T, F, a.gate8.ld_codes);
            m.codes(&P.d2, a.up8.codes, T, F, a.up8.ld_codes);
            P.scale_g = a.gate8.scales;
            P.scale_u = a.up8.scales;
            P.ld_scale = a.gate8.ld_scales;
        } else if (a.keep == DPO_KEEP_BF16) {
            m.bf16(&P.d1, a.gate, T, F, F);
            m.bf16(&P.d2, a.up, T, F, F);
        }
        P.keep = a.keep;
        P.act = a.act;
        if ((rc = run(what, *d, L, &s, 1, kGate, cg, m.ok, cuda_stream)) != DPO_OK)
            return rc;
    }
    const Shape s = {T, D, F, 1};
    Launch L{};
    Maps m;
    m.operand(&L.p[0].a[0], a.workspace, T, F, F, BM);
    m.operand(&L.p[0].b[0], a.w_down, D, F, F, BH);
    m.bf16(&L.p[0].d0, a.out, T, D, a.ld_out);
    return run(what, *d, L, &s, 1, kStore, form_of(*d, &s, 1, kStore), m.ok, cuda_stream);
}

extern "C" int dpo_ffn_backward(const dpo_ffn_backward_args *args, void *cuda_stream)
{
    const char *what = "dpo_ffn_backward";
    if (args == nullptr)
        return call_fail(DPO_EINVAL, "%s: no arguments", what);
    const dpo_ffn_backward_args &a = *args;
    int rc = check_sizes(what, a.tokens, a.dim, a.hidden);
    if (rc != DPO_OK)
        return rc;
    if ((a.act != DPO_ACT_SILU && a.act != DPO_ACT_GELU) ||
        (a.keep != DPO_KEEP_8BIT && a.keep != DPO_KEEP_BF16))
        return call_fail(DPO_EINVAL, "%s: act %d, keep %d", what, a.act, a.keep);
    if ((a.grad_dtype != DPO_F32 && a.grad_dtype != DPO_BF16) ||
        (a.gain != nullptr && a.gain_dtype != DPO_F32 && a.gain_dtype != DPO_BF16))
        return call_fail(DPO_EDTYPE, "%s: grad dtype %d, gain dtype %d", what, a.grad_dtype,
                         a.gain_dtype);
    const int64_t T = a.tokens, D = a.dim, F = a.hidden;
    const int64_t gsize = a.grad_dtype == DPO_F32 ? 4 : 2;
    Buffers b(what);
    b.add("dw_gate", a.dw_gate, F, D, D, gsize, 16, true);
    b.add("dw_up", a.dw_up, F, D, D, gsize, 16, true);
    b.add("dw_down", a.dw_down, D, F, F, gsize, 16, true);
    if (T == 0) {
        if ((rc = b.done()) != DPO_OK || a.accumulate)
            return rc;
        for (void *p : {a.dw_gate, a.dw_up, a.dw_down}) {
            const cudaError_t e = cudaMemsetAsync(p, 0, (size_t)(D * F * gsize),
                                                  static_cast<cudaStream_t>(cuda_stream));
            if (e != cudaSuccess)
                return call_fail(DPO_ECUDA, "%s: %s", what, cudaGetErrorString(e));
        }
        return DPO_OK;
    }
    const bool from_x8 = a.x == nullptr;
    const int64_t hb = hidden_bytes(T, F), need = 3 * hb + (from_x8 ? align_up(T * D * 2) : 0);
    if (a.workspace != nullptr && a.workspace_bytes < need)
        return call_fail(DPO_EINVAL, "%s: workspace of %lld bytes, %lld needed", what,
                         (long long)a.workspace_bytes, (long long)need);
    b.add("dout", a.dout, T, D, a.ld_dout, 2, 16, false);
    b.add("w_gate", a.w_gate, F, D, D, 2, 16, false);
    b.add("w_up", a.w_up, F, D, D, 2, 16, false);
    b.add("w_down", a.w_down, D, F, F, 2, 16, false);
    b.add("workspace", a.workspace, 1, need, need, 1, 256, true);
    if (from_x8) {
        b.packed("x8", a.x8, T, D, 1, false);
        if (a.gain != nullptr)
            b.add("gain", a.gain, 1, D, D, a.gain_dtype == DPO_F32 ? 4 : 2,
                  a.gain_dtype == DPO_F32 ? 4 : 2, false);
    } else {
        b.add("x", a.x, T, D, a.ld_x, 2, 16, false);
        if (b.rc == DPO_OK && a.gain != nullptr)
            b.rc = call_fail(DPO_EINVAL, "%s: a gain goes with x8, not with x", what);
    }
    if (a.keep == DPO_KEEP_8BIT) {
        b.packed("gate8", a.gate8, T, F, 16, false);
        b.packed("up8", a.up8, T, F, 16, false);
        if (b.rc == DPO_OK && (a.gate8.ld_scales != a.up8.ld_scales || a.gate8.ld_codes != a.up8.ld_codes))
            b.rc = call_fail(DPO_EINVAL, "%s: gate8 and up8 have different pitches", what);
    } else {
        b.add("gate", a.gate, T, F, F, 2, 16, false);
        b.add("up", a.up, T, F, F, 2, 16, false);
    }
    if (a.dx != nullptr)
        b.add("dx", a.dx, T, D, a.ld_dx, 2, 16, true);
    if ((rc = b.done()) != DPO_OK)
        return rc;
    const Device *d = nullptr;
    if ((rc = device_info(what, &d)) != DPO_OK)
        return rc;

    uint8_t *ws = static_cast<uint8_t *>(a.workspace);
    void *dg = ws, *du = ws + hb, *act = ws + 2 * hb;
    const void *x = a.x;
    int64_t ld_x = a.ld_x;
    if (from_x8) {
        if ((rc = dpo_unpack8(&a.x8, T, D, ws + 3 * hb, DPO_BF16, D, cuda_stream)) != DPO_OK)
            return rc;
        x = ws + 3 * hb;
        ld_x = D;
    }
    {
        const Shape s = {T, F, D, 1};
        Launch L{};
        Maps m;
        Product &P = L.p[0];
        m.operand(&P.a[0], a.dout, T, D, a.ld_dout, BM);
        m.operand(&P.b[0], a.w_down, D, F, F, kBoxK);
        P.b_mn = 1;
        m.bf16(&P.d0, dg, T, F, F);
        m.bf16(&P.d1, du, T, F, F);
        m.bf16(&P.d2, act, T, F, F);
        if (a.keep == DPO_KEEP_8BIT) {
            P.kept_g = a.gate8.codes;
            P.kept_u = a.up8.codes;
            P.ld_kept = a.gate8.ld_codes;
            P.scale_g = a.gate8.scales;
            P.scale_u = a.up8.scales;
            P.ld_scale = a.gate8.ld_scales;
        } else {
            P.kept_g = a.gate;
            P.kept_u = a.up;
            P.ld_kept = F;
        }
        P.keep = a.keep;
        P.act = a.act;
        if ((rc = run(what, *d, L, &s, 1, kGateBack, form_of(*d, &s, 1, kGateBack), m.ok,
                      cuda_stream)) != DPO_OK)
            return rc;
    }
    Launch L{};
    Shape s[kMaxProducts];
    Maps m;
    int n = 0;
    if (a.dx != nullptr) {
        Product &P = L.p[n];
        s[n++] = {T, D, F, 2};
        m.operand(&P.a[0], dg, T, F, F, BM);
        m.operand(&P.a[1], du, T, F, F, BM);
        m.operand(&P.b[0], a.w_gate, F, D, D, kBoxK);
        m.operand(&P.b[1], a.w_up, F, D, D, kBoxK);
        P.b_mn = 1;
        m.bf16(&P.d0, a.dx, T, D, a.ld_dx);
    }
    struct {
        const void *left, *right;
        int64_t ld_left, ld_right, rows, cols;
        void *dw;
        bool gain;
    } const dw[3] = {{dg, x, F, ld_x, F, D, a.dw_gate, true},
                     {du, x, F, ld_x, F, D, a.dw_up, true},
                     {a.dout, act, a.ld_dout, F, D, F, a.dw_down, false}};
    for (const auto &w : dw) {
        Product &P = L.p[n];
        s[n++] = {w.rows, w.cols, T, 1};
        m.operand(&P.a[0], w.left, T, w.rows, w.ld_left, kBoxK);
        m.operand(&P.b[0], w.right, T, w.cols, w.ld_right, kBoxK);
        P.a_mn = P.b_mn = 1;
        if (a.grad_dtype == DPO_F32)
            m.f32(&P.d0, w.dw, w.rows, w.cols, w.cols);
        else
            m.bf16(&P.d0, w.dw, w.rows, w.cols, w.cols);
        P.f32 = a.grad_dtype == DPO_F32;
        P.accumulate = a.accumulate != 0;
        P.old = w.dw;
        P.ld_old = w.cols;
        if (w.gain && from_x8) {
            P.gain = a.gain;
            P.gain_f32 = a.gain_dtype == DPO_F32;
        }
    }
    return run(what, *d, L, s, n, kStore, form_of(*d, s, n, kStore), m.ok, cuda_stream);
}

extern "C" int dpo_ffn_get_status(uint32_t *bits)
{
    const char *what = "dpo_ffn_get_status";
    if (bits == nullptr)
        return call_fail(DPO_EINVAL, "%s: no result", what);
    const Device *d = nullptr;
    const int rc = device_info(what, &d);
    if (rc != DPO_OK)
        return rc;
    cudaError_t e = cudaDeviceSynchronize();
    if (e == cudaSuccess)
        e = cudaMemcpy(bits, d->err, sizeof *bits, cudaMemcpyDeviceToHost);
    return e == cudaSuccess ? DPO_OK : call_fail(DPO_ECUDA, "%s: %s", what, cudaGetErrorString(e));
}

extern "C" int dpo_ffn_clear_status(void *cuda_stream)
{
    const char *what = "dpo_ffn_clear_status";
    const Device *d = nullptr;
    const int rc = device_info(what, &d);
    if (rc != DPO_OK)
        return rc;
    const cudaError_t e = cudaMemsetAsync(d->err, 0, sizeof(unsigned int),
                                          static_cast<cudaStream_t>(cuda_stream));
    return e == cudaSuccess ? DPO_OK : call_fail(DPO_ECUDA, "%s: %s", what, cudaGetErrorString(e));
}
