// dpo_ffn.cu -- the gated feed-forward block, forward and backward
// (dpo_ffn_forward, dpo_ffn_backward in include/dpo.h): argument checks and the
// launches of the tensor-core kernel of dpo_ffn_gemm.cuh.
//
// Forward, two launches:   A = act(x w_gate^T) (x w_up^T), both projections in one;
//                          out = A w_down^T
// Backward, two launches:  dG, dU, A from dA = dout w_down and what was kept;
//                          dx, dw_gate, dw_up, dw_down, one list of tiles
// (one more where dx is better off alone, and one to widen the 8-bit rows when the block's
// input was kept so).
// What passes from one launch to the next, A, dG and dU, is rounded to bf16, the operand type of
// the product that reads it: results are 0.0023 to 0.0025 off in the norm, where their own
// rounding alone leaves 0.0017. As pairs of bf16 numbers they would hold 16 bits, for twice
// the MMAs and bytes of the down product, of dx and of the weights' gradients.
#include "dpo.h"
#include "dpo_check.h"
#include "dpo_ffn_few.cuh"
#include "dpo_products.h"

#include <cuda_runtime.h>

#include <mutex>
#include <type_traits>

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
constexpr int kForms = 6;   // epilogues

// What the launches need to know of a device, found by its first call.
struct Device {
    bool ready = false;
    int sms = 0;
    unsigned int *err = nullptr;
    // what is resident of each kernel at once: pairs, single CTAs, and clusters that split a
    // tile's K by 1, 2, 4, 8
    int pairs[kForms] = {}, singles[kForms] = {}, clusters[4][kForms] = {};
};
constexpr int kMaxDevices = 64;
std::mutex g_mu;
Device g_devices[kMaxDevices];
EncodeTiled g_encode = nullptr;

// How a launch's tiles are taken: by CTA pairs (cg 2), by single CTAs (cg 1), or by
// clusters of `ways` CTAs that split a tile's K (thin).
struct Form {
    int cg;
    bool thin;
    int ways, a_rows, cols;       // rows of A a stage loads, a tile's columns
    int cluster() const { return cg * ways; }
    int bk() const { return thin ? Ring<true>::BK : Ring<false>::BK; }
    int smem() const { return thin ? Ring<true>::smem(a_rows, cols) : Ring<false>::smem(BM, BH); }
};
constexpr Form kPairs = {2, false, 1, BM, kTile(2)};
Form single(int a_rows) { return {1, false, 1, a_rows, kTile(1)}; }
Form thin(int ways, int a_rows, int cols) { return {1, true, ways, a_rows, cols}; }

int slots_of(const Device &d, Form f, int epi)
{
    return f.cg == 2 ? d.pairs[epi]
           : f.thin  ? d.clusters[__builtin_ctz((unsigned)f.ways)][epi] : d.singles[epi];
}

template <int CG, bool SPLIT> KernelFn kernel_of(int epi)
{
    if constexpr (!SPLIT) {
        if (epi == kShared)
            return ffn_gemm_kernel<CG, kShared, SPLIT>;
        if (epi == kHead)
            return ffn_gemm_kernel<CG, kHead, SPLIT>;
    }
    return epi == kGate         ? ffn_gemm_kernel<CG, kGate, SPLIT>
           : epi == kGateBack8  ? ffn_gemm_kernel<CG, kGateBack8, SPLIT>
           : epi == kGateBack16 ? ffn_gemm_kernel<CG, kGateBack16, SPLIT>
                                : ffn_gemm_kernel<CG, kStore, SPLIT>;
}
KernelFn kernel_of(Form f, int epi)
{
    return f.cg == 2 ? kernel_of<2, false>(epi) : f.thin ? kernel_of<1, true>(epi) : kernel_of<1, false>(epi);
}

cudaLaunchAttribute cluster_of(int n)
{
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)n;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    return attr;
}

// A launch of `ctas` CTAs in clusters, overlapping the tail of the one before it
// (launch_pdl of dpo_internal.h).
template <class A>
int launch_clusters(const char *what, void (*kernel)(A), int64_t ctas, int cluster, int threads,
                    size_t smem, void *stream, const typename std::remove_const<A>::type &args)
{
    cudaLaunchAttribute attr[2] = {cluster_of(cluster), {}};
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = static_cast<cudaStream_t>(stream);
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args);
    const cudaError_t last = cudaGetLastError();
    e = e != cudaSuccess ? e : last;
    return e == cudaSuccess ? DPO_OK : call_fail(DPO_ECUDA, "%s: %s", what, cudaGetErrorString(e));
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
    // (every form of a kernel has an SM to itself)
    for (const Form f : {kPairs, single(BM), thin(1, BM, BH), thin(2, BM, BH), thin(4, BM, BH),
                         thin(8, BM, BH)})
        for (int epi = 0; epi < kForms; ++epi) {
            if (f.thin && epi >= kShared)   // K is not split there
                continue;
            const void *k = reinterpret_cast<const void *>(kernel_of(f, epi));
            cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                 kMaxSmem);
            if (e != cudaSuccess)
                return e;
            cudaLaunchAttribute attr = cluster_of(f.cluster());
            cudaLaunchConfig_t cfg{};
            cfg.gridDim = dim3(1024);
            cfg.blockDim = dim3(kThreads);
            cfg.dynamicSmemBytes = (size_t)f.smem();
            cfg.attrs = &attr;
            cfg.numAttrs = 1;
            int &n = f.cg == 2 ? d.pairs[epi]
                     : f.thin  ? d.clusters[__builtin_ctz((unsigned)f.ways)][epi] : d.singles[epi];
            e = cudaOccupancyMaxActiveClusters(&n, k, &cfg);
            if (e != cudaSuccess)
                return e;
            if (n < 1)
                return cudaErrorInvalidConfiguration;
        }
    void *p = nullptr;
    cudaError_t e = cudaGetSymbolAddress(&p, g_ffn_err);
    int device = 0;
    if (e == cudaSuccess)
        e = cudaGetDevice(&device);
    if (e == cudaSuccess)
        e = cudaDeviceGetAttribute(&d.sms, cudaDevAttrMultiProcessorCount, device);
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

int64_t blocks_of(int64_t k, int bk) { return (k + bk - 1) / bk; }

// A product's sizes, before its operands.
struct Shape {
    int64_t m, n, k;    // kGate: n of one projection
    int segments;
    int ways = 1;       // shares of K, each a tile of its own (Product::ways)
};

int64_t m_tiles(const Shape &s, const Form &f) { return (s.m + kTile(f.cg) - 1) / kTile(f.cg); }
int64_t n_tiles(const Shape &s, const Form &f, int epi)
{
    const int64_t tn = epi == kGate ? f.cols / 2 : f.cols;
    return (s.n + tn - 1) / tn;
}
int64_t tiles_of(const Shape &s, const Form &f, int epi) { return m_tiles(s, f) * n_tiles(s, f, epi) * s.ways; }

// The form of a launch: the one with the smallest estimate of its time in ns, tiles dealt
// in rounds. A K block costs a single CTA the stage's bytes at 154 a ns, or its instructions,
// and a pair 500; the exchange of a split tile's sums adds to each round, with the CTAs that
// take part, and 3.2 us at the end. (The weights' way from HBM is the same for all forms.) In
// a list of products the tiles' stores may take longer than few K blocks. K is split only
// where a launch is one product. The numbers are fitted to GB300's measured alternatives, all
// forms forced in turn, 9 to 1001 tokens, four pairs of widths, each product of forward and
// backward: within 2.3 us of the best one, or 2 % of the block.
struct Choice {
    Form form;
    double time;
};
// whole: no split of K (outputs in fp32 or added, A M-contiguous); a_mn: A is M-contiguous, its boxes whole.
Choice form_of(const Device &d, const Shape *s, int n, int epi, bool whole = false, bool a_mn = false)
{
    const int a_rows = a_mn ? BM : s[0].m <= 32 ? 32 : s[0].m <= 64 ? 64 : BM;
    const Form forms[] = {single(n == 1 ? a_rows : BM), thin(1, a_rows, BH), thin(2, a_rows, BH),
                          thin(4, a_rows, BH), thin(8, a_rows, BH), thin(1, a_rows, BH / 2),
                          thin(2, a_rows, BH / 2), thin(4, a_rows, BH / 2),
                          thin(8, a_rows, BH / 2), kPairs};
    Choice best = {kPairs, 1e30};
    for (const Form &f : forms) {
        const double bytes = (double)(f.a_rows + f.cols) * f.bk() * 2;
        const double copy = bytes / 154.0, issue = f.thin ? 110.0 : 365.0;
        const double block = f.cg == 2 ? 500.0 : copy > issue ? copy : issue;
        const double epilogue = f.cg == 2 ? 370.0 : f.thin ? 3200.0 : 240.0;
        const double store = n == 1 ? 0.0 : f.cg == 2 ? 1850.0 : 1000.0;
        const double exchange = 400.0 + 73.0 * f.ways;
        const int64_t slots = slots_of(d, f, epi);
        int64_t tiles = 0;
        double work = 0.0, longest = 0.0;
        for (int i = 0; i < n; ++i)
            tiles += tiles_of(s[i], f, epi);
        if (f.thin && (whole || n > 1 || blocks_of(s[0].k, f.bk()) < 2 * f.ways))
            continue;
        for (int i = 0; i < n; ++i) {
            const int64_t blocks = (blocks_of(s[i].k, f.bk()) * s[i].segments + s[i].ways - 1) / s[i].ways;
            const double c = (double)((blocks + f.ways - 1) / f.ways) * block;
            const double each = f.thin ? c + exchange : c > store ? c : store;
            work += (double)tiles_of(s[i], f, epi) * each;
            longest = longest > each ? longest : each;
        }
        // whole rounds of equal tiles, or the longest one's end
        double time = n == 1 ? (double)((tiles + slots - 1) / slots) * longest : work / (double)slots;
        time = (time > longest ? time : longest) * 1.02 + epilogue;
        if (time < best.time)
            best = {f, time};
    }
    return best;
}

// The products of a call of T tokens, D dim and F hidden.
Shape gate_shape(int64_t T, int64_t D, int64_t F) { return {T, F, D, 1}; }   // its backward too
Shape down_shape(int64_t T, int64_t D, int64_t F) { return {T, D, F, 1}; }
struct Gradients {   // dx, then the weights'
    Shape s[kMaxProducts];
};
Gradients gradient_shapes(int64_t T, int64_t D, int64_t F)
{
    return {{{T, D, F, 2}, {F, D, T, 1}, {F, D, T, 1}, {D, F, T, 1}}};
}
// dx with the weights' gradients in one list, or, where its few long tiles would be what the
// list waits for, before them with K split (1B widths, 9 tokens: its tiles have 128 blocks,
// the gradients' one).
struct DxChoice {
    bool alone;
    Form form;      // of its own launch
};
DxChoice dx_form(const Device &d, const Gradients &g)
{
    const Choice all = form_of(d, g.s, 4, kStore), dx = form_of(d, g.s, 1, kStore);
    return {dx.form.thin && dx.time + form_of(d, g.s + 1, 3, kStore).time + 2000.0 < all.time, dx.form};
}
// The forward's products by streaming the weights (dpo_ffn_few.cuh). It has no 8-bit form: a
// scale's group of 32 columns lies in four of its CTAs. (1 token kept in 8 bits, by the
// forms of few tiles: 7B widths 59.7 us, 47.6 streamed with nothing kept; 1B 27.1, 20.1.)
bool streamed(int64_t tokens, int keep) { return tokens <= kFewTokens && keep != DPO_KEEP_8BIT; }

int run(const char *what, const Device &d, Launch &L, const Shape *s, int n, int epi, Form f,
        bool followed, bool maps_ok, void *stream)
{
    if (!maps_ok)
        return call_fail(DPO_ECUDA, "%s: a tensor map was refused", what);
    int64_t total = 0;
    for (int i = 0; i < n; ++i) {
        Product &P = L.p[i];
        P.m = (int)s[i].m;
        P.n = (int)s[i].n;
        P.k_blocks[0] = (int)blocks_of(s[i].k, f.bk());
        P.k_blocks[1] = s[i].segments == 2 ? P.k_blocks[0] : 0;
        P.m_tiles = (int)m_tiles(s[i], f);
        P.n_tiles = (int)n_tiles(s[i], f, epi);
        P.first = (int)total;
        P.ways = s[i].ways;
        total += tiles_of(s[i], f, epi);
    }
    L.n_products = n;
    L.n_tiles = (int)total;
    L.err = d.err;
    L.a_rows = f.a_rows;
    L.cols = f.cols;
    const int64_t slots = slots_of(d, f, epi);
    L.early = followed;
    return launch_clusters(what, kernel_of(f, epi), (total < slots ? total : slots) * f.cluster(),
                           f.cluster(), kThreads, (size_t)f.smem(), stream, L);
}

// ---- few tokens ----

// One product of the forward for at most kFewTokens tokens. K is split over a cluster as far
// as all CTAs are resident at once (one more doubling, 1 token: 7B 49.3 -> 51.4 us, 1B
// 20.6 -> 23.3; one less: 52.7, 22.7) and every warp keeps 64 of k.
int run_few(const char *what, FewArgs a, int epi, int sms, void *stream)
{
    const int rows = epi == kGate ? 8 : 16;
    const int64_t units = (a.rows + rows - 1) / rows;
    int split = 1;
    while (split < 8 && units * split * 2 <= (int64_t)sms * kFewCtas && a.k > split * kFewWarps * 64)
        split *= 2;
    const int64_t ctas = units * split, resident = (int64_t)sms * kFewCtas;
    a.ahead.ctas = (int)(ctas < resident ? ctas : resident);
    return launch_clusters(what, epi == kGate ? few_kernel<kGate> : few_kernel<kStore>,
                           ctas, split, kFewThreads, 0, stream, a);
}

// What the first product reads ahead of a weight matrix: up to 24 MB, evenly over its rows
// (1 and 8 tokens: 7B 49.4 -> 48.5 us, 53.5 -> 52.5; 1B 21.1 -> 20.5, 23.6 -> 22.5; 8 and 48 MB
// less of it. Before the split tiles of dpo_ffn_gemm.cuh it delays the first product by as
// much as the second one gains).
Ahead ahead_of(const void *w, int64_t rows, int64_t cols)
{
    constexpr int64_t kBytes = (int64_t)24 << 20;
    const int64_t share = kBytes / rows / 128 * 128, bytes = cols * 2 < share ? cols * 2 : share;
    return {static_cast<const uint8_t *>(w), cols * 2, bytes > 0 ? (int)rows : 0, (int)bytes, 0};
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
        fits = fits && tiles_of(q, kPairs, kGate) < ((int64_t)1 << 28);
    if (!fits)
        return call_fail(DPO_EINVAL, "%s: %lld x %lld x %lld is too large", what, (long long)tokens,
                         (long long)dim, (long long)hidden);
    return DPO_OK;
}

}  // namespace

namespace {

int64_t slab_rows(int64_t m) { return (m + kTile(2) - 1) / kTile(2) * kTile(2); }

}  // namespace

int dpo::product_ways(int64_t m, int64_t n, int64_t k)
{
    constexpr int64_t kPlanned = 76;
    const int64_t tiles = (m + 255) / 256 * ((n + 255) / 256), blocks = (k + 127) / 128;
    const int64_t other = (k + 255) / 256 * ((n + 255) / 256), each = (m + 127) / 128;
    const double all = (double)(tiles * blocks + other * (each > 4 ? each : 4)) / kPlanned;
    const int64_t ways = (int64_t)((double)blocks / (0.8 * all) + 0.999);
    const int64_t most = blocks / 8 < 16 ? blocks / 8 : 16;
    return ways < 1 || most < 2 ? 1 : (int)(ways < most ? ways : most);
}
int64_t dpo::product_share_bytes(int64_t m, int64_t n, int64_t k)
{
    const int ways = product_ways(m, n, k);
    return ways > 1 ? ways * slab_rows(m) * n * 4 : 0;
}

int dpo::store_products(const char *what, const StoreProduct *p, int n, void *stream)
{
    const Device *d = nullptr;
    int rc = device_info(what, &d);
    if (rc != DPO_OK)
        return rc;
    static_assert(kMaxStoreProducts == kMaxProducts, "products of a launch");
    if (n < 1 || n > kMaxStoreProducts || (p[0].shares != nullptr && (p[0].f32 || p[0].accumulate)))
        return call_fail(DPO_EINVAL, "%s: %d products", what, n);
    Shape s[kMaxProducts];
    auto whole = [&](int i) { return p[i].f32 || p[i].accumulate || p[i].a_mn; };
    for (int i = 0; i < n; ++i)
        s[i] = {p[i].m, p[i].n, p[i].k, 1};
    auto choose = [&](int i, int count) {
        bool a_mn = false;
        for (int j = i; j < i + count; ++j)
            a_mn = a_mn || p[j].a_mn;
        return form_of(*d, s + i, count, kStore, count > 1 || whole(i), a_mn);
    };
    Choice all = choose(0, n);
    // the first product, where its few long tiles would be what the list waits for, on its own with its
    // K split over clusters (dx_form), or in shares that are tiles of the list
    int first = 0;
    if (n > 1) {
        const Choice one = choose(0, 1), rest = choose(1, n - 1);
        const bool alone = one.form.thin && one.time + rest.time + 2000.0 < all.time;
        if (alone)
            all.time = one.time + rest.time + 2000.0;
        if (p[0].shares != nullptr) {
            s[0].ways = product_ways(p[0].m, p[0].n, p[0].k);
            const Choice shared = choose(0, n);
            const double sums = 4000.0 + (double)product_share_bytes(p[0].m, p[0].n, p[0].k) / 2500.0;
            if (s[0].ways > 1 && shared.time + sums < all.time)
                all = shared;
            else
                s[0].ways = 1;
        }
        if (alone && s[0].ways == 1) {
            if ((rc = store_products(what, p, 1, stream)) != DPO_OK)
                return rc;
            first = 1;
            all = rest;
        }
    }
    const Form f = all.form;
    Launch L{};
    Maps m;
    for (int i = first; i < n; ++i) {
        const StoreProduct &q = p[i];
        Product &P = L.p[i - first];
        P.a_mn = q.a_mn;
        P.b_mn = q.b_mn;
        if (q.a_mn)
            m.operand(&P.a[0], q.a, q.k, q.m, q.ld_a, f.bk());
        else
            m.operand(&P.a[0], q.a, q.m, q.k, q.ld_a, f.a_rows);
        if (q.b_mn)
            m.operand(&P.b[0], q.b, q.k, q.n, q.ld_b, f.bk());
        else
            m.operand(&P.b[0], q.b, q.n, q.k, q.ld_b, f.cg == 2 ? BH : f.cols);
        const bool shared = s[i].ways > 1;
        if (shared)
            m.f32(&P.d0, q.shares, s[i].ways * slab_rows(q.m), q.n, q.n);
        else if (q.f32)
            m.f32(&P.d0, q.out, q.m, q.n, q.ld_out);
        else
            m.bf16(&P.d0, q.out, q.m, q.n, q.ld_out);
        P.slab = shared ? (int)slab_rows(q.m) : 0;
        P.f32 = shared || q.f32;
        P.accumulate = q.accumulate;
        P.old = q.out;
        P.ld_old = P.ld_o = q.ld_out;
        P.o0 = static_cast<__nv_bfloat16 *>(q.out);
    }
    int epi = s[0].ways > 1 ? kShared : kStore;
    if (n - first == 2) {   // deal by length
        const int64_t slots = slots_of(*d, f, kShared), longs = tiles_of(s[first], f, kShared),
                      shorts = tiles_of(s[first + 1], f, kShared), fewer = longs % slots;
        const int64_t a = blocks_of(s[first].k, f.bk()) / s[first].ways, b = blocks_of(s[first + 1].k, f.bk());
        if (fewer > 0 && longs + shorts > slots && a >= 2 * b) {
            const int64_t most = shorts / (slots - fewer), want = a / (b > 4 ? b : 4);   // 4: its store
            L.longs = (int)longs;
            L.extra = (int)(want < most ? want : most);
            if (L.extra > 0)
                epi = kShared;
        }
    }
    if ((rc = run(what, *d, L, s + first, n - first, epi, f, false, m.ok, stream)) != DPO_OK ||
        s[0].ways == 1)
        return rc;
    const StoreProduct &q = p[0];
    return launch(what, sum_shares_kernel, (q.m * (q.n / 8) + kSumThreads - 1) / kSumThreads, kSumThreads, 0,
                  stream, static_cast<const float *>(q.shares), static_cast<__nv_bfloat16 *>(q.out), q.m, q.n,
                  q.ld_out, slab_rows(q.m) * q.n, s[0].ways);
}

int dpo::head_product(const char *what, const HeadProduct &h, void *stream)
{
    const Device *d = nullptr;
    int rc = device_info(what, &d);
    if (rc != DPO_OK)
        return rc;
    const Shape s = {h.tokens, h.vocab, h.dim, 1};
    const Form f = form_of(*d, &s, 1, kHead, true).form;
    Launch L{};
    Maps m;
    Product &P = L.p[0];
    m.operand(&P.a[0], h.x, h.tokens, h.dim, h.ld_x, f.a_rows);
    m.operand(&P.b[0], h.w, h.vocab, h.dim, h.dim, f.cg == 2 ? BH : f.cols);
    if (h.kept != nullptr)
        m.bf16(&P.d0, h.kept, blocks_of(h.vocab, kHeadStatCols) * h.kept_rows, kHeadStatCols, kHeadStatCols);
    if (h.logits != nullptr)
        m.f32(&P.d1, h.logits, h.tokens, h.vocab, h.ld);
    P.head = {h.ids, h.scale, h.target, h.maxima, h.sums, h.tokens, h.maxima != nullptr, h.kept != nullptr,
              h.logits != nullptr, (int)h.kept_rows};
    return run(what, *d, L, &s, 1, kHead, f, false, m.ok, stream);
}

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

    if (streamed(T, a.keep)) {
        using E = __nv_bfloat16;
        FewArgs f{};
        f.x = static_cast<const E *>(a.x);
        f.w0 = static_cast<const E *>(a.w_gate);
        f.w1 = static_cast<const E *>(a.w_up);
        f.out = static_cast<E *>(a.workspace);
        if (a.keep == DPO_KEEP_BF16) {
            f.keep0 = static_cast<E *>(a.gate);
            f.keep1 = static_cast<E *>(a.up);
        }
        f.ld_x = a.ld_x;
        f.ld_out = F;
        f.tokens = (int)T;
        f.rows = (int)F;
        f.k = (int)D;
        f.act = a.act;
        f.ahead = ahead_of(a.w_down, D, F);
        if ((rc = run_few(what, f, kGate, d->sms, cuda_stream)) != DPO_OK)
            return rc;
        FewArgs o{};
        o.x = f.out;
        o.w0 = static_cast<const E *>(a.w_down);
        o.out = static_cast<E *>(a.out);
        o.ld_x = F;
        o.ld_out = a.ld_out;
        o.tokens = (int)T;
        o.rows = (int)D;
        o.k = (int)F;
        return run_few(what, o, kStore, d->sms, cuda_stream);
    }
    {
        const Shape s = gate_shape(T, D, F);
        const Form form = form_of(*d, &s, 1, kGate).form;
        const int rows_w = form.cg == 2 ? BH : form.cols / 2;   // a box of either projection
        Launch L{};
        Maps m;
        Product &P = L.p[0];
        m.operand(&P.a[0], a.x, T, D, a.ld_x, form.a_rows);
        m.operand(&P.b[0], a.w_gate, F, D, D, rows_w);
        m.operand(&P.b[1], a.w_up, F, D, D, rows_w);
        m.bf16(&P.d0, a.workspace, T, F, F);
        P.o0 = static_cast<__nv_bfloat16 *>(a.workspace);
        P.ld_o = F;
        if (a.keep == DPO_KEEP_8BIT) {
            m.codes(&P.d1, a.gate8.codes, T, F, a.gate8.ld_codes);
            m.codes(&P.d2, a.up8.codes, T, F, a.up8.ld_codes);
            P.scale_g = a.gate8.scales;
            P.scale_u = a.up8.scales;
            P.ld_scale = a.gate8.ld_scales;
            P.wide = reinterpret_cast<uintptr_t>(P.scale_g) % 2 == 0 &&
                     reinterpret_cast<uintptr_t>(P.scale_u) % 2 == 0 && P.ld_scale % 2 == 0;
            P.codes_g = a.gate8.codes;
            P.codes_u = a.up8.codes;
            P.ld_codes_g = a.gate8.ld_codes;
            P.ld_codes_u = a.up8.ld_codes;
        } else if (a.keep == DPO_KEEP_BF16) {
            m.bf16(&P.d1, a.gate, T, F, F);
            m.bf16(&P.d2, a.up, T, F, F);
            P.o1 = static_cast<__nv_bfloat16 *>(a.gate);
            P.o2 = static_cast<__nv_bfloat16 *>(a.up);
        }
        P.keep = a.keep;
        P.act = a.act;
        if ((rc = run(what, *d, L, &s, 1, kGate, form, true, m.ok, cuda_stream)) != DPO_OK)
            return rc;
    }
    const Shape s = down_shape(T, D, F);
    Launch L{};
    Maps m;
    const Form form = form_of(*d, &s, 1, kStore).form;
    m.operand(&L.p[0].a[0], a.workspace, T, F, F, form.a_rows);
    m.operand(&L.p[0].b[0], a.w_down, D, F, F, form.cg == 2 ? BH : form.cols);
    m.bf16(&L.p[0].d0, a.out, T, D, a.ld_out);
    L.p[0].o0 = static_cast<__nv_bfloat16 *>(a.out);
    L.p[0].ld_o = a.ld_out;
    return run(what, *d, L, &s, 1, kStore, form, false, m.ok, cuda_stream);
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
        // read in pieces of 8 codes; the forward's TMA stores want 16 bytes
        b.packed("gate8", a.gate8, T, F, 8, false);
        b.packed("up8", a.up8, T, F, 8, false);
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
    {
        const Shape s = gate_shape(T, D, F);
        const int epi = a.keep == DPO_KEEP_8BIT ? kGateBack8 : kGateBack16;
        const Form form = form_of(*d, &s, 1, epi).form;
        Launch L{};
        Maps m;
        Product &P = L.p[0];
        m.operand(&P.a[0], a.dout, T, D, a.ld_dout, form.a_rows);
        m.operand(&P.b[0], a.w_down, D, F, F, form.bk());
        P.b_mn = 1;
        m.bf16(&P.d0, dg, T, F, F);
        m.bf16(&P.d1, du, T, F, F);
        m.bf16(&P.d2, act, T, F, F);
        P.o0 = static_cast<__nv_bfloat16 *>(dg);
        P.o1 = static_cast<__nv_bfloat16 *>(du);
        P.o2 = static_cast<__nv_bfloat16 *>(act);
        P.ld_o = F;
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
        const int64_t size = a.keep == DPO_KEEP_8BIT ? 1 : 2;
        P.wide = F % 128 == 0 && reinterpret_cast<uintptr_t>(P.kept_g) % 32 == 0 &&
                 reinterpret_cast<uintptr_t>(P.kept_u) % 32 == 0 && P.ld_kept * size % 32 == 0 &&
                 (a.keep != DPO_KEEP_8BIT ||
                  (reinterpret_cast<uintptr_t>(P.scale_g) % 4 == 0 &&
                   reinterpret_cast<uintptr_t>(P.scale_u) % 4 == 0 && P.ld_scale % 4 == 0));
        if ((rc = run(what, *d, L, &s, 1, epi, form, true, m.ok, cuda_stream)) != DPO_OK)
            return rc;
    }
    if (from_x8) {   // needed by the next launch only: beside the one just made
        x = ws + 3 * hb;
        ld_x = D;
        if ((rc = unpack8_beside(a.x8, T, D, ws + 3 * hb, cuda_stream)) != DPO_OK)
            return rc;
    }
    Launch L{};
    const Gradients g = gradient_shapes(T, D, F);
    const Shape *const s = g.s;
    Maps m;
    int n = 0, first = 1;   // products of L, of s
    if (a.dx != nullptr) {
        const DxChoice dx = dx_form(*d, g);
        const bool alone = dx.alone;
        const Form f = alone ? dx.form : kPairs;
        Product &P = L.p[0];
        m.operand(&P.a[0], dg, T, F, F, f.a_rows);
        m.operand(&P.a[1], du, T, F, F, f.a_rows);
        m.operand(&P.b[0], a.w_gate, F, D, D, f.bk());
        m.operand(&P.b[1], a.w_up, F, D, D, f.bk());
        P.b_mn = 1;
        m.bf16(&P.d0, a.dx, T, D, a.ld_dx);
        P.o0 = static_cast<__nv_bfloat16 *>(a.dx);
        P.ld_o = a.ld_dx;
        if (!alone) {
            n = 1;
            first = 0;
        } else if ((rc = run(what, *d, L, s, 1, kStore, f, true, m.ok, cuda_stream)) != DPO_OK) {
            return rc;
        }
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
        Product &P = L.p[n++];
        P = Product{};
        m.operand(&P.a[0], w.left, T, w.rows, w.ld_left, kPairs.bk());
        m.operand(&P.b[0], w.right, T, w.cols, w.ld_right, kPairs.bk());
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
    return run(what, *d, L, s + first, n, kStore, form_of(*d, s + first, n, kStore).form, false, m.ok,
               cuda_stream);
}

extern "C" int dpo_ffn_test_forms(int64_t tokens, int64_t dim, int64_t hidden, int keep,
                                  const int *slots, dpo_ffn_form *forms)
{
    const char *what = "dpo_ffn_test_forms";
    int rc = check_sizes(what, tokens, dim, hidden);
    if (rc != DPO_OK)
        return rc;
    if (tokens == 0 || forms == nullptr ||
        (keep != DPO_KEEP_NONE && keep != DPO_KEEP_8BIT && keep != DPO_KEEP_BF16))
        return call_fail(DPO_EINVAL, "%s: tokens %lld, keep %d", what, (long long)tokens, keep);
    Device given;
    const Device *d = &given;
    if (slots == nullptr) {
        if ((rc = device_info(what, &d)) != DPO_OK)
            return rc;
    } else {
        for (int i = 0; i < 6; ++i)
            if (slots[i] < 1)
                return call_fail(DPO_EINVAL, "%s: %d slots", what, slots[i]);
        for (int e = 0; e < kForms; ++e) {
            given.pairs[e] = slots[0];
            given.singles[e] = slots[1];
            for (int i = 0; i < 4; ++i)
                given.clusters[i][e] = slots[2 + i];
        }
    }
    auto fill = [&](dpo_ffn_form &out, const Shape *s, int n, int epi, const Form &f) {
        int64_t tiles = 0;
        for (int i = 0; i < n; ++i)
            tiles += tiles_of(s[i], f, epi);
        out = {f.cg == 2 ? DPO_FFN_PAIRS : f.thin ? DPO_FFN_SPLIT : DPO_FFN_SINGLE, f.ways, f.cols, tiles,
               slots_of(*d, f, epi)};
    };
    const Shape gate = gate_shape(tokens, dim, hidden), down = down_shape(tokens, dim, hidden);
    if (streamed(tokens, keep)) {
        forms[0] = forms[1] = {DPO_FFN_STREAM, 0, 0, 0, 0};
    } else {
        fill(forms[0], &gate, 1, kGate, form_of(*d, &gate, 1, kGate).form);
        fill(forms[1], &down, 1, kStore, form_of(*d, &down, 1, kStore).form);
    }
    const int back = keep == DPO_KEEP_8BIT ? kGateBack8 : kGateBack16;
    fill(forms[2], &gate, 1, back, form_of(*d, &gate, 1, back).form);
    const Gradients g = gradient_shapes(tokens, dim, hidden);
    const DxChoice dx = dx_form(*d, g);
    forms[3] = {DPO_FFN_NO_LAUNCH, 0, 0, 0, 0};
    if (dx.alone)
        fill(forms[3], g.s, 1, kStore, dx.form);
    const int first = dx.alone ? 1 : 0, n = kMaxProducts - first;
    fill(forms[4], g.s + first, n, kStore, form_of(*d, g.s + first, n, kStore).form);
    return DPO_OK;
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
