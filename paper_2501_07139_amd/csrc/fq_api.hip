// C-ABI entry points of the device half: argument checks, dispatch, and the
// block/stack driver that applies a hybrid model's configuration vector
// (FlexQuant, arXiv 2501.07139, Section "EQM Generation Philosophy": each
// module takes its parameters from one stored quantized model).
#include "fq.h"
#include "fq_internal.h"

#include <hip/hip_runtime.h>

#include <mutex>

// Scratch of the entry point that must not allocate (fq_stack_forward_noalloc): the activations of a decode
// stack forward for up to 16 rows of up to 16384 elements.  Every device the library runs on holds its own
// copy of this array until the process ends.  In host code the array's name is only a handle: the device
// address comes from hipGetSymbolAddress (static_scratch below) and is what kernels and copies are given.
constexpr int kNoallocMaxM = 16, kNoallocMaxDim = 16384;
constexpr size_t kNoallocScratchBytes = (size_t)13 * kNoallocMaxM * kNoallocMaxDim * 2 + fq_decode_sync_bytes;
static __device__ __align__(256) unsigned char scratch[kNoallocScratchBytes];

namespace {

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int check_hip(int e, const char *what)
{
    if (e == 0)
        return FQ_OK;
    return fq_fail(FQ_ERR_HIP, "%s: %s", what, hipGetErrorString((hipError_t)e));
}

int check_matrix(const char *fn, const void *packed, const void *scales, const void *zeros, int N, int K,
                 int bits, int group)
{
    if (!packed || !scales || !zeros)
        return fq_fail(FQ_ERR_NULL, "%s: NULL weight pointer", fn);
    if (fq_bits_index(bits) < 0)
        return fq_fail(FQ_ERR_BITS, "%s: bits=%d not in {2,3,4,8}", fn, bits);
    if (group != 128)
        return fq_fail(FQ_ERR_GROUP, "%s: group=%d, only 128 is supported", fn, group);
    if (N <= 0 || K <= 0 || K % 128 != 0)
        return fq_fail(FQ_ERR_SHAPE, "%s: N=%d K=%d (K must be a positive multiple of 128)", fn, N, K);
    if (!aligned16(packed) || !aligned16(scales) || !aligned16(zeros))
        return fq_fail(FQ_ERR_ALIGN, "%s: weight pointers must be 16-byte aligned", fn);
    return FQ_OK;
}

// The tile kernels (M > 16) address each array through 32-bit byte offsets.
bool below_4gib(size_t a, size_t b, size_t elem_bytes) { return a * b * elem_bytes < ((size_t)1 << 32); }

int qlinear_checked(const void *x, int M, const fq_packed_ref &w, void *out, fq_stream st, int tile_rows = 0)
{
    if (M > 16 && (!below_4gib(M, w.K, 2) || !below_4gib(((size_t)w.N + 63) / 64 * 8, w.K, w.bits)))
        return fq_fail(FQ_ERR_SHAPE, "fq_qlinear: M=%d N=%d K=%d: activations and packed weights must each stay "
                       "below 4 GiB", M, w.N, w.K);
    int e = (M <= 16) ? fq_launch_gemv(x, M, w, out, st) : fq_launch_gemm(x, M, w, out, st, tile_rows);
    return check_hip(e, "fq_qlinear launch");
}

// The linears that share an input (q/k/v, gate/up) in one launch of the few-row or a tile kernel.
int qlinear_multi_checked(const void *x, int M, const fq_packed_ref *w, void *const *outs, int count, fq_stream st)
{
    for (int i = 0; i < count; ++i)
        if (!below_4gib(M, w[i].K, 2) || !below_4gib(((size_t)w[i].N + 63) / 64 * 8, w[i].K, w[i].bits))
            return fq_fail(FQ_ERR_SHAPE, "fq_stack_forward: M=%d N=%d K=%d: activations and packed weights must each "
                           "stay below 4 GiB", M, w[i].N, w[i].K);
    return check_hip(fq_launch_gemm_multi(x, M, w, outs, count, st), "fq_stack_forward linears");
}

constexpr int kMaxGlueH = 16384;

size_t align_up(size_t v) { return (v + 255) & ~(size_t)255; }

// Device address of `scratch` on the current device, looked up once per device with that device current.
int static_scratch(void **out)
{
    static void *ptr[16] = {};
    static std::mutex guard;
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess)
        return (int)e;
    if (dev < 0 || dev >= 16)
        return (int)hipErrorInvalidDevice;
    std::lock_guard<std::mutex> lock(guard);
    if (!ptr[dev]) {
        void *p = nullptr;
        e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
        if (e != hipSuccess)
            return (int)e;
        if (!p)
            return (int)hipErrorInvalidSymbol;
        ptr[dev] = p;
    }
    *out = ptr[dev];
    return 0;
}

} // namespace

extern "C" int fq_dequant(const void *packed, const void *scales, const void *zeros, int N, int K, int bits,
                          int group, void *out, int out_is_fp16, void *stream)
{
    if (int rc = check_matrix("fq_dequant", packed, scales, zeros, N, K, bits, group))
        return rc;
    if (!out)
        return fq_fail(FQ_ERR_NULL, "fq_dequant: NULL output");
    fq_packed_ref w{packed, scales, zeros, N, K, bits};
    return check_hip(fq_launch_dequant(w, out, out_is_fp16, static_cast<fq_stream>(stream)), "fq_dequant launch");
}

extern "C" int fq_qlinear(const void *x, int M, const void *packed, const void *scales, const void *zeros,
                          int N, int K, int bits, int group, void *out, void *stream)
{
    return fq_qlinear_tile(x, M, packed, scales, zeros, N, K, bits, group, out, 0, stream);
}

extern "C" int fq_qlinear_tile(const void *x, int M, const void *packed, const void *scales, const void *zeros,
                               int N, int K, int bits, int group, void *out, int tile_rows, void *stream)
{
    if (tile_rows != 0 && tile_rows != 128 && tile_rows != 256)
        return fq_fail(FQ_ERR_SHAPE, "fq_qlinear_tile: tile_rows=%d (0, 128 or 256)", tile_rows);
    if (int rc = check_matrix("fq_qlinear", packed, scales, zeros, N, K, bits, group))
        return rc;
    if (!x || !out)
        return fq_fail(FQ_ERR_NULL, "fq_qlinear: NULL activation or output pointer");
    if (M <= 0)
        return fq_fail(FQ_ERR_SHAPE, "fq_qlinear: M=%d", M);
    if (!aligned16(x) || !aligned16(out))
        return fq_fail(FQ_ERR_ALIGN, "fq_qlinear: x and out must be 16-byte aligned");
    fq_packed_ref w{packed, scales, zeros, N, K, bits};
    return qlinear_checked(x, M, w, out, static_cast<fq_stream>(stream), tile_rows);
}

namespace {

// The matrices of a launch as fq_qlinear_route and fq_qlinear_tall_tile are given them.
int route_matrices(const char *fn, int M, const int *N, const int *bits, int count, int K, fq_packed_ref *w)
{
    if (M <= 0 || count < 1 || count > 3 || K <= 0 || K % 128 != 0)
        return fq_fail(FQ_ERR_SHAPE, "%s: M=%d count=%d K=%d", fn, M, count, K);
    for (int i = 0; i < count; ++i) {
        if (N[i] <= 0 || fq_bits_index(bits[i]) < 0)
            return fq_fail(N[i] <= 0 ? FQ_ERR_SHAPE : FQ_ERR_BITS, "%s: N=%d bits=%d", fn, N[i], bits[i]);
        w[i] = fq_packed_ref{nullptr, nullptr, nullptr, N[i], K, bits[i]};
    }
    return FQ_OK;
}

} // namespace

extern "C" int fq_qlinear_route(int M, const int *N, const int *bits, int count, int K, int *route_out)
{
    if (!N || !bits || !route_out)
        return fq_fail(FQ_ERR_NULL, "fq_qlinear_route: NULL argument");
    fq_packed_ref w[3];
    if (int rc = route_matrices("fq_qlinear_route", M, N, bits, count, K, w))
        return rc;
    bool stream = true;
    for (int i = 0; i < count; ++i)
        stream = stream && fq_gemv_can_stream(M, K, bits[i], 0);
    route_out[1] = route_out[2] = 0;
    if (M <= 16 && !fq_skinny_pays(M, w, count)) {
        route_out[0] = stream ? FQ_ROUTE_STREAM : FQ_ROUTE_GENERIC;
        return FQ_OK;
    }
    const fq_gemm_plan plan = fq_plan_gemm(M, w, count);
    route_out[0] = plan.tile_rows == 0 ? FQ_ROUTE_FEW_ROWS : (plan.tile_rows == 256 ? FQ_ROUTE_TILES_256 : FQ_ROUTE_TILES_128);
    route_out[1] = plan.tile_rows == 0 ? 16 * plan.few.mb : plan.height;
    route_out[2] = plan.tile_rows == 0 ? 16 << plan.few.s_log2 : 128;
    return FQ_OK;
}

extern "C" int fq_qlinear_tall_tile(int M, const int *N, const int *bits, int count, int K, int row_tile, int *out4)
{
    if (!N || !bits || !out4)
        return fq_fail(FQ_ERR_NULL, "fq_qlinear_tall_tile: NULL argument");
    fq_packed_ref w[3];
    if (int rc = route_matrices("fq_qlinear_tall_tile", M, N, bits, count, K, w))
        return rc;
    if (!below_4gib(M, K, 2))
        return fq_fail(FQ_ERR_SHAPE, "fq_qlinear_tall_tile: M=%d K=%d: activations must stay below 4 GiB", M, K);
    out4[0] = fq_gemm_tall_tile(M, w, count, row_tile, &out4[1], &out4[2], &out4[3]);
    if (row_tile < 0 || row_tile >= out4[0])
        return fq_fail(FQ_ERR_SHAPE, "fq_qlinear_tall_tile: row_tile=%d of %d", row_tile, out4[0]);
    return FQ_OK;
}

extern "C" int fq_qlinear_mixed(const void *x, int M, const fq_segment *segments, int count, int K, int group,
                                void *out, void *stream)
{
    if (!segments || !x || !out)
        return fq_fail(FQ_ERR_NULL, "fq_qlinear_mixed: NULL argument");
    if (count < 1 || count > FQ_MAX_SEGMENTS)
        return fq_fail(FQ_ERR_SHAPE, "fq_qlinear_mixed: %d segments (1..%d)", count, FQ_MAX_SEGMENTS);
    if (M <= 0)
        return fq_fail(FQ_ERR_SHAPE, "fq_qlinear_mixed: M=%d", M);
    if (!aligned16(x) || !aligned16(out))
        return fq_fail(FQ_ERR_ALIGN, "fq_qlinear_mixed: x and out must be 16-byte aligned");
    long total = 0;
    for (int i = 0; i < count; ++i) {
        const fq_segment &sg = segments[i];
        if (int rc = check_matrix("fq_qlinear_mixed", sg.packed, sg.scales, sg.zeros, sg.N, K, sg.bits, group))
            return rc;
        if (M > 16 && (!below_4gib(M, K, 2) || !below_4gib(((size_t)sg.N + 63) / 64 * 8, K, sg.bits)))
            return fq_fail(FQ_ERR_SHAPE, "fq_qlinear_mixed: M=%d N=%d K=%d: activations and packed weights must each "
                           "stay below 4 GiB", M, sg.N, K);
        total += sg.N;
    }
    if (total > (1L << 30))
        return fq_fail(FQ_ERR_SHAPE, "fq_qlinear_mixed: %ld output columns", total);
    fq_stream st = static_cast<fq_stream>(stream);
    fq_packed_ref w[FQ_MAX_SEGMENTS];
    void *outs[FQ_MAX_SEGMENTS];
    bool stream_all = M <= 16;
    long col = 0;
    for (int i = 0; i < count; ++i) {
        w[i] = fq_packed_ref{segments[i].packed, segments[i].scales, segments[i].zeros, segments[i].N, K,
                             segments[i].bits, (int)total};
        outs[i] = static_cast<_Float16 *>(out) + col; // row 0 of the segment's column range; rows are `total` apart
        col += segments[i].N;
        stream_all = stream_all && fq_gemv_can_stream(M, K, segments[i].bits, 0);
    }
    // up to three segments share a launch (they share x): the same multi-matrix launches q/k/v and gate/up use
    for (int i = 0; i < count; i += 3) {
        const int n = count - i < 3 ? count - i : 3;
        int e = 0;
        if (M > 16)
            e = fq_launch_gemm_multi(x, M, &w[i], &outs[i], n, st);
        else if (fq_skinny_pays(M, &w[i], n))
            e = fq_launch_skinny(x, M, &w[i], &outs[i], n, fq_plan_skinny(M, &w[i], n), st);
        else if (stream_all)
            e = fq_launch_gemv_multi(fq_gemv_input{x, nullptr, nullptr, nullptr, 0}, M, &w[i], &outs[i], n, st);
        else
            for (int j = i; j < i + n && e == 0; ++j)
                e = fq_launch_gemv(x, M, w[j], outs[j], st);
        if (int rc = check_hip(e, "fq_qlinear_mixed launch"))
            return rc;
    }
    return FQ_OK;
}

extern "C" int fq_init(void)
{
    if (int rc = check_hip(fq_gemv_prepare(), "fq_init"))
        return rc;
    if (int rc = check_hip(fq_decode_prepare(), "fq_init: decode kernel"))
        return rc;
    void *p = nullptr;
    return check_hip(static_scratch(&p), "fq_init: static scratch");
}

extern "C" int fq_dense_f16(const void *x, int M, const void *W, int N, int K, void *out, void *stream)
{
    return fq_dense_f16_tile(x, M, W, N, K, out, 0, stream);
}

extern "C" int fq_dense_f16_tile(const void *x, int M, const void *W, int N, int K, void *out, int tile_rows,
                                 void *stream)
{
    if (!x || !W || !out)
        return fq_fail(FQ_ERR_NULL, "fq_dense_f16: NULL argument");
    if (M <= 0 || N <= 0 || K <= 0 || K % 128 != 0)
        return fq_fail(FQ_ERR_SHAPE, "fq_dense_f16: M=%d N=%d K=%d (K must be a positive multiple of 128)", M, N, K);
    if (!aligned16(x) || !aligned16(W) || !aligned16(out))
        return fq_fail(FQ_ERR_ALIGN, "fq_dense_f16: pointers must be 16-byte aligned");
    if (!below_4gib(M, K, 2) || !below_4gib(N, K, 2))
        return fq_fail(FQ_ERR_SHAPE, "fq_dense_f16: M=%d N=%d K=%d: x and W must each stay below 4 GiB", M, N, K);
    if (tile_rows != 0 && tile_rows != 128 && tile_rows != 256)
        return fq_fail(FQ_ERR_SHAPE, "fq_dense_f16_tile: tile_rows=%d not in {0, 128, 256}", tile_rows);
    auto *launch = tile_rows == 0 ? fq_launch_dense_planned : (tile_rows == 256 ? fq_launch_dense_tiled : fq_launch_dense);
    return check_hip(launch(x, M, W, N, K, out, static_cast<fq_stream>(stream)), "fq_dense_f16 launch");
}

extern "C" int fq_dense_route(int M, int N, int K, int loss, int *route_out)
{
    if (!route_out)
        return fq_fail(FQ_ERR_NULL, "fq_dense_route: NULL argument");
    if (M <= 0 || N <= 0 || K <= 0 || K % 128 != 0)
        return fq_fail(FQ_ERR_SHAPE, "fq_dense_route: M=%d N=%d K=%d (K must be a positive multiple of 128)", M, N, K);
    fq_dense_plan(M, N, K, loss != 0, &route_out[0], &route_out[1], &route_out[2]);
    return FQ_OK;
}

extern "C" int fq_glue(int op, const void *a, const void *b, const void *c, int M, int H, void *out, void *stream)
{
    if (op < 0 || op > 5)
        return fq_fail(FQ_ERR_SHAPE, "fq_glue: op=%d not in 0..5", op);
    if (!a || !out || (op != 0 && !b) || (op == 1 && !c))
        return fq_fail(FQ_ERR_NULL, "fq_glue: NULL argument for op %d", op);
    if (M <= 0 || H <= 0 || H % 8 != 0 || H > kMaxGlueH)
        return fq_fail(FQ_ERR_SHAPE, "fq_glue: M=%d H=%d (H must be a multiple of 8, at most %d)", M, H, kMaxGlueH);
    if (!aligned16(a) || !aligned16(out) || (b && !aligned16(b)) || (c && !aligned16(c)))
        return fq_fail(FQ_ERR_ALIGN, "fq_glue: pointers must be 16-byte aligned");
    return check_hip(fq_launch_glue(op, a, b, c, M, H, out, static_cast<fq_stream>(stream)), "fq_glue launch");
}

extern "C" int fq_token_nll(const void *logits, const int32_t *labels, int M, int V, float *nll_out, void *stream)
{
    if (!logits || !labels || !nll_out)
        return fq_fail(FQ_ERR_NULL, "fq_token_nll: NULL argument");
    if (M <= 0 || V <= 0)
        return fq_fail(FQ_ERR_SHAPE, "fq_token_nll: M=%d V=%d", M, V);
    if (!aligned16(logits))
        return fq_fail(FQ_ERR_ALIGN, "fq_token_nll: logits must be 16-byte aligned");
    return check_hip(fq_launch_nll(logits, labels, M, V, nll_out, static_cast<fq_stream>(stream)), "fq_token_nll launch");
}

extern "C" size_t fq_head_nll_workspace_bytes(int M, int V)
{
    if (M <= 0 || V <= 0)
        return 0;
    return (fq_head_nll_scratch_bytes(M, V) + 15) / 16 * 16;
}

extern "C" int fq_head_nll(const void *x, int M, const void *W, int V, int K, const int32_t *labels, float *nll_out,
                           void *workspace, size_t workspace_bytes, void *stream)
{
    if (!x || !W || !labels || !nll_out)
        return fq_fail(FQ_ERR_NULL, "fq_head_nll: NULL argument");
    if (M <= 0 || V <= 0 || K <= 0 || K % 128 != 0)
        return fq_fail(FQ_ERR_SHAPE, "fq_head_nll: M=%d V=%d K=%d (K must be a positive multiple of 128)", M, V, K);
    if (!below_4gib(M, K, 2) || !below_4gib(V, K, 2))
        return fq_fail(FQ_ERR_SHAPE, "fq_head_nll: M=%d V=%d K=%d: x and W must each stay below 4 GiB", M, V, K);
    if (!workspace || workspace_bytes < fq_head_nll_workspace_bytes(M, V))
        return fq_fail(FQ_ERR_WORKSPACE, "fq_head_nll: workspace of %zu bytes, need %zu", workspace ? workspace_bytes : 0,
                       fq_head_nll_workspace_bytes(M, V));
    if (!aligned16(x) || !aligned16(W) || !aligned16(workspace))
        return fq_fail(FQ_ERR_ALIGN, "fq_head_nll: x, W and workspace must be 16-byte aligned");
    return check_hip(fq_launch_head_nll(x, M, W, V, K, labels, nll_out, workspace, static_cast<fq_stream>(stream)),
                     "fq_head_nll launch");
}

extern "C" int fq_logit_l2(const void *a, const void *b, int M, int V, float *dist_out, void *stream)
{
    if (!a || !b || !dist_out)
        return fq_fail(FQ_ERR_NULL, "fq_logit_l2: NULL argument");
    if (M <= 0 || V <= 0)
        return fq_fail(FQ_ERR_SHAPE, "fq_logit_l2: M=%d V=%d", M, V);
    if (!aligned16(a) || !aligned16(b))
        return fq_fail(FQ_ERR_ALIGN, "fq_logit_l2: a and b must be 16-byte aligned");
    return check_hip(fq_launch_logit_l2(a, b, M, V, dist_out, static_cast<fq_stream>(stream)), "fq_logit_l2 launch");
}

extern "C" int fq_stream_read(const void *src, size_t bytes, uint32_t *sink, void *stream)
{
    if (!src || !sink)
        return fq_fail(FQ_ERR_NULL, "fq_stream_read: NULL argument");
    if (bytes == 0 || bytes % 16 != 0)
        return fq_fail(FQ_ERR_SHAPE, "fq_stream_read: %zu bytes (a positive multiple of 16)", bytes);
    if (!aligned16(src))
        return fq_fail(FQ_ERR_ALIGN, "fq_stream_read: src must be 16-byte aligned");
    return check_hip(fq_launch_stream_read(src, bytes, sink, FQ_STREAM_READ_WORDS, static_cast<fq_stream>(stream)),
                     "fq_stream_read launch");
}

// Shapes of the block's seven matrices and the selected packing of each, checked before anything is launched.
static int validate_layers(const char *fn, const fq_layer *layers, int L, const uint8_t *bitvec, int *H_out, int *F_out)
{
    const int H = layers[0].m[0].K, F = layers[0].m[4].N;
    if (H <= 0 || F <= 0 || H % 128 != 0 || F % 128 != 0 || H > kMaxGlueH || F > kMaxGlueH)
        return fq_fail(FQ_ERR_SHAPE, "%s: hidden=%d ffn=%d must be multiples of 128, at most %d", fn, H, F, kMaxGlueH);
    for (int l = 0; l < L; ++l)
        for (int j = 0; j < 7; ++j) {
            const fq_matrix &mx = layers[l].m[j];
            const int wantN = (j == 4 || j == 5) ? F : H, wantK = (j == 6) ? F : H;
            if (mx.N != wantN || mx.K != wantK)
                return fq_fail(FQ_ERR_SHAPE, "%s: layer %d matrix %d is %dx%d, expected %dx%d", fn, l, j, mx.N, mx.K,
                               wantN, wantK);
            const int bi = fq_bits_index(bitvec[7 * l + j]);
            if (bi < 0)
                return fq_fail(FQ_ERR_BITS, "%s: bitvec[%d]=%d not in {2,3,4,8}", fn, 7 * l + j, (int)bitvec[7 * l + j]);
            if (!mx.packed[bi] || !mx.scales[bi] || !mx.zeros[bi])
                return fq_fail(FQ_ERR_NULL, "%s: layer %d matrix %d has no %d-bit packing", fn, l, j,
                               (int)bitvec[7 * l + j]);
            if (!aligned16(mx.packed[bi]) || !aligned16(mx.scales[bi]) || !aligned16(mx.zeros[bi]))
                return fq_fail(FQ_ERR_ALIGN, "%s: layer %d matrix %d is not 16-byte aligned", fn, l, j);
        }
    *H_out = H;
    *F_out = F;
    return FQ_OK;
}

// Workspace: u, q, k, v, a, o, x1, u2, d, xcur (hidden wide), g, p, m (ffn wide), then the counters of the
// persistent decode kernel's grid barrier.
extern "C" size_t fq_stack_workspace_bytes(int M, int hidden, int ffn)
{
    if (M <= 0 || hidden <= 0 || ffn <= 0)
        return 0;
    const size_t h = align_up((size_t)M * hidden * 2), f = align_up((size_t)M * ffn * 2);
    return 10 * h + 3 * f + fq_decode_sync_bytes;
}

static const char kGaveUp[] = "an earlier decode kernel gave up waiting at its grid barrier (its results are invalid); "
                              "fq_clear_async_error() re-arms the library";

extern "C" int fq_set_decode_mode(int mode) { return fq_decode_set_mode(mode); }
extern "C" unsigned long long fq_decode_give_up_ticks(unsigned long long ticks) { return fq_decode_set_give_up_ticks(ticks); }
extern "C" int fq_decode_persistent(int hidden, int ffn) { return fq_decode_available(hidden, ffn); }
extern "C" unsigned long long fq_decode_persistent_launches(void) { return fq_decode_launches(); }
extern "C" int fq_async_error(void) { return fq_decode_async_error() ? FQ_ERR_HIP : FQ_OK; }
extern "C" void fq_clear_async_error(void) { fq_decode_clear_async_error(); }

extern "C" int fq_decode_partition(const uint8_t *bits7, int phase, int N, int wg, int grid, int *units_out)
{
    if (!bits7 || !units_out)
        return fq_fail(FQ_ERR_NULL, "fq_decode_partition: NULL argument");
    if (phase < 0 || phase > 3 || N <= 0 || grid <= 0 || wg < 0 || wg >= grid)
        return fq_fail(FQ_ERR_SHAPE, "fq_decode_partition: phase=%d N=%d wg=%d grid=%d", phase, N, wg, grid);
    unsigned bits4 = 0;
    for (int j = 0; j < 7; ++j) {
        if (fq_bits_index(bits7[j]) < 0)
            return fq_fail(FQ_ERR_BITS, "fq_decode_partition: bits=%d not in {2,3,4,8}", (int)bits7[j]);
        bits4 |= (unsigned)bits7[j] << (4 * j);
    }
    fq_decode_partition_of(bits4, phase, N, wg, grid, units_out);
    return FQ_OK;
}

static int stack_forward_checked(const fq_layer *layers, int L, const uint8_t *bitvec, const void *x_in, int M,
                                 void *x_out, void *workspace, int H, int F, bool may_allocate, fq_stream st);

extern "C" int fq_stack_forward(const fq_layer *layers, int L, const uint8_t *bitvec, const void *x_in, int M,
                                void *x_out, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!layers || !bitvec || !x_in || !x_out || !workspace)
        return fq_fail(FQ_ERR_NULL, "fq_stack_forward: NULL argument");
    if (L <= 0 || M <= 0)
        return fq_fail(FQ_ERR_SHAPE, "fq_stack_forward: L=%d M=%d", L, M);
    int H = 0, F = 0;
    if (int rc = validate_layers("fq_stack_forward", layers, L, bitvec, &H, &F))
        return rc;
    if (workspace_bytes < fq_stack_workspace_bytes(M, H, F))
        return fq_fail(FQ_ERR_WORKSPACE, "fq_stack_forward: workspace of %zu bytes, need %zu", workspace_bytes,
                       fq_stack_workspace_bytes(M, H, F));
    if (!aligned16(x_in) || !aligned16(x_out) || !aligned16(workspace))
        return fq_fail(FQ_ERR_ALIGN, "fq_stack_forward: x_in, x_out and workspace must be 16-byte aligned");
    if (fq_decode_async_error())
        return fq_fail(FQ_ERR_HIP, "fq_stack_forward: %s", kGaveUp);
    return stack_forward_checked(layers, L, bitvec, x_in, M, x_out, workspace, H, F, true, static_cast<fq_stream>(stream));
}

extern "C" int fq_stack_forward_noalloc(const fq_layer *layers, int L, const uint8_t *bitvec, const void *x_in, int M,
                                        void *x_out, void *stream)
{
    if (!layers || !bitvec || !x_in || !x_out)
        return fq_fail(FQ_ERR_NULL, "fq_stack_forward_noalloc: NULL argument");
    if (L <= 0 || M <= 0)
        return fq_fail(FQ_ERR_SHAPE, "fq_stack_forward_noalloc: L=%d M=%d", L, M);
    if (M > kNoallocMaxM)
        return fq_fail(FQ_ERR_SHAPE, "fq_stack_forward_noalloc: M=%d exceeds the %d rows the library's own scratch "
                       "holds; use fq_stack_forward with a workspace", M, kNoallocMaxM);
    int H = 0, F = 0;
    if (int rc = validate_layers("fq_stack_forward_noalloc", layers, L, bitvec, &H, &F))
        return rc;
    if (H > kNoallocMaxDim || F > kNoallocMaxDim || fq_stack_workspace_bytes(M, H, F) > kNoallocScratchBytes)
        return fq_fail(FQ_ERR_SHAPE, "fq_stack_forward_noalloc: hidden=%d ffn=%d exceed the %d elements per row the "
                       "library's own scratch holds; use fq_stack_forward with a workspace", H, F, kNoallocMaxDim);
    if (!aligned16(x_in) || !aligned16(x_out))
        return fq_fail(FQ_ERR_ALIGN, "fq_stack_forward_noalloc: x_in and x_out must be 16-byte aligned");
    void *ws = nullptr;
    if (int rc = check_hip(static_scratch(&ws), "fq_stack_forward_noalloc: static scratch"))
        return rc;
    if (fq_decode_async_error())
        return fq_fail(FQ_ERR_HIP, "fq_stack_forward_noalloc: %s", kGaveUp);
    return stack_forward_checked(layers, L, bitvec, x_in, M, x_out, ws, H, F, false, static_cast<fq_stream>(stream));
}

// The launches of a stack forward; every argument has been validated and the workspace holds
// fq_stack_workspace_bytes(M, H, F) bytes.
static int stack_forward_checked(const fq_layer *layers, int L, const uint8_t *bitvec, const void *x_in, int M,
                                 void *x_out, void *workspace, int H, int F, bool may_allocate, fq_stream st)
{
    fq_packed_ref sel[7];
    const size_t hb = align_up((size_t)M * H * 2), fb = align_up((size_t)M * F * 2);
    char *ws = static_cast<char *>(workspace);
    void *u = ws, *q = ws + hb, *k = ws + 2 * hb, *v = ws + 3 * hb, *a = ws + 4 * hb, *o = ws + 5 * hb,
         *x1 = ws + 6 * hb, *u2 = ws + 7 * hb, *d = ws + 8 * hb, *xc = ws + 9 * hb;
    void *g = ws + 10 * hb, *p = ws + 10 * hb + fb, *mm = ws + 10 * hb + 2 * fb;

    // One token: the whole stack in one persistent launch where that kernel applies.
    if (M == 1) {
        const fq_decode_buffers bufs = {q, k, v, o, g, p, d, x1, ws + 10 * hb + 3 * fb};
        const int e = fq_launch_decode_persist(layers, L, bitvec, H, F, x_in, x_out, bufs, may_allocate, st);
        if (e == 0)
            return FQ_OK;
        if (e > 0)
            return check_hip(e, "decode (persistent kernel)");
    }

    // Decode of up to three rows: four launches per block.  q/k/v and gate/up share a launch each, and every
    // row-wise step is folded into the input staging of the linear that consumes it.  The staging takes the rows one
    // after another, so from four rows on the linears and the row-wise steps are launches of their own (us per
    // block, hidden 1024 / ffn 2816: 35 and 34 at three rows, 40 against 29 at four, 106 against 29 at sixteen; rows of
    // 4096 / 11008 elements do not fit the staging from four rows on: 64 us at four rows against 60 at three).
    bool decode = M <= 3;
    static const int stack_mode[7] = {5, 5, 5, 2, 3, 3, 4}; // input transform of each linear (mode 1 needs no more than 5)
    for (int l = 0; l < L && decode; ++l)
        for (int j = 0; j < 7; ++j)
            decode = decode && fq_gemv_can_stream(M, layers[l].m[j].K, bitvec[7 * l + j], stack_mode[j]);

    const void *xcur = x_in;
    for (int l = 0; l < L; ++l) {
        for (int j = 0; j < 7; ++j) {
            const fq_matrix &mx = layers[l].m[j];
            const int bits = bitvec[7 * l + j], bi = fq_bits_index(bits);
            sel[j] = fq_packed_ref{mx.packed[bi], mx.scales[bi], mx.zeros[bi], mx.N, mx.K, bits};
        }
        void *xnext = (l == L - 1) ? x_out : xc;
        void *const qkv[3] = {q, k, v};
        void *const gp[2] = {g, p};
        int rc;
#define FQ_STEP(call) \
    do { \
        if ((rc = (call)) != FQ_OK) \
            return rc; \
    } while (0)
        if (decode) {
            // the previous block's x_next = rms(x1 + d) is produced (into xc) by this block's first launch
            const fq_gemv_input in_qkv = (l == 0) ? fq_gemv_input{x_in, nullptr, nullptr, nullptr, 1}
                                                  : fq_gemv_input{x1, d, nullptr, xc, 5};
            if (l > 0)
                xcur = xc;
            FQ_STEP(check_hip(fq_launch_gemv_multi(in_qkv, M, &sel[0], qkv, 3, st), "decode q/k/v"));
            FQ_STEP(check_hip(fq_launch_gemv_multi(fq_gemv_input{q, k, v, nullptr, 2}, M, &sel[3], &o, 1, st),
                              "decode o"));
            FQ_STEP(check_hip(fq_launch_gemv_multi(fq_gemv_input{xcur, o, nullptr, x1, 3}, M, &sel[4], gp, 2, st),
                              "decode gate/up"));
            FQ_STEP(check_hip(fq_launch_gemv_multi(fq_gemv_input{g, p, nullptr, nullptr, 4}, M, &sel[6], &d, 1, st),
                              "decode down"));
            if (l == L - 1)
                FQ_STEP(check_hip(fq_launch_glue(4, x1, d, nullptr, M, H, x_out, st), "glue rms(add)"));
            continue;
        }
        // otherwise the row-wise steps are kernels of their own, two of them per pass where one feeds the other
        // (the residual sum with the norm that reads it; a block's output with the next block's first norm)
        if (l == 0) {
            FQ_STEP(check_hip(fq_launch_glue(0, xcur, nullptr, nullptr, M, H, u, st), "glue rms"));
        }
        FQ_STEP(qlinear_multi_checked(u, M, &sel[0], qkv, 3, st));
        FQ_STEP(check_hip(fq_launch_glue(1, q, k, v, M, H, a, st), "glue rms(q+k+v)"));
        FQ_STEP(qlinear_checked(a, M, sel[3], o, st));
        FQ_STEP(check_hip(fq_launch_glue2(6, xcur, o, M, H, x1, u2, st), "glue add, rms"));
        FQ_STEP(qlinear_multi_checked(u2, M, &sel[4], gp, 2, st));
        FQ_STEP(check_hip(fq_launch_glue(3, g, p, nullptr, M, F, mm, st), "glue rms(silu*mul)"));
        FQ_STEP(qlinear_checked(mm, M, sel[6], d, st));
        if (l == L - 1) {
            FQ_STEP(check_hip(fq_launch_glue(4, x1, d, nullptr, M, H, xnext, st), "glue rms(add)"));
        } else {
            FQ_STEP(check_hip(fq_launch_glue2(7, x1, d, M, H, xnext, u, st), "glue rms(add), rms"));
        }
#undef FQ_STEP
        xcur = xnext;
    }
    return FQ_OK;
}

// Workspace: q, k, v, a, o, x1, d, x (hidden wide), g, p (ffn wide), then the attention's split results.
extern "C" size_t fq_decode_workspace_bytes(int hidden, int ffn, int Tmax)
{
    if (hidden <= 0 || ffn <= 0 || Tmax <= 0 || hidden % 128 != 0)
        return 0;
    return 8 * align_up((size_t)hidden * 2) + 2 * align_up((size_t)ffn * 2) + align_up(fq_attn_scratch_bytes(Tmax, hidden / 128));
}

extern "C" size_t fq_attn_workspace_bytes(int Tmax, int n_heads)
{
    if (Tmax <= 0 || n_heads <= 0)
        return 0;
    return align_up(fq_attn_scratch_bytes(Tmax, n_heads));
}

extern "C" int fq_attn_decode(const void *q, const void *k, const void *v, void *k_cache, void *v_cache, int pos,
                              int Tmax, int n_heads, const float *rope, void *out, void *workspace,
                              size_t workspace_bytes, void *stream)
{
    if (!q || !k || !v || !k_cache || !v_cache || !rope || !out || !workspace)
        return fq_fail(FQ_ERR_NULL, "fq_attn_decode: NULL argument");
    if (n_heads <= 0 || Tmax <= 0 || Tmax > fq_attn_max_positions() || pos < 0 || pos >= Tmax)
        return fq_fail(FQ_ERR_SHAPE, "fq_attn_decode: n_heads=%d Tmax=%d pos=%d (need 0 <= pos < Tmax <= %d)", n_heads, Tmax,
                       pos, fq_attn_max_positions());
    if (workspace_bytes < fq_attn_scratch_bytes(Tmax, n_heads))
        return fq_fail(FQ_ERR_WORKSPACE, "fq_attn_decode: workspace of %zu bytes, need %zu", workspace_bytes,
                       fq_attn_scratch_bytes(Tmax, n_heads));
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(k_cache) || !aligned16(v_cache) ||
        !aligned16(rope) || !aligned16(out) || !aligned16(workspace))
        return fq_fail(FQ_ERR_ALIGN, "fq_attn_decode: pointers must be 16-byte aligned");
    return check_hip(fq_launch_attn_decode(q, k, v, k_cache, v_cache, pos, Tmax, n_heads, rope, out, workspace,
                                           static_cast<fq_stream>(stream)), "fq_attn_decode launch");
}

extern "C" int fq_decode_step(const fq_layer *layers, int L, const uint8_t *bitvec, const void *x_in, void *x_out,
                              void *k_cache, void *v_cache, int pos, int Tmax, const float *rope, void *workspace,
                              size_t workspace_bytes, void *stream)
{
    if (!layers || !bitvec || !x_in || !x_out || !k_cache || !v_cache || !rope || !workspace)
        return fq_fail(FQ_ERR_NULL, "fq_decode_step: NULL argument");
    if (L <= 0 || Tmax <= 0 || Tmax > fq_attn_max_positions() || pos < 0 || pos >= Tmax)
        return fq_fail(FQ_ERR_SHAPE, "fq_decode_step: L=%d Tmax=%d pos=%d (need 0 <= pos < Tmax <= %d)", L, Tmax, pos,
                       fq_attn_max_positions());
    int H = 0, F = 0;
    if (int rc = validate_layers("fq_decode_step", layers, L, bitvec, &H, &F))
        return rc;
    for (int l = 0; l < L; ++l)
        for (int j = 0; j < 7; ++j)
            if (!fq_gemv_can_stream(1, layers[l].m[j].K, bitvec[7 * l + j], j == 6 ? 6 : (j == 3 ? 0 : 3)))
                return fq_fail(FQ_ERR_SHAPE, "fq_decode_step: rows of %d elements do not fit the decode kernel",
                               layers[l].m[j].K);
    if (workspace_bytes < fq_decode_workspace_bytes(H, F, Tmax))
        return fq_fail(FQ_ERR_WORKSPACE, "fq_decode_step: workspace of %zu bytes, need %zu", workspace_bytes,
                       fq_decode_workspace_bytes(H, F, Tmax));
    if (!aligned16(x_in) || !aligned16(x_out) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(rope) ||
        !aligned16(workspace))
        return fq_fail(FQ_ERR_ALIGN, "fq_decode_step: pointers must be 16-byte aligned");

    fq_stream st = static_cast<fq_stream>(stream);
    const int n_heads = H / 128;
    const size_t hb = align_up((size_t)H * 2), fb = align_up((size_t)F * 2), layer_cache = (size_t)Tmax * H * 2;
    char *ws = static_cast<char *>(workspace);
    void *q = ws, *k = ws + hb, *v = ws + 2 * hb, *a = ws + 3 * hb, *o = ws + 4 * hb, *x1 = ws + 5 * hb,
         *d = ws + 6 * hb, *xc = ws + 7 * hb, *g = ws + 8 * hb, *p = ws + 8 * hb + fb, *attn = ws + 8 * hb + 2 * fb;
    fq_packed_ref sel[7];
    const void *xres = x_in;
    for (int l = 0; l < L; ++l) {
        for (int j = 0; j < 7; ++j) {
            const fq_matrix &mx = layers[l].m[j];
            const int bits = bitvec[7 * l + j], bi = fq_bits_index(bits);
            sel[j] = fq_packed_ref{mx.packed[bi], mx.scales[bi], mx.zeros[bi], mx.N, mx.K, bits};
        }
        void *const qkv[3] = {q, k, v};
        void *const gp[2] = {g, p};
        int rc;
#define FQ_STEP(call) \
    do { \
        if ((rc = (call)) != FQ_OK) \
            return rc; \
    } while (0)
        // the previous block's output x1 + d is formed (into xc) by this block's first launch
        const fq_gemv_input in_qkv = (l == 0) ? fq_gemv_input{x_in, nullptr, nullptr, nullptr, 1}
                                              : fq_gemv_input{x1, d, nullptr, xc, 3};
        if (l > 0)
            xres = xc;
        FQ_STEP(check_hip(fq_launch_gemv_multi(in_qkv, 1, &sel[0], qkv, 3, st), "decode q/k/v"));
        FQ_STEP(check_hip(fq_launch_attn_decode(q, k, v, static_cast<char *>(k_cache) + l * layer_cache,
                                                static_cast<char *>(v_cache) + l * layer_cache, pos, Tmax, n_heads, rope, a,
                                                attn, st), "decode attention"));
        FQ_STEP(check_hip(fq_launch_gemv_multi(fq_gemv_input{a, nullptr, nullptr, nullptr, 0}, 1, &sel[3], &o, 1, st),
                          "decode o"));
        FQ_STEP(check_hip(fq_launch_gemv_multi(fq_gemv_input{xres, o, nullptr, x1, 3}, 1, &sel[4], gp, 2, st),
                          "decode gate/up"));
        FQ_STEP(check_hip(fq_launch_gemv_multi(fq_gemv_input{g, p, nullptr, nullptr, 6}, 1, &sel[6], &d, 1, st),
                          "decode down"));
#undef FQ_STEP
    }
    return check_hip(fq_launch_glue(2, x1, d, nullptr, 1, H, x_out, st), "glue add");
}

extern "C" size_t fq_attn_prefill_workspace_bytes(int T, int n_heads)
{
    if (T <= 0 || n_heads <= 0)
        return 0;
    return align_up(fq_attn_prefill_scratch_bytes(T, n_heads));
}

extern "C" int fq_attn_prefill(const void *q, const void *k, const void *v, int T, void *k_cache, void *v_cache,
                               int Tmax, int n_heads, const float *rope, void *out, void *workspace,
                               size_t workspace_bytes, void *stream)
{
    if (!q || !k || !v || !k_cache || !v_cache || !rope || !out || !workspace)
        return fq_fail(FQ_ERR_NULL, "fq_attn_prefill: NULL argument");
    if (n_heads <= 0 || T <= 0 || T > Tmax || Tmax > fq_attn_max_positions() || !below_4gib(T, (size_t)n_heads * 128, 2))
        return fq_fail(FQ_ERR_SHAPE, "fq_attn_prefill: n_heads=%d T=%d Tmax=%d (need 0 < T <= Tmax <= %d)", n_heads, T, Tmax,
                       fq_attn_max_positions());
    if (workspace_bytes < fq_attn_prefill_workspace_bytes(T, n_heads))
        return fq_fail(FQ_ERR_WORKSPACE, "fq_attn_prefill: workspace of %zu bytes, need %zu", workspace_bytes,
                       fq_attn_prefill_workspace_bytes(T, n_heads));
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(k_cache) || !aligned16(v_cache) ||
        !aligned16(rope) || !aligned16(out) || !aligned16(workspace))
        return fq_fail(FQ_ERR_ALIGN, "fq_attn_prefill: pointers must be 16-byte aligned");
    return check_hip(fq_launch_attn_prefill(q, k, v, T, k_cache, v_cache, Tmax, n_heads, rope, out, workspace,
                                            static_cast<fq_stream>(stream)), "fq_attn_prefill launch");
}

// Workspace: u, q, k, v, a, o, x1, d, x (hidden wide), g, p, m (ffn wide), then the attention's scratch.
extern "C" size_t fq_prefill_workspace_bytes(int T, int hidden, int ffn)
{
    if (T <= 0 || hidden <= 0 || ffn <= 0 || hidden % 128 != 0)
        return 0;
    return 9 * align_up((size_t)T * hidden * 2) + 3 * align_up((size_t)T * ffn * 2) +
           align_up(fq_attn_prefill_scratch_bytes(T, hidden / 128));
}

extern "C" int fq_prefill_forward(const fq_layer *layers, int L, const uint8_t *bitvec, const void *x_in, int T,
                                  void *x_out, void *k_cache, void *v_cache, int Tmax, const float *rope,
                                  void *workspace, size_t workspace_bytes, void *stream)
{
    if (!layers || !bitvec || !x_in || !x_out || !k_cache || !v_cache || !rope || !workspace)
        return fq_fail(FQ_ERR_NULL, "fq_prefill_forward: NULL argument");
    if (L <= 0 || T <= 0 || T > Tmax || Tmax > fq_attn_max_positions())
        return fq_fail(FQ_ERR_SHAPE, "fq_prefill_forward: L=%d T=%d Tmax=%d (need 0 < T <= Tmax <= %d)", L, T, Tmax,
                       fq_attn_max_positions());
    int H = 0, F = 0;
    if (int rc = validate_layers("fq_prefill_forward", layers, L, bitvec, &H, &F))
        return rc;
    if (workspace_bytes < fq_prefill_workspace_bytes(T, H, F))
        return fq_fail(FQ_ERR_WORKSPACE, "fq_prefill_forward: workspace of %zu bytes, need %zu", workspace_bytes,
                       fq_prefill_workspace_bytes(T, H, F));
    if (!aligned16(x_in) || !aligned16(x_out) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(rope) ||
        !aligned16(workspace))
        return fq_fail(FQ_ERR_ALIGN, "fq_prefill_forward: pointers must be 16-byte aligned");

    fq_stream st = static_cast<fq_stream>(stream);
    const int n_heads = H / 128, M = T;
    const size_t hb = align_up((size_t)T * H * 2), fb = align_up((size_t)T * F * 2), layer_cache = (size_t)Tmax * H * 2;
    char *ws = static_cast<char *>(workspace);
    void *u = ws, *q = ws + hb, *k = ws + 2 * hb, *v = ws + 3 * hb, *a = ws + 4 * hb, *o = ws + 5 * hb,
         *x1 = ws + 6 * hb, *d = ws + 7 * hb, *xc = ws + 8 * hb;
    void *g = ws + 9 * hb, *p = ws + 9 * hb + fb, *mm = ws + 9 * hb + 2 * fb, *attn = ws + 9 * hb + 3 * fb;
    fq_packed_ref sel[7];
    const void *xcur = x_in;
    for (int l = 0; l < L; ++l) {
        for (int j = 0; j < 7; ++j) {
            const fq_matrix &mx = layers[l].m[j];
            const int bits = bitvec[7 * l + j], bi = fq_bits_index(bits);
            sel[j] = fq_packed_ref{mx.packed[bi], mx.scales[bi], mx.zeros[bi], mx.N, mx.K, bits};
        }
        void *xnext = (l == L - 1) ? x_out : xc;
        void *const qkv[3] = {q, k, v};
        void *const gp[2] = {g, p};
        int rc;
#define FQ_STEP(call) \
    do { \
        if ((rc = (call)) != FQ_OK) \
            return rc; \
    } while (0)
        FQ_STEP(check_hip(fq_launch_glue(0, xcur, nullptr, nullptr, M, H, u, st), "glue rms"));
        if (M > 16 || fq_skinny_pays(M, &sel[0], 3)) {
            FQ_STEP(qlinear_multi_checked(u, M, &sel[0], qkv, 3, st));
        } else {
            for (int j = 0; j < 3; ++j)
                FQ_STEP(qlinear_checked(u, M, sel[j], qkv[j], st));
        }
        FQ_STEP(check_hip(fq_launch_attn_prefill(q, k, v, T, static_cast<char *>(k_cache) + l * layer_cache,
                                                 static_cast<char *>(v_cache) + l * layer_cache, Tmax, n_heads, rope, a,
                                                 attn, st), "prefill attention"));
        FQ_STEP(qlinear_checked(a, M, sel[3], o, st));
        FQ_STEP(check_hip(fq_launch_glue2(6, xcur, o, M, H, x1, u, st), "glue add, rms"));
        if (M > 16 || fq_skinny_pays(M, &sel[4], 2)) {
            FQ_STEP(qlinear_multi_checked(u, M, &sel[4], gp, 2, st));
        } else {
            for (int j = 0; j < 2; ++j)
                FQ_STEP(qlinear_checked(u, M, sel[4 + j], gp[j], st));
        }
        FQ_STEP(check_hip(fq_launch_glue(5, g, p, nullptr, M, F, mm, st), "glue silu*mul"));
        FQ_STEP(qlinear_checked(mm, M, sel[6], d, st));
        FQ_STEP(check_hip(fq_launch_glue(2, x1, d, nullptr, M, H, xnext, st), "glue add"));
#undef FQ_STEP
        xcur = xnext;
    }
    return FQ_OK;
}

// ------------------------------------------------------------------ paged cache
namespace {

int page_log2(int page) // 4..8, or -1
{
    for (int l = 4; l <= 8; ++l)
        if (page == 1 << l)
            return l;
    return -1;
}

int check_pool(const char *fn, int page, int pages, int n_kv_heads)
{
    if (page_log2(page) < 0)
        return fq_fail(FQ_ERR_SHAPE, "%s: pages of %d positions (16, 32, 64, 128 or 256)", fn, page);
    if (pages <= 0 || (long long)pages * page > INT32_MAX)
        return fq_fail(FQ_ERR_SHAPE, "%s: %d pages of %d positions (at most 2^31 - 1 positions)", fn, pages, page);
    if (n_kv_heads <= 0 || n_kv_heads > 65535)
        return fq_fail(FQ_ERR_SHAPE, "%s: n_kv_heads=%d", fn, n_kv_heads);
    return FQ_OK;
}

int check_heads(const char *fn, int tokens, int n_heads, int n_kv_heads)
{
    if (n_kv_heads <= 0 || n_heads <= 0 || n_heads % n_kv_heads != 0 || (long long)tokens * n_heads >= 1 << 26)
        return fq_fail(FQ_ERR_SHAPE, "%s: tokens=%d n_heads=%d n_kv_heads=%d (n_heads a multiple of n_kv_heads, tokens * n_heads "
                       "below 2^26)", fn, tokens, n_heads, n_kv_heads);
    return FQ_OK;
}

int check_batch(const char *fn, const fq_paged_batch *b, int n_kv_heads)
{
    if (!b || !b->q_start || !b->seq_len || !b->table)
        return fq_fail(FQ_ERR_NULL, "%s: NULL batch or array of it", fn);
    if (int rc = check_pool(fn, b->page, b->pages, n_kv_heads))
        return rc;
    if (b->seqs <= 0 || b->seqs > 65535 || b->tokens < 0 || b->max_q < 0 || b->max_q > b->tokens || (long long)b->max_q * b->seqs < b->tokens)
        return fq_fail(FQ_ERR_SHAPE, "%s: seqs=%d tokens=%d max_q=%d (need max_q <= tokens <= seqs * max_q)", fn, b->seqs, b->tokens, b->max_q);
    if ((long long)b->seqs * n_kv_heads >= 1 << 23)
        return fq_fail(FQ_ERR_SHAPE, "%s: seqs=%d n_kv_heads=%d (their product must be below 2^23)", fn, b->seqs, n_kv_heads);
    if (b->table_stride <= 0 || b->max_len < 0 || b->max_len > (1 << 24) || b->max_len > (long long)b->table_stride * b->page)
        return fq_fail(FQ_ERR_SHAPE, "%s: max_len=%d table_stride=%d (need max_len <= table_stride * page, at most 2^24)", fn, b->max_len,
                       b->table_stride);
    return FQ_OK;
}

bool overlap(const void *a, size_t a_bytes, const void *b, size_t b_bytes)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + b_bytes && y < x + a_bytes;
}

// The same of two arrays of as many rows, `stride` bytes apart and `row` of them used: rows of one may lie between those of the other.
bool rows_overlap(const void *a, const void *b, size_t rows, size_t stride, size_t row)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b), d = x < y ? y - x : x - y;
    const size_t at = d / stride, off = d % stride; // the later array's first row, in rows of the earlier one
    return (at < rows && off < row) || (at + 1 < rows && stride - off < row);
}

// Whether rows of `row` bytes, `stride` (at least that) apart, reach into a run of bytes.
bool rows_in(const void *a, size_t rows, size_t stride, size_t row, const void *run, size_t bytes)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(run);
    const size_t first = y < x + row ? 0 : (y - x - row) / stride + 1; // the first row that ends behind the run's start
    return first < rows && x + first * stride < y + bytes;
}

bool stride_ok(int ld, int width) { return ld >= width && ld % 8 == 0; }

} // namespace

extern "C" int fq_qk_norm_rope(const void *q, int ldq, const void *k, int ldk, const void *v, int ldv, int tokens, int n_heads, int n_kv_heads,
                               const int32_t *positions, const int32_t *slots, const float *rope, int rope_rows, const void *q_gain,
                               const void *k_gain, float eps, void *q_out, void *k_pages, void *v_pages, int page, int pages, void *stream)
{
    const char *fn = "fq_qk_norm_rope";
    if (!q || !k || !v || !positions || !slots || !rope || !q_out || !k_pages || !v_pages)
        return fq_fail(FQ_ERR_NULL, "%s: NULL argument", fn);
    if (int rc = check_pool(fn, page, pages, n_kv_heads))
        return rc;
    if (int rc = check_heads(fn, tokens, n_heads, n_kv_heads))
        return rc;
    if (tokens < 0 || n_heads > 65535 || rope_rows <= 0 || !(eps >= 0.f))
        return fq_fail(FQ_ERR_SHAPE, "%s: tokens=%d n_heads=%d rope_rows=%d eps=%g", fn, tokens, n_heads, rope_rows, eps);
    if (!stride_ok(ldq, n_heads * 128) || !stride_ok(ldk, n_kv_heads * 128) || !stride_ok(ldv, n_kv_heads * 128))
        return fq_fail(FQ_ERR_SHAPE, "%s: ldq=%d ldk=%d ldv=%d (at least the row, multiples of 8)", fn, ldq, ldk, ldv);
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(rope) || !aligned16(q_gain) || !aligned16(k_gain) || !aligned16(q_out) ||
        !aligned16(k_pages) || !aligned16(v_pages))
        return fq_fail(FQ_ERR_ALIGN, "%s: pointers must be 16-byte aligned", fn);
    const size_t row = (size_t)n_heads * 128 * 2;
    if (tokens > 0 && !(q_out == q && (ldq == n_heads * 128 || tokens == 1)) && overlap(q, (size_t)(tokens - 1) * ldq * 2 + row, q_out, tokens * row))
        return fq_fail(FQ_ERR_SHAPE, "%s: q_out overlaps q other than row by row", fn);
    const size_t kv_row = (size_t)n_kv_heads * 128 * 2;
    if (tokens > 0 && (rows_in(k, tokens, (size_t)ldk * 2, kv_row, q_out, tokens * row) || rows_in(v, tokens, (size_t)ldv * 2, kv_row, q_out, tokens * row)))
        return fq_fail(FQ_ERR_SHAPE, "%s: q_out overlaps k or v", fn);
    if (tokens == 0)
        return FQ_OK;
    return check_hip(fq_launch_qk_norm_rope(q, ldq, k, ldk, v, ldv, tokens, n_heads, n_kv_heads, positions, slots, rope, rope_rows, q_gain, k_gain,
                                            eps, q_out, k_pages, v_pages, page_log2(page), pages, static_cast<fq_stream>(stream)),
                     "fq_qk_norm_rope launch");
}

extern "C" size_t fq_attn_paged_workspace_bytes(const fq_paged_batch *batch, int n_heads, int n_kv_heads, int with_weights)
{
    const char *fn = "fq_attn_paged_workspace_bytes";
    if (check_batch(fn, batch, n_kv_heads) || check_heads(fn, batch->tokens, n_heads, n_kv_heads))
        return 0;
    return align_up(fq_attn_paged_scratch_bytes(*batch, n_heads, n_kv_heads, with_weights != 0));
}

extern "C" int fq_attn_paged_route(const fq_paged_batch *batch, int n_heads, int n_kv_heads, int *route_out)
{
    const char *fn = "fq_attn_paged_route";
    if (!route_out)
        return fq_fail(FQ_ERR_NULL, "%s: NULL output", fn);
    if (int rc = check_batch(fn, batch, n_kv_heads))
        return rc;
    if (int rc = check_heads(fn, batch->tokens, n_heads, n_kv_heads))
        return rc;
    fq_attn_paged_plan(*batch, n_heads, n_kv_heads, &route_out[0], &route_out[1], &route_out[2]);
    return FQ_OK;
}

extern "C" int fq_attn_paged(const fq_paged_batch *batch, const void *q, int ldq, int n_heads, int n_kv_heads, const void *k_pages,
                             const void *v_pages, float scale, void *out, float *lse, const float *weights, float *weights_out,
                             int weights_stride, void *workspace, size_t workspace_bytes, void *stream)
{
    const char *fn = "fq_attn_paged";
    if (int rc = check_batch(fn, batch, n_kv_heads))
        return rc;
    if (int rc = check_heads(fn, batch->tokens, n_heads, n_kv_heads))
        return rc;
    if (!k_pages || !v_pages || (batch->tokens > 0 && (!q || !out)))
        return fq_fail(FQ_ERR_NULL, "%s: NULL argument", fn);
    if (!stride_ok(ldq, n_heads * 128))
        return fq_fail(FQ_ERR_SHAPE, "%s: ldq=%d (at least the row, a multiple of 8)", fn, ldq);
    if (!(scale > 0.f) || scale > 1e30f)
        return fq_fail(FQ_ERR_SHAPE, "%s: scale=%g (must be positive and finite)", fn, scale);
    if (weights && !weights_out)
        return fq_fail(FQ_ERR_NULL, "%s: weights without weights_out", fn);
    if (weights_out && (weights_stride < batch->max_len || (long long)batch->max_len * n_kv_heads >= 1 << 28))
        return fq_fail(FQ_ERR_SHAPE, "%s: weights_stride=%d max_len=%d n_kv_heads=%d (need weights_stride >= max_len, max_len * n_kv_heads "
                       "below 2^28)", fn, weights_stride, batch->max_len, n_kv_heads);
    if (weights && weights != weights_out && batch->max_len > 0 &&
        rows_overlap(weights, weights_out, (size_t)batch->seqs * n_kv_heads, (size_t)weights_stride * 4, (size_t)batch->max_len * 4))
        return fq_fail(FQ_ERR_SHAPE, "%s: weights_out overlaps weights other than place by place", fn);
    const size_t need = fq_attn_paged_scratch_bytes(*batch, n_heads, n_kv_heads, weights_out != nullptr);
    if (need > 0 && (!workspace || workspace_bytes < need))
        return fq_fail(FQ_ERR_WORKSPACE, "%s: workspace of %zu bytes, need %zu", fn, workspace ? workspace_bytes : (size_t)0, need);
    if (!aligned16(q) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(out) || !aligned16(workspace))
        return fq_fail(FQ_ERR_ALIGN, "%s: pointers must be 16-byte aligned", fn);
    const size_t row = (size_t)n_heads * 128 * 2;
    if (batch->tokens > 0 && overlap(q, (size_t)(batch->tokens - 1) * ldq * 2 + row, out, batch->tokens * row))
        return fq_fail(FQ_ERR_SHAPE, "%s: out overlaps q, which every part of the call reads", fn);
    return check_hip(fq_launch_attn_paged(*batch, q, ldq, n_heads, n_kv_heads, k_pages, v_pages, scale, out, lse, weights, weights_out,
                                          weights_stride, workspace, static_cast<fq_stream>(stream)), "fq_attn_paged launch");
}

extern "C" int fq_cache_evict(const fq_paged_batch *batch, const void *k_pages, const void *v_pages, int n_kv_heads, const float *weights,
                              int weights_stride, int keep, int recent, const int32_t *dst_table, int dst_stride, int dst_pages, void *k_out,
                              void *v_out, int32_t *kept, int32_t *new_len, float *weights_out, int weights_out_stride, void *stream)
{
    const char *fn = "fq_cache_evict";
    if (int rc = check_batch(fn, batch, n_kv_heads))
        return rc;
    if (!k_pages || !v_pages || !weights || !dst_table || !k_out || !v_out || !kept || !new_len)
        return fq_fail(FQ_ERR_NULL, "%s: NULL argument", fn);
    if (keep <= 0 || keep > (1 << 30) || recent < 0 || recent > keep)
        return fq_fail(FQ_ERR_SHAPE, "%s: keep=%d recent=%d (need 0 <= recent <= keep, 0 < keep)", fn, keep, recent);
    if (int rc = check_pool(fn, batch->page, dst_pages, n_kv_heads))
        return rc;
    const int most = batch->max_len < keep ? batch->max_len : keep;
    if (weights_stride < batch->max_len || (weights_out && weights_out_stride < most) || dst_stride <= 0 ||
        (long long)dst_stride * batch->page < most)
        return fq_fail(FQ_ERR_SHAPE, "%s: weights_stride=%d weights_out_stride=%d dst_stride=%d for %d positions cut to %d", fn, weights_stride,
                       weights_out_stride, dst_stride, batch->max_len, most);
    if (!aligned16(k_pages) || !aligned16(v_pages) || !aligned16(k_out) || !aligned16(v_out))
        return fq_fail(FQ_ERR_ALIGN, "%s: pointers must be 16-byte aligned", fn);
    const size_t rows = (size_t)batch->seqs * n_kv_heads - 1;
    if (weights_out && (weights_out == weights || overlap(weights, (rows * weights_stride + batch->max_len) * 4, weights_out,
                                                          (rows * weights_out_stride + most) * 4)))
        return fq_fail(FQ_ERR_SHAPE, "%s: weights_out must not be weights", fn);
    if (overlap(batch->seq_len, (size_t)batch->seqs * 4, new_len, (size_t)batch->seqs * 4))
        return fq_fail(FQ_ERR_SHAPE, "%s: new_len must not be seq_len", fn);
    return check_hip(fq_launch_cache_evict(*batch, k_pages, v_pages, n_kv_heads, weights, weights_stride, keep, recent, dst_table, dst_stride,
                                           dst_pages, k_out, v_out, kept, new_len, weights_out, weights_out_stride,
                                           static_cast<fq_stream>(stream)), "fq_cache_evict launch");
}

// ------------------------------------------------------------------ trees of tokens
extern "C" int fq_paged_plan(const fq_paged_batch *batch, const int32_t *new_tokens, const int32_t *cached, const int32_t *next_position,
                             const int32_t *parents, const int32_t *held, int32_t *held_out, int32_t *free_pages, const int32_t *free_count,
                             int32_t *free_out, int32_t *lacking, int32_t *positions, int32_t *slots, uint64_t *mask, int mask_words, void *stream)
{
    const char *fn = "fq_paged_plan";
    if (int rc = check_batch(fn, batch, 1))
        return rc;
    if (!new_tokens || !cached || !held || !held_out || !free_pages || !free_count || !free_out || !lacking || (batch->tokens > 0 && (!positions || !slots)))
        return fq_fail(FQ_ERR_NULL, "%s: NULL argument", fn);
    if (batch->tokens >= 1 << 28)
        return fq_fail(FQ_ERR_SHAPE, "%s: tokens=%d (below 2^28)", fn, batch->tokens);
    if (mask && !parents)
        return fq_fail(FQ_ERR_NULL, "%s: a mask without parents", fn);
    if (mask ? mask_words <= 0 || mask_words > FQ_TREE_WORDS || batch->max_q > 64 * mask_words : mask_words != 0)
        return fq_fail(FQ_ERR_SHAPE, "%s: mask_words=%d for trees of up to %d tokens (64 a word, at most %d words; 0 without a mask)", fn, mask_words,
                       batch->max_q, FQ_TREE_WORDS);
    if (parents && batch->max_q > 64 * FQ_TREE_WORDS)
        return fq_fail(FQ_ERR_SHAPE, "%s: trees of up to %d tokens (at most %d)", fn, batch->max_q, 64 * FQ_TREE_WORDS);
    if (reinterpret_cast<uintptr_t>(mask) & 7)
        return fq_fail(FQ_ERR_ALIGN, "%s: mask must be 8-byte aligned", fn);
    // Everything that is written is an array of its own, but for what may be changed in place.
    const size_t n = batch->seqs, m = batch->tokens;
    struct Run {
        const void *at;
        size_t bytes;
    };
    const Run out[] = {{batch->q_start, (n + 1) * 4}, {batch->seq_len, n * 4}, {batch->table, n * batch->table_stride * 4}, {held_out, n * 4},
                       {free_pages, (size_t)batch->pages * 4}, {free_out, 4}, {lacking, 4}, {positions, m * 4}, {slots, m * 4}, {mask, m * mask_words * 8}};
    const Run in[] = {{new_tokens, n * 4}, {cached, n * 4}, {next_position, n * 4}, {parents, m * 4}, {held, n * 4}, {free_count, 4}};
    for (const Run &o : out) {
        for (const Run &i : in) {
            const bool in_place = (i.at == cached && o.at == batch->seq_len) || (i.at == held && o.at == held_out) || (i.at == free_count && o.at == free_out);
            if (i.at && o.at && o.bytes && i.bytes && overlap(o.at, o.bytes, i.at, i.bytes) && !(in_place && i.at == o.at))
                return fq_fail(FQ_ERR_SHAPE, "%s: an output overlaps an input (cached may be seq_len, held held_out, free_count free_out)", fn);
        }
        for (const Run &x : out)
            if (&x < &o && x.at && o.at && x.bytes && o.bytes && overlap(o.at, o.bytes, x.at, x.bytes))
                return fq_fail(FQ_ERR_SHAPE, "%s: two outputs overlap", fn);
    }
    const fq_plan_arrays a{new_tokens, cached, next_position, parents, held, held_out, free_pages, free_count, free_out, lacking, positions, slots, mask, mask_words};
    return check_hip(fq_launch_paged_plan(*batch, a, static_cast<fq_stream>(stream)), "fq_paged_plan launch");
}

extern "C" size_t fq_attn_tree_workspace_bytes(const fq_paged_batch *batch, int n_heads, int n_kv_heads)
{
    const char *fn = "fq_attn_tree_workspace_bytes";
    if (check_batch(fn, batch, n_kv_heads) || check_heads(fn, batch->tokens, n_heads, n_kv_heads))
        return 0;
    return align_up(fq_attn_paged_scratch_bytes(*batch, n_heads, n_kv_heads, false, true));
}

extern "C" int fq_attn_tree(const fq_paged_batch *batch, const uint64_t *mask, int mask_words, const int32_t *tail, const void *q, int ldq, int n_heads,
                            int n_kv_heads, const void *k_pages, const void *v_pages, float scale, void *out, float *lse, void *workspace,
                            size_t workspace_bytes, void *stream)
{
    const char *fn = "fq_attn_tree";
    if (int rc = check_batch(fn, batch, n_kv_heads))
        return rc;
    if (int rc = check_heads(fn, batch->tokens, n_heads, n_kv_heads))
        return rc;
    if (!k_pages || !v_pages || (batch->tokens > 0 && (!q || !out || !mask)))
        return fq_fail(FQ_ERR_NULL, "%s: NULL argument", fn);
    if (mask_words <= 0 || mask_words > FQ_TREE_WORDS)
        return fq_fail(FQ_ERR_SHAPE, "%s: mask_words=%d (1 to %d)", fn, mask_words, FQ_TREE_WORDS);
    if (!stride_ok(ldq, n_heads * 128))
        return fq_fail(FQ_ERR_SHAPE, "%s: ldq=%d (at least the row, a multiple of 8)", fn, ldq);
    if (!(scale > 0.f) || scale > 1e30f)
        return fq_fail(FQ_ERR_SHAPE, "%s: scale=%g (must be positive and finite)", fn, scale);
    const size_t need = fq_attn_paged_scratch_bytes(*batch, n_heads, n_kv_heads, false, true);
    if (need > 0 && (!workspace || workspace_bytes < need))
        return fq_fail(FQ_ERR_WORKSPACE, "%s: workspace of %zu bytes, need %zu", fn, workspace ? workspace_bytes : (size_t)0, need);
    if (!aligned16(q) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(out) || !aligned16(workspace) || (reinterpret_cast<uintptr_t>(mask) & 7))
        return fq_fail(FQ_ERR_ALIGN, "%s: pointers must be 16-byte aligned, the mask 8-byte", fn);
    const size_t row = (size_t)n_heads * 128 * 2;
    if (batch->tokens > 0 && overlap(q, (size_t)(batch->tokens - 1) * ldq * 2 + row, out, batch->tokens * row))
        return fq_fail(FQ_ERR_SHAPE, "%s: out overlaps q, which every part of the call reads", fn);
    if (batch->tokens == 0)
        return FQ_OK;
    return check_hip(fq_launch_attn_paged(*batch, q, ldq, n_heads, n_kv_heads, k_pages, v_pages, scale, out, lse, nullptr, nullptr, 0, workspace,
                                          static_cast<fq_stream>(stream), mask, mask_words, tail), "fq_attn_tree launch");
}

extern "C" int fq_tree_commit(const fq_paged_batch *batch, const int32_t *tail, const int32_t *parents, const int32_t *drafted, const int32_t *following,
                              void *k_pages, void *v_pages, int layers, int n_kv_heads, int32_t *path, int path_stride, int32_t *accepted,
                              int32_t *bonus, int32_t *new_len, void *stream)
{
    const char *fn = "fq_tree_commit";
    if (int rc = check_batch(fn, batch, n_kv_heads))
        return rc;
    if (!k_pages || !v_pages || !path || !accepted || !new_len)
        return fq_fail(FQ_ERR_NULL, "%s: NULL argument", fn);
    const bool walk = parents || drafted || following;
    if (walk && (!parents || !drafted || !following))
        return fq_fail(FQ_ERR_NULL, "%s: parents, drafted and following go together", fn);
    if (walk ? tail != nullptr : bonus != nullptr)
        return fq_fail(FQ_ERR_SHAPE, walk ? "%s: the tail of a tree that is checked is the tokens of the call" : "%s: bonus without a tree to check", fn);
    if (layers <= 0 || layers > 65535 || (long long)layers * n_kv_heads * batch->seqs >= 1 << 24 || path_stride <= 0 || path_stride > 1 << 24)
        return fq_fail(FQ_ERR_SHAPE, "%s: layers=%d n_kv_heads=%d seqs=%d path_stride=%d (product of the first three below 2^24)", fn, layers, n_kv_heads,
                       batch->seqs, path_stride);
    if (!aligned16(k_pages) || !aligned16(v_pages))
        return fq_fail(FQ_ERR_ALIGN, "%s: pools must be 16-byte aligned", fn);
    const size_t pool = (size_t)layers * batch->pages * n_kv_heads * batch->page * 256, n = batch->seqs;
    if (overlap(k_pages, pool, v_pages, pool))
        return fq_fail(FQ_ERR_SHAPE, "%s: the pools overlap", fn);
    // what every part of the call reads is not what one of them writes
    const void *const written[] = {path, accepted, bonus, new_len};
    const size_t size[] = {n * path_stride * 4, n * 4, n * 4, n * 4};
    const void *const read[] = {batch->q_start, batch->seq_len, batch->table, tail, parents, drafted, following};
    const size_t read_size[] = {(n + 1) * 4, n * 4, n * batch->table_stride * 4, n * 4, (size_t)batch->tokens * 4, (size_t)batch->tokens * 4,
                                (size_t)batch->tokens * 4};
    for (int i = 0; i < 4; ++i) {
        for (int j = 0; j < 7; ++j)
            if (written[i] && read[j] && read_size[j] && overlap(written[i], size[i], read[j], read_size[j]))
                return fq_fail(FQ_ERR_SHAPE, "%s: an output overlaps an input", fn);
        for (int j = 0; j < i; ++j)
            if (written[i] && written[j] && overlap(written[i], size[i], written[j], size[j]))
                return fq_fail(FQ_ERR_SHAPE, "%s: two of path, accepted, bonus and new_len overlap", fn);
    }
    return check_hip(fq_launch_tree_commit(*batch, tail, parents, drafted, following, k_pages, v_pages, layers, n_kv_heads, path, path_stride, accepted,
                                           bonus, new_len, static_cast<fq_stream>(stream)), "fq_tree_commit launch");
}

namespace {

int check_beams(const char *fn, int requests, int beams, int vocab, int width)
{
    if (requests <= 0 || beams <= 0 || beams > 64 || width <= 0 || width > 64 || vocab <= 0 || vocab > 1 << 18 ||
        (long long)requests * beams * ((vocab + 8191) / 8192) >= 1 << 24) // a grid has less than 2^32 threads
        return fq_fail(FQ_ERR_SHAPE, "%s: requests=%d beams=%d vocab=%d width=%d (beams and width 1 to 64, vocab up to 2^18, requests * beams for each 8192 "
                       "of it below 2^24)", fn, requests, beams, vocab, width);
    return FQ_OK;
}

} // namespace

extern "C" size_t fq_beam_step_workspace_bytes(int requests, int beams, int vocab, int width)
{
    if (check_beams("fq_beam_step_workspace_bytes", requests, beams, vocab, width))
        return 0;
    return align_up(fq_beam_scratch_bytes(requests, beams, vocab, width));
}

extern "C" int fq_beam_step(const void *logits, int64_t ld, const float *scores, const int32_t *done, int eos, int requests, int beams, int vocab, int width,
                            int32_t *parent, int32_t *token, float *scores_out, int32_t *done_out, const uint64_t *mask, uint64_t *mask_out,
                            int mask_words, const int32_t *tail, void *workspace, size_t workspace_bytes, void *stream)
{
    const char *fn = "fq_beam_step";
    if (int rc = check_beams(fn, requests, beams, vocab, width))
        return rc;
    if (!logits || !scores || !parent || !token || !scores_out)
        return fq_fail(FQ_ERR_NULL, "%s: NULL argument", fn);
    if (ld < vocab || ld > 1ll << 32)
        return fq_fail(FQ_ERR_SHAPE, "%s: ld=%lld for rows of %d", fn, (long long)ld, vocab);
    if (eos >= vocab || (done && eos < 0))
        return fq_fail(FQ_ERR_SHAPE, "%s: eos=%d of %d tokens%s", fn, eos, vocab, done ? ", which ended beams go on with" : "");
    if (mask_out ? mask_words <= 0 || mask_words > FQ_TREE_WORDS : mask || mask_words != 0)
        return fq_fail(FQ_ERR_SHAPE, "%s: mask_words=%d (1 to %d with mask_out, 0 without, and no mask then)", fn, mask_words, FQ_TREE_WORDS);
    const size_t need = fq_beam_scratch_bytes(requests, beams, vocab, width);
    if (!workspace || workspace_bytes < need)
        return fq_fail(FQ_ERR_WORKSPACE, "%s: workspace of %zu bytes, need %zu", fn, workspace ? workspace_bytes : (size_t)0, need);
    if (!aligned16(workspace) || (reinterpret_cast<uintptr_t>(logits) & 1) || ((reinterpret_cast<uintptr_t>(mask) | reinterpret_cast<uintptr_t>(mask_out)) & 7))
        return fq_fail(FQ_ERR_ALIGN, "%s: the workspace must be 16-byte aligned, masks 8-byte, logits 2-byte", fn);
    const size_t in = (size_t)requests * beams, n = (size_t)requests * width;
    const void *const written[] = {parent, token, scores_out, done_out, mask_out, workspace};
    const size_t size[] = {n * 4, n * 4, n * 4, n * 4, n * mask_words * 8, need};
    const void *const read[] = {logits, scores, done, mask, tail};
    const size_t read_size[] = {((in - 1) * ld + vocab) * 2, in * 4, in * 4, in * mask_words * 8, (size_t)requests * 4};
    for (int i = 0; i < 6; ++i) {
        for (int j = 0; j < 5; ++j)
            if (written[i] && read[j] && overlap(written[i], size[i], read[j], read_size[j]))
                return fq_fail(FQ_ERR_SHAPE, "%s: an output or the workspace overlaps an input", fn);
        for (int j = 0; j < i; ++j)
            if (written[i] && written[j] && overlap(written[i], size[i], written[j], size[j]))
                return fq_fail(FQ_ERR_SHAPE, "%s: two outputs, or one and the workspace, overlap", fn);
    }
    const fq_beam_arrays a{scores, done, tail, parent, token, done_out, scores_out, mask, mask_out, eos, mask_words};
    return check_hip(fq_launch_beam_step(logits, ld, requests, beams, vocab, width, a, workspace, static_cast<fq_stream>(stream)), "fq_beam_step launch");
}
