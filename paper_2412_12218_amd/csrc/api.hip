// C ABI of libftc: host-side argument validation and dispatch.  See include/ftc.h for the
// contract of every entry point.
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <mutex>

#include "ftc_common.hpp"

namespace ftc {

static thread_local char g_err[512] = "";

void set_error(const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof(g_err), fmt, ap);
    va_end(ap);
}

int32_t launch_status(const char *what)
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return FTC_OK;
    set_error("%s: HIP error %d (%s)", what, static_cast<int>(e), hipGetErrorString(e));
    return FTC_EHIP;
}

static int32_t fail(int32_t code, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof(g_err), fmt, ap);
    va_end(ap);
    return code;
}

static int32_t check_csr(const ftc_csr *g, const char *who)
{
    if (!g) return fail(FTC_EINVAL, "%s: graph is NULL", who);
    if (g->n < 0 || g->nnz < 0) return fail(FTC_EINVAL, "%s: negative n or nnz", who);
    if (!g->row_ptr) return fail(FTC_EINVAL, "%s: row_ptr is NULL", who);
    if (g->nnz > 0 && !g->col_idx) return fail(FTC_EINVAL, "%s: col_idx is NULL", who);
    if (g->n == 0 && g->nnz != 0) return fail(FTC_EINVAL, "%s: nnz > 0 with n == 0", who);
    return FTC_OK;
}

static int32_t check_windows(const ftc_csr *g, const ftc_windows *w, const char *who, bool need_arrays)
{
    if (!w) return fail(FTC_EINVAL, "%s: window index is NULL", who);
    if (w->blk_h < 1 || w->blk_h > 64 || w->blk_w < 1)
        return fail(FTC_EUNSUPPORTED, "%s: need 1 <= blk_h <= 64 and blk_w >= 1", who);
    if (w->n_windows != (g->n + w->blk_h - 1) / w->blk_h)
        return fail(FTC_EINVAL, "%s: n_windows != ceil(n / blk_h)", who);
    if (need_arrays) {
        if (!w->win_col_ptr || !w->summary || (w->n_windows > 0 && !w->block_partition))
            return fail(FTC_EINVAL, "%s: window arrays are NULL", who);
        if (g->nnz > 0 && (!w->edge_to_row || !w->edge_to_col || !w->win_cols))
            return fail(FTC_EINVAL, "%s: window edge arrays are NULL", who);
    }
    return FTC_OK;
}

static int32_t check_dense(const void *p, int ld, int dtype, int D, const char *who, const char *name)
{
    if (!p) return fail(FTC_EINVAL, "%s: %s is NULL", who, name);
    if (!valid_dtype(dtype)) return fail(FTC_EUNSUPPORTED, "%s: unknown dtype for %s", who, name);
    if (D < 1 || ld < D) return fail(FTC_EINVAL, "%s: need D >= 1 and ld >= D for %s", who, name);
    if (reinterpret_cast<uintptr_t>(p) % elem_size(dtype) != 0)
        return fail(FTC_EALIGN, "%s: %s is not aligned to its element size", who, name);
    return FTC_OK;
}

}  // namespace ftc

using namespace ftc;

// FTC_PATH_AUTO sends a window to the matrix cores when it has at least this many edges per
// condensed column (average reuse of a gathered row).  Values are the measured crossovers of the
// density sweep (bench.py --sweep, fp16, 2^18 nodes, 8.4 M edges): the vector path wins at every
// density up to completely full tiles for D <= 128 (both operations) and for SpMM at D = 256;
// SDDMM at D = 256 crosses over between 2.3 and 2.8 edges per condensed column.  A negative
// value means "never".
static float spmm_mfma_reuse(int D) { (void)D; return -1.f; }
static float sddmm_mfma_reuse(int D) { return D >= 256 ? 2.6f : -1.f; }
// Larger windows (hub rows) always stay on the edge-balanced vector kernels.
static constexpr int MFMA_MAX_WINDOW_EDGES = 4096;
// |beta| up to which the single-pass AGNN kernels (forward and backward) are used
static constexpr float AGNN_FUSED_MAX_BETA = 43.f;
// |beta| up to which the single pass also gives the probabilities; above, the three kernels, whose weights are relative to
// the row's maximum.  A row whose neighbours all point away has weights of exp(-2 |beta|) here, and the products with H
// must not become subnormal before they are divided by the row's sum: exp(-32) h is a normal number for |h| above 1e-24,
// which is 1e-12 of the smallest norm that is not clamped.  Error of the single pass against the three kernels in such rows:
// at 42 5e-5 / 1e-6 with features of 1e-3 and 6e-3 / 1e-6 with 1e-5, at 36 1e-2 / 1e-6 with 3e-11, at 16 7e-7 / 6e-7 with any.
static constexpr float AGNN_EDGE_P_MAX_BETA = 16.f;


#define FTC_TRY(expr)                   \
    do {                                \
        const int32_t st__ = (expr);    \
        if (st__ != FTC_OK) return st__; \
    } while (0)

extern "C" {

int32_t ftc_version(void) { return 100; }

const char *ftc_last_error(void) { return g_err; }

int32_t ftc_validate_csr(const ftc_csr *g, int32_t *flag, void *stream)
{
    FTC_TRY(check_csr(g, "ftc_validate_csr"));
    if (!flag) return fail(FTC_EINVAL, "ftc_validate_csr: flag is NULL");
    return launch_validate(*g, flag, static_cast<hipStream_t>(stream));
}

size_t ftc_build_windows_workspace_bytes(int32_t n, int32_t nnz, int32_t blk_h, int32_t blk_w)
{
    if (n < 0 || nnz < 0 || blk_h < 1 || blk_w < 1) return 0;
    return build_windows_ws(n, nnz, blk_h, blk_w);
}

int32_t ftc_build_windows_concurrent(const ftc_csr *g, ftc_windows *out, void *ws, size_t ws_bytes,
                                     const ftc_side_streams *side, void *stream)
{
    FTC_TRY(check_csr(g, "ftc_build_windows"));
    FTC_TRY(check_windows(g, out, "ftc_build_windows", true));
    const size_t need = build_windows_ws(g->n, g->nnz, out->blk_h, out->blk_w);
    if (!ws || ws_bytes < need)
        return fail(FTC_EWORKSPACE, "ftc_build_windows: workspace of %zu bytes needed, %zu given", need,
                    ws ? ws_bytes : static_cast<size_t>(0));
    if (reinterpret_cast<uintptr_t>(ws) % 256 != 0)
        return fail(FTC_EALIGN, "ftc_build_windows: workspace must be 256-byte aligned");
    if (side) {
        bool ok = side->fork != nullptr;
        for (int i = 0; i < 3; ++i) {
            ok = ok && side->stream[i] && side->join[i] && side->stream[i] != stream;
            for (int j = 0; j < i; ++j) ok = ok && side->stream[i] != side->stream[j] && side->join[i] != side->join[j];
            ok = ok && side->join[i] != side->fork;
        }
        if (!ok)
            return fail(FTC_EINVAL, "ftc_build_windows_concurrent: side needs three distinct streams other than `stream` and "
                                    "four distinct events");
    }
    return launch_build_windows(*g, *out, ws, ws_bytes, side, static_cast<hipStream_t>(stream));
}

int32_t ftc_build_windows(const ftc_csr *g, ftc_windows *out, void *ws, size_t ws_bytes, void *stream)
{
    return ftc_build_windows_concurrent(g, out, ws, ws_bytes, nullptr, stream);
}

int32_t ftc_gcn_norm(const ftc_csr *g, const ftc_windows *w, float *vals, float *dinv, void *stream)
{
    FTC_TRY(check_csr(g, "ftc_gcn_norm"));
    if (w) {
        FTC_TRY(check_windows(g, w, "ftc_gcn_norm", false));
        if (g->nnz > 0 && !w->edge_to_row) return fail(FTC_EINVAL, "ftc_gcn_norm: edge_to_row is NULL");
    }
    return launch_gcn_norm(*g, w, vals, dinv, static_cast<hipStream_t>(stream));
}

// What a call needs at least (`least`), or with room for the shorter ranges of small graphs and for odd widths: that is
// what the *_workspace_bytes queries return; a call that gets less than that but at least the former runs with long ranges.
static size_t spmm_ws(int32_t n, int32_t nnz, int32_t D, bool least) { return spmm_seg_ws(n, nnz, D, least) + flag_bytes(n); }

size_t ftc_spmm_workspace_bytes(int32_t n, int32_t nnz, int32_t D)
{
    if (n < 0 || nnz < 0 || D < 1) return 0;
    return spmm_ws(n, nnz, D, false);
}

int32_t ftc_spmm(const ftc_csr *g, const ftc_windows *w, const float *vals, const void *X, int32_t ldx,
                 int32_t x_dtype, int32_t D, void *out, int32_t ldo, int32_t out_dtype, const float *out_scale,
                 int32_t relu, int32_t path, void *ws, size_t ws_bytes, void *stream)
{
    const Epi epi{relu, out_scale};
    FTC_TRY(check_csr(g, "ftc_spmm"));
    if (g->n == 0) return FTC_OK;
    FTC_TRY(check_dense(X, ldx, x_dtype, D, "ftc_spmm", "X"));
    FTC_TRY(check_dense(out, ldo, out_dtype, D, "ftc_spmm", "out"));
    if (out == X) return fail(FTC_EINVAL, "ftc_spmm: out aliases X");
    if (w) FTC_TRY(check_windows(g, w, "ftc_spmm", true));
    if (path != FTC_PATH_AUTO && path != FTC_PATH_VALU && path != FTC_PATH_MFMA)
        return fail(FTC_EINVAL, "ftc_spmm: unknown path %d", path);
    int vec, lpr;
    const bool rows16 = aligned16(X) && aligned16(out) &&
                        (static_cast<int64_t>(ldx) * elem_size(x_dtype)) % 16 == 0 &&
                        (static_cast<int64_t>(ldo) * elem_size(out_dtype)) % 16 == 0;
    const bool seg_ok = w && rows16 && seg_shape(x_dtype, D, &vec, &lpr);
    const bool mfma_ok = seg_ok && w->blk_h == 16 && mfma_shape_ok(x_dtype, D);
    if (path == FTC_PATH_MFMA && !mfma_ok)
        return fail(FTC_EUNSUPPORTED,
                    "ftc_spmm: the matrix-core path needs a window index with blk_h = 16, fp16/bf16 "
                    "features with D a multiple of 8 (<= 256) and 16-byte aligned rows");
    // a graph without entries only has its output rows cleared, whatever the path
    const bool can_seg = seg_ok && g->nnz > 0, can_mfma = mfma_ok && g->nnz > 0;
    hipStream_t hs = static_cast<hipStream_t>(stream);
    if (can_seg) {
        const size_t need = spmm_ws(g->n, g->nnz, D, true);
        if (!ws || ws_bytes < need)
            return fail(FTC_EWORKSPACE, "ftc_spmm: workspace of %zu bytes needed, %zu given", need,
                        ws ? ws_bytes : static_cast<size_t>(0));
        if (reinterpret_cast<uintptr_t>(ws) % 256 != 0)
            return fail(FTC_EALIGN, "ftc_spmm: workspace must be 256-byte aligned");
        if (path != FTC_PATH_MFMA && spmm_group_ok(g->n, static_cast<int64_t>(ldx) * elem_size(x_dtype), D * elem_size(x_dtype), g->nnz))
            return launch_spmm_group(*g, vals, X, ldx, x_dtype, D, out, ldo, out_dtype, epi, hs);
        uint8_t *flags = nullptr;
        const size_t fb = flag_bytes(g->n);  // the flags take the end of the workspace, the carried pieces the rest
        const float reuse = path == FTC_PATH_MFMA ? 0.f : spmm_mfma_reuse(D);
        if (can_mfma && path != FTC_PATH_VALU && reuse >= 0.f) {
            flags = reinterpret_cast<uint8_t *>(static_cast<char *>(ws) + (ws_bytes - fb) / 256 * 256);
            FTC_TRY(launch_classify(*g, *w, reuse, MFMA_MAX_WINDOW_EDGES, flags, hs));
        }
        FTC_TRY(launch_spmm_seg(*g, *w, vals, X, ldx, x_dtype, D, out, ldo, out_dtype, epi, ws, (ws_bytes - fb) / 256 * 256,
                                flags, hs));
        if (flags) return launch_spmm_mfma(*g, *w, vals, X, ldx, x_dtype, D, out, ldo, out_dtype, epi, flags, hs);
        return FTC_OK;
    }
    // Widths that are no multiple of a lane's piece, or rows that are not 16-byte aligned (7 classes, say): on small graphs a
    // kernel of its own that takes no scratch memory, else the edge-balanced kernels again, at element alignment, wherever the
    // workspace holds their carried pieces.  The row-wise kernels below give a row to a thread per column, one after the
    // other over its entries (fp32, 10 columns, power-law graph with 100 000 nodes: 305 us against 36).
    if (w && g->nnz > 0) {
        const bool x16 = aligned16(X) && (static_cast<int64_t>(ldx) * elem_size(x_dtype)) % 16 == 0;
        const size_t any = spmm_any_width_ws(x_dtype, D, g->n, g->nnz, x16 && spmm_lane_shape(x_dtype, D, ldx));
        if (any > 0 && spmm_small_ok(D, g->nnz))
            return launch_spmm_small(*g, vals, X, ldx, x_dtype, D, out, ldo, out_dtype, epi, hs);
        if (any > 0 && ws && reinterpret_cast<uintptr_t>(ws) % 256 == 0 && ws_bytes >= any)
            return launch_spmm_seg(*g, *w, vals, X, ldx, x_dtype, D, out, ldo, out_dtype, epi, ws, ws_bytes, nullptr, hs);
    }
    return launch_spmm_rows(*g, vals, X, ldx, x_dtype, D, out, ldo, out_dtype, epi, hs);
}

// ftc_spmm for callers that can neither allocate nor hand over a workspace: the scratch memory of the
// aggregation kernels (carry rows of the cut rows, window flags) lives in this file-scope device array,
// one copy per GPU, held until the process ends.  In host code the array's name is only a stand-in; its
// device address is asked for once per device and kept.
}  // extern "C"
namespace {
static __device__ __align__(256) unsigned char scratch[NOALLOC_SCRATCH_BYTES];
constexpr int NOALLOC_MAX_DEVICES = 64;
void *g_scratch_ptr[NOALLOC_MAX_DEVICES];  // device address of `scratch` on every device that has asked
std::mutex g_scratch_mutex;

int32_t scratch_of_current_device(void **ptr)
{
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= NOALLOC_MAX_DEVICES) {
        (void)hipGetLastError();
        return fail(FTC_EHIP, "ftc_spmm_noalloc: no current device (or a device index beyond %d)", NOALLOC_MAX_DEVICES - 1);
    }
    std::lock_guard<std::mutex> lock(g_scratch_mutex);
    if (!g_scratch_ptr[dev]) {
        void *p = nullptr;
        const hipError_t e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
        if (e != hipSuccess || !p) {
            (void)hipGetLastError();
            return fail(FTC_EHIP, "ftc_spmm_noalloc: hipGetSymbolAddress failed (%d: %s)", static_cast<int>(e),
                        hipGetErrorString(e));
        }
        g_scratch_ptr[dev] = p;
    }
    *ptr = g_scratch_ptr[dev];
    return FTC_OK;
}
}  // namespace
extern "C" {

int32_t ftc_spmm_noalloc(const ftc_csr *g, const ftc_windows *w, const float *vals, const void *X, int32_t ldx,
                         int32_t x_dtype, int32_t D, void *out, int32_t ldo, int32_t out_dtype, const float *out_scale,
                         int32_t relu, int32_t path, void *stream)
{
    FTC_TRY(check_csr(g, "ftc_spmm_noalloc"));
    if (D < 1) return fail(FTC_EINVAL, "ftc_spmm_noalloc: need D >= 1");
    const size_t need = ftc_spmm_workspace_bytes(g->n, g->nnz, D);
    if (need > NOALLOC_SCRATCH_BYTES)
        return fail(FTC_EWORKSPACE,
                    "ftc_spmm_noalloc: this graph and width need %zu bytes of scratch memory, the built-in buffer holds "
                    "%zu; use ftc_spmm with a workspace",
                    need, NOALLOC_SCRATCH_BYTES);
    void *ptr = nullptr;
    FTC_TRY(scratch_of_current_device(&ptr));
    return ftc_spmm(g, w, vals, X, ldx, x_dtype, D, out, ldo, out_dtype, out_scale, relu, path, ptr, NOALLOC_SCRATCH_BYTES,
                    stream);
}

size_t ftc_sddmm_workspace_bytes(int32_t n, int32_t nnz, int32_t D)
{
    if (n < 0 || nnz < 0 || D < 1) return 0;
    // window flags of the per-window dispatch, then two arrays of inverse row norms (cosine mode on
    // the paths that do not recompute the norms from the rows)
    return align_up(flag_bytes(n), 256) + 2 * align_up(static_cast<size_t>(n) * sizeof(float), 256);
}

int32_t ftc_sddmm(const ftc_csr *g, const ftc_windows *w, const void *X, const void *Y, int32_t ld,
                  int32_t dtype, int32_t D, const float *row_scale, const float *col_scale, float alpha,
                  int32_t cosine, float *edge_out, int32_t path, void *ws, size_t ws_bytes, void *stream)
{
    FTC_TRY(check_csr(g, "ftc_sddmm"));
    if (g->n == 0 || g->nnz == 0) return FTC_OK;
    FTC_TRY(check_dense(X, ld, dtype, D, "ftc_sddmm", "X"));
    FTC_TRY(check_dense(Y, ld, dtype, D, "ftc_sddmm", "Y"));
    if (!edge_out) return fail(FTC_EINVAL, "ftc_sddmm: edge_out is NULL");
    if (cosine && (row_scale || col_scale))
        return fail(FTC_EINVAL, "ftc_sddmm: cosine mode takes no row_scale / col_scale");
    if (w) FTC_TRY(check_windows(g, w, "ftc_sddmm", true));
    if (path != FTC_PATH_AUTO && path != FTC_PATH_VALU && path != FTC_PATH_MFMA)
        return fail(FTC_EINVAL, "ftc_sddmm: unknown path %d", path);
    int vec, lpr;
    const bool can_edges = w && aligned16(X) && aligned16(Y) &&
                           (static_cast<int64_t>(ld) * elem_size(dtype)) % 16 == 0 && seg_shape(dtype, D, &vec, &lpr);
    const bool can_mfma = can_edges && w->blk_h == 16 && mfma_shape_ok(dtype, D);
    if (path == FTC_PATH_MFMA && !can_mfma)
        return fail(FTC_EUNSUPPORTED,
                    "ftc_sddmm: the matrix-core path needs a window index with blk_h = 16, fp16/bf16 "
                    "features with D a multiple of 8 (<= 256) and 16-byte aligned rows");
    hipStream_t hs = static_cast<hipStream_t>(stream);
    const float reuse = path == FTC_PATH_MFMA ? 0.f : sddmm_mfma_reuse(D);
    const bool use_mfma = can_mfma && path != FTC_PATH_VALU && reuse >= 0.f;
    const bool need_ws = use_mfma || (cosine && !can_edges);
    if (need_ws) {
        const size_t need = ftc_sddmm_workspace_bytes(g->n, g->nnz, D);
        if (!ws || ws_bytes < need)
            return fail(FTC_EWORKSPACE, "ftc_sddmm: workspace of %zu bytes needed, %zu given", need,
                        ws ? ws_bytes : static_cast<size_t>(0));
        if (reinterpret_cast<uintptr_t>(ws) % 256 != 0)
            return fail(FTC_EALIGN, "ftc_sddmm: workspace must be 256-byte aligned");
    }
    // Cosine mode: the edge-parallel vector kernel recomputes the norms from the rows it holds; the
    // other kernels take them as scale arrays, which are produced here.
    if (cosine && (use_mfma || !can_edges)) {
        char *p = static_cast<char *>(ws) + align_up(flag_bytes(g->n), 256);
        float *rx = reinterpret_cast<float *>(p);
        float *ry = X == Y ? rx : reinterpret_cast<float *>(p + align_up(static_cast<size_t>(g->n) * sizeof(float), 256));
        FTC_TRY(launch_row_rnorm(g->n, X, ld, dtype, D, rx, hs));
        if (ry != rx) FTC_TRY(launch_row_rnorm(g->n, Y, ld, dtype, D, ry, hs));
        row_scale = rx;
        col_scale = ry;
    }
    if (can_edges) {
        uint8_t *flags = nullptr;
        if (use_mfma) {
            flags = static_cast<uint8_t *>(ws);
            FTC_TRY(launch_classify(*g, *w, reuse, MFMA_MAX_WINDOW_EDGES, flags, hs));
        }
        FTC_TRY(launch_sddmm_edges(*g, *w, X, Y, ld, dtype, D, row_scale, col_scale, alpha, edge_out, flags,
                                   cosine != 0, hs));
        if (flags)
            return launch_sddmm_mfma(*g, *w, X, Y, ld, dtype, D, row_scale, col_scale, alpha, edge_out, flags, hs);
        return FTC_OK;
    }
    return launch_sddmm_rows(*g, X, Y, ld, dtype, D, row_scale, col_scale, alpha, edge_out, hs);
}

int32_t ftc_row_rnorm(int32_t n, const void *H, int32_t ld, int32_t dtype, int32_t D, float *rinv,
                      void *stream)
{
    if (n < 0) return fail(FTC_EINVAL, "ftc_row_rnorm: negative n");
    if (n == 0) return FTC_OK;
    FTC_TRY(check_dense(H, ld, dtype, D, "ftc_row_rnorm", "H"));
    if (!rinv) return fail(FTC_EINVAL, "ftc_row_rnorm: rinv is NULL");
    return launch_row_rnorm(n, H, ld, dtype, D, rinv, static_cast<hipStream_t>(stream));
}

size_t ftc_edge_softmax_workspace_bytes(int32_t n, int32_t nnz)
{
    if (n < 0 || nnz < 0) return 0;
    return softmax_seg_ws(n, nnz);
}

int32_t ftc_edge_softmax(const ftc_csr *g, const ftc_windows *w, const float *e_in, float *p_out, void *ws,
                         size_t ws_bytes, void *stream)
{
    FTC_TRY(check_csr(g, "ftc_edge_softmax"));
    if (g->n == 0 || g->nnz == 0) return FTC_OK;
    if (!e_in || !p_out) return fail(FTC_EINVAL, "ftc_edge_softmax: NULL edge array");
    if (!w) return launch_softmax(*g, e_in, p_out, static_cast<hipStream_t>(stream));
    FTC_TRY(check_windows(g, w, "ftc_edge_softmax", false));
    if (!w->edge_to_row) return fail(FTC_EINVAL, "ftc_edge_softmax: edge_to_row is NULL");
    const size_t need = softmax_seg_ws(g->n, g->nnz);
    if (!ws || ws_bytes < need)
        return fail(FTC_EWORKSPACE, "ftc_edge_softmax: workspace of %zu bytes needed, %zu given", need,
                    ws ? ws_bytes : static_cast<size_t>(0));
    if (reinterpret_cast<uintptr_t>(ws) % 256 != 0)
        return fail(FTC_EALIGN, "ftc_edge_softmax: workspace must be 256-byte aligned");
    return launch_softmax_seg(*g, *w, e_in, p_out, ws, static_cast<hipStream_t>(stream));
}

int32_t ftc_update_gemm(int32_t n, const void *X, int32_t ldx, int32_t dtype, int32_t d_in, const void *W,
                        int32_t d_out, void *Z, int32_t ldz, int32_t z_dtype, const float *row_scale, int32_t relu,
                        void *stream)
{
    if (n < 0) return fail(FTC_EINVAL, "ftc_update_gemm: negative n");
    if (n == 0) return FTC_OK;
    FTC_TRY(check_dense(X, ldx, dtype, d_in, "ftc_update_gemm", "X"));
    FTC_TRY(check_dense(Z, ldz, z_dtype, d_out, "ftc_update_gemm", "Z"));
    if (!W) return fail(FTC_EINVAL, "ftc_update_gemm: W is NULL");
    if (Z == X) return fail(FTC_EINVAL, "ftc_update_gemm: Z aliases X");
    return launch_gemm(n, X, ldx, dtype, d_in, W, d_out, Z, ldz, z_dtype, Epi{relu, row_scale},
                       static_cast<hipStream_t>(stream));
}

// The intermediate Z = X * W: fp16 when the inputs are fp16 (halves the gathered bytes; its rounding,
// 2^-11 relative, stays far below the 16-bit tolerance), fp32 otherwise (a bf16 Z would round at
// 2^-9, the size of the tolerance itself).  Rows padded to 16 bytes.
static int z_dtype_for(int dtype) { return dtype == FTC_F16 ? FTC_F16 : FTC_F32; }
static int z_ld(int d_out, int zdt) { return zdt == FTC_F32 ? (d_out + 3) / 4 * 4 : (d_out + 7) / 8 * 8; }

static size_t gcn_layer_ws(int32_t n, int32_t nnz, int32_t d_out, bool least)
{
    if (n < 0 || nnz < 0 || d_out < 1) return 0;
    // sized for the fp32 intermediate, which covers the fp16 one
    const int ldz = z_ld(d_out, FTC_F32);
    return align_up(static_cast<size_t>(n) * ldz * sizeof(float), 256) + spmm_ws(n, nnz, d_out, least);
}

size_t ftc_gcn_layer_workspace_bytes(int32_t n, int32_t nnz, int32_t d_in, int32_t d_out)
{
    (void)d_in;
    return gcn_layer_ws(n, nnz, d_out, false);
}

int32_t ftc_gcn_layer(const ftc_csr *g, const ftc_windows *w, const float *vals, const float *dinv,
                      const void *X, int32_t ldx, int32_t dtype, int32_t d_in, const void *W, int32_t d_out,
                      int32_t relu, void *out, int32_t ldo, int32_t out_dtype, int32_t path, void *ws,
                      size_t ws_bytes, void *stream)
{
    FTC_TRY(check_csr(g, "ftc_gcn_layer"));
    if (g->n == 0) return FTC_OK;
    const size_t need = gcn_layer_ws(g->n, g->nnz, d_out, true);
    if (!ws || ws_bytes < need)
        return fail(FTC_EWORKSPACE, "ftc_gcn_layer: workspace of %zu bytes needed", need);
    if (reinterpret_cast<uintptr_t>(ws) % 256 != 0)
        return fail(FTC_EALIGN, "ftc_gcn_layer: workspace must be 256-byte aligned");
    if (!valid_dtype(dtype)) return fail(FTC_EUNSUPPORTED, "ftc_gcn_layer: unknown dtype");
    const int zdt = z_dtype_for(dtype);
    const int ldz = z_ld(d_out, zdt);
    void *Z = ws;
    const size_t zbytes = align_up(static_cast<size_t>(g->n) * z_ld(d_out, FTC_F32) * sizeof(float), 256);
    // factored normalisation: rows of X*W are scaled by dinv[j] as they are written, the aggregation
    // runs without edge values and scales output row i by dinv[i]
    FTC_TRY(ftc_update_gemm(g->n, X, ldx, dtype, d_in, W, d_out, Z, ldz, zdt, dinv, 0, stream));
    return ftc_spmm(g, w, dinv ? nullptr : vals, Z, ldz, zdt, d_out, out, ldo, out_dtype, dinv, relu, path,
                    static_cast<char *>(ws) + zbytes, ws_bytes - zbytes, stream);
}

static size_t agnn_unfused_bytes(int32_t n, int32_t nnz, int32_t D, bool least)
{
    return align_up(static_cast<size_t>(nnz) * sizeof(float), 256) +
           align_up(ftc_sddmm_workspace_bytes(n, nnz, D), 256) +
           align_up(ftc_edge_softmax_workspace_bytes(n, nnz), 256) + spmm_ws(n, nnz, D, least);
}

static size_t agnn_layer_ws(int32_t n, int32_t nnz, int32_t D, bool least)
{
    if (n < 0 || nnz < 0 || D < 1) return 0;
    // the single pass, and the rows' sums when the probabilities are asked for
    const size_t a = agnn_unfused_bytes(n, nnz, D, least);
    const size_t b = agnn_fused_ws(nnz, D, least) + (least ? 0 : align_up(static_cast<size_t>(n) * sizeof(float), 256));
    return a > b ? a : b;
}

size_t ftc_agnn_layer_workspace_bytes(int32_t n, int32_t nnz, int32_t D) { return agnn_layer_ws(n, nnz, D, false); }

int32_t ftc_agnn_layer(const ftc_csr *g, const ftc_windows *w, const void *H, int32_t ld, int32_t dtype,
                       int32_t D, float beta, void *out, int32_t ldo, int32_t out_dtype, float *edge_p, float *row_z,
                       float *out_f32, int32_t ld_f32, int32_t path, void *ws, size_t ws_bytes, void *stream)
{
    FTC_TRY(check_csr(g, "ftc_agnn_layer"));
    if (g->n == 0) return FTC_OK;
    FTC_TRY(check_dense(H, ld, dtype, D, "ftc_agnn_layer", "H"));
    FTC_TRY(check_dense(out, ldo, out_dtype, D, "ftc_agnn_layer", "out"));
    if (out == H) return fail(FTC_EINVAL, "ftc_agnn_layer: out aliases H");
    if (w) FTC_TRY(check_windows(g, w, "ftc_agnn_layer", true));
    const size_t need = agnn_layer_ws(g->n, g->nnz, D, true);
    if (!ws || ws_bytes < need)
        return fail(FTC_EWORKSPACE, "ftc_agnn_layer: workspace of %zu bytes needed", need);
    if (reinterpret_cast<uintptr_t>(ws) % 256 != 0)
        return fail(FTC_EALIGN, "ftc_agnn_layer: workspace must be 256-byte aligned");
    char *p = static_cast<char *>(ws);

    // One pass over the edges when the vector path applies.
    int vec, lpr;
    const bool rows16 = aligned16(H) && aligned16(out) && (static_cast<int64_t>(ld) * elem_size(dtype)) % 16 == 0 &&
                        (static_cast<int64_t>(ldo) * elem_size(out_dtype)) % 16 == 0;
    if (out_f32) {
        FTC_TRY(check_dense(out_f32, ld_f32, FTC_F32, D, "ftc_agnn_layer", "out_f32"));
        if (!aligned16(out_f32) || ld_f32 % 4 != 0)
            return fail(FTC_EALIGN, "ftc_agnn_layer: rows of out_f32 must be 16-byte aligned");
        if (static_cast<void *>(out_f32) == out || static_cast<const void *>(out_f32) == H)
            return fail(FTC_EINVAL, "ftc_agnn_layer: out_f32 aliases out or H");
    }
    const bool keep = row_z || out_f32;
    // the single pass shifts the softmax by |beta| instead of the row maximum: exp(-2 |beta|) must stay a
    // normal fp32 number; beyond that the chain with the row-wise softmax takes over
    const bool beta_ok = fabsf(beta) < AGNN_FUSED_MAX_BETA;
    if (!edge_p && w && beta_ok && (g->nnz > 0 || keep) && path != FTC_PATH_MFMA && rows16 &&
        seg_shape(dtype, D, &vec, &lpr)) {
        if (agnn_group_ok(g->n, static_cast<int64_t>(ld) * elem_size(dtype), D * elem_size(dtype), g->nnz))
            return launch_agnn_group(*g, H, ld, dtype, D, beta, out, ldo, out_dtype, row_z, out_f32, ld_f32, nullptr,
                                     static_cast<hipStream_t>(stream));
        return launch_agnn_fused(*g, *w, H, ld, dtype, D, beta, out, ldo, out_dtype, row_z, out_f32, ld_f32, nullptr, p,
                                 ws_bytes, static_cast<hipStream_t>(stream));
    }
    // The probabilities come from the same pass; the rows' sums take the end of the workspace.  (The size that was checked
    // above is at least that of the three kernels, which counts the scores and two arrays of n floats: the carried pieces of
    // ranges of SEG_R entries and the sums fit into that.)
    const size_t z_bytes = align_up(static_cast<size_t>(g->n) * sizeof(float), 256);
    if (edge_p && !keep && w && fabsf(beta) <= AGNN_EDGE_P_MAX_BETA && g->nnz > 0 && path != FTC_PATH_MFMA && rows16 &&
        seg_shape(dtype, D, &vec, &lpr)) {
        if (agnn_group_ok(g->n, static_cast<int64_t>(ld) * elem_size(dtype), D * elem_size(dtype), g->nnz))
            return launch_agnn_group(*g, H, ld, dtype, D, beta, out, ldo, out_dtype, nullptr, nullptr, 0, edge_p,
                                     static_cast<hipStream_t>(stream));
        const size_t at = (ws_bytes - z_bytes) / 256 * 256;
        return launch_agnn_fused(*g, *w, H, ld, dtype, D, beta, out, ldo, out_dtype, reinterpret_cast<float *>(p + at), nullptr, 0,
                                 edge_p, p, at, static_cast<hipStream_t>(stream));
    }
    if (keep)
        return fail(FTC_EUNSUPPORTED,
                    "ftc_agnn_layer: |beta| < 43 is needed, and row_z and out_f32 come from the single-pass route only (window index, no edge_p, not "
                    "FTC_PATH_MFMA, 16-byte aligned rows, a width the edge-balanced kernels cover)");

    float *scores = edge_p ? edge_p : reinterpret_cast<float *>(p);
    p += align_up(static_cast<size_t>(g->nnz) * sizeof(float), 256);
    const size_t sd = align_up(ftc_sddmm_workspace_bytes(g->n, g->nnz, D), 256);
    void *ws_sddmm = p;
    p += sd;
    const size_t sm = align_up(ftc_edge_softmax_workspace_bytes(g->n, g->nnz), 256);
    void *ws_softmax = p;
    p += sm;
    const size_t rest = ws_bytes - static_cast<size_t>(p - static_cast<char *>(ws));
    FTC_TRY(ftc_sddmm(g, w, H, H, ld, dtype, D, nullptr, nullptr, beta, 1, scores, path, ws_sddmm, sd, stream));
    FTC_TRY(ftc_edge_softmax(g, w, scores, scores, ws_softmax, sm, stream));
    return ftc_spmm(g, w, scores, H, ld, dtype, D, out, ldo, out_dtype, nullptr, 0, path, p, rest, stream);
}

// ---------------------------------------------------------------------------------------------------
// Backward pass (gradients are fp32)

int32_t ftc_transpose_index(const ftc_csr *g, const ftc_windows *w, int32_t *T, int32_t *flag, void *stream)
{
    FTC_TRY(check_csr(g, "ftc_transpose_index"));
    if (!flag) return fail(FTC_EINVAL, "ftc_transpose_index: flag is NULL");
    if (g->nnz > 0 && !T) return fail(FTC_EINVAL, "ftc_transpose_index: T is NULL");
    const int32_t *e2r = nullptr;
    if (w) {
        FTC_TRY(check_windows(g, w, "ftc_transpose_index", false));
        e2r = w->edge_to_row;
    }
    return launch_transpose_index(*g, e2r, T, flag, static_cast<hipStream_t>(stream));
}

int32_t ftc_edge_softmax_backward(const ftc_csr *g, const ftc_windows *w, const float *p, const float *dp, float *ds,
                                  void *ws, size_t ws_bytes, void *stream)
{
    FTC_TRY(check_csr(g, "ftc_edge_softmax_backward"));
    if (g->n == 0 || g->nnz == 0) return FTC_OK;
    if (!p || !dp || !ds) return fail(FTC_EINVAL, "ftc_edge_softmax_backward: NULL edge array");
    if (!w) return launch_softmax_backward(*g, p, dp, ds, static_cast<hipStream_t>(stream));
    FTC_TRY(check_windows(g, w, "ftc_edge_softmax_backward", false));
    if (!w->edge_to_row) return fail(FTC_EINVAL, "ftc_edge_softmax_backward: edge_to_row is NULL");
    const size_t need = softmax_seg_ws(g->n, g->nnz);
    if (!ws || ws_bytes < need)
        return fail(FTC_EWORKSPACE, "ftc_edge_softmax_backward: workspace of %zu bytes needed, %zu given", need,
                    ws ? ws_bytes : static_cast<size_t>(0));
    if (reinterpret_cast<uintptr_t>(ws) % 256 != 0)
        return fail(FTC_EALIGN, "ftc_edge_softmax_backward: workspace must be 256-byte aligned");
    return launch_softmax_backward_seg(*g, *w, p, dp, ds, ws, static_cast<hipStream_t>(stream));
}

size_t ftc_weight_grad_workspace_bytes(int32_t n, int32_t d_in, int32_t d_out)
{
    if (n < 0 || d_in < 1 || d_out < 1) return 0;
    return weight_grad_ws(n, d_in, d_out);
}

int32_t ftc_weight_grad(int32_t n, const void *X, int32_t ldx, int32_t x_dtype, int32_t d_in, const float *G,
                        int32_t ldg, int32_t d_out, float *dW, void *ws, size_t ws_bytes, void *stream)
{
    if (n < 0) return fail(FTC_EINVAL, "ftc_weight_grad: negative n");
    FTC_TRY(check_dense(X, ldx, x_dtype, d_in, "ftc_weight_grad", "X"));
    FTC_TRY(check_dense(G, ldg, FTC_F32, d_out, "ftc_weight_grad", "G"));
    if (!dW) return fail(FTC_EINVAL, "ftc_weight_grad: dW is NULL");
    if (d_in < 1 || d_out < 1 || weight_grad_group(d_in, d_out) == 0)
        return fail(FTC_EUNSUPPORTED, "ftc_weight_grad: d_out too wide (8 input columns next to it must fit: d_out <= 504)");
    const size_t need = weight_grad_ws(n, d_in, d_out);
    if (!ws || ws_bytes < need) return fail(FTC_EWORKSPACE, "ftc_weight_grad: workspace of %zu bytes needed", need);
    return launch_weight_grad(n, X, ldx, x_dtype, d_in, G, ldg, d_out, nullptr, 0, FTC_F32, dW, ws, static_cast<hipStream_t>(stream));
}

static int pad4(int d) { return (d + 3) / 4 * 4; }

size_t ftc_update_gemm_backward_workspace_bytes(int32_t n, int32_t d_in, int32_t d_out)
{
    if (n < 0 || d_in < 1 || d_out < 1) return 0;
    return align_up(static_cast<size_t>(n) * pad4(d_out) * sizeof(float), 256) + weight_grad_ws(n, d_in, d_out);
}

int32_t ftc_update_gemm_backward(int32_t n, const void *X, int32_t ldx, int32_t dtype, int32_t d_in, const void *W,
                                 int32_t d_out, const void *Z, int32_t ldz, int32_t z_dtype, const float *dZ,
                                 int32_t lddz, void *dX, int32_t lddx, int32_t dx_dtype, float *dW, void *ws,
                                 size_t ws_bytes, void *stream)
{
    if (n < 0) return fail(FTC_EINVAL, "ftc_update_gemm_backward: negative n");
    if (n == 0) return FTC_OK;
    FTC_TRY(check_dense(X, ldx, dtype, d_in, "ftc_update_gemm_backward", "X"));
    FTC_TRY(check_dense(dZ, lddz, FTC_F32, d_out, "ftc_update_gemm_backward", "dZ"));
    if (Z) FTC_TRY(check_dense(Z, ldz, z_dtype, d_out, "ftc_update_gemm_backward", "Z"));
    if (dX) FTC_TRY(check_dense(dX, lddx, dx_dtype, d_in, "ftc_update_gemm_backward", "dX"));
    if (!W || !dW) return fail(FTC_EINVAL, "ftc_update_gemm_backward: W or dW is NULL");
    if (dX == X) return fail(FTC_EINVAL, "ftc_update_gemm_backward: dX aliases X");
    if (weight_grad_group(d_in, d_out) == 0) return fail(FTC_EUNSUPPORTED, "ftc_update_gemm_backward: need d_out <= 504");
    const size_t need = ftc_update_gemm_backward_workspace_bytes(n, d_in, d_out);
    if (!ws || ws_bytes < need)
        return fail(FTC_EWORKSPACE, "ftc_update_gemm_backward: workspace of %zu bytes needed", need);
    if (reinterpret_cast<uintptr_t>(ws) % 256 != 0)
        return fail(FTC_EALIGN, "ftc_update_gemm_backward: workspace must be 256-byte aligned");
    hipStream_t hs = static_cast<hipStream_t>(stream);
    const float *dP = dZ;
    int ldp = lddz;
    char *p = static_cast<char *>(ws);
    // ReLU: the gradient passes where the output was positive.  Only the input gradient needs the masked matrix.
    if (Z && dX) {
        float *masked = reinterpret_cast<float *>(p);
        ldp = pad4(d_out);
        FTC_TRY(launch_mask_scale(n, d_out, dZ, lddz, Z, ldz, z_dtype, nullptr, masked, ldp, hs));
        dP = masked;
    }
    void *ws_wg = p + align_up(static_cast<size_t>(n) * pad4(d_out) * sizeof(float), 256);
    FTC_TRY(launch_weight_grad(n, X, ldx, dtype, d_in, dP, ldp, d_out, Z && !dX ? Z : nullptr, ldz, z_dtype, dW, ws_wg, hs));
    if (dX)
        FTC_TRY(launch_input_grad(n, dP, ldp, d_out, W, dtype, d_in, dX, lddx, dx_dtype, hs));
    return FTC_OK;
}

static size_t gcn_backward_ws(int32_t n, int32_t nnz, int32_t d_in, int32_t d_out, bool least)
{
    if (n < 0 || nnz < 0 || d_in < 1 || d_out < 1) return 0;
    const size_t mat = align_up(static_cast<size_t>(n) * pad4(d_out) * sizeof(float), 256);
    return 2 * mat + align_up(spmm_ws(n, nnz, d_out, least), 256) + weight_grad_ws(n, d_in, d_out);
}

size_t ftc_gcn_layer_backward_workspace_bytes(int32_t n, int32_t nnz, int32_t d_in, int32_t d_out)
{
    return gcn_backward_ws(n, nnz, d_in, d_out, false);
}

int32_t ftc_gcn_layer_backward(const ftc_csr *gT, const ftc_windows *wT, const float *valsT, const float *dinv,
                               const void *X, int32_t ldx, int32_t dtype, int32_t d_in, const void *W, int32_t d_out,
                               const void *Y, int32_t ldy, int32_t y_dtype, const float *dY, int32_t lddy, float *dX,
                               int32_t lddx, float *dW, int32_t path, void *ws, size_t ws_bytes, void *stream)
{
    FTC_TRY(check_csr(gT, "ftc_gcn_layer_backward"));
    if (gT->n == 0) return FTC_OK;
    FTC_TRY(check_dense(X, ldx, dtype, d_in, "ftc_gcn_layer_backward", "X"));
    FTC_TRY(check_dense(dY, lddy, FTC_F32, d_out, "ftc_gcn_layer_backward", "dY"));
    if (Y) FTC_TRY(check_dense(Y, ldy, y_dtype, d_out, "ftc_gcn_layer_backward", "Y"));
    if (dX) FTC_TRY(check_dense(dX, lddx, FTC_F32, d_in, "ftc_gcn_layer_backward", "dX"));
    if (!W || !dW) return fail(FTC_EINVAL, "ftc_gcn_layer_backward: W or dW is NULL");
    if (weight_grad_group(d_in, d_out) == 0) return fail(FTC_EUNSUPPORTED, "ftc_gcn_layer_backward: need d_out <= 504");
    const size_t need = gcn_backward_ws(gT->n, gT->nnz, d_in, d_out, true);
    if (!ws || ws_bytes < need)
        return fail(FTC_EWORKSPACE, "ftc_gcn_layer_backward: workspace of %zu bytes needed", need);
    if (reinterpret_cast<uintptr_t>(ws) % 256 != 0)
        return fail(FTC_EALIGN, "ftc_gcn_layer_backward: workspace must be 256-byte aligned");
    hipStream_t hs = static_cast<hipStream_t>(stream);
    const int n = gT->n, ldp = pad4(d_out);
    const size_t mat = align_up(static_cast<size_t>(n) * ldp * sizeof(float), 256);
    char *p = static_cast<char *>(ws);
    float *dP = reinterpret_cast<float *>(p);
    float *dZ = reinterpret_cast<float *>(p + mat);
    void *ws_spmm = p + 2 * mat;
    const bool least = ws_bytes < gcn_backward_ws(n, gT->nnz, d_in, d_out, false);
    const size_t spmm_bytes = align_up(spmm_ws(n, gT->nnz, d_out, least), 256);
    void *ws_wg = p + 2 * mat + spmm_bytes;
    // dP = dY where the output was positive, rows scaled by dinv in the factored form
    FTC_TRY(launch_mask_scale(n, d_out, dY, lddy, Y, ldy, y_dtype, dinv, dP, ldp, hs));
    // dZ = A^T dP on the transposed graph the caller hands over
    FTC_TRY(ftc_spmm(gT, wT, dinv ? nullptr : valsT, dP, ldp, FTC_F32, d_out, dZ, ldp, FTC_F32, dinv, 0, path,
                     ws_spmm, spmm_bytes, stream));
    FTC_TRY(launch_weight_grad(n, X, ldx, dtype, d_in, dZ, ldp, d_out, nullptr, 0, FTC_F32, dW, ws_wg, hs));
    if (dX)
        FTC_TRY(launch_input_grad(n, dZ, ldp, d_out, W, dtype, d_in, dX, lddx, FTC_F32, hs));
    return FTC_OK;
}

static size_t agnn_backward_ws(int32_t n, int32_t nnz, int32_t D, bool least)
{
    if (n < 0 || nnz < 0 || D < 1) return 0;
    const size_t edge = align_up(static_cast<size_t>(nnz) * sizeof(float), 256);
    return 3 * edge + align_up(static_cast<size_t>(n) * sizeof(float), 256) +
           2 * align_up(static_cast<size_t>(n) * pad4(D) * sizeof(float), 256) +
           align_up(ftc_sddmm_workspace_bytes(n, nnz, D), 256) + align_up(spmm_ws(n, nnz, D, least), 256) +
           align_up(softmax_seg_ws(n, nnz), 256) + edge_dot_ws();
}

size_t ftc_agnn_layer_backward_workspace_bytes(int32_t n, int32_t nnz, int32_t D) { return agnn_backward_ws(n, nnz, D, false); }

int32_t ftc_agnn_layer_backward(const ftc_csr *g, const ftc_windows *w, const int32_t *T, const void *H, int32_t ld,
                                int32_t dtype, int32_t D, float beta, const float *p, const void *dY, int32_t lddy,
                                void *dH, int32_t lddh, int32_t dh_dtype, float *dbeta, int32_t path, void *ws,
                                size_t ws_bytes, void *stream)
{
    FTC_TRY(check_csr(g, "ftc_agnn_layer_backward"));
    if (g->n == 0) return FTC_OK;
    FTC_TRY(check_dense(H, ld, dtype, D, "ftc_agnn_layer_backward", "H"));
    FTC_TRY(check_dense(dY, lddy, dtype, D, "ftc_agnn_layer_backward", "dY"));
    FTC_TRY(check_dense(dH, lddh, dh_dtype, D, "ftc_agnn_layer_backward", "dH"));
    if (!dbeta) return fail(FTC_EINVAL, "ftc_agnn_layer_backward: dbeta is NULL");
    if (g->nnz > 0 && (!T || !p)) return fail(FTC_EINVAL, "ftc_agnn_layer_backward: T or p is NULL");
    if (dH == H || dH == dY) return fail(FTC_EINVAL, "ftc_agnn_layer_backward: dH aliases an input");
    if (ld != lddy) return fail(FTC_EINVAL, "ftc_agnn_layer_backward: H and dY need the same leading dimension");
    const size_t need = agnn_backward_ws(g->n, g->nnz, D, true);
    if (!ws || ws_bytes < need)
        return fail(FTC_EWORKSPACE, "ftc_agnn_layer_backward: workspace of %zu bytes needed", need);
    if (reinterpret_cast<uintptr_t>(ws) % 256 != 0)
        return fail(FTC_EALIGN, "ftc_agnn_layer_backward: workspace must be 256-byte aligned");
    hipStream_t hs = static_cast<hipStream_t>(stream);
    const int n = g->n, nnz = g->nnz, ldq = pad4(D);
    const size_t edge = align_up(static_cast<size_t>(nnz) * sizeof(float), 256);
    char *q8 = static_cast<char *>(ws);
    float *c = reinterpret_cast<float *>(q8); q8 += edge;       // cosines
    float *ds = reinterpret_cast<float *>(q8); q8 += edge;      // dL/dp, then dL/ds
    float *v = reinterpret_cast<float *>(q8); q8 += edge;       // edge values of the two transposed products
    float *rinv = reinterpret_cast<float *>(q8); q8 += align_up(static_cast<size_t>(n) * sizeof(float), 256);
    float *q = reinterpret_cast<float *>(q8); q8 += align_up(static_cast<size_t>(n) * ldq * sizeof(float), 256);
    float *agg = reinterpret_cast<float *>(q8); q8 += align_up(static_cast<size_t>(n) * ldq * sizeof(float), 256);
    void *ws_sd = q8; const size_t sd = align_up(ftc_sddmm_workspace_bytes(n, nnz, D), 256); q8 += sd;
    void *ws_sp = q8; const size_t sp = align_up(spmm_ws(n, nnz, D, ws_bytes < agnn_backward_ws(n, nnz, D, false)), 256); q8 += sp;
    void *ws_sm = q8; const size_t sm = align_up(softmax_seg_ws(n, nnz), 256); q8 += sm;
    void *ws_dot = q8;
    FTC_TRY(launch_row_rnorm(n, H, ld, dtype, D, rinv, hs));
    // c_e = cos(h_i, h_j);  dp_e = <dY_i, h_j>  (y_i = sum_e p_e h_j)
    FTC_TRY(ftc_sddmm(g, w, H, H, ld, dtype, D, nullptr, nullptr, 1.f, 1, c, path, ws_sd, sd, stream));
    FTC_TRY(ftc_sddmm(g, w, dY, H, ld, dtype, D, nullptr, nullptr, 1.f, 0, ds, path, ws_sd, sd, stream));
    FTC_TRY(ftc_edge_softmax_backward(g, w, p, ds, ds, ws_sm, sm, stream));
    FTC_TRY(launch_edge_dot(nnz, ds, c, dbeta, ws_dot, hs));  // s = beta * c, so dL/dbeta = sum_e ds_e c_e
    // gradient with respect to the normalised rows: q_i = sum_e (dc_e + dc_T(e)) hn_j, dc = beta * ds,
    // hn_j = rinv_j h_j folded into the edge values so that H itself is the gathered matrix
    FTC_TRY(launch_edge_combine(nnz, ds, T, 1.f, 1.f, beta, rinv, g->col_idx, v, hs));
    FTC_TRY(ftc_spmm(g, w, v, H, ld, dtype, D, q, ldq, FTC_F32, nullptr, 0, path, ws_sp, sp, stream));
    // through the aggregated rows: dH = P^T dY, (P^T)_e = p_T(e) on the symmetric pattern
    FTC_TRY(launch_edge_combine(nnz, p, T, 0.f, 1.f, 1.f, nullptr, g->col_idx, v, hs));
    FTC_TRY(ftc_spmm(g, w, v, dY, lddy, dtype, D, agg, ldq, FTC_F32, nullptr, 0, path, ws_sp, sp, stream));
    // ... plus the derivative of the normalisation, rounded once to the requested type
    return launch_cos_backward_rows(n, H, ld, dtype, D, rinv, q, ldq, agg, ldq, dH, lddh, dh_dtype, hs);
}

size_t ftc_agnn_layer_backward_fused_workspace_bytes(int32_t n, int32_t nnz, int32_t D)
{
    if (n < 0 || nnz < 0 || D < 1) return 0;
    return agnn_backward_fused_ws(n, nnz, D, false);
}

int32_t ftc_agnn_layer_backward_fused(const ftc_csr *g, const ftc_windows *w, const void *H, int32_t ld, int32_t dtype,
                                      int32_t D, float beta, const float *row_z, const void *Y, int32_t ldy,
                                      int32_t y_dtype, const void *dY, int32_t lddy, void *dH, int32_t lddh,
                                      int32_t dh_dtype, float *dbeta, const int32_t *pattern_flag, void *ws,
                                      size_t ws_bytes, void *stream)
{
    FTC_TRY(check_csr(g, "ftc_agnn_layer_backward_fused"));
    if (g->n == 0) return FTC_OK;
    FTC_TRY(check_dense(H, ld, dtype, D, "ftc_agnn_layer_backward_fused", "H"));
    FTC_TRY(check_dense(dY, lddy, dtype, D, "ftc_agnn_layer_backward_fused", "dY"));
    FTC_TRY(check_dense(Y, ldy, y_dtype, D, "ftc_agnn_layer_backward_fused", "Y"));
    FTC_TRY(check_dense(dH, lddh, dh_dtype, D, "ftc_agnn_layer_backward_fused", "dH"));
    if (!dbeta || !row_z) return fail(FTC_EINVAL, "ftc_agnn_layer_backward_fused: dbeta or row_z is NULL");
    if (dH == H || dH == dY || dH == Y) return fail(FTC_EINVAL, "ftc_agnn_layer_backward_fused: dH aliases an input");
    if (ld != lddy)
        return fail(FTC_EINVAL, "ftc_agnn_layer_backward_fused: H and dY need the same leading dimension");
    if (!w) return fail(FTC_EINVAL, "ftc_agnn_layer_backward_fused: the window index is required");
    FTC_TRY(check_windows(g, w, "ftc_agnn_layer_backward_fused", false));
    if (g->nnz > 0 && !w->edge_to_row) return fail(FTC_EINVAL, "ftc_agnn_layer_backward_fused: edge_to_row is NULL");
    const bool rows16 = aligned16(H) && aligned16(dY) && (static_cast<int64_t>(ld) * elem_size(dtype)) % 16 == 0;
    if (!rows16 || !agnn_backward_fused_shape(dtype, D) || !(fabsf(beta) < AGNN_FUSED_MAX_BETA))
        return fail(FTC_EUNSUPPORTED,
                    "ftc_agnn_layer_backward_fused: needs |beta| < 43, 16-byte aligned rows and a width the "
                    "edge-balanced kernels cover with 2 * D <= 256 padded slots; use ftc_agnn_layer_backward");
    const size_t need = agnn_backward_fused_ws(g->n, g->nnz, D, true);
    if (!ws || ws_bytes < need)
        return fail(FTC_EWORKSPACE, "ftc_agnn_layer_backward_fused: workspace of %zu bytes needed", need);
    if (reinterpret_cast<uintptr_t>(ws) % 256 != 0)
        return fail(FTC_EALIGN, "ftc_agnn_layer_backward_fused: workspace must be 256-byte aligned");
    // pattern_flag not zero, not a symmetric pattern: NaN instead of a gradient of nothing
    return launch_agnn_backward_fused(*g, *w, H, dY, ld, dtype, D, beta, row_z, Y, ldy, y_dtype, dH, lddh, dh_dtype, dbeta,
                                      pattern_flag, ws, ws_bytes, static_cast<hipStream_t>(stream));
}

// ---- graph transformer ---------------------------------------------------------------------------
static int32_t check_ws(const char *who, size_t need, const void *ws, size_t ws_bytes)
{
    if (need == 0) return FTC_OK;
    if (!ws || ws_bytes < need)
        return fail(FTC_EWORKSPACE, "%s: workspace of %zu bytes needed, %zu given", who, need, ws ? ws_bytes : static_cast<size_t>(0));
    if (reinterpret_cast<uintptr_t>(ws) % 256 != 0) return fail(FTC_EALIGN, "%s: workspace must be 256-byte aligned", who);
    return FTC_OK;
}

static int32_t check_out_type(const char *who, const char *name, int32_t dtype, int32_t out_dtype)
{
    if (out_dtype != FTC_F32 && out_dtype != dtype)
        return fail(FTC_EUNSUPPORTED, "%s: %s is fp32 or of the type of the inputs", who, name);
    return FTC_OK;
}

// Counts and widths: indexes of a whole tile, its end behind the last row included, are int32.
static constexpr int32_t MOST_ROWS = 1 << 30;
static int32_t check_sizes(const char *who, int32_t a, int32_t b, int32_t c, LaunchSize (*size)(int, int, int))
{
    if (a > MOST_ROWS || b > MOST_ROWS || c > MOST_ROWS) return fail(FTC_EUNSUPPORTED, "%s: counts and widths are at most 2^30", who);
    if (!size(a, b, c).fits()) return fail(FTC_EUNSUPPORTED, "%s: too large for one launch", who);
    return FTC_OK;
}
static LaunchSize lookup_size(int n, int, int D) { return embedding_size(n, D); }

int32_t ftc_embedding(int32_t n, const int32_t *ids, int32_t vocab, const void *E, int32_t lde, int32_t dtype, int32_t D,
                      float scale, void *out, int32_t ldo, int32_t out_dtype, void *stream)
{
    const char *who = "ftc_embedding";
    if (n < 0 || vocab < 0) return fail(FTC_EINVAL, "%s: negative n or vocab", who);
    if (n == 0) return FTC_OK;
    if (!ids) return fail(FTC_EINVAL, "%s: ids is NULL", who);
    if (vocab > 0) FTC_TRY(check_dense(E, lde, dtype, D, who, "E"));
    if (!valid_dtype(dtype)) return fail(FTC_EUNSUPPORTED, "%s: unknown dtype for E", who);
    FTC_TRY(check_dense(out, ldo, out_dtype, D, who, "out"));
    if (out == E) return fail(FTC_EINVAL, "%s: out aliases E", who);
    FTC_TRY(check_sizes(who, n, vocab, D, lookup_size));
    return launch_embedding(n, ids, vocab, E, lde, dtype, D, scale, out, ldo, out_dtype, static_cast<hipStream_t>(stream));
}

size_t ftc_embedding_backward_workspace_bytes(int32_t n, int32_t vocab, int32_t D)
{
    if (n < 0 || vocab < 0 || D < 1) return 0;
    return embedding_backward_ws(n, vocab, D);
}

int32_t ftc_embedding_backward(int32_t n, const int32_t *ids, int32_t vocab, const void *dOut, int32_t lddo, int32_t dtype,
                               int32_t D, float scale, void *dE, int32_t ldde, int32_t de_dtype, void *ws, size_t ws_bytes,
                               void *stream)
{
    const char *who = "ftc_embedding_backward";
    if (n < 0 || vocab < 0) return fail(FTC_EINVAL, "%s: negative n or vocab", who);
    if (vocab == 0) return FTC_OK;
    if (n > 0) {
        if (!ids) return fail(FTC_EINVAL, "%s: ids is NULL", who);
        FTC_TRY(check_dense(dOut, lddo, dtype, D, who, "dOut"));
    }
    if (!valid_dtype(dtype)) return fail(FTC_EUNSUPPORTED, "%s: unknown dtype for dOut", who);
    FTC_TRY(check_dense(dE, ldde, de_dtype, D, who, "dE"));
    if (dE == dOut) return fail(FTC_EINVAL, "%s: dE aliases dOut", who);
    FTC_TRY(check_sizes(who, n, vocab, D, embedding_backward_size));
    FTC_TRY(check_ws(who, embedding_backward_ws(n, vocab, D), ws, ws_bytes));
    return launch_embedding_backward(n, ids, vocab, dOut, lddo, dtype, D, scale, dE, ldde, de_dtype, ws,
                                     static_cast<hipStream_t>(stream));
}

size_t ftc_linear_workspace_bytes(int32_t n, int32_t d_in, int32_t d_out)
{
    if (n < 0 || d_in < 1 || d_out < 1) return 0;
    return linear_ws(n, d_in, d_out);
}

static int32_t check_linear(const char *who, const LinearShape &p)
{
    FTC_TRY(check_dense(p.X, p.ldx, p.dtype, p.d_in, who, "X"));
    FTC_TRY(check_dense(p.W, p.d_out, p.dtype, p.d_out, who, "W"));
    FTC_TRY(check_dense(p.Z, p.ldz, p.z_dtype, p.d_out, who, "Z"));
    FTC_TRY(check_out_type(who, "Z", p.dtype, p.z_dtype));
    if (p.bias) FTC_TRY(check_dense(p.bias, p.d_out, p.dtype, p.d_out, who, "bias"));
    if (p.residual) FTC_TRY(check_dense(p.residual, p.ldr, p.dtype, p.d_out, who, "residual"));
    if (p.slope) {
        if (p.lds < p.d_out) return fail(FTC_EINVAL, "%s: need ld >= D for slope", who);
        if (reinterpret_cast<uintptr_t>(p.slope) % elem_size(p.dtype) != 0)
            return fail(FTC_EALIGN, "%s: slope is not aligned to its element size", who);
    }
    if (p.Z == p.X || p.Z == p.W || p.Z == p.bias || p.Z == p.slope ||
        (p.slope && (p.slope == p.X || p.slope == p.W || p.slope == p.bias || p.slope == p.residual)))
        return fail(FTC_EINVAL, "%s: an output aliases an input or the other output", who);
    if (p.Z == p.residual && (p.ldz != p.ldr || p.z_dtype != p.dtype))
        return fail(FTC_EINVAL, "%s: Z on top of the residual needs its leading dimension and type", who);
    return FTC_OK;
}

int32_t ftc_linear(int32_t n, const void *X, int32_t ldx, int32_t dtype, int32_t d_in, const void *W, int32_t d_out,
                   const void *bias, int32_t act, const void *residual, int32_t ldr, void *slope, int32_t lds, void *Z,
                   int32_t ldz, int32_t z_dtype, void *ws, size_t ws_bytes, void *stream)
{
    const char *who = "ftc_linear";
    if (n < 0) return fail(FTC_EINVAL, "%s: negative n", who);
    if (act < FTC_ACT_NONE || act > FTC_ACT_SILU) return fail(FTC_EINVAL, "%s: unknown activation %d", who, act);
    if (n == 0) return FTC_OK;
    const LinearShape p = {n, d_in, d_out, dtype, X, W, bias, residual, slope, Z, ldx, ldr, lds, ldz, act, z_dtype};
    FTC_TRY(check_linear(who, p));
    FTC_TRY(check_sizes(who, n, d_in, d_out, linear_size));
    FTC_TRY(check_ws(who, linear_ws(n, d_in, d_out), ws, ws_bytes));
    return launch_linear(p, ws, static_cast<hipStream_t>(stream));
}

size_t ftc_linear_backward_workspace_bytes(int32_t n, int32_t d_in, int32_t d_out)
{
    if (n < 0 || d_in < 1 || d_out < 1) return 0;
    return linear_backward_ws(n, d_in, d_out);
}

static int32_t check_linear_backward(const char *who, const LinearShape &p, const LinearGrads &g)
{
    if (p.n < 0 || p.d_in < 1 || p.d_out < 1) return fail(FTC_EINVAL, "%s: negative n, or a width below 1", who);
    if (!valid_dtype(p.dtype)) return fail(FTC_EUNSUPPORTED, "%s: unknown dtype for X", who);
    if (p.n > 0) {
        if (g.dW) FTC_TRY(check_dense(p.X, p.ldx, p.dtype, p.d_in, who, "X"));
        if (g.dX) FTC_TRY(check_dense(p.W, p.d_out, p.dtype, p.d_out, who, "W"));
        FTC_TRY(check_dense(g.dZ, g.lddz, p.dtype, p.d_out, who, "dZ"));
        if (p.slope && p.lds < p.d_out) return fail(FTC_EINVAL, "%s: need ld >= D for slope", who);
        if (reinterpret_cast<uintptr_t>(p.slope) % elem_size(p.dtype) != 0)
            return fail(FTC_EALIGN, "%s: slope is not aligned to its element size", who);
        if (g.dX) {
            FTC_TRY(check_dense(g.dX, g.lddx, g.dx_dtype, p.d_in, who, "dX"));
            FTC_TRY(check_out_type(who, "dX", p.dtype, g.dx_dtype));
            if (g.dX_add) FTC_TRY(check_dense(g.dX_add, g.ldda, p.dtype, p.d_in, who, "dX_add"));
            if (g.dX_add == g.dX && (g.ldda != g.lddx || g.dx_dtype != p.dtype))
                return fail(FTC_EINVAL, "%s: dX on top of dX_add needs its leading dimension and type", who);
        }
    }
    if (g.dW) FTC_TRY(check_dense(g.dW, p.d_out, g.dw_dtype, p.d_out, who, "dW"));
    if (g.db) FTC_TRY(check_dense(g.db, p.d_out, g.dw_dtype, p.d_out, who, "db"));
    if (g.dW || g.db) FTC_TRY(check_out_type(who, "dW", p.dtype, g.dw_dtype));
    const void *outs[3] = {g.dX, g.dW, g.db}, *ins[4] = {p.X, p.W, p.slope, g.dZ};
    for (int i = 0; i < 3; ++i) {
        for (int j = 0; j < 4; ++j)
            if (outs[i] && outs[i] == ins[j]) return fail(FTC_EINVAL, "%s: an output aliases an input", who);
        for (int j = 0; j < i; ++j)
            if (outs[i] && outs[i] == outs[j]) return fail(FTC_EINVAL, "%s: two outputs are the same", who);
    }
    if (g.dX_add && (g.dX_add == g.dW || g.dX_add == g.db)) return fail(FTC_EINVAL, "%s: an output aliases an input", who);
    return FTC_OK;
}

int32_t ftc_linear_backward(int32_t n, const void *X, int32_t ldx, int32_t dtype, int32_t d_in, const void *W, int32_t d_out,
                            const void *slope, int32_t lds, const void *dZ, int32_t lddz, const void *dX_add, int32_t ldda, void *dX,
                            int32_t lddx, int32_t dx_dtype, void *dW, void *db, int32_t dw_dtype, void *ws, size_t ws_bytes,
                            void *stream)
{
    const char *who = "ftc_linear_backward";
    const LinearShape p = {n, d_in, d_out, dtype, X, W, nullptr, nullptr, const_cast<void *>(slope), nullptr, ldx, 0, lds, 0, FTC_ACT_NONE, dtype};
    const LinearGrads g = {dZ, dX_add, dX, dW, db, lddz, ldda, lddx, dx_dtype, dw_dtype};
    FTC_TRY(check_linear_backward(who, p, g));
    FTC_TRY(check_sizes(who, n, d_in, d_out, linear_backward_size));
    FTC_TRY(check_ws(who, linear_backward_ws(n, d_in, d_out), ws, ws_bytes));
    return launch_linear_backward(p, g, ws, static_cast<hipStream_t>(stream));
}

// ---- dense layers with weights for each group of rows
static constexpr int32_t GROUPED_MOST = 1 << 20;  // of groups and of each width
static bool grouped_sizes_ok(int32_t n, int32_t n_groups, int32_t d_in, int32_t d_out)
{
    return n >= 0 && n <= MOST_ROWS && n_groups >= 0 && n_groups <= GROUPED_MOST && d_in >= 1 && d_in <= GROUPED_MOST && d_out >= 1 && d_out <= GROUPED_MOST;
}
static int32_t check_groups(const char *who, int32_t n, const int32_t *group_ptr, int32_t n_groups, int32_t d_in, int32_t d_out)
{
    if (n < 0 || n_groups < 0) return fail(FTC_EINVAL, "%s: negative n or n_groups", who);
    if (d_in < 1 || d_out < 1) return fail(FTC_EINVAL, "%s: a width below 1", who);
    if (n_groups > 0 && !group_ptr) return fail(FTC_EINVAL, "%s: group_ptr is NULL", who);
    if (reinterpret_cast<uintptr_t>(group_ptr) % sizeof(int32_t) != 0) return fail(FTC_EALIGN, "%s: group_ptr is not aligned to its element size", who);
    if (!grouped_sizes_ok(n, n_groups, d_in, d_out)) return fail(FTC_EUNSUPPORTED, "%s: n is at most 2^30, n_groups and widths 2^20", who);
    return FTC_OK;
}

size_t ftc_grouped_linear_workspace_bytes(int32_t n, int32_t n_groups, int32_t d_in, int32_t d_out)
{
    return grouped_sizes_ok(n, n_groups, d_in, d_out) ? grouped_linear_ws(n, n_groups, d_in, d_out) : 0;
}

int32_t ftc_grouped_linear(int32_t n, const int32_t *group_ptr, int32_t n_groups, const void *X, int32_t ldx, int32_t dtype, int32_t d_in, const void *W,
                           int32_t d_out, const void *bias, int32_t act, const void *residual, int32_t ldr, void *slope, int32_t lds, void *Z, int32_t ldz,
                           int32_t z_dtype, void *ws, size_t ws_bytes, void *stream)
{
    const char *who = "ftc_grouped_linear";
    FTC_TRY(check_groups(who, n, group_ptr, n_groups, d_in, d_out));
    if (act < FTC_ACT_NONE || act > FTC_ACT_SILU) return fail(FTC_EINVAL, "%s: unknown activation %d", who, act);
    if (n == 0 || n_groups == 0) return FTC_OK;
    const LinearShape p = {n, d_in, d_out, dtype, X, W, bias, residual, slope, Z, ldx, ldr, lds, ldz, act, z_dtype};
    FTC_TRY(check_linear(who, p));
    if (!grouped_linear_size(n, n_groups, d_in, d_out).fits()) return fail(FTC_EUNSUPPORTED, "%s: too large for one launch", who);
    FTC_TRY(check_ws(who, grouped_linear_ws(n, n_groups, d_in, d_out), ws, ws_bytes));
    return launch_grouped_linear(p, group_ptr, n_groups, ws, static_cast<hipStream_t>(stream));
}

size_t ftc_grouped_linear_backward_workspace_bytes(int32_t n, int32_t n_groups, int32_t d_in, int32_t d_out)
{
    return grouped_sizes_ok(n, n_groups, d_in, d_out) ? grouped_linear_backward_ws(n, n_groups, d_in, d_out) : 0;
}

int32_t ftc_grouped_linear_backward(int32_t n, const int32_t *group_ptr, int32_t n_groups, const void *X, int32_t ldx, int32_t dtype, int32_t d_in, const void *W,
                                    int32_t d_out, const void *slope, int32_t lds, const void *dZ, int32_t lddz, const void *dX_add, int32_t ldda, void *dX,
                                    int32_t lddx, int32_t dx_dtype, void *dW, void *db, int32_t dw_dtype, void *ws, size_t ws_bytes, void *stream)
{
    const char *who = "ftc_grouped_linear_backward";
    FTC_TRY(check_groups(who, n, group_ptr, n_groups, d_in, d_out));
    if (n_groups == 0) return FTC_OK;
    const LinearShape p = {n, d_in, d_out, dtype, X, W, nullptr, nullptr, const_cast<void *>(slope), nullptr, ldx, 0, lds, 0, FTC_ACT_NONE, dtype};
    const LinearGrads g = {dZ, dX_add, dX, dW, db, lddz, ldda, lddx, dx_dtype, dw_dtype};
    FTC_TRY(check_linear_backward(who, p, g));
    if (!grouped_linear_backward_size(n, n_groups, d_in, d_out).fits()) return fail(FTC_EUNSUPPORTED, "%s: too large for one launch", who);
    FTC_TRY(check_ws(who, grouped_linear_backward_ws(n, n_groups, d_in, d_out), ws, ws_bytes));
    return launch_grouped_linear_backward(p, g, group_ptr, n_groups, ws, static_cast<hipStream_t>(stream));
}

// ---- the norm over all gradients
static constexpr int32_t GRAD_MOST = 1 << 20;  // gradients of a call
static int32_t check_grads(const char *who, const ftc_grad *grads, int32_t count, double scale, const float *norm, bool out)
{
    if (count < 0) return fail(FTC_EINVAL, "%s: negative count", who);
    if (count > 0 && !grads) return fail(FTC_EINVAL, "%s: grads is NULL", who);
    if (count > GRAD_MOST) return fail(FTC_EUNSUPPORTED, "%s: at most 2^20 gradients", who);
    if (!std::isfinite(scale)) return fail(FTC_EINVAL, "%s: scale is not finite", who);
    if (!norm) return fail(FTC_EINVAL, "%s: norm is NULL", who);
    if (reinterpret_cast<uintptr_t>(norm) % sizeof(float) != 0) return fail(FTC_EALIGN, "%s: norm is not aligned to its element size", who);
    for (int32_t i = 0; i < count; ++i) {
        const ftc_grad &g = grads[i];
        if (g.rows < 0 || g.cols < 0) return fail(FTC_EINVAL, "%s: gradient %d has a negative size", who, i);
        if (!valid_dtype(g.dtype)) return fail(FTC_EUNSUPPORTED, "%s: unknown dtype for gradient %d", who, i);
        if (g.rows == 0 || g.cols == 0) continue;
        if (g.rows > (1ll << 38) / g.cols) return fail(FTC_EUNSUPPORTED, "%s: gradient %d has more than 2^38 numbers", who, i);
        if (!g.grad || (out && !g.out)) return fail(FTC_EINVAL, "%s: gradient %d is NULL", who, i);
        const void *const both[2] = {g.grad, out ? g.out : nullptr};
        for (const void *p : both)
            if (reinterpret_cast<uintptr_t>(p) % elem_size(g.dtype) != 0) return fail(FTC_EALIGN, "%s: gradient %d is not aligned to its element size", who, i);
        if (g.rows == 1) continue;
        if (g.ld < g.cols || (out && g.ldo < g.cols)) return fail(FTC_EINVAL, "%s: need ld >= cols for gradient %d", who, i);
        if (out && g.out == g.grad && g.ldo != g.ld) return fail(FTC_EINVAL, "%s: out on top of gradient %d needs its leading dimension", who, i);
        if (!grad_whole(g, out) && (g.rows > INT32_MAX / g.cols || g.ld > INT32_MAX || (out && g.ldo > INT32_MAX)))
            return fail(FTC_EUNSUPPORTED, "%s: gradient %d is not contiguous and has rows of more than 2^31 - 1 numbers", who, i);
    }
    return FTC_OK;
}

size_t ftc_grad_norm_workspace_bytes(int32_t count) { return count < 0 || count > GRAD_MOST ? 0 : grad_norm_ws(count); }

int32_t ftc_grad_norm(const ftc_grad *grads, int32_t count, double scale, float *norm, void *ws, size_t ws_bytes, void *stream)
{
    const char *who = "ftc_grad_norm";
    FTC_TRY(check_grads(who, grads, count, scale, norm, false));
    FTC_TRY(check_ws(who, grad_norm_ws(count), ws, ws_bytes));
    return launch_grad_norm(grads, count, scale, norm, ws, static_cast<hipStream_t>(stream));
}

int32_t ftc_clip_grad_norm(const ftc_grad *grads, int32_t count, double max_norm, double scale, float *norm, void *ws, size_t ws_bytes, void *stream)
{
    const char *who = "ftc_clip_grad_norm";
    FTC_TRY(check_grads(who, grads, count, scale, norm, true));
    if (!(max_norm >= 0)) return fail(FTC_EINVAL, "%s: max_norm is negative or NaN", who);
    FTC_TRY(check_ws(who, grad_norm_ws(count), ws, ws_bytes));
    return launch_clip_grad_norm(grads, count, max_norm, scale, norm, ws, static_cast<hipStream_t>(stream));
}

static int32_t check_block(const char *who, const ftc_block *b)
{
    if (!b) return fail(FTC_EINVAL, "%s: block is NULL", who);
    if (b->n < 0 || b->d < 1) return fail(FTC_EINVAL, "%s: negative n, or d below 1", who);
    if (!valid_dtype(b->dtype)) return fail(FTC_EUNSUPPORTED, "%s: unknown dtype", who);
    if (b->post < FTC_NORM_NONE || b->post > FTC_NORM_LAYER || b->pre < FTC_NORM_NONE || b->pre > FTC_NORM_LAYER)
        return fail(FTC_EINVAL, "%s: unknown norm", who);
    if (b->d > BLOCK_NORM_WIDEST || b->n > MOST_ROWS) return fail(FTC_EUNSUPPORTED, "%s: d is at most %d, n 2^30", who, BLOCK_NORM_WIDEST);
    if (!(b->eps > 0.f) || !std::isfinite(b->eps)) return fail(FTC_EINVAL, "%s: eps is not a positive number", who);
    if (!std::isfinite(b->x_scale)) return fail(FTC_EINVAL, "%s: x_scale is not finite", who);
    if (b->n > 0 && !b->F && (b->post != FTC_NORM_NONE || b->gate)) return fail(FTC_EINVAL, "%s: a norm or gate of F without F", who);
    if (b->post == FTC_NORM_NONE && (b->post_w || b->post_b)) return fail(FTC_EINVAL, "%s: post_w or post_b without a norm", who);
    if (b->pre == FTC_NORM_NONE && (b->pre_w || b->pre_b)) return fail(FTC_EINVAL, "%s: pre_w or pre_b without a norm", who);
    if (b->n > 0) {
        FTC_TRY(check_dense(b->X, b->ldx, b->dtype, b->d, who, "X"));
        if (b->F) FTC_TRY(check_dense(b->F, b->ldf, b->dtype, b->d, who, "F"));
    }
    if (b->gate) FTC_TRY(check_dense(b->gate, b->ldg == 0 ? b->d : b->ldg, b->dtype, b->d, who, "gate"));
    const void *const vectors[4] = {b->post_w, b->post_b, b->pre_w, b->pre_b};
    for (const void *v : vectors)
        if (v) FTC_TRY(check_dense(v, b->d, b->dtype, b->d, who, "a weight or bias"));
    return FTC_OK;
}

// Whether `out` is one of the block's inputs, X aside.
static bool block_has(const ftc_block &b, const void *out)
{
    return out == b.F || out == b.gate || out == b.post_w || out == b.post_b || out == b.pre_w || out == b.pre_b;
}

int32_t ftc_block_norm(const ftc_block *b, void *H, int32_t ldh, void *U, int32_t ldu, float *stats, void *stream)
{
    const char *who = "ftc_block_norm";
    FTC_TRY(check_block(who, b));
    if (b->n == 0) return FTC_OK;
    if (!H && !U) return fail(FTC_EINVAL, "%s: neither H nor U is given", who);
    if (U && b->pre == FTC_NORM_NONE) return fail(FTC_EINVAL, "%s: U without a norm", who);
    if (H) FTC_TRY(check_dense(H, ldh, b->dtype, b->d, who, "H"));
    if (U) FTC_TRY(check_dense(U, ldu, b->dtype, b->d, who, "U"));
    if ((H && block_has(*b, H)) || (U && (U == b->X || U == H || block_has(*b, U))) || (stats && (stats == b->X || stats == H || stats == U || block_has(*b, stats))))
        return fail(FTC_EINVAL, "%s: an output aliases an input or another output", who);
    if (H == b->X && ldh != b->ldx) return fail(FTC_EINVAL, "%s: H on top of X needs its leading dimension", who);
    if (!aligned16(stats)) return fail(FTC_EALIGN, "%s: stats must be 16-byte aligned", who);
    return launch_block_norm(*b, H, ldh, U, ldu, stats, static_cast<hipStream_t>(stream));
}

size_t ftc_block_norm_backward_workspace_bytes(int32_t n, int32_t d)
{
    if (n < 0 || d < 1 || d > BLOCK_NORM_WIDEST || n > MOST_ROWS) return 0;
    return block_norm_backward_ws(n, d);
}

int32_t ftc_block_norm_backward(const ftc_block *b, const float *stats, const void *dH, int32_t lddh, const void *dU, int32_t lddu,
                                const ftc_block_grads *g, void *ws, size_t ws_bytes, void *stream)
{
    const char *who = "ftc_block_norm_backward";
    FTC_TRY(check_block(who, b));
    if (!g) return fail(FTC_EINVAL, "%s: grads is NULL", who);
    if (dU && b->pre == FTC_NORM_NONE) return fail(FTC_EINVAL, "%s: dU without a norm", who);
    if ((b->n > 0 && g->dF && !b->F) || (g->dgate && !b->gate) || (g->dpost_w && !b->post_w) || (g->dpre_w && !b->pre_w) || (g->dpost_b && b->post == FTC_NORM_NONE) ||
        (g->dpre_b && b->pre == FTC_NORM_NONE))
        return fail(FTC_EINVAL, "%s: a gradient of what the block does not have", who);
    const bool gates = b->gate && b->ldg != 0;  // one a row
    if (b->n > 0) {
        if ((b->pre != FTC_NORM_NONE || b->post != FTC_NORM_NONE) && !stats) return fail(FTC_EINVAL, "%s: stats is NULL", who);
        if (!aligned16(stats)) return fail(FTC_EALIGN, "%s: stats must be 16-byte aligned", who);
        if (dH) FTC_TRY(check_dense(dH, lddh, b->dtype, b->d, who, "dH"));
        if (dU) FTC_TRY(check_dense(dU, lddu, b->dtype, b->d, who, "dU"));
        if (g->dX) FTC_TRY(check_dense(g->dX, g->lddx, b->dtype, b->d, who, "dX"));
        if (g->dF) FTC_TRY(check_dense(g->dF, g->lddf, b->dtype, b->d, who, "dF"));
        if (g->dgate && gates) FTC_TRY(check_dense(g->dgate, g->lddg, b->dtype, b->d, who, "dgate"));
    }
    const void *sums[5] = {gates ? nullptr : g->dgate, g->dpost_w, g->dpost_b, g->dpre_w, g->dpre_b};
    for (const void *v : sums)
        if (v) {
            FTC_TRY(check_dense(v, b->d, g->dw_dtype, b->d, who, "the gradient of a weight or bias"));
            FTC_TRY(check_out_type(who, "the gradient of a weight or bias", b->dtype, g->dw_dtype));
        }
    const void *outs[7] = {g->dX, g->dF, g->dgate, g->dpost_w, g->dpost_b, g->dpre_w, g->dpre_b};
    for (int i = 0; i < 7; ++i) {
        if (!outs[i]) continue;
        if (outs[i] == b->X || block_has(*b, outs[i]) || outs[i] == stats || outs[i] == dU || (i > 0 && outs[i] == dH))
            return fail(FTC_EINVAL, "%s: an output aliases an input", who);
        for (int j = 0; j < i; ++j)
            if (outs[i] == outs[j]) return fail(FTC_EINVAL, "%s: two outputs are the same", who);
    }
    if (g->dX && g->dX == dH && g->lddx != lddh) return fail(FTC_EINVAL, "%s: dX on top of dH needs its leading dimension", who);
    FTC_TRY(check_ws(who, block_norm_backward_ws(b->n, b->d), ws, ws_bytes));
    return launch_block_norm_backward(*b, stats, dH, lddh, dU, lddu, *g, ws, static_cast<hipStream_t>(stream));
}

static constexpr int64_t ATTENTION_MOST_ROWS = 1 << 30;  // rows and heads of a matrix together, counted in int32
static constexpr int32_t ATTENTION_MOST_HEADS = 65535;   // of K and V: far more than any model has; what fits a launch is attention_size()'s to say

static bool attention_sizes_ok(int32_t n_q, int32_t n_kv, int32_t n_graphs, int32_t heads, int32_t kv_heads, int32_t D)
{
    return n_q >= 0 && n_kv >= 0 && n_graphs >= 0 && n_graphs <= ATTENTION_MOST_ROWS && heads >= 1 && kv_heads >= 1 &&
           kv_heads <= ATTENTION_MOST_HEADS && heads % kv_heads == 0 && D >= 1 && D <= 128 &&
           static_cast<int64_t>(n_q) * heads <= ATTENTION_MOST_ROWS && static_cast<int64_t>(n_kv) * kv_heads <= ATTENTION_MOST_ROWS;
}

static int32_t check_attention(const char *who, const AttnShape &p)
{
    if (p.n_q < 0 || p.n_kv < 0 || p.graphs < 0) return fail(FTC_EINVAL, "%s: negative n_q, n_kv or n_graphs", who);
    if (p.heads < 1 || p.kv_heads < 1 || p.heads % p.kv_heads != 0)
        return fail(FTC_EINVAL, "%s: heads must be a multiple of kv_heads, both at least 1", who);
    if (p.D < 1) return fail(FTC_EINVAL, "%s: need D >= 1", who);
    if (!std::isfinite(p.scale)) return fail(FTC_EINVAL, "%s: scale is not finite", who);
    if (!attention_sizes_ok(p.n_q, p.n_kv, p.graphs, p.heads, p.kv_heads, p.D))
        return fail(FTC_EUNSUPPORTED, "%s: D is at most 128, kv_heads 65535, n_q * heads and n_kv * kv_heads 2^30", who);
    if (!attention_size(p.n_q, p.n_kv, p.graphs, p.heads, p.kv_heads, p.D).fits())
        return fail(FTC_EUNSUPPORTED, "%s: too many graphs and heads for one launch", who);
    if (!valid_dtype(p.dtype)) return fail(FTC_EUNSUPPORTED, "%s: unknown dtype", who);
    if (p.graphs > 0 && (!p.q_ptr || !p.kv_ptr)) return fail(FTC_EINVAL, "%s: q_ptr or kv_ptr is NULL", who);
    if (static_cast<int64_t>(p.heads) * p.D > INT32_MAX) return fail(FTC_EUNSUPPORTED, "%s: heads * D does not fit 32 bits", who);
    if (p.n_q > 0) FTC_TRY(check_dense(p.Q, p.ldq, p.dtype, p.heads * p.D, who, "Q"));
    if (p.n_kv > 0) {
        FTC_TRY(check_dense(p.K, p.ldk, p.dtype, p.kv_heads * p.D, who, "K"));
        FTC_TRY(check_dense(p.V, p.ldv, p.dtype, p.kv_heads * p.D, who, "V"));
    }
    return FTC_OK;
}

size_t ftc_graph_attention_workspace_bytes(int32_t n_q, int32_t n_kv, int32_t n_graphs, int32_t heads, int32_t kv_heads, int32_t D)
{
    if (!attention_sizes_ok(n_q, n_kv, n_graphs, heads, kv_heads, D)) return 0;
    return attention_ws(n_q, n_kv, n_graphs, heads, kv_heads, D);
}

int32_t ftc_graph_attention(int32_t n_q, const int32_t *q_ptr, int32_t n_kv, const int32_t *kv_ptr, int32_t n_graphs,
                            int32_t heads, int32_t kv_heads, int32_t D, int32_t dtype, const void *Q, int32_t ldq, const void *K,
                            int32_t ldk, const void *V, int32_t ldv, const uint8_t *kv_mask, float scale, void *out, int32_t ldo,
                            float *lse, void *ws, size_t ws_bytes, void *stream)
{
    const char *who = "ftc_graph_attention";
    const AttnShape p = {n_q, n_kv, n_graphs, heads, kv_heads, D, dtype, Q, K, V, ldq, ldk, ldv, q_ptr, kv_ptr, kv_mask, scale};
    FTC_TRY(check_attention(who, p));
    if (n_q == 0 || n_graphs == 0) return FTC_OK;
    FTC_TRY(check_dense(out, ldo, dtype, heads * D, who, "out"));
    if (out == Q || out == K || out == V) return fail(FTC_EINVAL, "%s: out aliases an input", who);
    FTC_TRY(check_ws(who, attention_ws(n_q, n_kv, n_graphs, heads, kv_heads, D), ws, ws_bytes));
    return launch_attention(p, out, ldo, lse, ws, static_cast<hipStream_t>(stream));
}

size_t ftc_graph_attention_backward_workspace_bytes(int32_t n_q, int32_t n_kv, int32_t n_graphs, int32_t heads, int32_t kv_heads,
                                                    int32_t D)
{
    if (!attention_sizes_ok(n_q, n_kv, n_graphs, heads, kv_heads, D)) return 0;
    return attention_backward_ws(n_q, n_kv, n_graphs, heads, kv_heads, D);
}

int32_t ftc_graph_attention_backward(int32_t n_q, const int32_t *q_ptr, int32_t n_kv, const int32_t *kv_ptr, int32_t n_graphs,
                                     int32_t heads, int32_t kv_heads, int32_t D, int32_t dtype, const void *Q, int32_t ldq,
                                     const void *K, int32_t ldk, const void *V, int32_t ldv, const uint8_t *kv_mask, float scale,
                                     const void *out, int32_t ldo, const float *lse, const void *dOut, int32_t lddo, void *dQ,
                                     int32_t lddq, void *dK, int32_t lddk, void *dV, int32_t lddv, void *ws, size_t ws_bytes,
                                     void *stream)
{
    const char *who = "ftc_graph_attention_backward";
    const AttnShape p = {n_q, n_kv, n_graphs, heads, kv_heads, D, dtype, Q, K, V, ldq, ldk, ldv, q_ptr, kv_ptr, kv_mask, scale};
    FTC_TRY(check_attention(who, p));
    if (n_graphs == 0 || (n_q == 0 && n_kv == 0)) return FTC_OK;
    if (n_q > 0) {
        FTC_TRY(check_dense(out, ldo, dtype, heads * D, who, "out"));
        FTC_TRY(check_dense(dOut, lddo, dtype, heads * D, who, "dOut"));
        FTC_TRY(check_dense(dQ, lddq, dtype, heads * D, who, "dQ"));
        if (!lse) return fail(FTC_EINVAL, "%s: lse is NULL", who);
    }
    if (n_kv > 0) {
        FTC_TRY(check_dense(dK, lddk, dtype, kv_heads * D, who, "dK"));
        FTC_TRY(check_dense(dV, lddv, dtype, kv_heads * D, who, "dV"));
    }
    const void *outs[3] = {n_q > 0 ? dQ : nullptr, n_kv > 0 ? dK : nullptr, n_kv > 0 ? dV : nullptr}, *ins[6] = {Q, K, V, out, dOut, lse};
    for (int i = 0; i < 3; ++i) {
        for (int j = 0; j < 6; ++j)
            if (outs[i] && outs[i] == ins[j]) return fail(FTC_EINVAL, "%s: an output aliases an input", who);
        for (int j = 0; j < i; ++j)
            if (outs[i] && outs[i] == outs[j]) return fail(FTC_EINVAL, "%s: two outputs are the same", who);
    }
    FTC_TRY(check_ws(who, attention_backward_ws(n_q, n_kv, n_graphs, heads, kv_heads, D), ws, ws_bytes));
    return launch_attention_backward(p, out, ldo, lse, dOut, lddo, dQ, lddq, dK, lddk, dV, lddv, ws, static_cast<hipStream_t>(stream));
}

// ---- locality reordering (preprocessing) ---------------------------------------------------------
size_t ftc_reorder_workspace_bytes(int32_t n, int32_t nnz)
{
    if (n < 0 || nnz < 0) return 0;
    return reorder_ws(n, nnz);
}

static int32_t check_reorder_ws(const char *who, int n, int nnz, void *ws, size_t ws_bytes)
{
    const size_t need = reorder_ws(n, nnz);
    if (!ws || ws_bytes < need) return fail(FTC_EWORKSPACE, "%s: workspace of %zu bytes needed", who, need);
    if (reinterpret_cast<uintptr_t>(ws) % 256 != 0) return fail(FTC_EALIGN, "%s: workspace must be 256-byte aligned", who);
    return FTC_OK;
}

int32_t ftc_degree_order(const ftc_csr *g, int32_t mode, int32_t *perm, int32_t *inv, void *ws, size_t ws_bytes,
                         void *stream)
{
    FTC_TRY(check_csr(g, "ftc_degree_order"));
    if (mode != FTC_ORDER_DEGREE && mode != FTC_ORDER_DEGREE_CLASSES)
        return fail(FTC_EINVAL, "ftc_degree_order: unknown mode %d", mode);
    if (g->n == 0) return FTC_OK;
    if (!perm || !inv) return fail(FTC_EINVAL, "ftc_degree_order: perm or inv is NULL");
    FTC_TRY(check_reorder_ws("ftc_degree_order", g->n, g->nnz, ws, ws_bytes));
    return launch_degree_order(*g, mode, perm, inv, ws, static_cast<hipStream_t>(stream));
}

int32_t ftc_order_by_key(int32_t n, const int32_t *keys, int32_t *perm, int32_t *inv, int32_t *flag, void *ws,
                         size_t ws_bytes, void *stream)
{
    if (n < 0) return fail(FTC_EINVAL, "ftc_order_by_key: negative n");
    if (!flag) return fail(FTC_EINVAL, "ftc_order_by_key: flag is NULL");
    if (n > 0 && (!keys || !perm || !inv)) return fail(FTC_EINVAL, "ftc_order_by_key: keys, perm or inv is NULL");
    FTC_TRY(check_reorder_ws("ftc_order_by_key", n, 0, ws, ws_bytes));
    return launch_order_by_key(n, keys, perm, inv, flag, ws, static_cast<hipStream_t>(stream));
}

int32_t ftc_label_propagation(const ftc_csr *g, int32_t rounds, int32_t *labels, void *ws, size_t ws_bytes, void *stream)
{
    FTC_TRY(check_csr(g, "ftc_label_propagation"));
    if (rounds < 0) return fail(FTC_EINVAL, "ftc_label_propagation: negative number of rounds");
    if (g->n == 0) return FTC_OK;
    if (!labels) return fail(FTC_EINVAL, "ftc_label_propagation: labels is NULL");
    FTC_TRY(check_reorder_ws("ftc_label_propagation", g->n, g->nnz, ws, ws_bytes));
    return launch_label_propagation(*g, rounds, labels, ws, static_cast<hipStream_t>(stream));
}

int32_t ftc_permute_graph(const ftc_csr *g, const int32_t *perm, const int32_t *inv, int32_t *row_ptr_out,
                          int32_t *col_idx_out, int32_t *flag, void *ws, size_t ws_bytes, void *stream)
{
    FTC_TRY(check_csr(g, "ftc_permute_graph"));
    if (!flag) return fail(FTC_EINVAL, "ftc_permute_graph: flag is NULL");
    if (!row_ptr_out) return fail(FTC_EINVAL, "ftc_permute_graph: row_ptr_out is NULL");
    if (g->n > 0 && (!perm || !inv)) return fail(FTC_EINVAL, "ftc_permute_graph: perm or inv is NULL");
    if (g->nnz > 0 && !col_idx_out) return fail(FTC_EINVAL, "ftc_permute_graph: col_idx_out is NULL");
    if (row_ptr_out == g->row_ptr || (col_idx_out && col_idx_out == g->col_idx))
        return fail(FTC_EINVAL, "ftc_permute_graph: the output aliases the input graph");
    FTC_TRY(check_reorder_ws("ftc_permute_graph", g->n, g->nnz, ws, ws_bytes));
    return launch_permute_graph(*g, perm, inv, row_ptr_out, col_idx_out, flag, ws, static_cast<hipStream_t>(stream));
}

int32_t ftc_permute_rows(int32_t n, const void *X, int32_t ldx, int32_t dtype, int32_t D, const int32_t *map, void *out,
                         int32_t ldo, void *stream)
{
    if (n < 0) return fail(FTC_EINVAL, "ftc_permute_rows: negative n");
    if (n == 0) return FTC_OK;
    FTC_TRY(check_dense(X, ldx, dtype, D, "ftc_permute_rows", "X"));
    FTC_TRY(check_dense(out, ldo, dtype, D, "ftc_permute_rows", "out"));
    if (!map) return fail(FTC_EINVAL, "ftc_permute_rows: map is NULL");
    if (out == X) return fail(FTC_EINVAL, "ftc_permute_rows: out aliases X");
    return launch_permute_rows(n, X, ldx, dtype, D, map, out, ldo, static_cast<hipStream_t>(stream));
}

// ---- per-graph plan --------------------------------------------------------------------------------
int32_t ftc_degree_stats(const ftc_csr *g, int64_t *stats, void *stream)
{
    FTC_TRY(check_csr(g, "ftc_degree_stats"));
    if (!stats) return fail(FTC_EINVAL, "ftc_degree_stats: stats is NULL");
    return launch_degree_stats(*g, stats, static_cast<hipStream_t>(stream));
}

// Thresholds of the plan, from measurements on the benchmark graphs (bench.py --reorder, --sweep):
// relabelling by degree class paid 5 to 17 % on the gather kernels of the graphs with skew 7.8, 9.3
// and 70 and nothing on those with skew 1.03 and 1.1; it cannot pay while the whole feature matrix
// fits the 4 MiB L2 of one XCD.  With flat degrees only a community ordering can help (block-model
// graph: -28 to -52 % after ten rounds of label propagation); whether the graph has communities is
// not visible in these statistics, so the plan proposes a trial.
static constexpr double PLAN_SKEW_MIN = 2.0;
static constexpr double PLAN_L2_BYTES = 4.0 * 1024 * 1024;

int32_t ftc_plan_graph(int32_t n, int32_t nnz, int64_t sum_deg_sq, int64_t sum_uniq, int32_t D, int32_t dtype,
                       ftc_plan *plan)
{
    if (!plan) return fail(FTC_EINVAL, "ftc_plan_graph: plan is NULL");
    if (n < 0 || nnz < 0 || D < 1 || !valid_dtype(dtype) || sum_deg_sq < 0 || sum_uniq < 0 || sum_uniq > nnz)
        return fail(FTC_EINVAL, "ftc_plan_graph: bad argument");
    plan->skew = nnz > 0 ? static_cast<double>(n) * static_cast<double>(sum_deg_sq) /
                               (static_cast<double>(nnz) * static_cast<double>(nnz))
                         : 0.0;
    plan->reuse = sum_uniq > 0 ? static_cast<double>(nnz) / static_cast<double>(sum_uniq) : 0.0;
    const double feature_bytes = static_cast<double>(n) * D * elem_size(dtype);
    plan->reorder = FTC_ORDER_NONE;
    if (feature_bytes > PLAN_L2_BYTES) {
        if (plan->skew >= PLAN_SKEW_MIN) plan->reorder = FTC_ORDER_DEGREE_CLASSES;
        else if (nnz >= 8.0 * n) plan->reorder = FTC_ORDER_COMMUNITIES;  // flat degrees: only communities can help
    }
    int vec, lpr;
    const bool seg = seg_shape(dtype, D, &vec, &lpr);
    plan->agnn_single_pass = seg ? 1 : 0;
    plan->agnn_backward_single_pass = agnn_backward_fused_shape(dtype, D) ? 1 : 0;
    // FTC_PATH_AUTO splits the windows between the two kernels only where the matrix cores can win
    plan->spmm_mfma_windows = (mfma_shape_ok(dtype, D) && spmm_mfma_reuse(D) >= 0.f) ? 1 : 0;
    plan->sddmm_mfma_windows = (mfma_shape_ok(dtype, D) && sddmm_mfma_reuse(D) >= 0.f) ? 1 : 0;
    plan->mfma_min_reuse = sddmm_mfma_reuse(D);
    return FTC_OK;
}

}  // extern "C"
