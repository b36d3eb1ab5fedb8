// C ABI of libtfg: host-side argument checks, then the launchers.
// Every entry point validates before it touches the GPU, so a rejected call
// enqueues nothing.  See include/tfg.h for the contract of each call.
#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <memory>
#include <new>

#include "common.cuh"

// NVTX ranges (header-only NVTX 3; no-ops unless a profiler is attached):
// every entry point opens a range named after itself around its host work
// and launches, so ncu / nsys timelines show which call enqueued which
// kernels.  TFG_NVTX=0 compiles them out.
#ifndef TFG_NVTX
#define TFG_NVTX 1
#endif
#if TFG_NVTX
#include <nvtx3/nvToolsExt.h>
namespace {
struct NvtxRange {
    explicit NvtxRange(const char *name) { nvtxRangePushA(name); }
    ~NvtxRange() { nvtxRangePop(); }
    NvtxRange(const NvtxRange &) = delete;
    NvtxRange &operator=(const NvtxRange &) = delete;
};
}  // namespace
#define TFG_RANGE(name) NvtxRange tfg_nvtx_range_(name)
#else
#define TFG_RANGE(name) \
    do {                \
    } while (0)
#endif

// Helpers of the bounds-checked debug build (check_bounds.cu), the CSR
// build over an int32 edge list (csr_build.cu) and the max backward with
// win marks (backward.cu).
namespace tfg {
size_t max_backward_workspace_bytes(int64_t n, int64_t e, int64_t f);
cudaError_t launch_build_csr32(const int32_t *edge_index, int64_t e, int64_t n, int32_t *rowptr,
                               int32_t *col, int32_t *perm, int32_t *in_degree, void *ws,
                               int32_t *status, cudaStream_t s, bool by_source);
bool allocation_range(const void *p, uintptr_t *base, size_t *size);
cudaError_t csr_ends(const int32_t *rowptr, int64_t n, int32_t *first, int32_t *last,
                     cudaStream_t s);
cudaError_t validate_csr(const int32_t *rowptr, const int32_t *col, const int32_t *perm,
                         int64_t n, int64_t e, int *flags, cudaStream_t s);
}  // namespace tfg

namespace {

thread_local char g_err[512];

int fail(int code, const char *fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof(g_err), fmt, ap);
    va_end(ap);
    return code;
}

int ok() {
    g_err[0] = '\0';
    return TFG_OK;
}

int cuda_result(cudaError_t e, const char *where) {
    if (e != cudaSuccess) return fail(TFG_ERR_CUDA, "%s: %s", where, cudaGetErrorString(e));
    return ok();
}

constexpr int64_t kIndexLimit = int64_t(1) << 31;  // CSR ids are int32

int check_counts(const char *fn, int64_t n, int64_t e) {
    if (n < 0 || e < 0) return fail(TFG_ERR_INVALID_ARG, "%s: negative size (N=%lld, E=%lld)", fn,
                                    (long long)n, (long long)e);
    if (n >= kIndexLimit || e >= kIndexLimit)
        return fail(TFG_ERR_TOO_LARGE, "%s: N and E must be < 2^31 (N=%lld, E=%lld)", fn,
                    (long long)n, (long long)e);
    if (e > 0 && n == 0) return fail(TFG_ERR_INVALID_ARG, "%s: edges given but N == 0", fn);
    return TFG_OK;
}

int check_features(const char *fn, int64_t n, int64_t f) {
    if (f < 1 || f > (int64_t(1) << 24))
        return fail(TFG_ERR_INVALID_ARG, "%s: feature count must be in [1, 2^24] (F=%lld)", fn,
                    (long long)f);
    if (n * f >= (int64_t(1) << 46))
        return fail(TFG_ERR_TOO_LARGE, "%s: N*F too large", fn);
    return TFG_OK;
}

int check_dtype(const char *fn, int dtype) {
    if (dtype != TFG_F32 && dtype != TFG_BF16)
        return fail(TFG_ERR_INVALID_ARG, "%s: unknown dtype %d", fn, dtype);
    return TFG_OK;
}

#define TFG_TRY(expr)                    \
    do {                                 \
        int rc_ = (expr);                \
        if (rc_ != TFG_OK) return rc_;   \
    } while (0)

#define TFG_NEED(ptr, cond, fn, name)                                                  \
    do {                                                                               \
        if ((cond) && (ptr) == nullptr)                                                \
            return fail(TFG_ERR_INVALID_ARG, "%s: %s must not be NULL", fn, name);    \
    } while (0)

// ---- bounds-checked debug build (TFG_CHECK_BOUNDS=1) ----------------------
// Before any launch, every device buffer is checked against the allocation
// that holds it (the bytes the call will touch must lie inside it), and every
// caller-built index array is read once on the device: rowptr[0] = 0,
// rowptr[N] = E, rowptr non-decreasing, col ids in [0, N), perm ids in
// [0, E).  A violation returns TFG_ERR_INDEX_RANGE with the reason and
// launches nothing, so no kernel reads out of bounds.  Each check copies a
// few values to the host and synchronises the stream: a debugging aid, not a
// production mode.  The default build compiles none of it.
#ifndef TFG_CHECK_BOUNDS
#define TFG_CHECK_BOUNDS 0
#endif

#if TFG_CHECK_BOUNDS
int debug_extent(const char *fn, const char *name, const void *p, size_t bytes) {
    if (p == nullptr || bytes == 0) return TFG_OK;
    uintptr_t base = 0;
    size_t size = 0;
    if (!tfg::allocation_range(p, &base, &size))
        return fail(TFG_ERR_INVALID_ARG, "%s: %s is not device memory of the current context", fn,
                    name);
    const uintptr_t a = reinterpret_cast<uintptr_t>(p);
    if (a + bytes > base + size)
        return fail(TFG_ERR_INDEX_RANGE,
                    "%s: %s must hold %zu bytes, its allocation ends %zu bytes after it", fn, name,
                    bytes, static_cast<size_t>(base + size - a));
    return TFG_OK;
}

// rowptr [N + 1] (or NULL: col ids only, E = e_given), col [E] and perm [E]
// each NULL when the call does not read it (a NULL col that the call reads
// is refused when E > 0); e_given < 0 takes E from rowptr[N].  E is returned
// in *e_out.
int debug_csr(const char *fn, const char *which, const int32_t *rowptr, const int32_t *col,
              const int32_t *perm, int64_t n, int64_t e_given, int64_t *e_out,
              tfg_stream_t stream, bool col_read = true) {
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    int64_t e = e_given;
    if (rowptr) {
        TFG_TRY(debug_extent(fn, "rowptr", rowptr, sizeof(int32_t) * size_t(n + 1)));
        int32_t first = 0, last = 0;
        cudaError_t err = tfg::csr_ends(rowptr, n, &first, &last, s);
        if (err != cudaSuccess) return cuda_result(err, fn);
        if (first != 0 || last < 0 || (e_given >= 0 && last != e_given))
            return fail(TFG_ERR_INDEX_RANGE, "%s: %s rowptr[0] = %d, rowptr[N] = %d (E = %lld)",
                        fn, which, first, last, (long long)e_given);
        e = last;
    }
    if (e_out) *e_out = e;
    if (e > 0 && col_read && col == nullptr)
        return fail(TFG_ERR_INVALID_ARG, "%s: %s is NULL but the graph has %lld edges", fn, which,
                    (long long)e);
    if (e > 0) {
        TFG_TRY(debug_extent(fn, "col", col, sizeof(int32_t) * size_t(e)));
        TFG_TRY(debug_extent(fn, "perm", perm, sizeof(int32_t) * size_t(e)));
    }
    int flags = 0;
    cudaError_t err = tfg::validate_csr(rowptr, col, perm, n, e, &flags, s);
    if (err != cudaSuccess) return cuda_result(err, fn);
    if (flags & 1) return fail(TFG_ERR_INDEX_RANGE, "%s: %s rowptr decreases", fn, which);
    if (flags & 2) return fail(TFG_ERR_INDEX_RANGE, "%s: a %s id lies outside [0, N)", fn, which);
    if (flags & 4) return fail(TFG_ERR_INDEX_RANGE, "%s: a %s perm id lies outside [0, E)", fn, which);
    return TFG_OK;
}
#define TFG_DEBUG(expr) TFG_TRY(expr)

#else
#define TFG_DEBUG(expr) \
    do {                \
    } while (0)
#endif

size_t elem_bytes(int dtype) { return dtype == TFG_BF16 ? 2 : 4; }

// Whether [a, a + na) and [b, b + nb) share a byte.
bool overlap(const void *a, size_t na, const void *b, size_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return na > 0 && nb > 0 && x < y + nb && y < x + na;
}

int check_workspace(const char *fn, const void *ws, size_t given, size_t need, size_t align) {
    if (need == 0) return TFG_OK;
    if (ws == nullptr || given < need)
        return fail(TFG_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need, ws ? given : size_t(0));
    if (reinterpret_cast<uintptr_t>(ws) % align != 0)
        return fail(TFG_ERR_INVALID_ARG, "%s: workspace must be %zu-byte aligned", fn, align);
    return TFG_OK;
}

int check_element(const char *fn, const char *name, const void *p, int dtype) {
    if (reinterpret_cast<uintptr_t>(p) % elem_bytes(dtype) != 0)
        return fail(TFG_ERR_INVALID_ARG, "%s: %s is not aligned to its element", fn, name);
    return TFG_OK;
}

int aggregate_common(const char *fn, int mode, const int32_t *rowptr, const int32_t *col,
                     const float *w, const float *dinv, const void *x, int dtype, int64_t n,
                     int64_t f, int add_self, float fill, float *out, tfg_stream_t stream) {
    TFG_RANGE(fn);
    TFG_TRY(check_counts(fn, n, 0));
    TFG_TRY(check_features(fn, n, f));
    TFG_TRY(check_dtype(fn, dtype));
    TFG_NEED(rowptr, true, fn, "rowptr");
    TFG_NEED(x, n > 0, fn, "x");
    TFG_NEED(out, n > 0, fn, "out");
    TFG_NEED(dinv, mode == 3 && n > 0, fn, "dinv");
#if TFG_CHECK_BOUNDS
    {
        int64_t e = 0;
        TFG_DEBUG(debug_csr(fn, "col", rowptr, col, nullptr, n, -1, &e, stream));
        TFG_DEBUG(debug_extent(fn, "w_csr", w, sizeof(float) * size_t(e)));
        TFG_DEBUG(debug_extent(fn, "dinv", dinv, sizeof(float) * size_t(n)));
        TFG_DEBUG(debug_extent(fn, "x", x, elem_bytes(dtype) * size_t(n * f)));
        TFG_DEBUG(debug_extent(fn, "out", out, sizeof(float) * size_t(n * f)));
    }
#endif
    return cuda_result(tfg::launch_aggregate(mode, rowptr, col, w, dinv, x, dtype, n, f, add_self,
                                             fill, out, reinterpret_cast<cudaStream_t>(stream)),
                       fn);
}

constexpr int kMaxHops = 1024;

int propagate_common(const char *fn, const int32_t *rowptr, const int32_t *col, const float *dinv,
                     const float *w, const void *x0, int dtype, int64_t n, int64_t f, int64_t hops,
                     float alpha, int add_self, float fill, float *out, void *ws, size_t ws_bytes,
                     tfg_stream_t stream) {
    TFG_RANGE(fn);
    TFG_TRY(check_counts(fn, n, 0));
    TFG_TRY(check_features(fn, n, f));
    TFG_TRY(check_dtype(fn, dtype));
    if (hops < 0 || hops > kMaxHops)
        return fail(TFG_ERR_INVALID_ARG, "%s: num_hops must be in [0, %d]", fn, kMaxHops);
    if (!(alpha >= 0.f && alpha <= 1.f))
        return fail(TFG_ERR_INVALID_ARG, "%s: alpha must be in [0, 1]", fn);
    TFG_NEED(rowptr, hops > 0, fn, "rowptr");
    TFG_NEED(dinv, hops > 0 && n > 0, fn, "dinv");
    TFG_NEED(x0, n > 0, fn, "x0");
    TFG_NEED(out, n > 0, fn, "out");
    const size_t need = tfg::propagate_workspace_bytes(n, f, hops);
    if (need > 0) {
        if (ws == nullptr || ws_bytes < need)
            return fail(TFG_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need,
                        ws ? ws_bytes : size_t(0));
        if (reinterpret_cast<uintptr_t>(ws) % 16 != 0)
            return fail(TFG_ERR_INVALID_ARG, "%s: workspace must be 16-byte aligned", fn);
    }
#if TFG_CHECK_BOUNDS
    if (hops > 0) {
        int64_t e = 0;
        TFG_DEBUG(debug_csr(fn, "col", rowptr, col, nullptr, n, -1, &e, stream));
        TFG_DEBUG(debug_extent(fn, "w_csr", w, sizeof(float) * size_t(e)));
        TFG_DEBUG(debug_extent(fn, "dinv", dinv, sizeof(float) * size_t(n)));
    }
    TFG_DEBUG(debug_extent(fn, "x0", x0, elem_bytes(dtype) * size_t(n * f)));
    TFG_DEBUG(debug_extent(fn, "out", out, sizeof(float) * size_t(n * f)));
    TFG_DEBUG(debug_extent(fn, "workspace", ws, need));
#endif
    return cuda_result(tfg::launch_propagate(rowptr, col, w, dinv, x0, dtype, n, f, hops, alpha,
                                             add_self, fill, out, ws,
                                             reinterpret_cast<cudaStream_t>(stream)),
                       fn);
}

}  // namespace

namespace tfg {
int sm_count() {
    thread_local int sms = 0, sms_dev = -1;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) dev = 0;
    if (sms == 0 || sms_dev != dev) {
        if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms <= 0)
            sms = 148;
        sms_dev = dev;
    }
    return sms;
}

int balanced_grid(int64_t n, int64_t e, int64_t min_work) {
    const int sms = sm_count();
    const int64_t by_work = (n + e + min_work - 1) / min_work;
    const int64_t cap = int64_t(sms) * 16;
    const int64_t g = by_work < cap ? by_work : cap;
    return static_cast<int>(g < 1 ? 1 : g);
}
}  // namespace tfg

extern "C" {

int tfg_version(void) { return 300; }

int tfg_check_bounds_enabled(void) { return TFG_CHECK_BOUNDS; }

const char *tfg_last_error(void) { return g_err; }

int tfg_build_csr_workspace_size(int64_t num_nodes, int64_t num_edges, size_t *bytes) {
    const char *fn = "tfg_build_csr_workspace_size";
    TFG_RANGE(fn);
    TFG_TRY(check_counts(fn, num_nodes, num_edges));
    TFG_NEED(bytes, true, fn, "bytes");
    *bytes = tfg::csr_workspace_bytes(num_nodes, num_edges);
    return ok();
}

namespace {
// edge_index: int64 [2, E], or int32 [2, E] when id32
int build_csr_common(const char *fn, bool by_source, const void *edge_index, bool id32, int64_t num_edges,
                     int64_t num_nodes, int32_t *rowptr, int32_t *col, int32_t *perm,
                     int32_t *in_degree, void *workspace, size_t workspace_bytes, int32_t *status,
                     tfg_stream_t stream) {
    TFG_RANGE(fn);
    TFG_TRY(check_counts(fn, num_nodes, num_edges));
    TFG_NEED(edge_index, num_edges > 0, fn, "edge_index");
    TFG_NEED(rowptr, true, fn, "rowptr");
    TFG_NEED(col, num_edges > 0, fn, "col");
    TFG_NEED(perm, num_edges > 0, fn, "perm");
    TFG_NEED(in_degree, num_nodes > 0, fn, "in_degree");
    TFG_NEED(status, true, fn, "status");
    const size_t need = tfg::csr_workspace_bytes(num_nodes, num_edges);
    if (num_edges > 0) {
        if (workspace == nullptr || workspace_bytes < need)
            return fail(TFG_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need,
                        workspace ? workspace_bytes : size_t(0));
        if (reinterpret_cast<uintptr_t>(workspace) % 256 != 0)
            return fail(TFG_ERR_INVALID_ARG, "%s: workspace must be 256-byte aligned", fn);
    }
    TFG_DEBUG(debug_extent(fn, "edge_index", edge_index,
                           (id32 ? sizeof(int32_t) : sizeof(int64_t)) * 2 * size_t(num_edges)));
    TFG_DEBUG(debug_extent(fn, "rowptr", rowptr, sizeof(int32_t) * size_t(num_nodes + 1)));
    TFG_DEBUG(debug_extent(fn, "col", col, sizeof(int32_t) * size_t(num_edges)));
    TFG_DEBUG(debug_extent(fn, "perm", perm, sizeof(int32_t) * size_t(num_edges)));
    TFG_DEBUG(debug_extent(fn, "in_degree", in_degree, sizeof(int32_t) * size_t(num_nodes)));
    TFG_DEBUG(debug_extent(fn, "workspace", num_edges > 0 ? workspace : nullptr, need));
    const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    return cuda_result(
        id32 ? tfg::launch_build_csr32(static_cast<const int32_t *>(edge_index), num_edges,
                                       num_nodes, rowptr, col, perm, in_degree, workspace, status,
                                       s, by_source)
             : tfg::launch_build_csr(static_cast<const int64_t *>(edge_index), num_edges,
                                     num_nodes, rowptr, col, perm, in_degree, workspace, status,
                                     s, by_source),
        fn);
}
}  // namespace

int tfg_build_csr(const int64_t *edge_index, int64_t num_edges, int64_t num_nodes,
                  int32_t *rowptr, int32_t *col, int32_t *perm, int32_t *in_degree,
                  void *workspace, size_t workspace_bytes, int32_t *status,
                  tfg_stream_t stream) {
    return build_csr_common("tfg_build_csr", false, edge_index, false, num_edges, num_nodes, rowptr,
                            col, perm, in_degree, workspace, workspace_bytes, status, stream);
}

int tfg_build_csr32(const int32_t *edge_index, int64_t num_edges, int64_t num_nodes,
                    int32_t *rowptr, int32_t *col, int32_t *perm, int32_t *in_degree,
                    void *workspace, size_t workspace_bytes, int32_t *status,
                    tfg_stream_t stream) {
    return build_csr_common("tfg_build_csr32", false, edge_index, true, num_edges, num_nodes,
                            rowptr, col, perm, in_degree, workspace, workspace_bytes, status,
                            stream);
}

int tfg_build_csr32_by_source(const int32_t *edge_index, int64_t num_edges, int64_t num_nodes,
                              int32_t *rowptr_src, int32_t *col_src, int32_t *perm_src,
                              int32_t *out_degree, void *workspace, size_t workspace_bytes,
                              int32_t *status, tfg_stream_t stream) {
    return build_csr_common("tfg_build_csr32_by_source", true, edge_index, true, num_edges,
                            num_nodes, rowptr_src, col_src, perm_src, out_degree, workspace,
                            workspace_bytes, status, stream);
}

int tfg_build_csr_by_source(const int64_t *edge_index, int64_t num_edges, int64_t num_nodes,
                            int32_t *rowptr_src, int32_t *col_src, int32_t *perm_src,
                            int32_t *out_degree, void *workspace, size_t workspace_bytes,
                            int32_t *status, tfg_stream_t stream) {
    return build_csr_common("tfg_build_csr_by_source", true, edge_index, false, num_edges, num_nodes,
                            rowptr_src, col_src, perm_src, out_degree, workspace, workspace_bytes,
                            status, stream);
}

int tfg_gcn_norm(const int32_t *rowptr, const int32_t *col, const int32_t *perm,
                 const float *edge_weight, int64_t num_nodes, int64_t num_edges,
                 int add_self_loops, float self_loop_fill, float *dinv, float *w_csr,
                 tfg_stream_t stream) {
    const char *fn = "tfg_gcn_norm";
    TFG_RANGE(fn);
    TFG_TRY(check_counts(fn, num_nodes, num_edges));
    TFG_NEED(rowptr, true, fn, "rowptr");
    TFG_NEED(dinv, num_nodes > 0, fn, "dinv");
    TFG_NEED(col, w_csr != nullptr && num_edges > 0, fn, "col");
    TFG_NEED(perm, (w_csr != nullptr || edge_weight != nullptr) && num_edges > 0, fn, "perm");
    TFG_DEBUG(debug_csr(fn, "col", rowptr, w_csr ? col : nullptr, w_csr || edge_weight ? perm : nullptr,
                        num_nodes, num_edges, nullptr, stream, w_csr != nullptr));
    TFG_DEBUG(debug_extent(fn, "edge_weight", edge_weight, sizeof(float) * size_t(num_edges)));
    TFG_DEBUG(debug_extent(fn, "dinv", dinv, sizeof(float) * size_t(num_nodes)));
    TFG_DEBUG(debug_extent(fn, "w_csr", w_csr, sizeof(float) * size_t(num_edges)));
    return cuda_result(tfg::launch_gcn_norm(rowptr, col, perm, edge_weight, num_nodes,
                                            add_self_loops, self_loop_fill, dinv, w_csr,
                                            reinterpret_cast<cudaStream_t>(stream)),
                       fn);
}

int tfg_aggregate_sum(const int32_t *rowptr, const int32_t *col, const float *w_csr,
                      const void *x, int x_dtype, int64_t num_nodes, int64_t num_features,
                      float *out, tfg_stream_t stream) {
    return aggregate_common("tfg_aggregate_sum", 0, rowptr, col, w_csr, nullptr, x, x_dtype,
                            num_nodes, num_features, 0, 0.f, out, stream);
}

int tfg_aggregate_mean(const int32_t *rowptr, const int32_t *col, const float *w_csr,
                       const void *x, int x_dtype, int64_t num_nodes, int64_t num_features,
                       float *out, tfg_stream_t stream) {
    return aggregate_common("tfg_aggregate_mean", 1, rowptr, col, w_csr, nullptr, x, x_dtype,
                            num_nodes, num_features, 0, 0.f, out, stream);
}

int tfg_aggregate_max(const int32_t *rowptr, const int32_t *col, const float *w_csr,
                      const void *x, int x_dtype, int64_t num_nodes, int64_t num_features,
                      float *out, tfg_stream_t stream) {
    return aggregate_common("tfg_aggregate_max", 2, rowptr, col, w_csr, nullptr, x, x_dtype,
                            num_nodes, num_features, 0, 0.f, out, stream);
}

int tfg_gcn_aggregate_sum(const int32_t *rowptr, const int32_t *col, const float *dinv,
                          const float *w_csr, const void *x, int x_dtype, int64_t num_nodes,
                          int64_t num_features, int add_self_loops, float self_loop_fill,
                          float *out, tfg_stream_t stream) {
    return aggregate_common("tfg_gcn_aggregate_sum", 3, rowptr, col, w_csr, dinv, x, x_dtype,
                            num_nodes, num_features, add_self_loops, self_loop_fill, out, stream);
}

int tfg_aggregate_backward_workspace_size(int reduce, int64_t num_edges, size_t *bytes) {
    const char *fn = "tfg_aggregate_backward_workspace_size";
    TFG_RANGE(fn);
    TFG_TRY(check_counts(fn, 1, num_edges));
    if (reduce != TFG_SUM && reduce != TFG_MEAN)
        return fail(TFG_ERR_INVALID_ARG, "%s: reduce must be TFG_SUM or TFG_MEAN", fn);
    TFG_NEED(bytes, true, fn, "bytes");
    *bytes = tfg::backward_workspace_bytes(reduce, num_edges);
    return ok();
}

int tfg_aggregate_backward(int reduce, const int32_t *rowptr_src, const int32_t *col_src,
                           const int32_t *perm_src, const float *edge_weight,
                           const int32_t *in_degree, const float *grad_out, int64_t num_nodes,
                           int64_t num_edges, int64_t num_features, float *grad_x,
                           void *workspace, size_t workspace_bytes, tfg_stream_t stream) {
    const char *fn = "tfg_aggregate_backward";
    TFG_RANGE(fn);
    TFG_TRY(check_counts(fn, num_nodes, num_edges));
    TFG_TRY(check_features(fn, num_nodes, num_features));
    if (reduce != TFG_SUM && reduce != TFG_MEAN)
        return fail(TFG_ERR_INVALID_ARG, "%s: reduce must be TFG_SUM or TFG_MEAN", fn);
    TFG_NEED(rowptr_src, true, fn, "rowptr_src");
    TFG_NEED(col_src, num_edges > 0, fn, "col_src");
    TFG_NEED(perm_src, num_edges > 0 && (edge_weight != nullptr || reduce == TFG_MEAN), fn,
             "perm_src");
    TFG_NEED(in_degree, reduce == TFG_MEAN && num_edges > 0, fn, "in_degree");
    TFG_NEED(grad_out, num_nodes > 0, fn, "grad_out");
    TFG_NEED(grad_x, num_nodes > 0, fn, "grad_x");
    const bool weighted = num_edges > 0 && (edge_weight != nullptr || reduce == TFG_MEAN);
    const size_t need = weighted ? tfg::backward_workspace_bytes(reduce, num_edges) : 0;
    if (need > 0 && (workspace == nullptr || workspace_bytes < need))
        return fail(TFG_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need,
                    workspace ? workspace_bytes : size_t(0));
    TFG_DEBUG(debug_csr(fn, "col_src", rowptr_src, col_src, weighted ? perm_src : nullptr, num_nodes,
                        num_edges, nullptr, stream));
    TFG_DEBUG(debug_extent(fn, "edge_weight", edge_weight, sizeof(float) * size_t(num_edges)));
    TFG_DEBUG(debug_extent(fn, "in_degree", reduce == TFG_MEAN ? in_degree : nullptr,
                           sizeof(int32_t) * size_t(num_nodes)));
    TFG_DEBUG(debug_extent(fn, "grad_out", grad_out, sizeof(float) * size_t(num_nodes * num_features)));
    TFG_DEBUG(debug_extent(fn, "grad_x", grad_x, sizeof(float) * size_t(num_nodes * num_features)));
    TFG_DEBUG(debug_extent(fn, "workspace", need ? workspace : nullptr, need));
    return cuda_result(tfg::launch_aggregate_backward(reduce, rowptr_src, col_src, perm_src,
                                                      edge_weight, in_degree, grad_out, num_nodes,
                                                      num_edges, num_features, grad_x, workspace,
                                                      reinterpret_cast<cudaStream_t>(stream)),
                       fn);
}

int tfg_gcn_aggregate_backward(const int32_t *rowptr_src, const int32_t *col_src,
                               const float *dinv, const float *grad_out, int64_t num_nodes,
                               int64_t num_features, int add_self_loops, float self_loop_fill,
                               float *grad_x, tfg_stream_t stream) {
    return aggregate_common("tfg_gcn_aggregate_backward", 3, rowptr_src, col_src, nullptr, dinv,
                            grad_out, TFG_F32, num_nodes, num_features, add_self_loops,
                            self_loop_fill, grad_x, stream);
}

int tfg_aggregate_max_argmax(const int32_t *rowptr, const int32_t *col, const int32_t *perm,
                             const float *w_csr, const void *x, int x_dtype, int64_t num_nodes,
                             int64_t num_features, float *out, int32_t *argmax,
                             tfg_stream_t stream) {
    const char *fn = "tfg_aggregate_max_argmax";
    TFG_RANGE(fn);
    TFG_TRY(check_counts(fn, num_nodes, 0));
    TFG_TRY(check_features(fn, num_nodes, num_features));
    TFG_TRY(check_dtype(fn, x_dtype));
    TFG_NEED(rowptr, true, fn, "rowptr");
    TFG_NEED(perm, col != nullptr, fn, "perm");
    TFG_NEED(x, num_nodes > 0, fn, "x");
    TFG_NEED(out, num_nodes > 0, fn, "out");
    TFG_NEED(argmax, num_nodes > 0, fn, "argmax");
#if TFG_CHECK_BOUNDS
    {
        int64_t e = 0;
        TFG_DEBUG(debug_csr(fn, "col", rowptr, col, perm, num_nodes, -1, &e, stream));
        TFG_DEBUG(debug_extent(fn, "w_csr", w_csr, sizeof(float) * size_t(e)));
        TFG_DEBUG(debug_extent(fn, "x", x, elem_bytes(x_dtype) * size_t(num_nodes * num_features)));
        TFG_DEBUG(debug_extent(fn, "out", out, sizeof(float) * size_t(num_nodes * num_features)));
        TFG_DEBUG(debug_extent(fn, "argmax", argmax, sizeof(int32_t) * size_t(num_nodes * num_features)));
    }
#endif
    return cuda_result(tfg::launch_max_argmax(rowptr, col, perm, w_csr, x, x_dtype, num_nodes,
                                              num_features, out, argmax,
                                              reinterpret_cast<cudaStream_t>(stream)),
                       fn);
}

int tfg_aggregate_max_backward_workspace_size(int64_t num_nodes, int64_t num_edges,
                                              int64_t num_features, size_t *bytes) {
    const char *fn = "tfg_aggregate_max_backward_workspace_size";
    TFG_RANGE(fn);
    TFG_TRY(check_counts(fn, num_nodes, num_edges));
    TFG_TRY(check_features(fn, num_nodes, num_features));
    TFG_NEED(bytes, true, fn, "bytes");
    *bytes = tfg::max_backward_workspace_bytes(num_nodes, num_edges, num_features);
    return ok();
}

int tfg_aggregate_max_backward(const int32_t *rowptr_src, const int32_t *col_src,
                               const int32_t *perm_src, const int32_t *argmax,
                               const float *edge_weight, const float *grad_out,
                               int64_t num_nodes, int64_t num_edges, int64_t num_features,
                               float *grad_x, void *workspace, size_t workspace_bytes,
                               tfg_stream_t stream) {
    const char *fn = "tfg_aggregate_max_backward";
    TFG_RANGE(fn);
    TFG_TRY(check_counts(fn, num_nodes, num_edges));
    TFG_TRY(check_features(fn, num_nodes, num_features));
    TFG_NEED(rowptr_src, true, fn, "rowptr_src");
    TFG_NEED(col_src, num_edges > 0, fn, "col_src");
    TFG_NEED(perm_src, num_edges > 0, fn, "perm_src");
    TFG_NEED(argmax, num_nodes > 0, fn, "argmax");
    TFG_NEED(grad_out, num_nodes > 0, fn, "grad_out");
    TFG_NEED(grad_x, num_nodes > 0, fn, "grad_x");
    const size_t need =
        workspace ? tfg::max_backward_workspace_bytes(num_nodes, num_edges, num_features) : 0;
    if (need > 0 && workspace_bytes < need)
        return fail(TFG_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need,
                    workspace_bytes);
    if (need > 0 && reinterpret_cast<uintptr_t>(workspace) % 16 != 0)
        return fail(TFG_ERR_INVALID_ARG, "%s: workspace must be 16-byte aligned", fn);
    TFG_DEBUG(debug_csr(fn, "col_src", rowptr_src, col_src, perm_src, num_nodes, num_edges,
                        nullptr, stream));
    TFG_DEBUG(debug_extent(fn, "edge_weight", edge_weight, sizeof(float) * size_t(num_edges)));
    TFG_DEBUG(debug_extent(fn, "argmax", argmax, sizeof(int32_t) * size_t(num_nodes * num_features)));
    TFG_DEBUG(debug_extent(fn, "grad_out", grad_out, sizeof(float) * size_t(num_nodes * num_features)));
    TFG_DEBUG(debug_extent(fn, "grad_x", grad_x, sizeof(float) * size_t(num_nodes * num_features)));
    TFG_DEBUG(debug_extent(fn, "workspace", need ? workspace : nullptr, need));
    const int32_t *col = num_edges > 0 ? col_src : nullptr;
    const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    return cuda_result(
        tfg::launch_max_backward(rowptr_src, col, perm_src, argmax, edge_weight, grad_out, num_nodes,
                                 num_edges, num_features, grad_x, need ? workspace : nullptr, s),
        fn);
}

int tfg_propagate_workspace_size(int64_t num_nodes, int64_t num_features, int64_t num_hops,
                                 size_t *bytes) {
    const char *fn = "tfg_propagate_workspace_size";
    TFG_RANGE(fn);
    TFG_TRY(check_counts(fn, num_nodes, 0));
    TFG_TRY(check_features(fn, num_nodes, num_features));
    if (num_hops < 0 || num_hops > kMaxHops)
        return fail(TFG_ERR_INVALID_ARG, "%s: num_hops must be in [0, %d]", fn, kMaxHops);
    TFG_NEED(bytes, true, fn, "bytes");
    *bytes = tfg::propagate_workspace_bytes(num_nodes, num_features, num_hops);
    return ok();
}

int tfg_appnp_propagate(const int32_t *rowptr, const int32_t *col, const float *dinv,
                        const float *w_csr, const void *x0, int x_dtype, int64_t num_nodes,
                        int64_t num_features, int64_t num_hops, float alpha, int add_self_loops,
                        float self_loop_fill, float *out, void *workspace,
                        size_t workspace_bytes, tfg_stream_t stream) {
    return propagate_common("tfg_appnp_propagate", rowptr, col, dinv, w_csr, x0, x_dtype,
                            num_nodes, num_features, num_hops, alpha, add_self_loops,
                            self_loop_fill, out, workspace, workspace_bytes, stream);
}

int tfg_sgc_propagate(const int32_t *rowptr, const int32_t *col, const float *dinv,
                      const float *w_csr, const void *x0, int x_dtype, int64_t num_nodes,
                      int64_t num_features, int64_t num_hops, int add_self_loops,
                      float self_loop_fill, float *out, void *workspace, size_t workspace_bytes,
                      tfg_stream_t stream) {
    return propagate_common("tfg_sgc_propagate", rowptr, col, dinv, w_csr, x0, x_dtype,
                            num_nodes, num_features, num_hops, 0.f, add_self_loops,
                            self_loop_fill, out, workspace, workspace_bytes, stream);
}

int tfg_edge_softmax_workspace_size(int64_t num_nodes, int heads, size_t *bytes) {
    const char *fn = "tfg_edge_softmax_workspace_size";
    TFG_RANGE(fn);
    TFG_TRY(check_counts(fn, num_nodes, 0));
    if (heads < 1) return fail(TFG_ERR_INVALID_ARG, "%s: heads must be >= 1", fn);
    TFG_NEED(bytes, true, fn, "bytes");
    *bytes = tfg::softmax_workspace_bytes(num_nodes, heads);
    return ok();
}

int tfg_edge_softmax_aggregate(const int32_t *rowptr, const int32_t *col, const void *x,
                               int x_dtype, int64_t num_nodes, int64_t num_edges, int heads,
                               int channels,
                               const float *a_src, const float *a_dst, float negative_slope,
                               float *out, float *alpha, void *workspace,
                               size_t workspace_bytes, tfg_stream_t stream) {
    const char *fn = "tfg_edge_softmax_aggregate";
    TFG_RANGE(fn);
    TFG_TRY(check_counts(fn, num_nodes, num_edges));
    if (heads < 1 || channels < 1)
        return fail(TFG_ERR_INVALID_ARG, "%s: heads and channels must be >= 1", fn);
    TFG_TRY(check_features(fn, num_nodes, int64_t(heads) * channels));
    TFG_TRY(check_dtype(fn, x_dtype));
    TFG_NEED(rowptr, true, fn, "rowptr");
    TFG_NEED(col, num_edges > 0, fn, "col");
    TFG_NEED(x, num_nodes > 0, fn, "x");
    TFG_NEED(out, num_nodes > 0, fn, "out");
    TFG_NEED(a_src, true, fn, "a_src");
    TFG_NEED(a_dst, true, fn, "a_dst");
    const size_t need = tfg::softmax_workspace_bytes(num_nodes, heads);
    if (num_nodes > 0 && (workspace == nullptr || workspace_bytes < need))
        return fail(TFG_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need,
                    workspace ? workspace_bytes : size_t(0));
    TFG_DEBUG(debug_csr(fn, "col", rowptr, col, nullptr, num_nodes, num_edges, nullptr, stream));
    TFG_DEBUG(debug_extent(fn, "x", x, elem_bytes(x_dtype) * size_t(num_nodes * heads * channels)));
    TFG_DEBUG(debug_extent(fn, "out", out, sizeof(float) * size_t(num_nodes * heads * channels)));
    TFG_DEBUG(debug_extent(fn, "alpha", alpha, sizeof(float) * size_t(num_edges * heads)));
    TFG_DEBUG(debug_extent(fn, "a_src", a_src, sizeof(float) * size_t(heads * channels)));
    TFG_DEBUG(debug_extent(fn, "a_dst", a_dst, sizeof(float) * size_t(heads * channels)));
    TFG_DEBUG(debug_extent(fn, "workspace", num_nodes > 0 ? workspace : nullptr, need));
    return cuda_result(tfg::launch_edge_softmax(rowptr, num_edges > 0 ? col : nullptr, x, x_dtype,
                                                num_nodes, num_edges, heads, channels, a_src, a_dst,
                                                negative_slope, out, alpha, workspace,
                                                reinterpret_cast<cudaStream_t>(stream)),
                       fn);
}

int tfg_edge_softmax_backward_workspace_size(int64_t num_nodes, int heads, int channels,
                                             size_t *bytes) {
    const char *fn = "tfg_edge_softmax_backward_workspace_size";
    TFG_RANGE(fn);
    TFG_NEED(bytes, true, fn, "bytes");
    TFG_TRY(check_counts(fn, num_nodes, 0));
    if (!tfg::attention_backward_layout_ok(heads, channels))
        return fail(TFG_ERR_INVALID_ARG,
                    "%s: channels must be a power of two up to 32 or a multiple of 32, H*C <= 256",
                    fn);
    *bytes = tfg::attention_backward_workspace_bytes(num_nodes, heads, channels);
    return ok();
}

int tfg_edge_softmax_aggregate_backward(const int32_t *rowptr, const int32_t *col,
                                        const int32_t *rowptr_src, const int32_t *col_src,
                                        const void *x, int x_dtype, int64_t num_nodes,
                                        int64_t num_edges, int heads, int channels,
                                        const float *a_src, const float *a_dst,
                                        float negative_slope, const float *out,
                                        const float *grad_out, float *grad_x, float *grad_a_src,
                                        float *grad_a_dst, void *workspace,
                                        size_t workspace_bytes, tfg_stream_t stream) {
    const char *fn = "tfg_edge_softmax_aggregate_backward";
    TFG_RANGE(fn);
    TFG_TRY(check_counts(fn, num_nodes, num_edges));
    if (!tfg::attention_backward_layout_ok(heads, channels))
        return fail(TFG_ERR_INVALID_ARG,
                    "%s: channels must be a power of two up to 32 or a multiple of 32, H*C <= 256",
                    fn);
    TFG_TRY(check_features(fn, num_nodes, int64_t(heads) * channels));
    TFG_TRY(check_dtype(fn, x_dtype));
    TFG_NEED(rowptr, true, fn, "rowptr");
    TFG_NEED(rowptr_src, true, fn, "rowptr_src");
    TFG_NEED(col, num_edges > 0, fn, "col");
    TFG_NEED(col_src, num_edges > 0, fn, "col_src");
    TFG_NEED(x, num_nodes > 0, fn, "x");
    TFG_NEED(out, num_nodes > 0, fn, "out");
    TFG_NEED(grad_out, num_nodes > 0, fn, "grad_out");
    TFG_NEED(grad_x, num_nodes > 0, fn, "grad_x");
    TFG_NEED(a_src, true, fn, "a_src");
    TFG_NEED(a_dst, true, fn, "a_dst");
    TFG_NEED(grad_a_src, true, fn, "grad_a_src");
    TFG_NEED(grad_a_dst, true, fn, "grad_a_dst");
    const size_t need = tfg::attention_backward_workspace_bytes(num_nodes, heads, channels);
    if (workspace == nullptr || workspace_bytes < need)
        return fail(TFG_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need,
                    workspace ? workspace_bytes : size_t(0));
#if TFG_CHECK_BOUNDS
    {
        const size_t nf = size_t(num_nodes) * size_t(heads) * size_t(channels);
        TFG_DEBUG(debug_csr(fn, "col", rowptr, col, nullptr, num_nodes, num_edges, nullptr, stream));
        TFG_DEBUG(debug_csr(fn, "col_src", rowptr_src, col_src, nullptr, num_nodes, num_edges,
                            nullptr, stream));
        TFG_DEBUG(debug_extent(fn, "x", x, elem_bytes(x_dtype) * nf));
        TFG_DEBUG(debug_extent(fn, "out", out, sizeof(float) * nf));
        TFG_DEBUG(debug_extent(fn, "grad_out", grad_out, sizeof(float) * nf));
        TFG_DEBUG(debug_extent(fn, "grad_x", grad_x, sizeof(float) * nf));
        TFG_DEBUG(debug_extent(fn, "workspace", workspace, need));
    }
#endif
    return cuda_result(tfg::launch_edge_softmax_backward(
                           rowptr, col, rowptr_src, col_src, x, x_dtype, num_nodes,
                           num_edges, heads, channels, a_src, a_dst, negative_slope, out, grad_out, grad_x,
                           grad_a_src, grad_a_dst, workspace, reinterpret_cast<cudaStream_t>(stream)),
                       fn);
}

int tfg_dot_edge_softmax_backward_workspace_size(int64_t num_nodes, int heads, int channels,
                                                 size_t *bytes) {
    const char *fn = "tfg_dot_edge_softmax_backward_workspace_size";
    TFG_RANGE(fn);
    TFG_NEED(bytes, true, fn, "bytes");
    TFG_TRY(check_counts(fn, num_nodes, 0));
    if (!tfg::attention_backward_layout_ok(heads, channels))
        return fail(TFG_ERR_INVALID_ARG,
                    "%s: channels must be a power of two up to 32 or a multiple of 32, H*C <= 256",
                    fn);
    *bytes = tfg::dot_attention_backward_workspace_bytes(num_nodes, heads);
    return TFG_OK;
}

int tfg_dot_edge_softmax_aggregate_backward(const int32_t *rowptr, const int32_t *col,
                                            const int32_t *rowptr_src, const int32_t *col_src,
                                            const void *q, const void *k, const void *v,
                                            int x_dtype, int64_t num_nodes, int64_t num_edges,
                                            int heads, int channels, float scale,
                                            const float *out, const float *grad_out,
                                            float *grad_q, float *grad_k, float *grad_v,
                                            void *workspace, size_t workspace_bytes,
                                            tfg_stream_t stream) {
    const char *fn = "tfg_dot_edge_softmax_aggregate_backward";
    TFG_RANGE(fn);
    TFG_TRY(check_counts(fn, num_nodes, num_edges));
    if (!tfg::attention_backward_layout_ok(heads, channels))
        return fail(TFG_ERR_INVALID_ARG,
                    "%s: channels must be a power of two up to 32 or a multiple of 32, H*C <= 256",
                    fn);
    TFG_TRY(check_features(fn, num_nodes, int64_t(heads) * channels));
    TFG_TRY(check_dtype(fn, x_dtype));
    if (!(scale == scale) || scale == INFINITY || scale == -INFINITY)
        return fail(TFG_ERR_INVALID_ARG, "%s: scale must be finite", fn);
    TFG_NEED(rowptr, true, fn, "rowptr");
    TFG_NEED(rowptr_src, true, fn, "rowptr_src");
    TFG_NEED(col, num_edges > 0, fn, "col");
    TFG_NEED(col_src, num_edges > 0, fn, "col_src");
    TFG_NEED(q, num_nodes > 0, fn, "q");
    TFG_NEED(k, num_nodes > 0, fn, "k");
    TFG_NEED(v, num_nodes > 0, fn, "v");
    TFG_NEED(out, num_nodes > 0, fn, "out");
    TFG_NEED(grad_out, num_nodes > 0, fn, "grad_out");
    TFG_NEED(grad_q, num_nodes > 0, fn, "grad_q");
    TFG_NEED(grad_k, num_nodes > 0, fn, "grad_k");
    TFG_NEED(grad_v, num_nodes > 0, fn, "grad_v");
    const size_t need = tfg::dot_attention_backward_workspace_bytes(num_nodes, heads);
    if (workspace == nullptr || workspace_bytes < need)
        return fail(TFG_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need,
                    workspace ? workspace_bytes : size_t(0));
#if TFG_CHECK_BOUNDS
    {
        const size_t nf = size_t(num_nodes) * size_t(heads) * size_t(channels);
        TFG_DEBUG(debug_csr(fn, "col", rowptr, col, nullptr, num_nodes, num_edges, nullptr, stream));
        TFG_DEBUG(debug_csr(fn, "col_src", rowptr_src, col_src, nullptr, num_nodes, num_edges,
                            nullptr, stream));
        TFG_DEBUG(debug_extent(fn, "q", q, elem_bytes(x_dtype) * nf));
        TFG_DEBUG(debug_extent(fn, "k", k, elem_bytes(x_dtype) * nf));
        TFG_DEBUG(debug_extent(fn, "v", v, elem_bytes(x_dtype) * nf));
        TFG_DEBUG(debug_extent(fn, "out", out, sizeof(float) * nf));
        TFG_DEBUG(debug_extent(fn, "grad_out", grad_out, sizeof(float) * nf));
        TFG_DEBUG(debug_extent(fn, "grad_q", grad_q, sizeof(float) * nf));
        TFG_DEBUG(debug_extent(fn, "grad_k", grad_k, sizeof(float) * nf));
        TFG_DEBUG(debug_extent(fn, "grad_v", grad_v, sizeof(float) * nf));
        TFG_DEBUG(debug_extent(fn, "workspace", workspace, need));
    }
#endif
    return cuda_result(tfg::launch_dot_softmax_backward(
                           rowptr, col, rowptr_src, col_src, q, k, v, x_dtype, num_nodes,
                           num_edges, heads, channels, scale, out, grad_out, grad_q, grad_k,
                           grad_v, workspace, reinterpret_cast<cudaStream_t>(stream)),
                       fn);
}

int tfg_dot_edge_softmax_aggregate(const int32_t *rowptr, const int32_t *col, const void *q,
                                   const void *k, const void *v, int x_dtype, int64_t num_nodes,
                                   int64_t num_edges, int heads, int channels, float scale,
                                   float *out, float *alpha, tfg_stream_t stream) {
    const char *fn = "tfg_dot_edge_softmax_aggregate";
    TFG_RANGE(fn);
    TFG_TRY(check_counts(fn, num_nodes, num_edges));
    if (heads < 1 || channels < 1)
        return fail(TFG_ERR_INVALID_ARG, "%s: heads and channels must be >= 1", fn);
    if (channels > tfg::dot_softmax_max_channels())
        return fail(TFG_ERR_TOO_LARGE, "%s: at most %d channels per head", fn,
                    tfg::dot_softmax_max_channels());
    TFG_TRY(check_features(fn, num_nodes, int64_t(heads) * channels));
    TFG_TRY(check_dtype(fn, x_dtype));
    if (!(scale == scale) || scale == INFINITY || scale == -INFINITY)
        return fail(TFG_ERR_INVALID_ARG, "%s: scale must be finite", fn);
    TFG_NEED(rowptr, true, fn, "rowptr");
    TFG_NEED(col, num_edges > 0, fn, "col");
    TFG_NEED(q, num_nodes > 0, fn, "q");
    TFG_NEED(k, num_nodes > 0, fn, "k");
    TFG_NEED(v, num_nodes > 0, fn, "v");
    TFG_NEED(out, num_nodes > 0, fn, "out");
#if TFG_CHECK_BOUNDS
    {
        const size_t nf = size_t(num_nodes) * size_t(heads) * size_t(channels);
        TFG_DEBUG(debug_csr(fn, "col", rowptr, col, nullptr, num_nodes, num_edges, nullptr, stream));
        TFG_DEBUG(debug_extent(fn, "q", q, elem_bytes(x_dtype) * nf));
        TFG_DEBUG(debug_extent(fn, "k", k, elem_bytes(x_dtype) * nf));
        TFG_DEBUG(debug_extent(fn, "v", v, elem_bytes(x_dtype) * nf));
        TFG_DEBUG(debug_extent(fn, "out", out, sizeof(float) * nf));
        TFG_DEBUG(debug_extent(fn, "alpha", alpha, sizeof(float) * size_t(num_edges * heads)));
    }
#endif
    return cuda_result(tfg::launch_dot_softmax(rowptr, num_edges > 0 ? col : nullptr, q, k, v,
                                               x_dtype, num_nodes, num_edges, heads, channels,
                                               scale, out, alpha,
                                               reinterpret_cast<cudaStream_t>(stream)),
                       fn);
}

int tfg_edge_softmax_aggregate_noalloc(const int32_t *rowptr, const int32_t *col, const void *x,
                                       int x_dtype, int64_t num_nodes, int64_t num_edges,
                                       int heads, int channels, const float *a_src,
                                       const float *a_dst, float negative_slope, float *out,
                                       float *alpha, tfg_stream_t stream) {
    const char *fn = "tfg_edge_softmax_aggregate_noalloc";
    TFG_RANGE(fn);
    TFG_TRY(check_counts(fn, num_nodes, num_edges));
    if (heads < 1 || channels < 1)
        return fail(TFG_ERR_INVALID_ARG, "%s: heads and channels must be >= 1", fn);
    const int64_t limit = tfg::noalloc_softmax_max_node_heads();
    if (num_nodes * heads > limit)
        return fail(TFG_ERR_TOO_LARGE,
                    "%s: num_nodes * heads = %lld exceeds the built-in scratch of %lld node-head "
                    "pairs; use tfg_edge_softmax_aggregate with a caller workspace",
                    fn, (long long)(num_nodes * heads), (long long)limit);
    TFG_TRY(check_features(fn, num_nodes, int64_t(heads) * channels));
    TFG_TRY(check_dtype(fn, x_dtype));
    TFG_NEED(rowptr, true, fn, "rowptr");
    TFG_NEED(col, num_edges > 0, fn, "col");
    TFG_NEED(x, num_nodes > 0, fn, "x");
    TFG_NEED(out, num_nodes > 0, fn, "out");
    TFG_NEED(a_src, true, fn, "a_src");
    TFG_NEED(a_dst, true, fn, "a_dst");
    if (num_nodes == 0) return ok();
    TFG_DEBUG(debug_csr(fn, "col", rowptr, col, nullptr, num_nodes, num_edges, nullptr, stream));
    TFG_DEBUG(debug_extent(fn, "x", x, elem_bytes(x_dtype) * size_t(num_nodes * heads * channels)));
    TFG_DEBUG(debug_extent(fn, "out", out, sizeof(float) * size_t(num_nodes * heads * channels)));
    TFG_DEBUG(debug_extent(fn, "alpha", alpha, sizeof(float) * size_t(num_edges * heads)));
    void *scratch = nullptr;
    size_t scratch_bytes = 0;
    cudaError_t err = tfg::noalloc_softmax_scratch(&scratch, &scratch_bytes);
    if (err != cudaSuccess) return cuda_result(err, fn);
    if (tfg::softmax_workspace_bytes(num_nodes, heads) > scratch_bytes)
        return fail(TFG_ERR_TOO_LARGE, "%s: scratch too small", fn);
    return cuda_result(tfg::launch_edge_softmax(rowptr, num_edges > 0 ? col : nullptr, x, x_dtype,
                                                num_nodes, num_edges, heads, channels, a_src, a_dst,
                                                negative_slope, out, alpha, scratch,
                                                reinterpret_cast<cudaStream_t>(stream)),
                       fn);
}

int tfg_segment_pool_meanmax(const void *x, int x_dtype, const int64_t *batch,
                             int64_t num_nodes, int64_t num_graphs, int64_t num_features,
                             float *out, int32_t *status, tfg_stream_t stream) {
    const char *fn = "tfg_segment_pool_meanmax";
    TFG_RANGE(fn);
    if (num_nodes < 0 || num_graphs < 0)
        return fail(TFG_ERR_INVALID_ARG, "%s: negative size", fn);
    if (num_graphs >= kIndexLimit) return fail(TFG_ERR_TOO_LARGE, "%s: too many graphs", fn);
    TFG_TRY(check_features(fn, num_nodes > num_graphs ? num_nodes : num_graphs, num_features));
    TFG_TRY(check_dtype(fn, x_dtype));
    if (num_features > int64_t(65535) * 8)
        return fail(TFG_ERR_TOO_LARGE, "%s: at most %d features", fn, 65535 * 8);
    TFG_NEED(x, num_nodes > 0, fn, "x");
    TFG_NEED(batch, num_nodes > 0, fn, "batch");
    TFG_NEED(out, num_graphs > 0, fn, "out");
    TFG_NEED(status, true, fn, "status");
    TFG_DEBUG(debug_extent(fn, "x", x, elem_bytes(x_dtype) * size_t(num_nodes * num_features)));
    TFG_DEBUG(debug_extent(fn, "batch", batch, sizeof(int64_t) * size_t(num_nodes)));
    TFG_DEBUG(debug_extent(fn, "out", out, sizeof(float) * 2 * size_t(num_graphs * num_features)));
    return cuda_result(tfg::launch_segment_pool(x, x_dtype, batch, num_nodes, num_graphs,
                                                num_features, 3 /* mean | max */, out, status,
                                                reinterpret_cast<cudaStream_t>(stream)),
                       fn);
}

int tfg_batch_graphs_workspace_size(int64_t num_graphs, size_t *bytes) {
    const char *fn = "tfg_batch_graphs_workspace_size";
    TFG_RANGE(fn);
    if (num_graphs < 0) return fail(TFG_ERR_INVALID_ARG, "%s: negative size", fn);
    TFG_NEED(bytes, true, fn, "bytes");
    *bytes = tfg::batch_graphs_workspace_bytes(num_graphs);
    return ok();
}

int tfg_batch_graphs(int64_t num_graphs, const int64_t *node_counts, const int64_t *edge_counts,
                     const int64_t *edge_index, int64_t total_edges, int64_t total_nodes,
                     int64_t *out_edge_index, int64_t *batch, int64_t *node_offsets,
                     void *workspace, size_t workspace_bytes, int32_t *status,
                     tfg_stream_t stream) {
    const char *fn = "tfg_batch_graphs";
    TFG_RANGE(fn);
    TFG_TRY(check_counts(fn, total_nodes, total_edges));
    if (num_graphs < 0) return fail(TFG_ERR_INVALID_ARG, "%s: negative graph count", fn);
    if (num_graphs >= kIndexLimit) return fail(TFG_ERR_TOO_LARGE, "%s: too many graphs", fn);
    if (num_graphs == 0 && (total_nodes > 0 || total_edges > 0))
        return fail(TFG_ERR_INVALID_ARG, "%s: nodes or edges given for zero graphs", fn);
    TFG_NEED(node_counts, num_graphs > 0, fn, "node_counts");
    TFG_NEED(edge_counts, num_graphs > 0, fn, "edge_counts");
    TFG_NEED(edge_index, total_edges > 0, fn, "edge_index");
    TFG_NEED(out_edge_index, total_edges > 0, fn, "out_edge_index");
    TFG_NEED(batch, total_nodes > 0, fn, "batch");
    TFG_NEED(node_offsets, true, fn, "node_offsets");
    TFG_NEED(status, true, fn, "status");
    const size_t need = tfg::batch_graphs_workspace_bytes(num_graphs);
    if (workspace == nullptr || workspace_bytes < need)
        return fail(TFG_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need,
                    workspace ? workspace_bytes : size_t(0));
    TFG_DEBUG(debug_extent(fn, "node_counts", node_counts, sizeof(int64_t) * size_t(num_graphs)));
    TFG_DEBUG(debug_extent(fn, "edge_counts", edge_counts, sizeof(int64_t) * size_t(num_graphs)));
    TFG_DEBUG(debug_extent(fn, "edge_index", edge_index, sizeof(int64_t) * 2 * size_t(total_edges)));
    TFG_DEBUG(debug_extent(fn, "out_edge_index", out_edge_index,
                           sizeof(int64_t) * 2 * size_t(total_edges)));
    TFG_DEBUG(debug_extent(fn, "batch", batch, sizeof(int64_t) * size_t(total_nodes)));
    TFG_DEBUG(debug_extent(fn, "node_offsets", node_offsets, sizeof(int64_t) * size_t(num_graphs + 1)));
    return cuda_result(tfg::launch_batch_graphs(num_graphs, node_counts, edge_counts, edge_index,
                                                total_edges, total_nodes, out_edge_index, batch,
                                                node_offsets, workspace, status,
                                                reinterpret_cast<cudaStream_t>(stream)),
                       fn);
}

int tfg_segment_pool(const void *x, int x_dtype, const int64_t *batch, int64_t num_nodes,
                     int64_t num_graphs, int64_t num_features, int reduce, float *out,
                     int32_t *status, tfg_stream_t stream) {
    const char *fn = "tfg_segment_pool";
    TFG_RANGE(fn);
    if (num_nodes < 0 || num_graphs < 0)
        return fail(TFG_ERR_INVALID_ARG, "%s: negative size", fn);
    if (num_graphs >= kIndexLimit) return fail(TFG_ERR_TOO_LARGE, "%s: too many graphs", fn);
    TFG_TRY(check_features(fn, num_nodes > num_graphs ? num_nodes : num_graphs, num_features));
    TFG_TRY(check_dtype(fn, x_dtype));
    if (num_features > int64_t(65535) * 8)
        return fail(TFG_ERR_TOO_LARGE, "%s: at most %d features", fn, 65535 * 8);
    if (reduce != TFG_SUM && reduce != TFG_MEAN && reduce != TFG_MAX)
        return fail(TFG_ERR_INVALID_ARG, "%s: unknown reducer %d", fn, reduce);
    TFG_NEED(x, num_nodes > 0, fn, "x");
    TFG_NEED(batch, num_nodes > 0, fn, "batch");
    TFG_NEED(out, num_graphs > 0, fn, "out");
    TFG_NEED(status, true, fn, "status");
    TFG_DEBUG(debug_extent(fn, "x", x, elem_bytes(x_dtype) * size_t(num_nodes * num_features)));
    TFG_DEBUG(debug_extent(fn, "batch", batch, sizeof(int64_t) * size_t(num_nodes)));
    TFG_DEBUG(debug_extent(fn, "out", out, sizeof(float) * size_t(num_graphs * num_features)));
    return cuda_result(tfg::launch_segment_pool(x, x_dtype, batch, num_nodes, num_graphs,
                                                num_features, reduce, out, status,
                                                reinterpret_cast<cudaStream_t>(stream)),
                       fn);
}

// ---- embedding lookup and its gradient --------------------------------------------
namespace {
constexpr int64_t kMaxEmbeddingFeatures = int64_t(65535) * 128;

int check_embedding(const char *fn, int64_t num_ids, int64_t num_rows, int64_t num_features) {
    if (num_ids < 0 || num_rows < 0)
        return fail(TFG_ERR_INVALID_ARG, "%s: negative size (ids=%lld, rows=%lld)", fn, (long long)num_ids, (long long)num_rows);
    if (num_ids >= kIndexLimit - 1 || num_rows >= kIndexLimit - 1)
        return fail(TFG_ERR_TOO_LARGE, "%s: ids and rows must be < 2^31 - 1 (ids=%lld, rows=%lld)", fn, (long long)num_ids,
                    (long long)num_rows);
    if (num_features < 1) return fail(TFG_ERR_INVALID_ARG, "%s: feature count must be positive", fn);
    if (num_features > kMaxEmbeddingFeatures)
        return fail(TFG_ERR_TOO_LARGE, "%s: at most %lld features", fn, (long long)kMaxEmbeddingFeatures);
    if ((num_ids > num_rows ? num_ids : num_rows) * num_features >= (int64_t(1) << 46))
        return fail(TFG_ERR_TOO_LARGE, "%s: rows * features too large", fn);
    return TFG_OK;
}

int lookup_common(const char *fn, const void *ids, bool id32, int64_t num_ids, const void *table, int table_dtype,
                  int64_t num_rows, int64_t num_features, float scale, int64_t padding_id, void *out, int out_dtype,
                  int32_t *status, tfg_stream_t stream) {
    TFG_RANGE(fn);
    TFG_TRY(check_embedding(fn, num_ids, num_rows, num_features));
    TFG_TRY(check_dtype(fn, table_dtype));
    TFG_TRY(check_dtype(fn, out_dtype));
    TFG_NEED(ids, num_ids > 0, fn, "ids");
    TFG_NEED(table, num_rows > 0, fn, "table");
    TFG_NEED(out, num_ids > 0, fn, "out");
    TFG_NEED(status, true, fn, "status");
    TFG_TRY(check_element(fn, "table", table, table_dtype));
    TFG_TRY(check_element(fn, "out", out, out_dtype));
    const size_t id_bytes = (id32 ? sizeof(int32_t) : sizeof(int64_t)) * size_t(num_ids);
    const size_t table_bytes = elem_bytes(table_dtype) * size_t(num_rows * num_features);
    const size_t out_bytes = elem_bytes(out_dtype) * size_t(num_ids * num_features);
    if (overlap(out, out_bytes, table, table_bytes) || overlap(out, out_bytes, ids, id_bytes))
        return fail(TFG_ERR_INVALID_ARG, "%s: out overlaps an input", fn);
    TFG_DEBUG(debug_extent(fn, "ids", ids, id_bytes));
    TFG_DEBUG(debug_extent(fn, "table", table, table_bytes));
    TFG_DEBUG(debug_extent(fn, "out", out, out_bytes));
    return cuda_result(tfg::launch_embedding_lookup(ids, id32, num_ids, table, table_dtype, num_rows, num_features, scale,
                                                    padding_id, out, out_dtype, status,
                                                    reinterpret_cast<cudaStream_t>(stream)),
                       fn);
}

int group_ids_common(const char *fn, const void *ids, bool id32, int64_t num_ids, int64_t num_rows, int64_t padding_id,
                     int32_t *rowptr, int32_t *sorted_ids, int32_t *perm, void *workspace, size_t workspace_bytes,
                     int32_t *status, tfg_stream_t stream) {
    TFG_RANGE(fn);
    TFG_TRY(check_embedding(fn, num_ids, num_rows, 1));
    TFG_NEED(ids, num_ids > 0, fn, "ids");
    TFG_NEED(rowptr, true, fn, "rowptr");
    TFG_NEED(sorted_ids, num_ids > 0, fn, "sorted_ids");
    TFG_NEED(perm, num_ids > 0, fn, "perm");
    TFG_NEED(status, true, fn, "status");
    if (num_ids > 0)
        TFG_TRY(check_workspace(fn, workspace, workspace_bytes, tfg::group_ids_workspace_bytes(num_rows, num_ids), 256));
    TFG_DEBUG(debug_extent(fn, "ids", ids, (id32 ? sizeof(int32_t) : sizeof(int64_t)) * size_t(num_ids)));
    TFG_DEBUG(debug_extent(fn, "rowptr", rowptr, sizeof(int32_t) * size_t(num_rows + 1)));
    TFG_DEBUG(debug_extent(fn, "sorted_ids", sorted_ids, sizeof(int32_t) * size_t(num_ids)));
    TFG_DEBUG(debug_extent(fn, "perm", perm, sizeof(int32_t) * size_t(num_ids)));
    return cuda_result(tfg::launch_group_ids(ids, id32, num_ids, num_rows, padding_id, rowptr, sorted_ids, perm, workspace,
                                             status, reinterpret_cast<cudaStream_t>(stream)),
                       fn);
}
}  // namespace

int tfg_embedding_lookup(const int64_t *ids, int64_t num_ids, const void *table, int table_dtype, int64_t num_rows,
                         int64_t num_features, float scale, int64_t padding_id, void *out, int out_dtype,
                         int32_t *status, tfg_stream_t stream) {
    return lookup_common("tfg_embedding_lookup", ids, false, num_ids, table, table_dtype, num_rows, num_features, scale,
                         padding_id, out, out_dtype, status, stream);
}

int tfg_embedding_lookup32(const int32_t *ids, int64_t num_ids, const void *table, int table_dtype, int64_t num_rows,
                           int64_t num_features, float scale, int64_t padding_id, void *out, int out_dtype,
                           int32_t *status, tfg_stream_t stream) {
    return lookup_common("tfg_embedding_lookup32", ids, true, num_ids, table, table_dtype, num_rows, num_features, scale,
                         padding_id, out, out_dtype, status, stream);
}

int tfg_group_ids_workspace_size(int64_t num_rows, int64_t num_ids, size_t *bytes) {
    const char *fn = "tfg_group_ids_workspace_size";
    TFG_RANGE(fn);
    TFG_TRY(check_embedding(fn, num_ids, num_rows, 1));
    TFG_NEED(bytes, true, fn, "bytes");
    *bytes = tfg::group_ids_workspace_bytes(num_rows, num_ids);
    return ok();
}

int tfg_group_ids(const int64_t *ids, int64_t num_ids, int64_t num_rows, int64_t padding_id, int32_t *rowptr,
                  int32_t *sorted_ids, int32_t *perm, void *workspace, size_t workspace_bytes, int32_t *status,
                  tfg_stream_t stream) {
    return group_ids_common("tfg_group_ids", ids, false, num_ids, num_rows, padding_id, rowptr, sorted_ids, perm, workspace,
                            workspace_bytes, status, stream);
}

int tfg_group_ids32(const int32_t *ids, int64_t num_ids, int64_t num_rows, int64_t padding_id, int32_t *rowptr,
                    int32_t *sorted_ids, int32_t *perm, void *workspace, size_t workspace_bytes, int32_t *status,
                    tfg_stream_t stream) {
    return group_ids_common("tfg_group_ids32", ids, true, num_ids, num_rows, padding_id, rowptr, sorted_ids, perm, workspace,
                            workspace_bytes, status, stream);
}

int tfg_embedding_backward_workspace_size(int64_t num_features, size_t *bytes) {
    const char *fn = "tfg_embedding_backward_workspace_size";
    TFG_RANGE(fn);
    TFG_TRY(check_embedding(fn, 0, 0, num_features));
    TFG_NEED(bytes, true, fn, "bytes");
    *bytes = tfg::embedding_backward_workspace_bytes(num_features);
    return ok();
}

int tfg_embedding_backward(const int32_t *rowptr, const int32_t *sorted_ids, const int32_t *perm, const void *grad_out,
                           int grad_dtype, int64_t num_ids, int64_t num_rows, int64_t num_features, float scale,
                           float *grad_table, void *workspace, size_t workspace_bytes, tfg_stream_t stream) {
    const char *fn = "tfg_embedding_backward";
    TFG_RANGE(fn);
    TFG_TRY(check_embedding(fn, num_ids, num_rows, num_features));
    TFG_TRY(check_dtype(fn, grad_dtype));
    TFG_NEED(rowptr, true, fn, "rowptr");
    TFG_NEED(sorted_ids, num_ids > 0, fn, "sorted_ids");
    TFG_NEED(perm, num_ids > 0, fn, "perm");
    TFG_NEED(grad_out, num_ids > 0, fn, "grad_out");
    TFG_NEED(grad_table, num_rows > 0, fn, "grad_table");
    TFG_TRY(check_element(fn, "grad_out", grad_out, grad_dtype));
    TFG_TRY(check_element(fn, "grad_table", grad_table, TFG_F32));
    const size_t grad_bytes = elem_bytes(grad_dtype) * size_t(num_ids * num_features);
    const size_t table_bytes = sizeof(float) * size_t(num_rows * num_features);
    if (overlap(grad_table, table_bytes, grad_out, grad_bytes))
        return fail(TFG_ERR_INVALID_ARG, "%s: grad_table overlaps grad_out", fn);
    TFG_TRY(check_workspace(fn, workspace, workspace_bytes, tfg::embedding_backward_workspace_bytes(num_features), 16));
    TFG_DEBUG(debug_extent(fn, "rowptr", rowptr, sizeof(int32_t) * size_t(num_rows + 1)));
    TFG_DEBUG(debug_extent(fn, "sorted_ids", sorted_ids, sizeof(int32_t) * size_t(num_ids)));
    TFG_DEBUG(debug_extent(fn, "perm", perm, sizeof(int32_t) * size_t(num_ids)));
    TFG_DEBUG(debug_extent(fn, "grad_out", grad_out, grad_bytes));
    TFG_DEBUG(debug_extent(fn, "grad_table", grad_table, table_bytes));
    TFG_DEBUG(debug_extent(fn, "workspace", workspace, tfg::embedding_backward_workspace_bytes(num_features)));
    if (num_rows == 0) return ok();
    return cuda_result(tfg::launch_embedding_backward(rowptr, sorted_ids, perm, grad_out, grad_dtype, num_ids, num_rows,
                                                      num_features, scale, grad_table, workspace,
                                                      reinterpret_cast<cudaStream_t>(stream)),
                       fn);
}

// ---- group norm -------------------------------------------------------------------
namespace {
constexpr int64_t kMaxGroupChannels = 1024;       // a row of a group, value by value, in a team of at most 1,024 threads

int check_group_norm(const char *fn, int64_t num_nodes, int64_t num_graphs, int64_t num_features, int64_t num_groups) {
    TFG_TRY(check_counts(fn, num_nodes, 0));
    if (num_graphs < 0) return fail(TFG_ERR_INVALID_ARG, "%s: negative graph count", fn);
    if (num_graphs >= kIndexLimit) return fail(TFG_ERR_TOO_LARGE, "%s: too many graphs", fn);
    TFG_TRY(check_features(fn, num_nodes > num_graphs ? num_nodes : num_graphs, num_features));
    if (num_groups < 1 || num_features % num_groups != 0)
        return fail(TFG_ERR_INVALID_ARG, "%s: num_groups (%lld) must divide num_features (%lld)", fn, (long long)num_groups,
                    (long long)num_features);
    if (num_features / num_groups > kMaxGroupChannels)
        return fail(TFG_ERR_TOO_LARGE, "%s: at most %lld channels per group", fn, (long long)kMaxGroupChannels);
    // no more teams than graphs and rows, no more tiles than channels: most calls need no plan
    if ((num_nodes + num_graphs + 2) * num_features > int64_t(0x7f000000) &&
        !tfg::group_norm_fits(num_nodes, num_graphs, num_features, num_groups))
        return fail(TFG_ERR_TOO_LARGE, "%s: graphs * features too large", fn);
    return TFG_OK;
}

int check_activation(const char *fn, int activation) {
    if (activation < TFG_ACT_NONE || activation > TFG_ACT_GELU)
        return fail(TFG_ERR_INVALID_ARG, "%s: unknown activation %d", fn, activation);
    return TFG_OK;
}
}  // namespace

int tfg_group_norm_workspace_size(int64_t num_nodes, int64_t num_graphs, int64_t num_features, int64_t num_groups,
                                  size_t *bytes) {
    const char *fn = "tfg_group_norm_workspace_size";
    TFG_RANGE(fn);
    TFG_TRY(check_group_norm(fn, num_nodes, num_graphs, num_features, num_groups));
    TFG_NEED(bytes, true, fn, "bytes");
    *bytes = tfg::group_norm_workspace_bytes(num_nodes, num_graphs, num_features, num_groups);
    return ok();
}

int tfg_group_norm(const void *x, int x_dtype, const int64_t *node_offsets, int64_t num_nodes, int64_t num_graphs,
                   int64_t num_features, int64_t num_groups, const float *gamma, const float *beta, float eps,
                   int activation, void *out, int out_dtype, float *mean, float *rstd, void *workspace,
                   size_t workspace_bytes, int32_t *status, tfg_stream_t stream) {
    const char *fn = "tfg_group_norm";
    TFG_RANGE(fn);
    TFG_TRY(check_group_norm(fn, num_nodes, num_graphs, num_features, num_groups));
    TFG_TRY(check_dtype(fn, x_dtype));
    TFG_TRY(check_dtype(fn, out_dtype));
    TFG_TRY(check_activation(fn, activation));
    if (!(eps > 0.f) || !std::isfinite(eps)) return fail(TFG_ERR_INVALID_ARG, "%s: eps must be finite and positive", fn);
    TFG_NEED(x, num_nodes > 0, fn, "x");
    TFG_NEED(out, num_nodes > 0, fn, "out");
    TFG_NEED(node_offsets, num_graphs > 0, fn, "node_offsets");
    TFG_NEED(status, true, fn, "status");
    if ((mean == nullptr) != (rstd == nullptr))
        return fail(TFG_ERR_INVALID_ARG, "%s: mean and rstd are wanted both or neither", fn);
    TFG_TRY(check_element(fn, "x", x, x_dtype));
    TFG_TRY(check_element(fn, "out", out, out_dtype));
    const size_t x_bytes = elem_bytes(x_dtype) * size_t(num_nodes * num_features);
    const size_t out_bytes = elem_bytes(out_dtype) * size_t(num_nodes * num_features);
    if (overlap(out, out_bytes, x, x_bytes)) return fail(TFG_ERR_INVALID_ARG, "%s: out overlaps x", fn);
    const size_t need = tfg::group_norm_workspace_bytes(num_nodes, num_graphs, num_features, num_groups);
    TFG_TRY(check_workspace(fn, workspace, workspace_bytes, need, 16));
    TFG_DEBUG(debug_extent(fn, "x", x, x_bytes));
    TFG_DEBUG(debug_extent(fn, "out", out, out_bytes));
    TFG_DEBUG(debug_extent(fn, "node_offsets", node_offsets, sizeof(int64_t) * size_t(num_graphs + 1)));
    TFG_DEBUG(debug_extent(fn, "gamma", gamma, sizeof(float) * size_t(num_features)));
    TFG_DEBUG(debug_extent(fn, "beta", beta, sizeof(float) * size_t(num_features)));
    TFG_DEBUG(debug_extent(fn, "mean", mean, sizeof(float) * size_t(num_graphs * num_groups)));
    TFG_DEBUG(debug_extent(fn, "rstd", rstd, sizeof(float) * size_t(num_graphs * num_groups)));
    TFG_DEBUG(debug_extent(fn, "workspace", workspace, need));
    return cuda_result(tfg::launch_group_norm(x, x_dtype, node_offsets, num_nodes, num_graphs, num_features, num_groups,
                                              gamma, beta, eps, activation, out, out_dtype, mean, rstd, workspace, status,
                                              reinterpret_cast<cudaStream_t>(stream)),
                       fn);
}

int tfg_group_norm_backward_workspace_size(int64_t num_nodes, int64_t num_graphs, int64_t num_features, int64_t num_groups,
                                           size_t *bytes) {
    const char *fn = "tfg_group_norm_backward_workspace_size";
    TFG_RANGE(fn);
    TFG_TRY(check_group_norm(fn, num_nodes, num_graphs, num_features, num_groups));
    TFG_NEED(bytes, true, fn, "bytes");
    *bytes = tfg::group_norm_backward_workspace_bytes(num_nodes, num_graphs, num_features, num_groups);
    return ok();
}

int tfg_group_norm_backward(const void *x, int x_dtype, const int64_t *node_offsets, int64_t num_nodes,
                            int64_t num_graphs, int64_t num_features, int64_t num_groups, const float *gamma,
                            const float *beta, const float *mean, const float *rstd, int activation, const void *grad_out,
                            int grad_dtype, void *grad_x, float *grad_gamma, float *grad_beta, void *workspace,
                            size_t workspace_bytes, tfg_stream_t stream) {
    const char *fn = "tfg_group_norm_backward";
    TFG_RANGE(fn);
    TFG_TRY(check_group_norm(fn, num_nodes, num_graphs, num_features, num_groups));
    TFG_TRY(check_dtype(fn, x_dtype));
    TFG_TRY(check_dtype(fn, grad_dtype));
    TFG_TRY(check_activation(fn, activation));
    TFG_NEED(x, num_nodes > 0, fn, "x");
    TFG_NEED(grad_out, num_nodes > 0, fn, "grad_out");
    TFG_NEED(grad_x, num_nodes > 0, fn, "grad_x");
    TFG_NEED(node_offsets, num_graphs > 0, fn, "node_offsets");
    TFG_NEED(mean, num_graphs > 0, fn, "mean");
    TFG_NEED(rstd, num_graphs > 0, fn, "rstd");
    if ((grad_gamma == nullptr) != (grad_beta == nullptr))
        return fail(TFG_ERR_INVALID_ARG, "%s: grad_gamma and grad_beta are wanted both or neither", fn);
    TFG_TRY(check_element(fn, "x", x, x_dtype));
    TFG_TRY(check_element(fn, "grad_out", grad_out, grad_dtype));
    TFG_TRY(check_element(fn, "grad_x", grad_x, grad_dtype));
    const size_t x_bytes = elem_bytes(x_dtype) * size_t(num_nodes * num_features);
    const size_t g_bytes = elem_bytes(grad_dtype) * size_t(num_nodes * num_features);
    if (overlap(grad_x, g_bytes, x, x_bytes) || overlap(grad_x, g_bytes, grad_out, g_bytes))
        return fail(TFG_ERR_INVALID_ARG, "%s: grad_x overlaps an input", fn);
    const size_t need = tfg::group_norm_backward_workspace_bytes(num_nodes, num_graphs, num_features, num_groups);
    TFG_TRY(check_workspace(fn, workspace, workspace_bytes, need, 16));
    TFG_DEBUG(debug_extent(fn, "x", x, x_bytes));
    TFG_DEBUG(debug_extent(fn, "grad_out", grad_out, g_bytes));
    TFG_DEBUG(debug_extent(fn, "grad_x", grad_x, g_bytes));
    TFG_DEBUG(debug_extent(fn, "node_offsets", node_offsets, sizeof(int64_t) * size_t(num_graphs + 1)));
    TFG_DEBUG(debug_extent(fn, "gamma", gamma, sizeof(float) * size_t(num_features)));
    TFG_DEBUG(debug_extent(fn, "beta", beta, sizeof(float) * size_t(num_features)));
    TFG_DEBUG(debug_extent(fn, "mean", mean, sizeof(float) * size_t(num_graphs * num_groups)));
    TFG_DEBUG(debug_extent(fn, "rstd", rstd, sizeof(float) * size_t(num_graphs * num_groups)));
    TFG_DEBUG(debug_extent(fn, "grad_gamma", grad_gamma, sizeof(float) * size_t(num_features)));
    TFG_DEBUG(debug_extent(fn, "grad_beta", grad_beta, sizeof(float) * size_t(num_features)));
    TFG_DEBUG(debug_extent(fn, "workspace", workspace, need));
    return cuda_result(tfg::launch_group_norm_backward(x, x_dtype, node_offsets, num_nodes, num_graphs, num_features,
                                                       num_groups, gamma, beta, mean, rstd, activation, grad_out, grad_dtype,
                                                       grad_x, grad_gamma, grad_beta, workspace,
                                                       reinterpret_cast<cudaStream_t>(stream)),
                       fn);
}

// ---- layer norm of rows ---------------------------------------------------------------
namespace {
int check_rows(const char *fn, int64_t num_rows, int64_t num_features) {
    TFG_TRY(check_counts(fn, num_rows, 0));
    return check_features(fn, num_rows, num_features);
}
int check_eps(const char *fn, float eps) {
    if (!(eps > 0.f) || !std::isfinite(eps)) return fail(TFG_ERR_INVALID_ARG, "%s: eps must be finite and positive", fn);
    return TFG_OK;
}

// An array of rows that may begin further apart than they are long.
struct Rows {
    const char *name;
    const void *p;
    size_t stride, width, extent;        // bytes; extent: from the first byte to the last
    Rows(const char *nm, const void *ptr, int64_t n, int64_t ld, int64_t f, size_t elem)
        : name(nm), p(ptr), stride(size_t(ld) * elem), width(size_t(f) * elem),
          extent(n > 0 ? size_t(n - 1) * size_t(ld) * elem + size_t(f) * elem : 0) {}
};

// Whether rows of a and b share a byte; columns side by side in rows of one buffer do not.
bool rows_overlap(const Rows &a, const Rows &b) {
    if (a.p == nullptr || b.p == nullptr || !overlap(a.p, a.extent, b.p, b.extent)) return false;
    if (a.stride != b.stride) return true;
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a.p), pb = reinterpret_cast<uintptr_t>(b.p);
    const Rows &low = pa <= pb ? a : b, &high = pa <= pb ? b : a;
    const size_t off = (pa <= pb ? pb - pa : pa - pb) % a.stride;
    return !(off >= low.width && off + high.width <= a.stride);
}

// Every output against every input and every later output.
int check_apart(const char *fn, const Rows *outs, int num_outs, const Rows *ins, int num_ins) {
    for (int i = 0; i < num_outs; ++i) {
        for (int j = 0; j < num_ins; ++j)
            if (rows_overlap(outs[i], ins[j]))
                return fail(TFG_ERR_INVALID_ARG, "%s: %s overlaps %s", fn, outs[i].name, ins[j].name);
        for (int j = i + 1; j < num_outs; ++j)
            if (rows_overlap(outs[i], outs[j]))
                return fail(TFG_ERR_INVALID_ARG, "%s: %s overlaps %s", fn, outs[i].name, outs[j].name);
    }
    return TFG_OK;
}
}  // namespace

int tfg_layer_norm(const void *x, int x_dtype, const void *residual, int sum_dtype, void *sum, int64_t num_rows,
                   int64_t num_features, const float *gamma, const float *beta, float eps, void *out, int out_dtype,
                   float *mean, float *rstd, tfg_stream_t stream) {
    const char *fn = "tfg_layer_norm";
    TFG_RANGE(fn);
    TFG_TRY(check_rows(fn, num_rows, num_features));
    TFG_TRY(check_dtype(fn, x_dtype));
    TFG_TRY(check_dtype(fn, out_dtype));
    if (residual) TFG_TRY(check_dtype(fn, sum_dtype));
    TFG_TRY(check_eps(fn, eps));
    TFG_NEED(x, num_rows > 0, fn, "x");
    TFG_NEED(out, num_rows > 0, fn, "out");
    if (num_rows > 0 && (residual == nullptr) != (sum == nullptr))
        return fail(TFG_ERR_INVALID_ARG, "%s: residual and sum are given both or neither", fn);
    if ((mean == nullptr) != (rstd == nullptr))
        return fail(TFG_ERR_INVALID_ARG, "%s: mean and rstd are wanted both or neither", fn);
    const size_t values = size_t(num_rows * num_features);
    const size_t x_bytes = elem_bytes(x_dtype) * values, out_bytes = elem_bytes(out_dtype) * values;
    const size_t sum_bytes = residual ? elem_bytes(sum_dtype) * values : 0, w_bytes = sizeof(float) * size_t(num_features);
    TFG_TRY(check_element(fn, "x", x, x_dtype));
    TFG_TRY(check_element(fn, "out", out, out_dtype));
    if (residual) {
        TFG_TRY(check_element(fn, "residual", residual, sum_dtype));
        TFG_TRY(check_element(fn, "sum", sum, sum_dtype));
    }
    const int64_t n = num_rows, f = num_features;
    const size_t sum_elem = residual ? elem_bytes(sum_dtype) : 0;
    const Rows ins[] = {{"x", x, n, f, f, elem_bytes(x_dtype)}, {"residual", sum == residual ? nullptr : residual, n, f, f, sum_elem},
                        {"gamma", gamma, 1, f, f, 4}, {"beta", beta, 1, f, f, 4}};
    const Rows outs[] = {{"out", out, n, f, f, elem_bytes(out_dtype)}, {"sum", residual ? sum : nullptr, n, f, f, sum_elem},
                         {"mean", mean, 1, n, n, 4}, {"rstd", rstd, 1, n, n, 4}};
    TFG_TRY(check_apart(fn, outs, 4, ins, 4));
    TFG_DEBUG(debug_extent(fn, "x", x, x_bytes));
    TFG_DEBUG(debug_extent(fn, "residual", residual, sum_bytes));
    TFG_DEBUG(debug_extent(fn, "sum", sum, sum_bytes));
    TFG_DEBUG(debug_extent(fn, "out", out, out_bytes));
    TFG_DEBUG(debug_extent(fn, "gamma", gamma, w_bytes));
    TFG_DEBUG(debug_extent(fn, "beta", beta, w_bytes));
    TFG_DEBUG(debug_extent(fn, "mean", mean, sizeof(float) * size_t(num_rows)));
    TFG_DEBUG(debug_extent(fn, "rstd", rstd, sizeof(float) * size_t(num_rows)));
    return cuda_result(tfg::launch_layer_norm(x, x_dtype, residual, sum_dtype, sum, num_rows, num_features, gamma, beta, eps,
                                              out, out_dtype, mean, rstd, reinterpret_cast<cudaStream_t>(stream)),
                       fn);
}

int tfg_layer_norm_backward_workspace_size(int64_t num_rows, int64_t num_features, size_t *bytes) {
    const char *fn = "tfg_layer_norm_backward_workspace_size";
    TFG_RANGE(fn);
    TFG_TRY(check_rows(fn, num_rows, num_features));
    TFG_NEED(bytes, true, fn, "bytes");
    *bytes = tfg::layer_norm_backward_workspace_bytes(num_rows, num_features);
    return ok();
}

int tfg_layer_norm_backward(const void *sum, int sum_dtype, int64_t num_rows, int64_t num_features, const float *gamma,
                            const float *mean, const float *rstd, const void *grad_out, int grad_dtype, const void *grad_sum,
                            void *grad_s, int grad_sum_dtype, float *grad_gamma, float *grad_beta, void *workspace,
                            size_t workspace_bytes, tfg_stream_t stream) {
    const char *fn = "tfg_layer_norm_backward";
    TFG_RANGE(fn);
    TFG_TRY(check_rows(fn, num_rows, num_features));
    TFG_TRY(check_dtype(fn, sum_dtype));
    TFG_TRY(check_dtype(fn, grad_dtype));
    TFG_TRY(check_dtype(fn, grad_sum_dtype));
    TFG_NEED(sum, num_rows > 0, fn, "sum");
    TFG_NEED(mean, num_rows > 0, fn, "mean");
    TFG_NEED(rstd, num_rows > 0, fn, "rstd");
    TFG_NEED(grad_out, num_rows > 0, fn, "grad_out");
    TFG_NEED(grad_s, num_rows > 0, fn, "grad_s");
    if ((grad_gamma == nullptr) != (grad_beta == nullptr))
        return fail(TFG_ERR_INVALID_ARG, "%s: grad_gamma and grad_beta are wanted both or neither", fn);
    const size_t values = size_t(num_rows * num_features);
    const size_t s_bytes = elem_bytes(sum_dtype) * values, g_bytes = elem_bytes(grad_dtype) * values;
    const size_t gs_bytes = elem_bytes(grad_sum_dtype) * values, w_bytes = sizeof(float) * size_t(num_features);
    TFG_TRY(check_element(fn, "sum", sum, sum_dtype));
    TFG_TRY(check_element(fn, "grad_out", grad_out, grad_dtype));
    TFG_TRY(check_element(fn, "grad_sum", grad_sum, grad_sum_dtype));
    TFG_TRY(check_element(fn, "grad_s", grad_s, grad_sum_dtype));
    const int64_t n = num_rows, f = num_features;
    const size_t gs_elem = elem_bytes(grad_sum_dtype);
    const Rows ins[] = {{"sum", sum, n, f, f, elem_bytes(sum_dtype)}, {"grad_out", grad_out, n, f, f, elem_bytes(grad_dtype)},
                        {"grad_sum", grad_sum == grad_s ? nullptr : grad_sum, n, f, f, gs_elem}, {"gamma", gamma, 1, f, f, 4},
                        {"mean", mean, 1, n, n, 4}, {"rstd", rstd, 1, n, n, 4}};
    const Rows outs[] = {{"grad_s", grad_s, n, f, f, gs_elem}, {"grad_gamma", grad_gamma, 1, f, f, 4},
                         {"grad_beta", grad_beta, 1, f, f, 4}};
    TFG_TRY(check_apart(fn, outs, 3, ins, 6));
    const size_t need = grad_gamma ? tfg::layer_norm_backward_workspace_bytes(num_rows, num_features) : 0;
    TFG_TRY(check_workspace(fn, workspace, workspace_bytes, need, 16));
    TFG_DEBUG(debug_extent(fn, "sum", sum, s_bytes));
    TFG_DEBUG(debug_extent(fn, "grad_out", grad_out, g_bytes));
    TFG_DEBUG(debug_extent(fn, "grad_sum", grad_sum, gs_bytes));
    TFG_DEBUG(debug_extent(fn, "grad_s", grad_s, gs_bytes));
    TFG_DEBUG(debug_extent(fn, "gamma", gamma, w_bytes));
    TFG_DEBUG(debug_extent(fn, "mean", mean, sizeof(float) * size_t(num_rows)));
    TFG_DEBUG(debug_extent(fn, "rstd", rstd, sizeof(float) * size_t(num_rows)));
    TFG_DEBUG(debug_extent(fn, "grad_gamma", grad_gamma, w_bytes));
    TFG_DEBUG(debug_extent(fn, "grad_beta", grad_beta, w_bytes));
    TFG_DEBUG(debug_extent(fn, "workspace", workspace, need));
    return cuda_result(tfg::launch_layer_norm_backward(sum, sum_dtype, num_rows, num_features, gamma, mean, rstd, grad_out,
                                                       grad_dtype, grad_sum, grad_s, grad_sum_dtype, grad_gamma, grad_beta,
                                                       workspace, reinterpret_cast<cudaStream_t>(stream)),
                       fn);
}

// ---- gated linear recurrence ----------------------------------------------------------
namespace {
constexpr int64_t kMaxTiles = (int64_t(1) << 31) - (int64_t(1) << 16);

int check_recurrence(const char *fn, int64_t num_rows, int64_t num_sequences, int64_t num_features) {
    TFG_TRY(check_counts(fn, num_rows, 0));
    if (num_sequences < 0) return fail(TFG_ERR_INVALID_ARG, "%s: negative sequence count", fn);
    if (num_sequences >= kIndexLimit - 1) return fail(TFG_ERR_TOO_LARGE, "%s: too many sequences", fn);
    TFG_TRY(check_features(fn, num_rows > num_sequences ? num_rows : num_sequences, num_features));
    if (((num_rows + TFG_RECURRENCE_TILE_ROWS - 1) / TFG_RECURRENCE_TILE_ROWS) * ((num_features + 31) / 32) >= kMaxTiles)
        return fail(TFG_ERR_TOO_LARGE, "%s: num_rows * num_features too large", fn);
    return TFG_OK;
}

int gate_of(int gate_kind) { return gate_kind & ~TFG_GATE_ZERO_OUTSIDE; }
bool zeroes_of(int gate_kind) { return (gate_kind & TFG_GATE_ZERO_OUTSIDE) != 0; }
int check_gate(const char *fn, int gate_kind) {
    if (gate_of(gate_kind) != TFG_GATE_SIGMOID && gate_of(gate_kind) != TFG_GATE_EXP)
        return fail(TFG_ERR_INVALID_ARG, "%s: unknown gate %d", fn, gate_kind);
    return TFG_OK;
}

int check_stride(const char *fn, const char *name, int64_t num_rows, int64_t stride, int64_t num_features) {
    if (stride < num_features)
        return fail(TFG_ERR_INVALID_ARG, "%s: %s (%lld) must be at least num_features (%lld)", fn, name, (long long)stride,
                    (long long)num_features);
    if (num_rows > 0 && stride >= (int64_t(1) << 46) / num_rows)
        return fail(TFG_ERR_TOO_LARGE, "%s: %s too large", fn, name);
    return TFG_OK;
}

}  // namespace

int tfg_gated_recurrence_workspace_size(int64_t num_rows, int64_t num_features, size_t *bytes) {
    const char *fn = "tfg_gated_recurrence_workspace_size";
    TFG_RANGE(fn);
    TFG_TRY(check_recurrence(fn, num_rows, 0, num_features));
    TFG_NEED(bytes, true, fn, "bytes");
    *bytes = tfg::gated_recurrence_workspace_bytes(num_rows, num_features);
    return ok();
}

int tfg_gated_recurrence(const void *gate, int64_t gate_stride, const void *x, int64_t x_stride, int dtype,
                         const int64_t *node_offsets, int64_t num_rows, int64_t num_sequences, int64_t num_features,
                         int gate_kind, const float *initial, void *out, int out_dtype, float *final_state, float *entering,
                         void *workspace, size_t workspace_bytes, int32_t *status, tfg_stream_t stream) {
    const char *fn = "tfg_gated_recurrence";
    TFG_RANGE(fn);
    TFG_TRY(check_recurrence(fn, num_rows, num_sequences, num_features));
    TFG_TRY(check_dtype(fn, dtype));
    TFG_TRY(check_dtype(fn, out_dtype));
    TFG_TRY(check_gate(fn, gate_kind));
    TFG_TRY(check_stride(fn, "gate_stride", num_rows, gate_stride, num_features));
    TFG_TRY(check_stride(fn, "x_stride", num_rows, x_stride, num_features));
    TFG_NEED(gate, num_rows > 0, fn, "gate");
    TFG_NEED(x, num_rows > 0, fn, "x");
    TFG_NEED(out, num_rows > 0, fn, "out");
    TFG_NEED(node_offsets, num_sequences > 0, fn, "node_offsets");
    TFG_NEED(status, true, fn, "status");
    TFG_TRY(check_element(fn, "gate", gate, dtype));
    TFG_TRY(check_element(fn, "x", x, dtype));
    TFG_TRY(check_element(fn, "out", out, out_dtype));
    const int64_t n = num_rows, q = num_sequences, f = num_features;
    const int64_t tiles = (n + TFG_RECURRENCE_TILE_ROWS - 1) / TFG_RECURRENCE_TILE_ROWS;
    const Rows ins[] = {{"gate", gate, n, gate_stride, f, elem_bytes(dtype)}, {"x", x, n, x_stride, f, elem_bytes(dtype)},
                        {"initial", initial, q, f, f, 4}, {"node_offsets", node_offsets, 1, q + 1, q + 1, 8}};
    const Rows outs[] = {{"out", out, n, f, f, elem_bytes(out_dtype)}, {"final_state", final_state, q, f, f, 4},
                         {"entering", entering, tiles, f, f, 4}};
    TFG_TRY(check_apart(fn, outs, 3, ins, 4));
    const size_t need = tfg::gated_recurrence_workspace_bytes(n, f);
    TFG_TRY(check_workspace(fn, workspace, workspace_bytes, need, 16));
#if TFG_CHECK_BOUNDS
    for (const Rows &r : ins) TFG_DEBUG(debug_extent(fn, r.name, r.p, r.extent));
    for (const Rows &r : outs) TFG_DEBUG(debug_extent(fn, r.name, r.p, r.extent));
    TFG_DEBUG(debug_extent(fn, "workspace", workspace, need));
#endif
    return cuda_result(tfg::launch_gated_recurrence(gate, gate_stride, x, x_stride, dtype, node_offsets, n, q, f, gate_of(gate_kind),
                                                    zeroes_of(gate_kind), initial, out, out_dtype, final_state, entering, workspace, status,
                                                    reinterpret_cast<cudaStream_t>(stream)),
                       fn);
}

int tfg_gated_recurrence_backward(const void *gate, int64_t gate_stride, const void *x, int64_t x_stride, int dtype,
                                  const int64_t *node_offsets, int64_t num_rows, int64_t num_sequences, int64_t num_features,
                                  int gate_kind, const float *initial, const float *entering, const void *grad_out,
                                  int grad_dtype, const float *grad_final, void *grad_gate, int64_t grad_gate_stride,
                                  void *grad_x, int64_t grad_x_stride, float *grad_initial, void *workspace,
                                  size_t workspace_bytes, int32_t *status, tfg_stream_t stream) {
    const char *fn = "tfg_gated_recurrence_backward";
    TFG_RANGE(fn);
    TFG_TRY(check_recurrence(fn, num_rows, num_sequences, num_features));
    TFG_TRY(check_dtype(fn, dtype));
    TFG_TRY(check_dtype(fn, grad_dtype));
    TFG_TRY(check_gate(fn, gate_kind));
    TFG_TRY(check_stride(fn, "gate_stride", num_rows, gate_stride, num_features));
    TFG_TRY(check_stride(fn, "x_stride", num_rows, x_stride, num_features));
    TFG_TRY(check_stride(fn, "grad_gate_stride", num_rows, grad_gate_stride, num_features));
    TFG_TRY(check_stride(fn, "grad_x_stride", num_rows, grad_x_stride, num_features));
    TFG_NEED(gate, num_rows > 0, fn, "gate");
    TFG_NEED(x, num_rows > 0, fn, "x");
    TFG_NEED(entering, num_rows > 0, fn, "entering");
    TFG_NEED(grad_gate, num_rows > 0, fn, "grad_gate");
    TFG_NEED(grad_x, num_rows > 0, fn, "grad_x");
    TFG_NEED(node_offsets, num_sequences > 0, fn, "node_offsets");
    TFG_NEED(status, true, fn, "status");
    TFG_TRY(check_element(fn, "gate", gate, dtype));
    TFG_TRY(check_element(fn, "x", x, dtype));
    TFG_TRY(check_element(fn, "grad_out", grad_out, grad_dtype));
    TFG_TRY(check_element(fn, "grad_gate", grad_gate, dtype));
    TFG_TRY(check_element(fn, "grad_x", grad_x, dtype));
    const int64_t n = num_rows, q = num_sequences, f = num_features;
    const int64_t tiles = (n + TFG_RECURRENCE_TILE_ROWS - 1) / TFG_RECURRENCE_TILE_ROWS;
    const size_t elem = elem_bytes(dtype);
    const Rows ins[] = {{"gate", gate, n, gate_stride, f, elem}, {"x", x, n, x_stride, f, elem},
                        {"initial", initial, q, f, f, 4}, {"node_offsets", node_offsets, 1, q + 1, q + 1, 8},
                        {"entering", entering, tiles, f, f, 4}, {"grad_out", grad_out, n, f, f, elem_bytes(grad_dtype)},
                        {"grad_final", grad_final, q, f, f, 4}};
    const Rows outs[] = {{"grad_gate", grad_gate, n, grad_gate_stride, f, elem}, {"grad_x", grad_x, n, grad_x_stride, f, elem},
                         {"grad_initial", grad_initial, q, f, f, 4}};
    TFG_TRY(check_apart(fn, outs, 3, ins, 7));
    const size_t need = tfg::gated_recurrence_workspace_bytes(n, f);
    TFG_TRY(check_workspace(fn, workspace, workspace_bytes, need, 16));
#if TFG_CHECK_BOUNDS
    for (const Rows &r : ins) TFG_DEBUG(debug_extent(fn, r.name, r.p, r.extent));
    for (const Rows &r : outs) TFG_DEBUG(debug_extent(fn, r.name, r.p, r.extent));
    TFG_DEBUG(debug_extent(fn, "workspace", workspace, need));
#endif
    return cuda_result(tfg::launch_gated_recurrence_backward(gate, gate_stride, x, x_stride, dtype, node_offsets, n, q, f,
                                                             gate_of(gate_kind), zeroes_of(gate_kind), initial, entering, grad_out, grad_dtype, grad_final,
                                                             grad_gate, grad_gate_stride, grad_x, grad_x_stride, grad_initial,
                                                             workspace, status, reinterpret_cast<cudaStream_t>(stream)),
                       fn);
}

// ---- distillation loss ----------------------------------------------------------------
namespace {
constexpr int64_t kMaxTop = 1024;

struct Distil {
    const void *logits;
    int dtype;
    int64_t num_rows, num_classes;
    const void *ids;
    bool id32;
    const void *teacher;
    int teacher_dtype;
    int64_t top_k;
    float temperature;
    const float *row_weight;
};

int check_distillation(const char *fn, const Distil &a) {
    TFG_TRY(check_counts(fn, a.num_rows, 0));
    if (a.num_classes < 1) return fail(TFG_ERR_INVALID_ARG, "%s: at least one class", fn);
    if (a.num_classes >= kIndexLimit - 1 || (a.num_rows > 0 && a.num_classes >= (int64_t(1) << 46) / a.num_rows))
        return fail(TFG_ERR_TOO_LARGE, "%s: num_rows * num_classes too large", fn);
    if (a.top_k < 1) return fail(TFG_ERR_INVALID_ARG, "%s: top_k must be at least 1", fn);
    if (a.top_k > kMaxTop) return fail(TFG_ERR_TOO_LARGE, "%s: top_k at most %lld", fn, (long long)kMaxTop);
    TFG_TRY(check_dtype(fn, a.dtype));
    TFG_TRY(check_dtype(fn, a.teacher_dtype));
    if (!(a.temperature >= 1e-6f && a.temperature <= 1e6f))
        return fail(TFG_ERR_INVALID_ARG, "%s: temperature must be in [1e-6, 1e6]", fn);
    TFG_NEED(a.logits, a.num_rows > 0, fn, "logits");
    TFG_NEED(a.ids, a.num_rows > 0, fn, "ids");
    TFG_NEED(a.teacher, a.num_rows > 0, fn, "teacher");
    TFG_TRY(check_element(fn, "logits", a.logits, a.dtype));
    TFG_TRY(check_element(fn, "teacher", a.teacher, a.teacher_dtype));
    TFG_DEBUG(debug_extent(fn, "logits", a.logits, elem_bytes(a.dtype) * size_t(a.num_rows * a.num_classes)));
    TFG_DEBUG(debug_extent(fn, "ids", a.ids, (a.id32 ? 4 : 8) * size_t(a.num_rows * a.top_k)));
    TFG_DEBUG(debug_extent(fn, "teacher", a.teacher, elem_bytes(a.teacher_dtype) * size_t(a.num_rows * a.top_k)));
    TFG_DEBUG(debug_extent(fn, "row_weight", a.row_weight, sizeof(float) * size_t(a.num_rows)));
    return TFG_OK;
}

// Outputs against the inputs: stats are one or the other.
int check_distillation_apart(const char *fn, const Distil &a, const float *loss, const float *stats, const float *grad_loss,
                             const void *grad) {
    const int64_t n = a.num_rows, v = a.num_classes, k = a.top_k;
    TFG_TRY(check_element(fn, "grad_logits", grad, a.dtype));
    if (reinterpret_cast<uintptr_t>(stats) % 8 != 0) return fail(TFG_ERR_INVALID_ARG, "%s: stats must be 8-byte aligned", fn);
    const Rows all_stats{"stats", stats, n, 2, 2, 4}, none{"stats", nullptr, 0, 2, 2, 4};
    const Rows ins[] = {{"logits", a.logits, n, v, v, elem_bytes(a.dtype)}, {"ids", a.ids, n, k, k, a.id32 ? 4u : 8u},
                        {"teacher", a.teacher, n, k, k, elem_bytes(a.teacher_dtype)}, {"row_weight", a.row_weight, 1, n, n, 4},
                        {"grad_loss", grad_loss, 1, n, n, 4}, loss ? none : all_stats};
    const Rows outs[] = {{"grad_logits", grad, n, v, v, elem_bytes(a.dtype)}, {"loss", loss, 1, n, n, 4}, loss ? all_stats : none};
    TFG_TRY(check_apart(fn, outs, 3, ins, 6));
    TFG_DEBUG(debug_extent(fn, "grad_logits", grad, outs[0].extent));
    TFG_DEBUG(debug_extent(fn, "loss", loss, outs[1].extent));
    TFG_DEBUG(debug_extent(fn, "stats", stats, all_stats.extent));
    TFG_DEBUG(debug_extent(fn, "grad_loss", grad_loss, ins[4].extent));
    return TFG_OK;
}

int distillation_common(const char *fn, const Distil &a, int64_t padding_id, float *loss, float *stats, void *grad,
                        int32_t *status, tfg_stream_t stream) {
    TFG_RANGE(fn);
    TFG_TRY(check_distillation(fn, a));
    TFG_NEED(loss, a.num_rows > 0, fn, "loss");
    TFG_NEED(status, true, fn, "status");
    TFG_TRY(check_distillation_apart(fn, a, loss, stats, nullptr, grad));
    return cuda_result(tfg::launch_distillation(a.logits, a.dtype, a.num_rows, a.num_classes, a.ids, a.id32, a.teacher,
                                                a.teacher_dtype, static_cast<int>(a.top_k), padding_id, a.temperature,
                                                a.row_weight, loss, stats, grad, status, reinterpret_cast<cudaStream_t>(stream)),
                       fn);
}

int distillation_backward_common(const char *fn, const Distil &a, int64_t padding_id, const float *stats,
                                 const float *grad_loss, void *grad, tfg_stream_t stream) {
    TFG_RANGE(fn);
    TFG_TRY(check_distillation(fn, a));
    TFG_NEED(stats, a.num_rows > 0, fn, "stats");
    TFG_NEED(grad_loss, a.num_rows > 0, fn, "grad_loss");
    TFG_NEED(grad, a.num_rows > 0, fn, "grad_logits");
    TFG_TRY(check_distillation_apart(fn, a, nullptr, stats, grad_loss, grad));
    return cuda_result(tfg::launch_distillation_backward(a.logits, a.dtype, a.num_rows, a.num_classes, a.ids, a.id32, a.teacher,
                                                         a.teacher_dtype, static_cast<int>(a.top_k), padding_id, a.temperature,
                                                         a.row_weight, stats, grad_loss, grad,
                                                         reinterpret_cast<cudaStream_t>(stream)),
                       fn);
}
}  // namespace

int tfg_distillation_loss(const void *logits, int dtype, int64_t num_rows, int64_t num_classes, const int64_t *ids,
                          const void *teacher, int teacher_dtype, int64_t top_k, int64_t padding_id, float temperature,
                          const float *row_weight, float *loss, float *stats, void *grad_logits, int32_t *status,
                          tfg_stream_t stream) {
    return distillation_common("tfg_distillation_loss", {logits, dtype, num_rows, num_classes, ids, false, teacher, teacher_dtype,
                               top_k, temperature, row_weight}, padding_id, loss, stats, grad_logits, status, stream);
}

int tfg_distillation_loss32(const void *logits, int dtype, int64_t num_rows, int64_t num_classes, const int32_t *ids,
                            const void *teacher, int teacher_dtype, int64_t top_k, int64_t padding_id, float temperature,
                            const float *row_weight, float *loss, float *stats, void *grad_logits, int32_t *status,
                            tfg_stream_t stream) {
    return distillation_common("tfg_distillation_loss32", {logits, dtype, num_rows, num_classes, ids, true, teacher,
                               teacher_dtype, top_k, temperature, row_weight}, padding_id, loss, stats, grad_logits, status,
                               stream);
}

int tfg_distillation_loss_backward(const void *logits, int dtype, int64_t num_rows, int64_t num_classes, const int64_t *ids,
                                   const void *teacher, int teacher_dtype, int64_t top_k, int64_t padding_id,
                                   float temperature, const float *row_weight, const float *stats, const float *grad_loss,
                                   void *grad_logits, tfg_stream_t stream) {
    return distillation_backward_common("tfg_distillation_loss_backward", {logits, dtype, num_rows, num_classes, ids, false,
                                        teacher, teacher_dtype, top_k, temperature, row_weight}, padding_id, stats, grad_loss,
                                        grad_logits, stream);
}

int tfg_distillation_loss_backward32(const void *logits, int dtype, int64_t num_rows, int64_t num_classes, const int32_t *ids,
                                     const void *teacher, int teacher_dtype, int64_t top_k, int64_t padding_id,
                                     float temperature, const float *row_weight, const float *stats, const float *grad_loss,
                                     void *grad_logits, tfg_stream_t stream) {
    return distillation_backward_common("tfg_distillation_loss_backward32", {logits, dtype, num_rows, num_classes, ids, true,
                                        teacher, teacher_dtype, top_k, temperature, row_weight}, padding_id, stats, grad_loss,
                                        grad_logits, stream);
}

// ---- global norm and clipping -----------------------------------------------------
namespace {
constexpr int64_t kMaxTensors = int64_t(1) << 20;

int check_tensors(const char *fn, int64_t num_tensors, const void *const *tensors, const int64_t *sizes, const int *dtypes) {
    if (num_tensors < 0) return fail(TFG_ERR_INVALID_ARG, "%s: negative tensor count", fn);
    if (num_tensors > kMaxTensors) return fail(TFG_ERR_TOO_LARGE, "%s: at most %lld tensors", fn, (long long)kMaxTensors);
    TFG_NEED(tensors, num_tensors > 0, fn, "tensors");
    TFG_NEED(sizes, num_tensors > 0, fn, "sizes");
    TFG_NEED(dtypes, num_tensors > 0, fn, "dtypes");
    int64_t total = 0;
    for (int64_t i = 0; i < num_tensors; ++i) {
        if (sizes[i] < 0) return fail(TFG_ERR_INVALID_ARG, "%s: tensor %lld has a negative size", fn, (long long)i);
        if (sizes[i] >= (int64_t(1) << 46) || (total += sizes[i]) >= (int64_t(1) << 46))
            return fail(TFG_ERR_TOO_LARGE, "%s: too many values", fn);
        TFG_TRY(check_dtype(fn, dtypes[i]));
        if (sizes[i] > 0 && tensors[i] == nullptr)
            return fail(TFG_ERR_INVALID_ARG, "%s: tensor %lld must not be NULL", fn, (long long)i);
        TFG_TRY(check_element(fn, "a tensor", tensors[i], dtypes[i]));
        TFG_DEBUG(debug_extent(fn, "a tensor", tensors[i], elem_bytes(dtypes[i]) * size_t(sizes[i])));
    }
    return TFG_OK;
}

// The bytes of a tensor that a call reads, or writes (out).
struct Extent {
    uintptr_t at;
    size_t bytes;
    int64_t tensor;
    bool out;
};

// Outputs may share bytes with nothing but the very tensor they are scaled from.
int check_outs(const char *fn, int64_t num_tensors, const void *const *tensors, const int64_t *sizes, const int *dtypes,
               void *const *outs) {
    std::unique_ptr<Extent[]> all(new (std::nothrow) Extent[size_t(2 * num_tensors)]);
    if (!all) return fail(TFG_ERR_TOO_LARGE, "%s: no host memory for %lld tensors", fn, (long long)num_tensors);
    int64_t m = 0;
    for (int64_t i = 0; i < num_tensors; ++i) {
        if (sizes[i] == 0) continue;
        if (outs[i] == nullptr) return fail(TFG_ERR_INVALID_ARG, "%s: output %lld must not be NULL", fn, (long long)i);
        TFG_TRY(check_element(fn, "an output", outs[i], dtypes[i]));
        const size_t bytes = elem_bytes(dtypes[i]) * size_t(sizes[i]);
        TFG_DEBUG(debug_extent(fn, "an output", outs[i], bytes));
        if (outs[i] != tensors[i]) all[m++] = {reinterpret_cast<uintptr_t>(tensors[i]), bytes, i, false};
        all[m++] = {reinterpret_cast<uintptr_t>(outs[i]), bytes, i, true};
    }
    std::sort(all.get(), all.get() + m, [](const Extent &a, const Extent &b) { return a.at < b.at; });
    // in order of their begin, a range that reaches past another's begin overlaps it: it is
    // enough to keep the furthest end of the outputs and of all ranges so far
    uintptr_t end_out = 0, end_any = 0;
    for (int64_t i = 0; i < m; ++i) {
        if (all[i].at < end_out || (all[i].out && all[i].at < end_any))
            return fail(TFG_ERR_INVALID_ARG, "%s: output of tensor %lld overlaps another tensor", fn, (long long)all[i].tensor);
        const uintptr_t end = all[i].at + all[i].bytes;
        if (end > end_any) end_any = end;
        if (all[i].out && end > end_out) end_out = end;
    }
    return TFG_OK;
}
}  // namespace

int tfg_global_norm_workspace_size(int64_t num_tensors, size_t *bytes) {
    const char *fn = "tfg_global_norm_workspace_size";
    TFG_RANGE(fn);
    if (num_tensors < 0) return fail(TFG_ERR_INVALID_ARG, "%s: negative tensor count", fn);
    if (num_tensors > kMaxTensors) return fail(TFG_ERR_TOO_LARGE, "%s: at most %lld tensors", fn, (long long)kMaxTensors);
    TFG_NEED(bytes, true, fn, "bytes");
    *bytes = tfg::global_norm_workspace_bytes(num_tensors);
    return ok();
}

int tfg_global_norm(int64_t num_tensors, const void *const *tensors, const int64_t *sizes, const int *dtypes, float *norm,
                    void *workspace, size_t workspace_bytes, tfg_stream_t stream) {
    const char *fn = "tfg_global_norm";
    TFG_RANGE(fn);
    TFG_TRY(check_tensors(fn, num_tensors, tensors, sizes, dtypes));
    TFG_NEED(norm, true, fn, "norm");
    TFG_TRY(check_workspace(fn, workspace, workspace_bytes, tfg::global_norm_workspace_bytes(num_tensors), 16));
    TFG_DEBUG(debug_extent(fn, "norm", norm, sizeof(float)));
    TFG_DEBUG(debug_extent(fn, "workspace", workspace, tfg::global_norm_workspace_bytes(num_tensors)));
    return cuda_result(tfg::launch_global_norm(num_tensors, tensors, sizes, dtypes, 0.f, nullptr, norm, workspace,
                                               reinterpret_cast<cudaStream_t>(stream)),
                       fn);
}

int tfg_clip_by_global_norm(int64_t num_tensors, const void *const *tensors, const int64_t *sizes, const int *dtypes,
                            float clip_norm, void *const *outs, float *norm, void *workspace, size_t workspace_bytes,
                            tfg_stream_t stream) {
    const char *fn = "tfg_clip_by_global_norm";
    TFG_RANGE(fn);
    TFG_TRY(check_tensors(fn, num_tensors, tensors, sizes, dtypes));
    if (!(clip_norm > 0.f) || !std::isfinite(clip_norm))
        return fail(TFG_ERR_INVALID_ARG, "%s: clip_norm must be finite and positive", fn);
    TFG_NEED(outs, num_tensors > 0, fn, "outs");
    TFG_NEED(norm, true, fn, "norm");
    TFG_TRY(check_outs(fn, num_tensors, tensors, sizes, dtypes, outs));
    TFG_TRY(check_workspace(fn, workspace, workspace_bytes, tfg::global_norm_workspace_bytes(num_tensors), 16));
    TFG_DEBUG(debug_extent(fn, "norm", norm, sizeof(float)));
    TFG_DEBUG(debug_extent(fn, "workspace", workspace, tfg::global_norm_workspace_bytes(num_tensors)));
    void *none = nullptr;                         // no tensors: outs may be NULL, the norm is written all the same
    return cuda_result(tfg::launch_global_norm(num_tensors, tensors, sizes, dtypes, clip_norm, outs ? outs : &none, norm,
                                               workspace, reinterpret_cast<cudaStream_t>(stream)),
                       fn);
}

int tfg_gather_xor(const int32_t *col, int64_t num_edges, const void *x, int64_t num_nodes,
                   int64_t row_bytes, uint32_t *out, tfg_stream_t stream) {
    const char *fn = "tfg_gather_xor";
    TFG_RANGE(fn);
    TFG_TRY(check_counts(fn, num_nodes, num_edges));
    if (row_bytes < 16 || row_bytes > 512 || (row_bytes & (row_bytes - 1)) != 0)
        return fail(TFG_ERR_INVALID_ARG, "%s: row_bytes must be a power of two in [16, 512] (%lld)",
                    fn, (long long)row_bytes);
    TFG_NEED(col, num_edges > 0, fn, "col");
    TFG_NEED(x, num_edges > 0, fn, "x");
    TFG_NEED(out, true, fn, "out");
    if (reinterpret_cast<uintptr_t>(x) % 16 != 0)
        return fail(TFG_ERR_INVALID_ARG, "%s: x must be 16-byte aligned", fn);
    TFG_DEBUG(debug_csr(fn, "col", nullptr, col, nullptr, num_nodes, num_edges, nullptr, stream));
    TFG_DEBUG(debug_extent(fn, "x", num_edges > 0 ? x : nullptr, size_t(num_nodes) * size_t(row_bytes)));
    TFG_DEBUG(debug_extent(fn, "out", out, size_t(row_bytes)));
    return cuda_result(tfg::launch_gather_xor(col, num_edges, x, row_bytes, out,
                                              reinterpret_cast<cudaStream_t>(stream)),
                       fn);
}

}  // extern "C"
