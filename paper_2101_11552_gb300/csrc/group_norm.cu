// Group norm with an activation, forward: plan and dispatch (group_norm_forward.cuh: the
// kernels).
#include "group_norm.cuh"

namespace tfg {

cudaError_t launch_group_norm_f32(const NormArgs &p, int act, bool out_bf16, cudaStream_t s);
cudaError_t launch_group_norm_bf16(const NormArgs &p, int act, bool out_bf16, cudaStream_t s);

namespace {
NormPlan forward_plan(int64_t n, int64_t graphs, int64_t f, int64_t c, int elem, bool aligned) {
    const int vec = norm_vec(f, c, 16 / elem, aligned);
    return norm_plan(n, graphs, f, c, vec, 1, vec * elem);
}
}  // namespace

// Whether the teams of every type and alignment fit a grid.
bool group_norm_fits(int64_t n, int64_t graphs, int64_t f, int64_t groups) {
    for (const int elem : {4, 2}) {
        for (const bool aligned : {true, false}) {
            const NormPlan p = forward_plan(n, graphs, f, f / groups, elem, aligned);
            if ((graphs + p.shares) * p.tiles > 0x7fff0000) return false;
        }
    }
    return group_norm_backward_fits(n, graphs, f, groups);
}

// Bytes for any type and alignment of the inputs.
size_t group_norm_workspace_bytes(int64_t n, int64_t graphs, int64_t f, int64_t groups) {
    size_t most = 0;
    for (const int elem : {4, 2}) {
        for (const bool aligned : {true, false}) {
            const NormPlan p = forward_plan(n, graphs, f, f / groups, elem, aligned);
            const size_t bytes = size_t(p.shares) * (2 * sizeof(Piece) + 3 * size_t(groups) * sizeof(float4));
            if (bytes > most) most = bytes;
        }
    }
    return most;
}

cudaError_t launch_group_norm(const void *x, int x_dtype, const int64_t *offsets, int64_t n, int64_t graphs, int64_t f,
                              int64_t groups, const float *gamma, const float *beta, float eps, int act, void *out,
                              int out_dtype, float *mean, float *rstd, void *ws, int32_t *status, cudaStream_t s) {
    if (graphs == 0 || graphs > kStatusGraphs) {
        const cudaError_t err = cudaMemsetAsync(status, 0, sizeof(int32_t), s);
        if (err != cudaSuccess || graphs == 0) return err;
    }
    const bool aligned = ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(out) |
                           reinterpret_cast<uintptr_t>(gamma) | reinterpret_cast<uintptr_t>(beta)) & 15) == 0;
    const int64_t c = f / groups;
    NormArgs p{};
    p.x = x;
    p.offsets = offsets;
    p.n = n;
    p.graphs = graphs;
    p.f = f;
    p.groups = static_cast<int>(groups);
    p.c = static_cast<int>(c);
    p.gamma = gamma;
    p.beta = beta;
    p.eps = eps;
    p.mean = mean;
    p.rstd = rstd;
    (graphs > kStatusGraphs ? p.status : p.status_all) = status;
    p.out = out;
    p.p = forward_plan(n, graphs, f, c, x_dtype == TFG_BF16 ? 2 : 4, aligned);
    p.pieces = static_cast<Piece *>(ws);
    p.moments = reinterpret_cast<float4 *>(p.pieces + 2 * p.p.shares);
    p.joined_moments = p.moments + p.p.shares * 2 * groups;
    const bool out_bf16 = out_dtype == TFG_BF16;
    return x_dtype == TFG_BF16 ? launch_group_norm_bf16(p, act, out_bf16, s) : launch_group_norm_f32(p, act, out_bf16, s);
}

}  // namespace tfg
