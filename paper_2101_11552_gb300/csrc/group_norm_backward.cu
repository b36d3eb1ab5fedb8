// Group norm with an activation, backward: plan and dispatch (group_norm_backward.cuh: the
// kernels).
#include "group_norm.cuh"

namespace tfg {

cudaError_t launch_group_norm_backward_f32_f32(const NormArgs &p, int act, float *grad_gamma, float *grad_beta, cudaStream_t s);
cudaError_t launch_group_norm_backward_f32_bf16(const NormArgs &p, int act, float *grad_gamma, float *grad_beta, cudaStream_t s);
cudaError_t launch_group_norm_backward_bf16_f32(const NormArgs &p, int act, float *grad_gamma, float *grad_beta, cudaStream_t s);
cudaError_t launch_group_norm_backward_bf16_bf16(const NormArgs &p, int act, float *grad_gamma, float *grad_beta, cudaStream_t s);

namespace {

// Graphs of a batch: one, or so many that the batches of all tiles are twice what is
// resident at once (a batch leaves 8 bytes a channel).
int64_t back_batch(const NormPlan &p, int64_t graphs) {
    const int64_t resident = team_ctas(p.team, kBackResident) * (p.team == 32 ? kWarpTeams : 1) * 152;
    const int64_t batches = (2 * resident + p.tiles - 1) / p.tiles;
    return graphs <= batches ? 1 : (graphs + batches - 1) / batches;
}
int64_t back_batches(const NormPlan &p, int64_t graphs) {
    const int64_t b = back_batch(p, graphs);
    return (graphs + b - 1) / b;
}

struct BackLayout {       // of the workspace, in bytes
    size_t pieces, part, joined, channels;
    size_t all() const { return pieces + part + joined + channels; }
};
BackLayout back_layout(const NormPlan &p, int64_t graphs, int64_t f, int64_t groups) {
    const size_t shares = size_t(p.shares);
    return {shares * 2 * sizeof(Piece), shares * 2 * size_t(groups) * sizeof(float2), shares * size_t(groups) * sizeof(float2),
            size_t((back_batches(p, graphs) + p.shares) * f) * sizeof(float2)};
}

NormPlan back_plan(int64_t n, int64_t graphs, int64_t f, int64_t c, int elems, bool aligned) {
    const int vec = norm_vec(f, c, 4, aligned);
    return norm_plan(n, graphs, f, c, vec, 2, vec * elems);
}

}  // namespace

bool group_norm_backward_fits(int64_t n, int64_t graphs, int64_t f, int64_t groups) {
    for (const int elems : {8, 6, 4}) {
        for (const bool aligned : {true, false}) {
            const NormPlan p = back_plan(n, graphs, f, f / groups, elems, aligned);
            if ((back_batches(p, graphs) + p.shares) * p.tiles + (f + 3) / 4 > 0x7ff00000) return false;
        }
    }
    return true;
}

size_t group_norm_backward_workspace_bytes(int64_t n, int64_t graphs, int64_t f, int64_t groups) {
    size_t most = 0;
    for (const int elems : {8, 6, 4}) {
        for (const bool aligned : {true, false}) {
            const size_t bytes = back_layout(back_plan(n, graphs, f, f / groups, elems, aligned), graphs, f, groups).all();
            if (bytes > most) most = bytes;
        }
    }
    return most;
}

cudaError_t launch_group_norm_backward(const void *x, int x_dtype, const int64_t *offsets, int64_t n, int64_t graphs,
                                       int64_t f, int64_t groups, const float *gamma, const float *beta,
                                       const float *mean, const float *rstd, int act, const void *g, int g_dtype,
                                       void *grad_x, float *grad_gamma, float *grad_beta, void *ws, cudaStream_t s) {
    const bool aligned = ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(g) |
                           reinterpret_cast<uintptr_t>(grad_x) | reinterpret_cast<uintptr_t>(gamma) |
                           reinterpret_cast<uintptr_t>(beta)) & 15) == 0;
    if (graphs == 0 || n == 0) {
        if (!grad_gamma) return cudaSuccess;
        const cudaError_t err = cudaMemsetAsync(grad_gamma, 0, sizeof(float) * size_t(f), s);
        return err != cudaSuccess ? err : cudaMemsetAsync(grad_beta, 0, sizeof(float) * size_t(f), s);
    }
    NormArgs p{};
    p.x = x;
    p.offsets = offsets;
    p.n = n;
    p.graphs = graphs;
    p.f = f;
    p.groups = static_cast<int>(groups);
    p.c = static_cast<int>(f / groups);
    p.gamma = gamma;
    p.beta = beta;
    p.mean_in = mean;
    p.rstd_in = rstd;
    p.g = g;
    p.out = grad_x;
    p.p = back_plan(n, graphs, f, p.c, (x_dtype == TFG_BF16 ? 2 : 4) + (g_dtype == TFG_BF16 ? 2 : 4), aligned);
    p.batch = back_batch(p.p, graphs);
    p.batches = back_batches(p.p, graphs);
    const BackLayout l = back_layout(p.p, graphs, f, groups);
    char *at = static_cast<char *>(ws);
    p.pieces = reinterpret_cast<Piece *>(at);
    p.part = reinterpret_cast<float2 *>(at + l.pieces);
    p.joined = reinterpret_cast<float2 *>(at + l.pieces + l.part);
    p.channel_part = grad_gamma ? reinterpret_cast<float2 *>(at + l.pieces + l.part + l.joined) : nullptr;
    if (x_dtype == TFG_BF16)
        return g_dtype == TFG_BF16 ? launch_group_norm_backward_bf16_bf16(p, act, grad_gamma, grad_beta, s)
                                   : launch_group_norm_backward_bf16_f32(p, act, grad_gamma, grad_beta, s);
    return g_dtype == TFG_BF16 ? launch_group_norm_backward_f32_bf16(p, act, grad_gamma, grad_beta, s)
                               : launch_group_norm_backward_f32_f32(p, act, grad_gamma, grad_beta, s);
}

}  // namespace tfg
