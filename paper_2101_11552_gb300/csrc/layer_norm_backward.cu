// Layer norm of rows, backward: geometry, launch by type and the join of the columns' sums
// (layer_norm_backward.cuh: the kernels).
#include "layer_norm_backward.cuh"

namespace tfg {

cudaError_t launch_row_back_f32_f32(const RowBackArgs &p, cudaStream_t s);
cudaError_t launch_row_back_f32_bf16(const RowBackArgs &p, cudaStream_t s);
cudaError_t launch_row_back_bf16_f32(const RowBackArgs &p, cudaStream_t s);
cudaError_t launch_row_back_bf16_bf16(const RowBackArgs &p, cudaStream_t s);

namespace {

constexpr int kJoinLanes = 32, kJoinRows = 32;
constexpr int kBackResident = 3;          // CTAs of a multiprocessor at most (256 threads each)

// out[c] = sum over the CTAs of part[.][c], in 32 interleaved chains joined in order; V columns a thread.
template <int V>
__global__ void __launch_bounds__(kJoinLanes *kJoinRows) join_columns_kernel(const float *part, int ctas, int64_t f,
                                                                             float *gamma, float *beta) {
    __shared__ __align__(16) float s_part[kJoinRows][kJoinLanes * V];
    const int x = threadIdx.x % kJoinLanes, y = threadIdx.x / kJoinLanes;
    const int64_t c = (static_cast<int64_t>(blockIdx.x) * kJoinLanes + x) * V;
    float sum[V] = {};
    if (c < 2 * f) {
#pragma unroll 8
        for (int b = y; b < ctas; b += kJoinRows) {
            float v[V];
            VecLoad<float, V>::load(part + b * 2 * f + c, v);
#pragma unroll
            for (int q = 0; q < V; ++q) sum[q] += v[q];
        }
    }
#pragma unroll
    for (int q = 0; q < V; ++q) s_part[y][x * V + q] = sum[q];
    __syncthreads();
    const int64_t out = static_cast<int64_t>(blockIdx.x) * kJoinLanes * V + threadIdx.x;
    if (threadIdx.x < kJoinLanes * V && out < 2 * f) {
        float total = 0.f;
#pragma unroll
        for (int j = 0; j < kJoinRows; ++j) total += s_part[j][threadIdx.x];
        (out < f ? gamma[out] : beta[out - f]) = total;
    }
}

}  // namespace

cudaError_t join_columns(const float *part, int ctas, int64_t f, float *gamma, float *beta, cudaStream_t s) {
    // four columns a thread where that leaves a CTA for most multiprocessors
    if (f % 2 == 0 && f >= 8192) join_columns_kernel<4><<<ceil_div(2 * f, 4 * kJoinLanes), kJoinLanes * kJoinRows, 0, s>>>(part, ctas, f, gamma, beta);
    else join_columns_kernel<1><<<ceil_div(2 * f, kJoinLanes), kJoinLanes * kJoinRows, 0, s>>>(part, ctas, f, gamma, beta);
    return cudaGetLastError();
}

int back_ctas(int64_t n, int teams, int resident) {
    const int64_t rounds = (n + teams - 1) / teams, sms = sm_count();
    const int64_t few = rounds < sms ? rounds : sms, want = rounds / 4 > few ? rounds / 4 : few;
    return static_cast<int>(want < resident * sms ? want : resident * sms);
}

size_t layer_norm_backward_workspace_bytes(int64_t n, int64_t f) {
    return sizeof(float) * (2 * size_t(f) * size_t(back_ctas(n, 1, kBackResident)) + size_t(n));
}

cudaError_t launch_layer_norm_backward(const void *sum, int sum_dtype, int64_t n, int64_t f, const float *gamma,
                                       const float *mean, const float *rstd, const void *g, int g_dtype, const void *skip,
                                       void *grad_s, int out_dtype, float *grad_gamma, float *grad_beta, void *ws,
                                       cudaStream_t s) {
    if (n == 0) {
        if (!grad_gamma) return cudaSuccess;
        cudaError_t e = cudaMemsetAsync(grad_gamma, 0, sizeof(float) * size_t(f), s);
        return e != cudaSuccess ? e : cudaMemsetAsync(grad_beta, 0, sizeof(float) * size_t(f), s);
    }
    RowBackArgs p{sum, n, f, gamma, mean, rstd, g, skip, grad_s, nullptr, nullptr, grad_gamma, grad_beta, out_dtype, false, 1};
    const auto whole = [&](const void *q, int dtype) {
        return f * (dtype == TFG_BF16 ? 2 : 4) % 16 == 0 && reinterpret_cast<uintptr_t>(q) % 16 == 0;
    };
    p.bulk = whole(sum, sum_dtype) && whole(g, g_dtype) && whole(grad_s, out_dtype) && (!skip || whole(skip, out_dtype)) &&
             reinterpret_cast<uintptr_t>(gamma) % 16 == 0;
    if (grad_gamma) {
        p.part = static_cast<float *>(ws);
        p.shift = p.part + 2 * size_t(f) * size_t(back_ctas(n, 1, kBackResident));
    }
    if (sum_dtype == TFG_BF16) return g_dtype == TFG_BF16 ? launch_row_back_bf16_bf16(p, s) : launch_row_back_bf16_f32(p, s);
    return g_dtype == TFG_BF16 ? launch_row_back_f32_bf16(p, s) : launch_row_back_f32_f32(p, s);
}

}  // namespace tfg
