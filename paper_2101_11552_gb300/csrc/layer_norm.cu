// Layer norm of rows with the addition of the residual stream, forward.
//
//   s = x + residual, rounded to the stream's type and stored; s = x without a residual
//   m = mean of the row's F values of s, v = mean of (s - m)^2, r = 1 / sqrt(v + eps)
//   out = gamma (s - m) r + beta
//
// The norm is that of the stored stream, the one array that the next layer and the backward
// read.  One pass over memory: a team holds the row in registers, takes a first mean, then the
// sums of the deviations d from it and of their squares, m = first mean + mean d, v = mean d^2 - (mean
// d)^2.  The rounding of the first mean, a few u |m|, is in mean d and so costs nothing; what is
// left is a few u of the deviations.
//
// What bounds it: memory, in rows of up to 1,024 columns, a warp each: 131,072 rows of 1,024 in bf16 on an fp32 stream
// 228 us (1.61 GB, 7.1 TB/s).  8,192 rows of 8,192 bf16 95 us (537 MB, 5.7 TB/s): a CTA a row, which its two barriers
// leave waiting; with 512 threads of 16 values 104.  A few rows are bound by latency and spread over 128 threads each: 8
// rows of 1,024 3.1 us, a warp each 6.0.  Odd widths go value by value: 19,717 rows of 123 fp32 8.7 us (19 MB).
#include <type_traits>

#include "layer_norm.cuh"

namespace tfg {
namespace {

struct None {};           // no residual

struct RowNormArgs {
    const void *x;
    const void *residual;
    void *sum;
    int64_t n, f;
    const float *gamma, *beta;
    float eps;
    void *out;
    bool out_bf16;
    float *mean, *rstd;
};

template <typename RT>
constexpr bool kHasStream = !std::is_same<RT, None>::value;

// x and the residual of VEC values; the second keeps nothing where there is none.
template <typename XT, typename RT, int VEC>
__device__ __forceinline__ void load_terms(const RowNormArgs &p, int64_t at, float (&x)[VEC], float (&r)[VEC]) {
    load_row<VEC>(static_cast<const XT *>(p.x) + at, x);
    if constexpr (kHasStream<RT>) load_row<VEC>(static_cast<const RT *>(p.residual) + at, r);
}

// s of VEC values into x: added, rounded to the stream's type and stored.
template <typename RT, int VEC>
__device__ __forceinline__ void add_stream(const RowNormArgs &p, int64_t at, float (&x)[VEC], const float (&r)[VEC]) {
    if constexpr (kHasStream<RT>) {
        add_vec(x, r);
        store_vec<VEC>(static_cast<RT *>(p.sum) + at, x);
        if constexpr (sizeof(RT) == 2) {
#pragma unroll
            for (int q = 0; q < VEC; ++q) x[q] = bf16_lo(pack_bf16(x[q], 0.f));
        }
    }
}

// r of a row whose deviations from the first mean have the means d and d2 (squares).
__device__ __forceinline__ float row_rstd(float d, float d2, float eps) {
    const float v = fmaf(-d, d, d2);
    return rsqrtf((v < 0.f ? 0.f : v) + eps);                // rounding may take it below 0; a NaN stays
}

// 0: as many CTAs as the registers allow that the compiler takes by itself (told of one it takes 86 in place of 76, and two
// CTAs of 256 fit where three did: 8,192 rows of 8,192 bf16 115 us).
template <typename XT, typename RT, int VEC, int TT, int NV>
__global__ void __launch_bounds__(TT <= 32 ? 256 : TT, TT == 512 && VEC > 1 ? 2 : 0) row_norm(RowNormArgs p) {
    constexpr int kTeams = TT <= 32 ? 256 / TT : 1;
    __shared__ float s_sum[3 * (TT > 32 ? TT / 32 : 1)];
    const int t = threadIdx.x % TT;
    const int64_t row0 = static_cast<int64_t>(blockIdx.x) * kTeams + threadIdx.x / TT;
    const bool live = row0 < p.n;                            // a team without a row goes through the exchanges
    const int64_t row = live ? row0 : p.n - 1;
    const int cols = static_cast<int>(p.f);
    float v[NV][VEC], w[NV][VEC];
    float sum[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {                           // all loads before the first store
        const int c = (t + i * TT) * VEC;
        if (live && c < cols) {
            load_terms<XT, RT, VEC>(p, row * p.f + c, v[i], w[i]);
        } else {
#pragma unroll
            for (int q = 0; q < VEC; ++q) v[i][q] = 0.f;
        }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (t + i * TT) * VEC;
        if (live && c < cols) add_stream<RT, VEC>(p, row * p.f + c, v[i], w[i]);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int q = 0; q < VEC; ++q) sum[0] += v[i][q];
    team_sums<TT, 1, 1>(sum, s_sum);
    const float per = 1.f / static_cast<float>(p.f);
    const float first = sum[0] * per;
    float dev[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if ((t + i * TT) * VEC < cols) {
#pragma unroll
            for (int q = 0; q < VEC; ++q) {
                v[i][q] -= first;
                dev[0] += v[i][q];
                dev[1] = fmaf(v[i][q], v[i][q], dev[1]);
            }
        }
    team_sums<TT, 1, 2>(dev, s_sum + (TT > 32 ? TT / 32 : 1));
    if (!live) return;
    const float d = dev[0] * per, r = row_rstd(d, dev[1] * per, p.eps);
    if (t == 0 && p.mean) {
        p.mean[row] = first + d;
        p.rstd[row] = r;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (t + i * TT) * VEC;
        if (c < cols) {
            float g[VEC], b[VEC];
            row_weights(p.gamma, c, 1.f, g);
            row_weights(p.beta, c, 0.f, b);
#pragma unroll
            for (int q = 0; q < VEC; ++q) g[q] = fmaf((v[i][q] - d) * r, g[q], b[q]);
            store_row<VEC>(p.out, p.out_bf16, row * p.f + c, g);
        }
    }
}

// Rows that no team holds: three passes, the second and third over what L2 keeps of the row.
template <typename XT, typename RT, int VEC>
__global__ void __launch_bounds__(1024) row_norm_long(RowNormArgs p) {
    __shared__ float s_sum[3 * 32];
    constexpr bool kPlain = !kHasStream<RT>;
    using ST = typename std::conditional<kPlain, XT, RT>::type;
    const ST *s = static_cast<const ST *>(kPlain ? p.x : p.sum);
    const float per = 1.f / static_cast<float>(p.f);
    const int64_t at0 = blockIdx.x * p.f;
    const int64_t step = 1024 * VEC;
    float sum[1] = {0.f}, dev[2] = {0.f, 0.f};
    for (int64_t c = threadIdx.x * VEC; c < p.f; c += step) {
        float v[VEC], w[VEC], part = 0.f;
        load_terms<XT, RT, VEC>(p, at0 + c, v, w);
        add_stream<RT, VEC>(p, at0 + c, v, w);
#pragma unroll
        for (int q = 0; q < VEC; ++q) part += v[q];
        sum[0] += part;
    }
    team_sums<1024, 1, 1>(sum, s_sum);
    const float first = sum[0] * per;
    for (int64_t c = threadIdx.x * VEC; c < p.f; c += step) {   // each thread reads what it wrote
        float v[VEC], part[2] = {0.f, 0.f};
        load_row<VEC>(s + at0 + c, v);
#pragma unroll
        for (int q = 0; q < VEC; ++q) {
            v[q] -= first;
            part[0] += v[q];
            part[1] = fmaf(v[q], v[q], part[1]);
        }
        dev[0] += part[0];
        dev[1] += part[1];
    }
    team_sums<1024, 1, 2>(dev, s_sum + 32);
    const float d = dev[0] * per, r = row_rstd(d, dev[1] * per, p.eps);
    if (threadIdx.x == 0 && p.mean) {
        p.mean[blockIdx.x] = first + d;
        p.rstd[blockIdx.x] = r;
    }
    for (int64_t c = threadIdx.x * VEC; c < p.f; c += step) {
        float v[VEC], g[VEC], b[VEC];
        load_row<VEC>(s + at0 + c, v);
        row_weights(p.gamma, c, 1.f, g);
        row_weights(p.beta, c, 0.f, b);
#pragma unroll
        for (int q = 0; q < VEC; ++q) g[q] = fmaf(((v[q] - first) - d) * r, g[q], b[q]);
        store_row<VEC>(p.out, p.out_bf16, at0 + c, g);
    }
}

template <typename XT, typename RT, int VEC>
cudaError_t launch_vec(const RowNormArgs &p, cudaStream_t s) {
    constexpr int kHeld = VEC == 8 ? 4 : 8;                  // vectors that a thread holds
    const int64_t vecs = (p.f + VEC - 1) / VEC;
    const auto ctas = [&](int teams) { return static_cast<unsigned>((p.n + teams - 1) / teams); };
    // As many threads as hold the row in full vectors (250,000 rows of 128 bf16 42 us with 16, 70 with 32; 32,768 of 2,048
    // 88 us with 64, 171 with 256; 4,096 of 16,384 118 with two CTAs of 512 on a multiprocessor, 156 with one, 164 with
    // 1,024); a few rows spread over more of them.
    const bool few = p.n <= 4 * sm_count();
    if (vecs <= 4) row_norm<XT, RT, VEC, 4, 1><<<ctas(64), 256, 0, s>>>(p);
    else if (vecs <= 8) row_norm<XT, RT, VEC, 8, 1><<<ctas(32), 256, 0, s>>>(p);
    else if (vecs <= 16) row_norm<XT, RT, VEC, 16, 1><<<ctas(16), 256, 0, s>>>(p);
    else if (vecs <= 32) row_norm<XT, RT, VEC, 32, 1><<<ctas(8), 256, 0, s>>>(p);
    else if (few && vecs <= 128) row_norm<XT, RT, VEC, 128, 1><<<ctas(1), 128, 0, s>>>(p);
    else if (vecs <= 64) row_norm<XT, RT, VEC, 32, 2><<<ctas(8), 256, 0, s>>>(p);
    else if (vecs <= 32 * kHeld) row_norm<XT, RT, VEC, 32, kHeld><<<ctas(8), 256, 0, s>>>(p);
    else if (vecs <= 64 * kHeld) row_norm<XT, RT, VEC, 64, kHeld><<<ctas(1), 64, 0, s>>>(p);
    else if (vecs <= 128 * kHeld) row_norm<XT, RT, VEC, 128, kHeld><<<ctas(1), 128, 0, s>>>(p);
    else if (vecs <= 256 * kHeld) row_norm<XT, RT, VEC, 256, kHeld><<<ctas(1), 256, 0, s>>>(p);
    else if (vecs <= 512 * kHeld) row_norm<XT, RT, VEC, 512, kHeld><<<ctas(1), 512, 0, s>>>(p);
    else if (vecs <= 1024 * kHeld) row_norm<XT, RT, VEC, 1024, kHeld><<<ctas(1), 1024, 0, s>>>(p);
    else row_norm_long<XT, RT, VEC><<<ctas(1), 1024, 0, s>>>(p);
    return cudaGetLastError();
}

template <typename XT, typename RT>
cudaError_t launch_types(const RowNormArgs &p, int vec, cudaStream_t s) {
    if (vec == 8) return launch_vec<XT, RT, 8>(p, s);
    if (vec == 4) return launch_vec<XT, RT, 4>(p, s);
    return launch_vec<XT, RT, 1>(p, s);
}

}  // namespace

cudaError_t launch_layer_norm(const void *x, int x_dtype, const void *residual, int sum_dtype, void *sum, int64_t n,
                              int64_t f, const float *gamma, const float *beta, float eps, void *out, int out_dtype,
                              float *mean, float *rstd, cudaStream_t s) {
    if (n == 0) return cudaSuccess;
    const RowNormArgs p{x, residual, sum, n, f, gamma, beta, eps, out, out_dtype == TFG_BF16, mean, rstd};
    const auto fits = [&](int vec) {
        return vec_fits(x, x_dtype, f, vec) && vec_fits(out, out_dtype, f, vec) && weights_fit(gamma) && weights_fit(beta) &&
               (!residual || (vec_fits(residual, sum_dtype, f, vec) && vec_fits(sum, sum_dtype, f, vec)));
    };
    const int vec = fits(8) ? 8 : (fits(4) ? 4 : 1);
    if (x_dtype == TFG_BF16) {
        if (!residual) return launch_types<uint16_t, None>(p, vec, s);
        return sum_dtype == TFG_BF16 ? launch_types<uint16_t, uint16_t>(p, vec, s) : launch_types<uint16_t, float>(p, vec, s);
    }
    if (!residual) return launch_types<float, None>(p, vec, s);
    return sum_dtype == TFG_BF16 ? launch_types<float, uint16_t>(p, vec, s) : launch_types<float, float>(p, vec, s);
}

}  // namespace tfg
