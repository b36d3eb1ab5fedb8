// Layer norm of rows, backward: the kernels.  A translation unit for each type of the stream
// compiles them.
//
//   h = (s - m) r, d = gamma g
//   grad_s = r (d - mean d - h mean(d h)) + grad_sum
//   grad_gamma = sum over rows of g h, grad_beta = sum of g
//
// The reported mean is rounded to fp32, which would leave h off by up to |m| r 2^-24 in all of a
// row: with e = r mean(s - m) taken beside the other sums, h - e is right to a few u of itself,
// and mean(d (h - e)) = mean(d h) - e mean d needs no second pass.
//
// A CTA takes the rows b, b + CTAs, ..., keeps the sums of its columns for gamma and beta in
// registers and writes them once; a second kernel adds the CTAs' in order.
#pragma once

#include "layer_norm.cuh"

namespace tfg {

struct RowBackArgs {
    const void *s;
    int64_t n, f;
    const float *gamma, *mean, *rstd;
    const void *g;
    const void *skip;         // dL/ds by other ways, or null; of grad_s's type
    void *grad_s;
    float *part;              // [CTAs][2][f] sums for gamma and beta, or null
    float *shift;             // long rows: e of each row
    float *grad_gamma, *grad_beta;
    int out_dtype;            // of skip and grad_s
    int vec;
    int ctas;
};

namespace {

// The three sums of a row: d, d h, s - m.
template <int VEC>
__device__ __forceinline__ void row_terms(const float (&s)[VEC], const float (&g)[VEC], const float (&w)[VEC], float m, float r,
                                          float (&sum)[3]) {
#pragma unroll
    for (int q = 0; q < VEC; ++q) {
        const float c = s[q] - m, d = g[q] * w[q];
        sum[0] += d;
        sum[1] = fmaf(d, c, sum[1]);
        sum[2] += c;
    }
}

// What the sums make of a row: h = (s - m) r - e.
struct RowMeans {
    float d, dh, e;
    __device__ __forceinline__ RowMeans(const float (&sum)[3], float r, float per) {
        d = sum[0] * per;
        e = sum[2] * per * r;
        dh = fmaf(-e, d, sum[1] * r * per);
    }
};

template <typename ST, typename GT, typename DT, int VEC, int TT, int NV>
__global__ void __launch_bounds__(TT < 256 ? 256 : TT) row_norm_back(RowBackArgs p) {
    constexpr int kTeams = TT < 256 ? 256 / TT : 1;
    constexpr int kWarps = TT > 32 ? TT / 32 : 1;
    __shared__ float s_sum[2][3 * kWarps];
    const int t = threadIdx.x % TT, team = threadIdx.x / TT;
    const int cols = static_cast<int>(p.f);
    const float per = 1.f / static_cast<float>(p.f);
    float gg[NV][VEC] = {}, gb[NV][VEC] = {};
    int parity = 0;
    // every team of a CTA takes part in every round: the exchanges are by whole warps
    for (int64_t row0 = static_cast<int64_t>(blockIdx.x) * kTeams; row0 < p.n; row0 += static_cast<int64_t>(gridDim.x) * kTeams) {
        const bool live = row0 + team < p.n;
        const int64_t row = live ? row0 + team : p.n - 1;
        const float m = __ldg(p.mean + row), r = __ldg(p.rstd + row);
        float s[NV][VEC], g[NV][VEC], sum[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * TT) * VEC;
            if (live && c < cols) {
                VecLoad<ST, VEC>::load(static_cast<const ST *>(p.s) + row * p.f + c, s[i]);
                VecLoad<GT, VEC>::load(static_cast<const GT *>(p.g) + row * p.f + c, g[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * TT) * VEC;
            if (live && c < cols) {
                float w[VEC];
                row_weights(p.gamma, c, 1.f, w);
                row_terms<VEC>(s[i], g[i], w, m, r, sum);
            }
        }
        team_sums<TT, 3>(sum, s_sum[parity]);
        parity ^= 1;
        const RowMeans a(sum, r, per);
        if (!live) continue;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * TT) * VEC;
            if (c < cols) {
                float w[VEC], o[VEC];
                row_weights(p.gamma, c, 1.f, w);
                if (p.skip) {
                    load_row<VEC>(static_cast<const DT *>(p.skip) + row * p.f + c, o);
                } else {
#pragma unroll
                    for (int q = 0; q < VEC; ++q) o[q] = 0.f;
                }
#pragma unroll
                for (int q = 0; q < VEC; ++q) {
                    const float h = fmaf(s[i][q] - m, r, -a.e);
                    gg[i][q] = fmaf(g[i][q], h, gg[i][q]);
                    gb[i][q] += g[i][q];
                    o[q] = fmaf(fmaf(-h, a.dh, g[i][q] * w[q] - a.d), r, o[q]);
                }
                store_vec<VEC>(static_cast<DT *>(p.grad_s) + row * p.f + c, o);
            }
        }
    }
    if (!p.part) return;
    // the teams' sums, one team after the other
    float *part = p.part + static_cast<int64_t>(blockIdx.x) * 2 * p.f;
    if constexpr (kTeams == 1) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int q = 0; q < VEC; ++q) {
                const int c = (t + i * TT) * VEC + q;
                if (c < cols) {
                    part[c] = gg[i][q];
                    part[p.f + c] = gb[i][q];
                }
            }
    } else {
        constexpr int kCols = TT * NV * VEC;
        __shared__ float s_cols[2 * kCols];
        for (int j = 0; j < kTeams; ++j) {
            if (team == j) {
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int q = 0; q < VEC; ++q) {
                        const int c = (i * VEC + q) * TT + t;            // no two lanes on one bank
                        s_cols[c] = j ? s_cols[c] + gg[i][q] : gg[i][q];
                        s_cols[kCols + c] = j ? s_cols[kCols + c] + gb[i][q] : gb[i][q];
                    }
            }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < cols; c += 256) {
            const int v = c / VEC, at = ((v / TT) * VEC + c % VEC) * TT + v % TT;
            part[c] = s_cols[at];
            part[p.f + c] = s_cols[kCols + at];
        }
    }
}

// Rows that no team holds: sums, then the row again, and e of the row for the columns' kernel.
template <typename ST, typename GT, typename DT, int VEC>
__global__ void __launch_bounds__(1024) row_norm_back_long(RowBackArgs p) {
    __shared__ float s_sum[3 * 32];
    const float per = 1.f / static_cast<float>(p.f);
    const int64_t row = blockIdx.x, at0 = row * p.f, step = 1024 * VEC;
    const float m = __ldg(p.mean + row), r = __ldg(p.rstd + row);
    float sum[3] = {0.f, 0.f, 0.f};
    for (int64_t c = threadIdx.x * VEC; c < p.f; c += step) {
        float s[VEC], g[VEC], w[VEC], part[3] = {0.f, 0.f, 0.f};
        VecLoad<ST, VEC>::load(static_cast<const ST *>(p.s) + at0 + c, s);
        VecLoad<GT, VEC>::load(static_cast<const GT *>(p.g) + at0 + c, g);
        row_weights(p.gamma, c, 1.f, w);
        row_terms<VEC>(s, g, w, m, r, part);
#pragma unroll
        for (int k = 0; k < 3; ++k) sum[k] += part[k];
    }
    team_sums<1024, 3>(sum, s_sum);
    const RowMeans a(sum, r, per);
    if (threadIdx.x == 0 && p.shift) p.shift[row] = a.e;
    for (int64_t c = threadIdx.x * VEC; c < p.f; c += step) {
        float s[VEC], g[VEC], w[VEC], o[VEC];
        VecLoad<ST, VEC>::load(static_cast<const ST *>(p.s) + at0 + c, s);
        VecLoad<GT, VEC>::load(static_cast<const GT *>(p.g) + at0 + c, g);
        row_weights(p.gamma, c, 1.f, w);
        if (p.skip) {
            load_row<VEC>(static_cast<const DT *>(p.skip) + at0 + c, o);
        } else {
#pragma unroll
            for (int q = 0; q < VEC; ++q) o[q] = 0.f;
        }
#pragma unroll
        for (int q = 0; q < VEC; ++q) {
            const float h = fmaf(s[q] - m, r, -a.e);
            o[q] = fmaf(fmaf(-h, a.dh, g[q] * w[q] - a.d), r, o[q]);
        }
        store_vec<VEC>(static_cast<DT *>(p.grad_s) + at0 + c, o);
    }
}

// Their columns: a CTA adds 256 columns over its share of the rows.
template <typename ST, typename GT>
__global__ void __launch_bounds__(256) long_columns(RowBackArgs p) {
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (c >= p.f) return;
    float gg = 0.f, gb = 0.f;
    for (int64_t row = blockIdx.y; row < p.n; row += gridDim.y) {
        float s[1], g[1];
        VecLoad<ST, 1>::load(static_cast<const ST *>(p.s) + row * p.f + c, s);
        VecLoad<GT, 1>::load(static_cast<const GT *>(p.g) + row * p.f + c, g);
        const float r = __ldg(p.rstd + row), h = fmaf(s[0] - __ldg(p.mean + row), r, -__ldg(p.shift + row));
        gg = fmaf(g[0], h, gg);
        gb += g[0];
    }
    float *part = p.part + static_cast<int64_t>(blockIdx.y) * 2 * p.f;
    part[c] = gg;
    part[p.f + c] = gb;
}

}  // namespace

// The geometry of the first kernel, for the workspace and the launch.
constexpr int kBackVecs8 = 4, kBackVecs1 = 8;               // vectors that a thread holds, of 8 values, of fewer
inline int back_held(int vec) { return vec == 8 ? kBackVecs8 : kBackVecs1; }
inline bool back_long(int64_t f, int vec) { return (f + vec - 1) / vec > 256 * back_held(vec); }

namespace {

template <typename ST, typename GT, typename DT, int VEC>
cudaError_t launch_back_vec(const RowBackArgs &p, cudaStream_t s) {
    constexpr int kHeld = VEC == 8 ? kBackVecs8 : kBackVecs1;
    const int64_t vecs = (p.f + VEC - 1) / VEC;
    if (vecs <= 8) row_norm_back<ST, GT, DT, VEC, 8, 1><<<p.ctas, 256, 0, s>>>(p);
    else if (vecs <= 32) row_norm_back<ST, GT, DT, VEC, 32, 1><<<p.ctas, 256, 0, s>>>(p);
    else if (vecs <= 32 * kHeld) row_norm_back<ST, GT, DT, VEC, 32, kHeld><<<p.ctas, 256, 0, s>>>(p);
    else if (vecs <= 256 * kHeld) row_norm_back<ST, GT, DT, VEC, 256, kHeld><<<p.ctas, 256, 0, s>>>(p);
    else {
        row_norm_back_long<ST, GT, DT, VEC><<<static_cast<unsigned>(p.n), 1024, 0, s>>>(p);
        if (p.part) {
            const dim3 grid(static_cast<unsigned>((p.f + 255) / 256), p.ctas);
            long_columns<ST, GT><<<grid, 256, 0, s>>>(p);
        }
    }
    return cudaGetLastError();
}

template <typename ST, typename GT, typename DT>
cudaError_t launch_back_types(const RowBackArgs &p, cudaStream_t s) {
    if (p.vec == 8) return launch_back_vec<ST, GT, DT, 8>(p, s);
    if (p.vec == 4) return launch_back_vec<ST, GT, DT, 4>(p, s);
    return launch_back_vec<ST, GT, DT, 1>(p, s);
}

template <typename ST, typename GT>
cudaError_t launch_row_back(const RowBackArgs &p, cudaStream_t s) {
    return p.out_dtype == TFG_BF16 ? launch_back_types<ST, GT, uint16_t>(p, s) : launch_back_types<ST, GT, float>(p, s);
}

}  // namespace
}  // namespace tfg
