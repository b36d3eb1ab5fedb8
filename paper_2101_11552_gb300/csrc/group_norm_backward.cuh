// Group norm with an activation, backward: the kernels (group_norm.cuh: the work split).  A
// translation unit for each pair of types compiles them.
//
//   h = (x - m) r, y = gamma h + beta, d = g act'(y)
//   grad_beta = sum d, grad_gamma = sum d h                     over all rows
//   s1 = sum gamma d, s2 = sum gamma d h                        over the (graph, group)
//   grad_x = r (gamma d - (s1 + h s2) / M)
//
// A team takes a batch of graphs (or a piece of a large one), keeps its columns' sums for
// gamma and beta in registers from graph to graph and leaves them once; a last kernel adds
// those of all teams in order.
//
// What bounds it: as the forward, with the slope of the activation taken twice (in the sums
// and in grad_x: keeping it would halve the rows a team holds).  1,024 graphs of 110 rows, F =
// 128 fp32, SiLU: 50 us (173 MB, 3.5 TB/s; first kernel 41, channels' sums 8).  41 graphs of
// 232,965 rows, F = 128 bf16: 87 us (179 MB, 2.1 TB/s: 40, the join, 40 for the second read).  300
// ragged graphs of 19,717 rows, F = 123 fp32, GELU: 31 us.
#pragma once

#include "group_norm.cuh"

namespace tfg {
namespace {

// Shared memory of a team: sums and held rows, and at the end its channels' sums instead.
__host__ __device__ inline int back_bytes(const NormPlan &p, int sums, int vec, int row_bytes) {
    const int held = team_bytes(p, kBackBuffers, sums, row_bytes), channels = 2 * p.team * vec * 4;
    return held > channels ? held : channels;
}

template <int VEC, int S>
struct Column {           // what a thread's channels need
    float away[S], rstd[S], gamma[VEC], beta[VEC];          // away: minus the mean

    template <int TT>
    __device__ __forceinline__ void weights(const NormArgs &p, const Place<TT, VEC, S> &at) {
        channel_weights(at.on ? p.gamma : nullptr, at.c0, 1.f, gamma);
        channel_weights(at.on ? p.beta : nullptr, at.c0, 0.f, beta);
    }
    template <int TT>
    __device__ __forceinline__ void statistics(const NormArgs &p, const Place<TT, VEC, S> &at, int64_t graph) {
#pragma unroll
        for (int q = 0; q < S; ++q) {
            const int64_t i = graph * p.groups + at.group0 + at.grp[q];
            away[q] = at.on ? -__ldg(p.mean_in + i) : 0.f;
            rstd[q] = at.on ? __ldg(p.rstd_in + i) : 0.f;
        }
    }
    __device__ __forceinline__ void slopes(float (&slope)[VEC]) const {
#pragma unroll
        for (int q = 0; q < VEC; ++q) slope[q] = gamma[q];
        mul_vec(slope, rstd);
    }
    // e = x - m = h / r and d of row i; slope: gamma r
    template <int ACT, typename XH, typename GH>
    __device__ __forceinline__ void values(const XH &x, const GH &g, int i, const float (&slope)[VEC], float (&e)[VEC],
                                           float (&d)[VEC]) const {
        x.widen(i, e);
        g.widen(i, d);
        float y[VEC];
        add_vec(e, away);
        fma_vec(y, e, slope, beta);
        times_slope<ACT>(y, d);
    }
};

// Sums of gamma d and gamma d h over the held rows of each group, to every thread for its
// groups; weight adds up this thread's d h and d.
template <int ACT, typename XT, typename GT, int TT, int VEC, int S>
__device__ __forceinline__ void sums(const NormArgs &p, const Place<TT, VEC, S> &at, const Column<VEC, S> &c,
                                     const float (&slope)[VEC], const Held<XT, VEC, TT> &x, const Held<GT, VEC, TT> &g,
                                     int rows, float *smem, int buffer, float (&s)[2][S], float (&weight)[2][VEC]) {
    constexpr int kPer = VEC / S;
    float de[VEC] = {}, db[VEC] = {};
#pragma unroll 2
    for (int i = 0; i < rows; ++i) {
        float e[VEC], d[VEC];
        c.template values<ACT>(x, g, i, slope, e, d);
        fma_vec(de, d, e, de);
        add_vec(db, d);
    }
#pragma unroll
    for (int q = 0; q < S; ++q) s[0][q] = s[1][q] = 0.f;
#pragma unroll
    for (int q = 0; q < VEC; ++q) {
        s[0][q / kPer] = fmaf(c.gamma[q], db[q], s[0][q / kPer]);
        s[1][q / kPer] = fmaf(slope[q], de[q], s[1][q / kPer]);
        weight[0][q] = fmaf(c.rstd[q / kPer], de[q], weight[0][q]);
        weight[1][q] += db[q];
    }
    group_sums<TT, VEC, S, 2>(p, at, s, smem, buffer);
}

// grad_x of the held rows from row a on, gamma r d - r s1 - (r^2 s2) e; s: the sums over M.
template <int ACT, typename XT, typename GT, int TT, int VEC, int S>
__device__ __forceinline__ void gradient(const NormArgs &p, const Place<TT, VEC, S> &at, const Column<VEC, S> &c,
                                         const float (&slope)[VEC], const Held<XT, VEC, TT> &x, const Held<GT, VEC, TT> &g,
                                         int rows, int64_t a, const float (&s)[2][S]) {
    float s1[S], s2[S];
#pragma unroll
    for (int q = 0; q < S; ++q) {
        s1[q] = -c.rstd[q] * s[0][q];
        s2[q] = -c.rstd[q] * (c.rstd[q] * s[1][q]);
    }
    const int64_t step = p.p.rows_at_once * p.f;
    GT *to = static_cast<GT *>(p.out) + (a + at.rl) * p.f + at.c0;
#pragma unroll 2
    for (int i = 0; i < rows; ++i) {
        float e[VEC], d[VEC];
        c.template values<ACT>(x, g, i, slope, e, d);
        fma_vec(e, e, s2, s1);
        fma_vec(d, d, slope, e);
        store_vec<VEC>(to + i * step, d);
    }
}

template <typename XT, typename GT, int VEC, int TT, int S>
__device__ __forceinline__ void copy_rows(const NormArgs &p, const Place<TT, VEC, S> &at, const Held<XT, VEC, TT> &x,
                                          const Held<GT, VEC, TT> &g, int64_t a, int rows) {
    const int64_t first = (a + at.rl) * p.f + at.c0, step = p.p.rows_at_once * p.f;
    x.copy(static_cast<const XT *>(p.x) + first, rows, step);
    g.copy(static_cast<const GT *>(p.g) + first, rows, step);
}

template <int ACT, int TT, typename XT, typename GT, int VEC, int S>
__global__ void __launch_bounds__(Team<TT>::kThreads, team_ctas(TT, kBackResident)) norm_back_units(NormArgs p) {
    using M = Team<TT>;
    constexpr int kRowBytes = VEC * static_cast<int>(sizeof(XT) + sizeof(GT));
    extern __shared__ __align__(16) char s_all[];
    const uint32_t id = blockIdx.x * M::kPerCta + M::index();
    const int64_t row = id / static_cast<uint32_t>(p.p.tiles);   // a batch of graphs, then the shares
    const int tile = static_cast<int>(id - static_cast<uint32_t>(row) * p.p.tiles);
    if (row >= p.batches + p.p.shares) return;              // whole teams
    char *own = s_all + M::index() * back_bytes(p.p, S, VEC, kRowBytes);
    float *smem = reinterpret_cast<float *>(own);
    char *rows_at = own + sum_floats(p.p, kBackBuffers, S) * 4;
    const Held<XT, VEC, TT> x(rows_at);
    const Held<GT, VEC, TT> g(rows_at + p.p.held * TT * VEC * sizeof(XT));
    const Place<TT, VEC, S> at(p, tile);
    Column<VEC, S> c;
    float weight[2][VEC] = {}, s[2][S];
    const int64_t share = row - p.batches;
    c.weights(p, at);
    int buffer = 0;
    int64_t covered = 0;
    const int64_t first = row * p.batch, stop = share >= 0 ? first + 2 : min64(p.graphs, first + p.batch);
    bool any = share < 0;
#pragma unroll 1
    for (int64_t i = first; i < stop; ++i) {                // graphs, or the share's slots
        Piece piece{0, 0, i, 0};
        if (share < 0) {
            bool bad;
            const RowRange r = graph_rows(p.offsets, i, p.n, bad);
            if (r.b - r.a > p.p.most) continue;
            piece.a = r.a;
            piece.b = r.b;
        } else {
            piece = find_piece(p, share, static_cast<int>(i - first), covered);
            if (tile == 0 && M::thread() == 0) p.pieces[share * 2 + i - first] = piece;
        }
        if (piece.a == piece.b) continue;
        any = true;
        const int rows = at.rows(p, piece.a, piece.b);
        copy_rows(p, at, x, g, piece.a, rows);
        c.statistics(p, at, piece.graph);
        float slope[VEC];
        c.slopes(slope);
        copies_done();
        sums<ACT>(p, at, c, slope, x, g, rows, smem, buffer, s, weight);
        buffer ^= 2;
        if (share < 0) {
            const float per_value = 1.f / static_cast<float>((piece.b - piece.a) * p.c);
#pragma unroll
            for (int q = 0; q < S; ++q) {
                s[0][q] *= per_value;
                s[1][q] *= per_value;
            }
            gradient<ACT>(p, at, c, slope, x, g, rows, piece.a, s);
        } else {
#pragma unroll
            for (int q = 0; q < S; ++q)
                if (at.writes(p, q))
                    p.part[(share * 2 + i - first) * p.groups + at.group0 + at.grp[q]] = make_float2(s[0][q], s[1][q]);
        }
    }
    if (!any) return;                                       // a share without pieces: its channels' row is not read
    if (!p.channel_part) return;
    // this team's sums of every channel, over its row lanes in order
    const int t = M::thread(), cols = p.p.cols, rows = p.p.rows_at_once;
    M::sync();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        if (t < rows * p.p.row_vecs) {
#pragma unroll
            for (int q = 0; q < VEC; ++q) smem[(k * rows + at.rl) * cols + at.sub * VEC + q] = weight[k][q];
        }
    }
    M::sync();
    const int64_t c0 = static_cast<int64_t>(tile) * cols;
    for (int i = t; i < cols && c0 + i < p.f; i += TT) {
        float2 r = make_float2(0.f, 0.f);
        for (int j = 0; j < rows; ++j) {
            r.x += smem[j * cols + i];
            r.y += smem[(rows + j) * cols + i];
        }
        p.channel_part[row * p.f + c0 + i] = r;
    }
}

// Sums over M of a large graph (rows r, from share s on) for group k.
template <int TT>
__device__ __forceinline__ float2 join(const NormArgs &p, const JoinPlace<TT> &at, const RowRange &r, int64_t s, int k) {
    const float all = static_cast<float>((r.b - r.a) * p.c);
    float v[2] = {0.f, 0.f};
    Pieces<float2>(p, p.part, r, s, k).walk(at, [&](const float2 &w) {
        v[0] += w.x;
        v[1] += w.y;
    });
    at.sums(v);
    return make_float2(v[0] / all, v[1] / all);
}

__global__ void __launch_bounds__(kJoinThreads) norm_back_join(NormArgs p, int64_t per_cta) {
    join_graphs(p, per_cta, p.joined, [&](const auto &at, const RowRange &r, int64_t s, int k) {
        return join(p, at, r, s, k);
    });
}

// grad_gamma and grad_beta of four channels: the teams' sums, 64 interleaved in order.  Of
// the rows behind the batches, the shares', those without a piece were not written.
constexpr int kChannelCols = 4;
template <int TT>
__device__ __forceinline__ void channel_gradients(const NormArgs &p, int64_t c0, float2 (&s_sum)[TT],
                                                  float *__restrict__ grad_gamma, float *__restrict__ grad_beta) {
    constexpr int kLines = TT / kChannelCols;
    const int64_t c = c0 + threadIdx.x % kChannelCols;
    const int line = threadIdx.x / kChannelCols;
    float2 v = make_float2(0.f, 0.f);
    auto add = [&](int64_t row) {
        const float2 w = __ldg(p.channel_part + row * p.f + c);
        v.x += w.x;
        v.y += w.y;
    };
    if (c < p.f) {
#pragma unroll 8
        for (int64_t i = line; i < p.batches; i += kLines) add(i);
#pragma unroll 4
        for (int64_t i = line; i < p.p.shares; i += kLines)
            if (p.pieces[2 * i].a != p.pieces[2 * i].b || p.pieces[2 * i + 1].a != p.pieces[2 * i + 1].b) add(p.batches + i);
    }
    s_sum[threadIdx.x] = v;
    __syncthreads();
#pragma unroll
    for (int o = TT / 2; o >= kChannelCols; o >>= 1) {
        if (threadIdx.x < o) {
            s_sum[threadIdx.x].x += s_sum[threadIdx.x + o].x;
            s_sum[threadIdx.x].y += s_sum[threadIdx.x + o].y;
        }
        __syncthreads();
    }
    if (threadIdx.x < kChannelCols && c < p.f) {
        grad_gamma[c] = s_sum[threadIdx.x].x;
        grad_beta[c] = s_sum[threadIdx.x].y;
    }
}

// The first channel_ctas CTAs add up the channels' gradients, the others take the pieces of
// large graphs once more, a CTA a (share, tile), the last share first.
template <int ACT, int TT, typename XT, typename GT, int VEC, int S>
__global__ void __launch_bounds__(TT, team_ctas(TT, kBackResident))
norm_back_large(NormArgs p, int channel_ctas, float *grad_gamma, float *grad_beta) {
    extern __shared__ __align__(16) char s_all[];
    if (blockIdx.x < channel_ctas) {
        __shared__ float2 s_sum[TT];
        return channel_gradients<TT>(p, static_cast<int64_t>(blockIdx.x) * kChannelCols, s_sum, grad_gamma, grad_beta);
    }
    const Held<XT, VEC, TT> x(s_all);
    const Held<GT, VEC, TT> g(s_all + p.p.held * TT * VEC * sizeof(XT));
    float2 *s_stat = reinterpret_cast<float2 *>(s_all + p.p.held * TT * VEC * (sizeof(XT) + sizeof(GT)));   // [tile's groups]
    const uint32_t back = (blockIdx.x - channel_ctas) / static_cast<uint32_t>(p.p.tiles);
    const int tile = static_cast<int>(blockIdx.x - channel_ctas - back * p.p.tiles);
    const int64_t share = p.p.shares - 1 - back;
    if (no_piece(p, share)) return;
#pragma unroll 1
    for (int slot = 0; slot < 2; ++slot) {
        const Piece piece = p.pieces[share * 2 + slot];
        if (piece.a == piece.b) continue;
        const Place<TT, VEC, S> at(p, tile);
        const int rows = at.rows(p, piece.a, piece.b);
        copy_rows(p, at, x, g, piece.a, rows);
        Column<VEC, S> c;
        c.weights(p, at);
        c.statistics(p, at, piece.graph);
        float2 stat[S];
        joined_statistics<TT>(p, at, piece, p.joined, s_stat, stat,
                              [&](const auto &place, const RowRange &r, int64_t s, int k) { return join(p, place, r, s, k); });
        copies_done();
        float s[2][S];
#pragma unroll
        for (int q = 0; q < S; ++q) {
            s[0][q] = stat[q].x;
            s[1][q] = stat[q].y;
        }
        float slope[VEC];
        c.slopes(slope);
        gradient<ACT>(p, at, c, slope, x, g, rows, piece.a, s);
    }
}

template <int ACT, int TT, typename XT, typename GT, int VEC, int S>
cudaError_t launch_units(const NormArgs &p, cudaStream_t s) {
    using M = Team<TT>;
    const int smem = M::kPerCta * back_bytes(p.p, S, VEC, VEC * static_cast<int>(sizeof(XT) + sizeof(GT)));
    const cudaError_t err = allow_shared(norm_back_units<ACT, TT, XT, GT, VEC, S>, smem);
    if (err != cudaSuccess) return err;
    const int64_t teams = (p.batches + p.p.shares) * p.p.tiles;
    norm_back_units<ACT, TT, XT, GT, VEC, S>
        <<<static_cast<unsigned>((teams + M::kPerCta - 1) / M::kPerCta), M::kThreads, smem, s>>>(p);
    return cudaGetLastError();
}

template <int ACT, int TT, typename XT, typename GT, int VEC, int S>
cudaError_t launch_large(NormArgs p, float *grad_gamma, float *grad_beta, cudaStream_t s) {
    if (p.p.join_apart && p.p.shares > 0) {
        const JoinRange range = join_range(p.p, p.groups);
        norm_back_join<<<range.grid, kJoinThreads, 0, s>>>(p, range.per_cta);
        const cudaError_t launched = cudaGetLastError();
        if (launched != cudaSuccess) return launched;
    }
    set_rows_at_once(p.p, TT);
    p.p.held = static_cast<int>((p.p.share + p.p.rows_at_once - 1) / p.p.rows_at_once);
    if (p.p.shares == 0) p.p.held = 0;                      // channels alone
    const int channel_ctas = grad_gamma ? static_cast<int>((p.f + kChannelCols - 1) / kChannelCols) : 0;
    const int64_t ctas = channel_ctas + p.p.shares * p.p.tiles;
    const int smem = p.p.held * TT * VEC * static_cast<int>(sizeof(XT) + sizeof(GT)) + p.p.tile_groups * static_cast<int>(sizeof(float2));
    const cudaError_t err = allow_shared(norm_back_large<ACT, TT, XT, GT, VEC, S>, smem);
    if (err != cudaSuccess) return err;
    norm_back_large<ACT, TT, XT, GT, VEC, S><<<static_cast<unsigned>(ctas), TT, smem, s>>>(p, channel_ctas, grad_gamma, grad_beta);
    return cudaGetLastError();
}

template <int ACT, typename XT, typename GT, int VEC, int S>
cudaError_t launch_act(const NormArgs &p, float *gg, float *gb, cudaStream_t s) {
    const bool widest = VEC == 1 && p.p.team == 1024;
    cudaError_t err;
    if (widest) err = launch_units<ACT, VEC == 1 ? 1024 : 256, XT, GT, VEC, S>(p, s);
    else if (p.p.team == 32) err = launch_units<ACT, 32, XT, GT, VEC, S>(p, s);
    else if (p.p.team == 128) err = launch_units<ACT, 128, XT, GT, VEC, S>(p, s);
    else err = launch_units<ACT, 256, XT, GT, VEC, S>(p, s);
    if (err != cudaSuccess || (p.p.shares == 0 && !gg)) return err;
    return widest ? launch_large<ACT, VEC == 1 ? 1024 : 256, XT, GT, VEC, S>(p, gg, gb, s)
                  : launch_large<ACT, kLargeTeam, XT, GT, VEC, S>(p, gg, gb, s);
}

template <typename XT, typename GT, int VEC, int S>
cudaError_t launch_team(const NormArgs &p, int act, float *gg, float *gb, cudaStream_t s) {
    switch (act) {
        case kActRelu: return launch_act<kActRelu, XT, GT, VEC, S>(p, gg, gb, s);
        case kActSilu: return launch_act<kActSilu, XT, GT, VEC, S>(p, gg, gb, s);
        case kActGelu: return launch_act<kActGelu, XT, GT, VEC, S>(p, gg, gb, s);
        default: return launch_act<kActNone, XT, GT, VEC, S>(p, gg, gb, s);
    }
}

// S = 1 where a vector lies in one group.
template <typename XT, typename GT>
cudaError_t launch_back(const NormArgs &p, int act, float *gg, float *gb, cudaStream_t s) {
    if (p.p.vec == 1) return launch_team<XT, GT, 1, 1>(p, act, gg, gb, s);
    return p.c % 4 == 0 ? launch_team<XT, GT, 4, 1>(p, act, gg, gb, s) : launch_team<XT, GT, 4, 4>(p, act, gg, gb, s);
}

}  // namespace
}  // namespace tfg
