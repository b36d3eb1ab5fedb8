// Group norm with an activation, backward (group_norm.cuh: the work split).
//
//   h = (x - m) r, y = gamma h + beta, d = g act'(y)
//   grad_beta = sum d, grad_gamma = sum d h                     over all rows
//   s1 = sum gamma d, s2 = sum gamma d h                        over the (graph, group)
//   grad_x = r (gamma d - (s1 + h s2) / M)
//
// The units -- graphs, then shares of the large ones -- of a tile are dealt to a fixed
// number of teams, each of which keeps its columns' sums for gamma and beta in registers
// from unit to unit and leaves them once; a last kernel adds those of all teams in order.
#include "group_norm.cuh"

namespace tfg {
namespace {

#ifndef TFG_BACK_DEPTH
#define TFG_BACK_DEPTH 4
#endif
constexpr int kBackDepth = TFG_BACK_DEPTH;        // rows of x and of the gradient in flight per thread

template <int VEC, int S>
struct Column {           // what a thread's channels need
    float mean[S], rstd[S], gamma[VEC], beta[VEC];

    template <int TT>
    __device__ __forceinline__ void weights(const NormArgs &p, const Place<TT, VEC, S> &at) {
#pragma unroll
        for (int q = 0; q < VEC; ++q) {
            gamma[q] = at.on && p.gamma ? __ldg(p.gamma + at.c0 + q) : 1.f;
            beta[q] = at.on && p.beta ? __ldg(p.beta + at.c0 + q) : 0.f;
        }
    }
    template <int TT>
    __device__ __forceinline__ void statistics(const NormArgs &p, const Place<TT, VEC, S> &at, int64_t graph) {
#pragma unroll
        for (int q = 0; q < S; ++q) {
            const int64_t i = graph * p.groups + at.group0 + at.grp[q];
            mean[q] = at.on ? __ldg(p.mean_in + i) : 0.f;
            rstd[q] = at.on ? __ldg(p.rstd_in + i) : 0.f;
        }
    }
    // h and d of one vector
    template <int ACT, typename XV, typename GV>
    __device__ __forceinline__ void values(const XV &x, const GV &g, float (&h)[VEC], float (&d)[VEC]) const {
        x.widen(h);
        g.widen(d);
#pragma unroll
        for (int q = 0; q < VEC; ++q) {
            h[q] = (h[q] - mean[q / (VEC / S)]) * rstd[q / (VEC / S)];
            d[q] *= activation_slope<ACT>(fmaf(gamma[q], h[q], beta[q]));
        }
    }
};

// Calls each(row vector of x, of the gradient, offset of the row) for this thread's rows of
// [a, b) in order, kBackDepth rows of loads at a time.
template <typename XT, typename GT, int VEC, int TT, int S, typename Each>
__device__ __forceinline__ void for_rows(const NormArgs &p, const Place<TT, VEC, S> &at, int64_t a, int64_t b, Each each) {
    const int rows = at.rows(p, a, b);
    const int64_t step = p.p.rows_at_once * p.f;
    int64_t first = (a + at.rl) * p.f + at.c0;
#pragma unroll 1
    for (int i = 0; i < rows; i += kBackDepth) {
        RowVec<XT, VEC> x[kBackDepth];
        RowVec<GT, VEC> g[kBackDepth];
#pragma unroll
        for (int u = 0; u < kBackDepth; ++u) {
            if (i + u >= rows) continue;
            x[u].load(static_cast<const XT *>(p.x) + first + u * step);
            g[u].load(static_cast<const GT *>(p.g) + first + u * step);
        }
#pragma unroll
        for (int u = 0; u < kBackDepth; ++u) {
            if (i + u >= rows) break;
            each(x[u], g[u], first + u * step);
        }
        first += kBackDepth * step;
    }
}

// Sums of gamma d and gamma d h over rows [a, b) of each group, to every thread for its
// groups; weight adds up this thread's d h and d.
template <int ACT, typename XT, typename GT, int TT, int VEC, int S>
__device__ __forceinline__ void sums(const NormArgs &p, const Place<TT, VEC, S> &at, const Column<VEC, S> &c, int64_t a,
                                     int64_t b, float *smem, int buffer, float (&s)[2][S], float (&weight)[2][VEC]) {
    float dh[VEC] = {}, db[VEC] = {};
    for_rows<XT, GT>(p, at, a, b, [&](const auto &x, const auto &g, int64_t) {
        float h[VEC], d[VEC];
        c.template values<ACT>(x, g, h, d);
#pragma unroll
        for (int q = 0; q < VEC; ++q) {
            dh[q] = fmaf(d[q], h[q], dh[q]);
            db[q] += d[q];
        }
    });
#pragma unroll
    for (int q = 0; q < S; ++q) s[0][q] = s[1][q] = 0.f;
#pragma unroll
    for (int q = 0; q < VEC; ++q) {
        s[0][q / (VEC / S)] += c.gamma[q] * db[q];
        s[1][q / (VEC / S)] += c.gamma[q] * dh[q];
        weight[0][q] += dh[q];
        weight[1][q] += db[q];
    }
    group_sums<TT, VEC, S, 2>(p, at, s, smem, buffer);
}

// grad_x of rows [a, b); s: the sums over M.
template <int ACT, typename XT, typename GT, int TT, int VEC, int S>
__device__ __forceinline__ void gradient(const NormArgs &p, const Place<TT, VEC, S> &at, const Column<VEC, S> &c, int64_t a,
                                         int64_t b, const float (&s)[2][S]) {
    for_rows<XT, GT>(p, at, a, b, [&](const auto &x, const auto &g, int64_t to) {
        float h[VEC], d[VEC];
        c.template values<ACT>(x, g, h, d);
#pragma unroll
        for (int q = 0; q < VEC; ++q) {
            const int k = q / (VEC / S);
            d[q] = c.rstd[k] * (fmaf(c.gamma[q], d[q], -s[0][k]) - h[q] * s[1][k]);
        }
        store_vec<VEC>(static_cast<GT *>(p.out) + to, d);
    });
}

template <int ACT, int TT, typename XT, typename GT, int VEC, int S>
__global__ void __launch_bounds__(Team<TT>::kThreads, team_ctas(TT, TFG_BACK_RESIDENT)) norm_back_units(NormArgs p) {
    using M = Team<TT>;
    extern __shared__ __align__(16) float s_all[];
    const int64_t id = static_cast<int64_t>(blockIdx.x) * M::kPerCta + M::index();
    const int64_t chain = id / p.p.tiles;
    const int tile = static_cast<int>(id - chain * p.p.tiles);
    if (chain >= p.chains) return;                          // whole teams
    float *smem = s_all + M::index() * back_floats(p.p, S, VEC);
    const Place<TT, VEC, S> at(p, tile);
    Column<VEC, S> c;
    c.weights(p, at);
    float weight[2][VEC] = {}, s[2][S];
    int buffer = 0;
#pragma unroll 1
    for (int64_t unit = chain; unit < p.graphs + 2 * p.p.shares; unit += p.chains) {
        Piece rows{0, 0, 0, 0};
        if (unit < p.graphs) {
            bool bad;
            const RowRange r = graph_rows(p.offsets, unit, p.n, bad);
            if (r.b - r.a <= p.p.most) rows = {r.a, r.b, unit, 0};
        } else {
            rows = find_piece(p, (unit - p.graphs) >> 1, (unit - p.graphs) & 1);
            if (tile == 0 && M::thread() == 0) p.pieces[unit - p.graphs] = rows;
        }
        if (rows.a == rows.b) continue;
        c.statistics(p, at, rows.graph);
        sums<ACT, XT, GT>(p, at, c, rows.a, rows.b, smem, buffer, s, weight);
        buffer ^= 1;
        if (unit < p.graphs) {
            const float count = static_cast<float>((rows.b - rows.a) * p.c);
#pragma unroll
            for (int q = 0; q < S; ++q) {
                s[0][q] /= count;
                s[1][q] /= count;
            }
            gradient<ACT, XT, GT>(p, at, c, rows.a, rows.b, s);
        } else {
#pragma unroll
            for (int q = 0; q < S; ++q)
                if (at.writes(p, q)) p.part[(unit - p.graphs) * p.groups + at.group0 + at.grp[q]] = make_float2(s[0][q], s[1][q]);
        }
    }
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
        p.channel_part[chain * p.f + c0 + i] = r;
    }
}

// Sums over M of the large graph that begins in share blockIdx.x, a warp a group.
constexpr int kBackJoinWarps = 4;
__global__ void __launch_bounds__(kBackJoinWarps * 32) norm_back_join(NormArgs p) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t s = blockIdx.x;
    Piece piece = p.pieces[s * 2];
    if (piece.a == piece.b || piece.first_share != s) piece = p.pieces[s * 2 + 1];
    if (piece.a == piece.b || piece.first_share != s) return;
    bool bad;
    const RowRange r = graph_rows(p.offsets, piece.graph, p.n, bad);
    const int64_t s1 = (r.b - 1) / p.p.most;
    const float all = static_cast<float>((r.b - r.a) * p.c);
    for (int k = blockIdx.y * kBackJoinWarps + warp; k < p.groups; k += gridDim.y * kBackJoinWarps) {
        float x = 0.f, y = 0.f;
        for (int64_t i = s + lane; i <= s1; i += 32) {
            const float2 v = p.part[slot_at(p, r.a, i) * p.groups + k];
            x += v.x;
            y += v.y;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            x += lane_xor(x, o);
            y += lane_xor(y, o);
        }
        if (lane == 0) p.joined[s * p.groups + k] = make_float2(x / all, y / all);
    }
}

// The shares' large pieces once more, the last first: L2 still holds them.
template <int ACT, int TT, typename XT, typename GT, int VEC, int S>
__global__ void __launch_bounds__(Team<TT>::kThreads, team_ctas(TT, TFG_BACK_RESIDENT)) norm_back_apply(NormArgs p) {
    using M = Team<TT>;
    const int64_t id = static_cast<int64_t>(blockIdx.x) * M::kPerCta + M::index();
    const int64_t back = id / p.p.tiles;
    const int tile = static_cast<int>(id - back * p.p.tiles);
    if (back >= 2 * p.p.shares) return;
    const Piece piece = p.pieces[2 * p.p.shares - 1 - back];
    if (piece.a == piece.b) return;
    const Place<TT, VEC, S> at(p, tile);
    Column<VEC, S> c;
    c.weights(p, at);
    c.statistics(p, at, piece.graph);
    float s[2][S];
#pragma unroll
    for (int q = 0; q < S; ++q) {
        const float2 j = at.on ? __ldg(p.joined + piece.first_share * p.groups + at.group0 + at.grp[q]) : make_float2(0.f, 0.f);
        s[0][q] = j.x;
        s[1][q] = j.y;
    }
    gradient<ACT, XT, GT>(p, at, c, piece.a, piece.b, s);
}

// grad_gamma and grad_beta: the chains' sums of every channel, 32 interleaved in order.
constexpr int kChannelRows = 32;
__global__ void __launch_bounds__(32 * kChannelRows)
norm_channels(const float2 *__restrict__ part, int64_t chains, int64_t f, float *__restrict__ grad_gamma,
              float *__restrict__ grad_beta) {
    __shared__ float2 s_sum[kChannelRows][33];
    const int lane = threadIdx.x & 31, row = threadIdx.x >> 5;
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 32 + lane;
    float2 v = make_float2(0.f, 0.f);
    if (c < f) {
#pragma unroll 4
        for (int64_t i = row; i < chains; i += kChannelRows) {
            const float2 w = __ldg(part + i * f + c);
            v.x += w.x;
            v.y += w.y;
        }
    }
    s_sum[row][lane] = v;
    __syncthreads();
    v = s_sum[lane][row];                                   // channel `row`, chain `lane`
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        v.x += lane_xor(v.x, o);
        v.y += lane_xor(v.y, o);
    }
    const int64_t to = static_cast<int64_t>(blockIdx.x) * 32 + row;
    if (lane == 0 && to < f) {
        grad_gamma[to] = v.x;
        grad_beta[to] = v.y;
    }
}

// Teams a tile's units are dealt to: what is resident at once.
int64_t back_chains(const NormPlan &p, int64_t graphs) {
    const int64_t per_sm = team_ctas(p.team, TFG_BACK_RESIDENT) * (p.team == 32 ? kWarpTeams : 1);
    const int64_t at_once = (per_sm * 152 + p.tiles - 1) / p.tiles;
    const int64_t units = graphs + 2 * p.shares;
    return units < at_once ? units : at_once;
}

struct BackLayout {       // of the workspace, in bytes
    size_t pieces, part, joined, channels;
    size_t all() const { return pieces + part + joined + channels; }
};
BackLayout back_layout(const NormPlan &p, int64_t graphs, int64_t f, int64_t groups) {
    const size_t shares = size_t(p.shares);
    return {shares * 2 * sizeof(Piece), shares * 2 * size_t(groups) * sizeof(float2), shares * size_t(groups) * sizeof(float2),
            size_t(back_chains(p, graphs) * f) * sizeof(float2)};
}

template <int ACT, int TT, typename XT, typename GT, int VEC, int S>
cudaError_t launch_act(const NormArgs &p, float *grad_gamma, float *grad_beta, cudaStream_t s) {
    using M = Team<TT>;
    const int smem = M::kPerCta * back_floats(p.p, S, VEC) * static_cast<int>(sizeof(float));
    auto ctas = [](int64_t teams) { return static_cast<unsigned>((teams + M::kPerCta - 1) / M::kPerCta); };
    norm_back_units<ACT, TT, XT, GT, VEC, S><<<ctas(p.chains * p.p.tiles), M::kThreads, smem, s>>>(p);
    cudaError_t err = cudaGetLastError();
    if (err != cudaSuccess) return err;
    if (p.p.shares > 0) {
        const dim3 join(static_cast<unsigned>(p.p.shares),
                        static_cast<unsigned>(min64((p.groups + kBackJoinWarps - 1) / kBackJoinWarps, 65535)));
        norm_back_join<<<join, kBackJoinWarps * 32, 0, s>>>(p);
        err = cudaGetLastError();
        if (err != cudaSuccess) return err;
        norm_back_apply<ACT, TT, XT, GT, VEC, S><<<ctas(2 * p.p.shares * p.p.tiles), M::kThreads, 0, s>>>(p);
        err = cudaGetLastError();
        if (err != cudaSuccess) return err;
    }
    if (grad_gamma)
        norm_channels<<<static_cast<unsigned>((p.f + 31) / 32), 32 * kChannelRows, 0, s>>>(p.channel_part, p.chains, p.f,
                                                                                          grad_gamma, grad_beta);
    return cudaGetLastError();
}

template <int TT, typename XT, typename GT, int VEC, int S>
cudaError_t launch_back(const NormArgs &p, int act, float *gg, float *gb, cudaStream_t s) {
    switch (act) {
        case kActRelu: return launch_act<kActRelu, TT, XT, GT, VEC, S>(p, gg, gb, s);
        case kActSilu: return launch_act<kActSilu, TT, XT, GT, VEC, S>(p, gg, gb, s);
        case kActGelu: return launch_act<kActGelu, TT, XT, GT, VEC, S>(p, gg, gb, s);
        default: return launch_act<kActNone, TT, XT, GT, VEC, S>(p, gg, gb, s);
    }
}

template <typename XT, typename GT, int VEC, int S>
cudaError_t launch_team(const NormArgs &p, int act, float *gg, float *gb, cudaStream_t s) {
    if constexpr (VEC == 1) {
        if (p.p.team == 1024) return launch_back<1024, XT, GT, VEC, S>(p, act, gg, gb, s);
    }
    switch (p.p.team) {
        case 32: return launch_back<32, XT, GT, VEC, S>(p, act, gg, gb, s);
        case 128: return launch_back<128, XT, GT, VEC, S>(p, act, gg, gb, s);
        default: return launch_back<256, XT, GT, VEC, S>(p, act, gg, gb, s);
    }
}

NormPlan back_plan(int64_t n, int64_t graphs, int64_t f, int64_t c, bool aligned) {
    return norm_plan(n, graphs, f, c, norm_vec(f, c, 4, aligned));
}

}  // namespace

size_t group_norm_backward_workspace_bytes(int64_t n, int64_t graphs, int64_t f, int64_t groups) {
    size_t most = 0;
    for (const bool aligned : {true, false}) {
        const size_t bytes = back_layout(back_plan(n, graphs, f, f / groups, aligned), graphs, f, groups).all();
        if (bytes > most) most = bytes;
    }
    return most;
}

cudaError_t launch_group_norm_backward(const void *x, int x_dtype, const int64_t *offsets, int64_t n, int64_t graphs,
                                       int64_t f, int64_t groups, const float *gamma, const float *beta,
                                       const float *mean, const float *rstd, int act, const void *g, int g_dtype,
                                       void *grad_x, float *grad_gamma, float *grad_beta, void *ws, cudaStream_t s) {
    const bool aligned = ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(g) |
                           reinterpret_cast<uintptr_t>(grad_x)) & 15) == 0;
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
    p.p = back_plan(n, graphs, f, p.c, aligned);
    p.chains = back_chains(p.p, graphs);
    const BackLayout l = back_layout(p.p, graphs, f, groups);
    char *at = static_cast<char *>(ws);
    p.pieces = reinterpret_cast<Piece *>(at);
    p.part = reinterpret_cast<float2 *>(at + l.pieces);
    p.joined = reinterpret_cast<float2 *>(at + l.pieces + l.part);
    p.channel_part = grad_gamma ? reinterpret_cast<float2 *>(at + l.pieces + l.part + l.joined) : nullptr;
    auto types = [&](auto x_type, auto g_type) {
        using XT = decltype(x_type);
        using GT = decltype(g_type);
        if (p.p.vec == 1) return launch_team<XT, GT, 1, 1>(p, act, grad_gamma, grad_beta, s);
        return p.c % 4 == 0 ? launch_team<XT, GT, 4, 1>(p, act, grad_gamma, grad_beta, s)
                            : launch_team<XT, GT, 4, 4>(p, act, grad_gamma, grad_beta, s);
    };
    if (x_dtype == TFG_BF16)
        return g_dtype == TFG_BF16 ? types(uint16_t{}, uint16_t{}) : types(uint16_t{}, float{});
    return g_dtype == TFG_BF16 ? types(float{}, uint16_t{}) : types(float{}, float{});
}

}  // namespace tfg
