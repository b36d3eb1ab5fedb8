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

template <int VEC>
struct Column {           // what a thread's channels need
    float mean[VEC], rstd[VEC], gamma[VEC], beta[VEC];

    template <int TT>
    __device__ __forceinline__ void weights(const NormArgs &p, const Place<TT, VEC> &at) {
#pragma unroll
        for (int q = 0; q < VEC; ++q) {
            gamma[q] = at.on && p.gamma ? __ldg(p.gamma + at.c0 + q) : 1.f;
            beta[q] = at.on && p.beta ? __ldg(p.beta + at.c0 + q) : 0.f;
        }
    }
    template <int TT>
    __device__ __forceinline__ void statistics(const NormArgs &p, const Place<TT, VEC> &at, int64_t graph) {
#pragma unroll
        for (int q = 0; q < VEC; ++q) {
            const int64_t i = graph * p.groups + at.group0 + at.grp[q];
            mean[q] = at.on ? __ldg(p.mean_in + i) : 0.f;
            rstd[q] = at.on ? __ldg(p.rstd_in + i) : 0.f;
        }
    }
};

template <int TT, typename XT, typename GT, int VEC, int R>
struct Pair {             // rows of x and of the gradient
    RowVec<XT, VEC> x[R];
    RowVec<GT, VEC> g[R];

    __device__ __forceinline__ void load(const NormArgs &p, const Place<TT, VEC> &at, int64_t a, int64_t b) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int64_t row = a + i * p.p.rows_at_once + at.rl;
            if (at.on && row < b) {
                x[i].load(static_cast<const XT *>(p.x) + row * p.f + at.c0);
                g[i].load(static_cast<const GT *>(p.g) + row * p.f + at.c0);
            }
        }
    }
    __device__ __forceinline__ void next_pass() {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            x[i].renewed();
            g[i].renewed();
        }
    }
    // h and d of vector i
    template <int ACT>
    __device__ __forceinline__ void values(const Column<VEC> &c, int i, float (&h)[VEC], float (&d)[VEC]) const {
        x[i].widen(h);
        g[i].widen(d);
#pragma unroll
        for (int q = 0; q < VEC; ++q) {
            h[q] = (h[q] - c.mean[q]) * c.rstd[q];
            d[q] *= activation_slope<ACT>(fmaf(c.gamma[q], h[q], c.beta[q]));
        }
    }
};

// s[0], s[1]: this thread's sums of gamma d and gamma d h over rows [a, b); weight adds up
// d h and d.
template <int ACT, int TT, typename XT, typename GT, int VEC, int R>
__device__ __forceinline__ void sums(const NormArgs &p, const Place<TT, VEC> &at, const Pair<TT, XT, GT, VEC, R> &v,
                                     const Column<VEC> &c, int64_t a, int64_t b, float (&s)[2][VEC],
                                     float (&weight)[2][VEC]) {
    float dh[VEC] = {}, db[VEC] = {};
#pragma unroll
    for (int i = 0; i < R; ++i) {
        if (!at.on || a + i * p.p.rows_at_once + at.rl >= b) break;
        float h[VEC], d[VEC];
        v.template values<ACT>(c, i, h, d);
#pragma unroll
        for (int q = 0; q < VEC; ++q) {
            dh[q] = fmaf(d[q], h[q], dh[q]);
            db[q] += d[q];
        }
    }
#pragma unroll
    for (int q = 0; q < VEC; ++q) {
        s[0][q] = c.gamma[q] * db[q];
        s[1][q] = c.gamma[q] * dh[q];
        weight[0][q] += dh[q];
        weight[1][q] += db[q];
    }
}

// grad_x of rows [a, b); s1, s2: the sums over M.
template <int ACT, int TT, typename XT, typename GT, int VEC, int R>
__device__ __forceinline__ void gradient(const NormArgs &p, const Place<TT, VEC> &at, const Pair<TT, XT, GT, VEC, R> &v,
                                         const Column<VEC> &c, int64_t a, int64_t b, const float (&s1)[VEC],
                                         const float (&s2)[VEC]) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int64_t row = a + i * p.p.rows_at_once + at.rl;
        if (!at.on || row >= b) break;
        float h[VEC], d[VEC];
        v.template values<ACT>(c, i, h, d);
#pragma unroll
        for (int q = 0; q < VEC; ++q) d[q] = c.rstd[q] * (fmaf(c.gamma[q], d[q], -s1[q]) - h[q] * s2[q]);
        store_vec<VEC>(static_cast<GT *>(p.out) + row * p.f + at.c0, d);
    }
}

template <int ACT, int TT, typename XT, typename GT, int VEC, int R>
__global__ void __launch_bounds__(Team<TT>::kThreads, team_ctas(TT)) norm_back_units(NormArgs p) {
    using M = Team<TT>;
    extern __shared__ __align__(16) float s_all[];
    const int64_t id = static_cast<int64_t>(blockIdx.x) * M::kPerCta + M::index();
    const int64_t chain = id / p.p.tiles;
    const int tile = static_cast<int>(id - chain * p.p.tiles);
    if (chain >= p.chains) return;                          // whole teams
    float *smem = s_all + M::index() * team_floats<2>(p.p.rows_at_once, p.p.cols);
    const Place<TT, VEC> at(p, tile);
    Column<VEC> c;
    c.weights(p, at);
    float weight[2][VEC] = {}, *total[2];
    Pair<TT, XT, GT, VEC, R> v;
    auto one = [&](int64_t graph, int64_t a, int64_t b) {
        v.load(p, at, a, b);
        c.statistics(p, at, graph);
        float s[2][VEC];
        sums<ACT>(p, at, v, c, a, b, s, weight);
        M::sync();                                          // the last unit's sums have been read
        group_sums<TT, VEC, 2>(p, at, s, smem, total);
        v.next_pass();
    };
#pragma unroll 1
    for (int64_t unit = chain; unit < p.graphs + p.p.shares; unit += p.chains) {
        if (unit < p.graphs) {
            bool bad;
            const RowRange r = graph_rows(p.offsets, unit, p.n, bad);
            if (r.a == r.b || r.b - r.a > p.p.cap) continue;
            one(unit, r.a, r.b);
            const float count = static_cast<float>((r.b - r.a) * p.c);
            float s1[VEC], s2[VEC];
#pragma unroll
            for (int q = 0; q < VEC; ++q) {
                s1[q] = total[0][at.grp[q]] / count;
                s2[q] = total[1][at.grp[q]] / count;
            }
            gradient<ACT>(p, at, v, c, r.a, r.b, s1, s2);
            continue;
        }
        const int64_t share = unit - p.graphs;
#pragma unroll 1
        for (int slot = 0; slot < 2; ++slot) {
            const Piece piece = share_piece(p, share, slot);
            if (piece.a == piece.b) continue;
            one(piece.graph, piece.a, piece.b);
            for (int k = M::thread(); k < at.groups; k += TT)
                p.part[(share * 2 + slot) * p.groups + at.group0 + k] = make_float2(total[0][k], total[1][k]);
        }
    }
    if (!p.channel_part) return;
    float *chan[2];
    M::sync();
    channel_sums<TT, VEC, 2>(p, at, weight, smem, chan);
    const int64_t c0 = static_cast<int64_t>(tile) * p.p.cols;
    for (int i = M::thread(); i < p.p.cols && c0 + i < p.f; i += TT)
        p.channel_part[chain * p.f + c0 + i] = make_float2(chan[0][i], chan[1][i]);
}

// Sums over M of the large graph that begins in share blockIdx.x, a warp a group.
constexpr int kBackJoinWarps = 4;
__global__ void __launch_bounds__(kBackJoinWarps * 32) norm_back_join(NormArgs p) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t s = blockIdx.x;
    Piece piece = share_piece(p, s, 0);
    if (piece.a == piece.b || !piece.begins) {
        piece = share_piece(p, s, 1);
        if (piece.a == piece.b) return;
    }
    bool bad;
    const RowRange r = graph_rows(p.offsets, piece.graph, p.n, bad);
    const int64_t s1 = (r.b - 1) / p.p.share;
    const float all = static_cast<float>((r.b - r.a) * p.c);
    for (int k = blockIdx.y * kBackJoinWarps + warp; k < p.groups; k += gridDim.y * kBackJoinWarps) {
        float x = 0.f, y = 0.f;
        for (int64_t i = s + lane; i <= s1; i += 32) {
            const float2 v = p.part[(i * 2 + (r.a > i * p.p.share ? 1 : 0)) * p.groups + k];
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

template <int ACT, int TT, typename XT, typename GT, int VEC, int R>
__global__ void __launch_bounds__(Team<TT>::kThreads, team_ctas(TT)) norm_back_apply(NormArgs p) {
    using M = Team<TT>;
    const int64_t id = static_cast<int64_t>(blockIdx.x) * M::kPerCta + M::index();
    const int64_t back = id / p.p.tiles;
    const int tile = static_cast<int>(id - back * p.p.tiles);
    if (back >= p.p.shares) return;
    const int64_t share = p.p.shares - 1 - back;            // last share first: L2 still holds it
    const Place<TT, VEC> at(p, tile);
    Column<VEC> c;
    c.weights(p, at);
#pragma unroll 1
    for (int slot = 0; slot < 2; ++slot) {
        const Piece piece = share_piece(p, share, slot);
        if (piece.a == piece.b) continue;
        Pair<TT, XT, GT, VEC, R> v;
        v.load(p, at, piece.a, piece.b);
        c.statistics(p, at, piece.graph);
        float s1[VEC], s2[VEC];
#pragma unroll
        for (int q = 0; q < VEC; ++q) {
            const float2 j = at.on ? __ldg(p.joined + piece.first_share * p.groups + at.group0 + at.grp[q]) : make_float2(0.f, 0.f);
            s1[q] = j.x;
            s2[q] = j.y;
        }
        gradient<ACT>(p, at, v, c, piece.a, piece.b, s1, s2);
    }
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

constexpr int kBackVec = 4;

// Teams a tile's units are dealt to: what is resident at once.
int64_t back_chains(const NormPlan &p, int64_t graphs) {
    const int64_t per_sm = p.team == 32 ? 16 : team_ctas(p.team);
    const int64_t at_once = (per_sm * 152 + p.tiles - 1) / p.tiles;
    const int64_t units = graphs + p.shares;
    return units < at_once ? units : at_once;
}

struct BackLayout {       // of the workspace, in float2
    int64_t part, joined, channels;
};
BackLayout back_layout(const NormPlan &p, int64_t graphs, int64_t f, int64_t groups) {
    return {p.shares * 2 * groups, p.shares * groups, back_chains(p, graphs) * f};
}

template <int ACT, int TT, typename XT, typename GT, int VEC>
cudaError_t launch_act(const NormArgs &p, float *grad_gamma, float *grad_beta, cudaStream_t s) {
    using M = Team<TT>;
    constexpr int R = held_vectors(TT, VEC, true);
    const int smem = M::kPerCta * team_floats<2>(p.p.rows_at_once, p.p.cols) * static_cast<int>(sizeof(float));
    auto ctas = [](int64_t teams) { return static_cast<unsigned>((teams + M::kPerCta - 1) / M::kPerCta); };
    norm_back_units<ACT, TT, XT, GT, VEC, R><<<ctas(p.chains * p.p.tiles), M::kThreads, smem, s>>>(p);
    cudaError_t err = cudaGetLastError();
    if (err != cudaSuccess) return err;
    if (p.p.shares > 0) {
        const dim3 join(static_cast<unsigned>(p.p.shares),
                        static_cast<unsigned>(min64((p.groups + kBackJoinWarps - 1) / kBackJoinWarps, 65535)));
        norm_back_join<<<join, kBackJoinWarps * 32, 0, s>>>(p);
        err = cudaGetLastError();
        if (err != cudaSuccess) return err;
        norm_back_apply<ACT, TT, XT, GT, VEC, R><<<ctas(p.p.shares * p.p.tiles), M::kThreads, 0, s>>>(p);
        err = cudaGetLastError();
        if (err != cudaSuccess) return err;
    }
    if (grad_gamma)
        norm_channels<<<static_cast<unsigned>((p.f + 31) / 32), 32 * kChannelRows, 0, s>>>(p.channel_part, p.chains, p.f,
                                                                                          grad_gamma, grad_beta);
    return cudaGetLastError();
}

template <int TT, typename XT, typename GT, int VEC>
cudaError_t launch_back(const NormArgs &p, int act, float *gg, float *gb, cudaStream_t s) {
    switch (act) {
        case kActRelu: return launch_act<kActRelu, TT, XT, GT, VEC>(p, gg, gb, s);
        case kActSilu: return launch_act<kActSilu, TT, XT, GT, VEC>(p, gg, gb, s);
        case kActGelu: return launch_act<kActGelu, TT, XT, GT, VEC>(p, gg, gb, s);
        default: return launch_act<kActNone, TT, XT, GT, VEC>(p, gg, gb, s);
    }
}

template <typename XT, typename GT>
cudaError_t launch_types(const NormArgs &p, int act, float *gg, float *gb, cudaStream_t s) {
    if (p.p.vec == 1) {
        switch (p.p.team) {
            case 32: return launch_back<32, XT, GT, 1>(p, act, gg, gb, s);
            case 128: return launch_back<128, XT, GT, 1>(p, act, gg, gb, s);
            case 256: return launch_back<256, XT, GT, 1>(p, act, gg, gb, s);
            default: return launch_back<1024, XT, GT, 1>(p, act, gg, gb, s);
        }
    }
    switch (p.p.team) {
        case 32: return launch_back<32, XT, GT, kBackVec>(p, act, gg, gb, s);
        case 128: return launch_back<128, XT, GT, kBackVec>(p, act, gg, gb, s);
        default: return launch_back<256, XT, GT, kBackVec>(p, act, gg, gb, s);
    }
}

// Tiles by the wider of the two types: 128 bytes of the gradient or of x.
NormPlan back_plan(int64_t n, int64_t graphs, int64_t f, int64_t c, int elem, bool aligned) {
    return norm_plan(n, graphs, f, c, norm_vec(f, c, kBackVec, aligned), elem, true);
}

}  // namespace

size_t group_norm_backward_workspace_bytes(int64_t n, int64_t graphs, int64_t f, int64_t groups) {
    size_t most = 0;
    for (const int elem : {4, 2}) {
        for (const bool aligned : {true, false}) {
            const BackLayout l = back_layout(back_plan(n, graphs, f, f / groups, elem, aligned), graphs, f, groups);
            const size_t bytes = size_t(l.part + l.joined + l.channels) * sizeof(float2);
            if (bytes > most) most = bytes;
        }
    }
    return most;
}

cudaError_t launch_group_norm_backward(const void *x, int x_dtype, const int64_t *offsets, int64_t n, int64_t graphs,
                                       int64_t f, int64_t groups, const float *gamma, const float *beta,
                                       const float *mean, const float *rstd, int act, const void *g, int g_dtype,
                                       void *grad_x, float *grad_gamma, float *grad_beta, void *ws, cudaStream_t s) {
    const int elem = x_dtype == TFG_BF16 && g_dtype == TFG_BF16 ? 2 : 4;
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
    p.p = back_plan(n, graphs, f, p.c, elem, aligned);
    p.chains = back_chains(p.p, graphs);
    const BackLayout l = back_layout(p.p, graphs, f, groups);
    p.part = static_cast<float2 *>(ws);
    p.joined = p.part + l.part;
    p.channel_part = grad_gamma ? p.joined + l.joined : nullptr;
    if (x_dtype == TFG_BF16)
        return g_dtype == TFG_BF16 ? launch_types<uint16_t, uint16_t>(p, act, grad_gamma, grad_beta, s)
                                   : launch_types<uint16_t, float>(p, act, grad_gamma, grad_beta, s);
    return g_dtype == TFG_BF16 ? launch_types<float, uint16_t>(p, act, grad_gamma, grad_beta, s)
                               : launch_types<float, float>(p, act, grad_gamma, grad_beta, s);
}

}  // namespace tfg
