// Group norm with an activation, forward (group_norm.cuh: the work split).
//
//   m = sum x / M, v = sum (x - m)^2 / M, r = 1 / sqrt(v + eps)    M = n_g * C values
//   y = gamma (x - m) r + beta, out = act(y)
//
// The centred squares are summed in a second pass over the registers, so a mean far from
// zero costs no precision.
#include "group_norm.cuh"

namespace tfg {
namespace {

template <int TT, typename XT, int VEC, int R>
struct Tile {
    using V = VecLoad<XT, VEC>;
    typename V::Raw raw[R];

    // rows [a, b) of this thread's column, b - a <= the team's capacity
    __device__ __forceinline__ void load(const NormArgs &p, const Place<TT, VEC> &at, int64_t a, int64_t b) {
        const XT *x = static_cast<const XT *>(p.x) + at.c0;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int64_t row = a + i * p.p.rows_at_once + at.rl;
            raw[i] = V::zero();
            if (at.on && row < b) raw[i] = V::raw(x + row * p.f);
        }
    }
    __device__ __forceinline__ void next_pass() {
#pragma unroll
        for (int i = 0; i < R; ++i) renew(raw[i]);
    }
};

template <int ACT, int TT, typename XT, int VEC, int R>
__device__ __forceinline__ void apply(const NormArgs &p, const Place<TT, VEC> &at, Tile<TT, XT, VEC, R> &x,
                                      int64_t a, int64_t b, bool out_bf16, const float (&m)[VEC], const float (&r)[VEC]) {
    if (!at.on) return;
    float scale[VEC], shift[VEC];
#pragma unroll
    for (int q = 0; q < VEC; ++q) {
        scale[q] = p.gamma ? __ldg(p.gamma + at.c0 + q) * r[q] : r[q];
        shift[q] = p.beta ? __ldg(p.beta + at.c0 + q) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int64_t row = a + i * p.p.rows_at_once + at.rl;
        if (row >= b) break;
        float v[VEC];
        VecLoad<XT, VEC>::widen(x.raw[i], v);
#pragma unroll
        for (int q = 0; q < VEC; ++q) v[q] = activate<ACT>(fmaf(v[q] - m[q], scale[q], shift[q]));
        if (out_bf16) store_vec<VEC>(static_cast<uint16_t *>(p.out) + row * p.f + at.c0, v);
        else store_vec<VEC>(static_cast<float *>(p.out) + row * p.f + at.c0, v);
    }
}

template <int TT, typename XT, int VEC, int R>
__device__ __forceinline__ void apply_act(const NormArgs &p, const Place<TT, VEC> &at, Tile<TT, XT, VEC, R> &x,
                                          int64_t a, int64_t b, int act, bool out_bf16, const float (&m)[VEC],
                                          const float (&r)[VEC]) {
    switch (act) {
        case kActRelu: return apply<kActRelu>(p, at, x, a, b, out_bf16, m, r);
        case kActSilu: return apply<kActSilu>(p, at, x, a, b, out_bf16, m, r);
        case kActGelu: return apply<kActGelu>(p, at, x, a, b, out_bf16, m, r);
        default: return apply<kActNone>(p, at, x, a, b, out_bf16, m, r);
    }
}

// Means and centred squares of rows [a, b) of the tile in registers: total[k] of group k.
template <int TT, typename XT, int VEC, int R>
__device__ __forceinline__ void statistics(const NormArgs &p, const Place<TT, VEC> &at, Tile<TT, XT, VEC, R> &x,
                                           int64_t a, int64_t b, float *smem, float (&mean)[VEC], float *&squares) {
    const float count = static_cast<float>((b - a) * p.c);
    float v[1][VEC] = {}, *total[1];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        float w[VEC];
        VecLoad<XT, VEC>::widen(x.raw[i], w);               // zeros behind the last row
#pragma unroll
        for (int q = 0; q < VEC; ++q) v[0][q] += w[q];
    }
    group_sums<TT, VEC, 1>(p, at, v, smem, total);
    x.next_pass();
#pragma unroll
    for (int q = 0; q < VEC; ++q) {
        mean[q] = total[0][at.grp[q]] / count;
        v[0][q] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
        if (a + i * p.p.rows_at_once + at.rl >= b) break;
        float w[VEC];
        VecLoad<XT, VEC>::widen(x.raw[i], w);
#pragma unroll
        for (int q = 0; q < VEC; ++q) v[0][q] = fmaf(w[q] - mean[q], w[q] - mean[q], v[0][q]);
    }
    Team<TT>::sync();                                       // the means have been read
    group_sums<TT, VEC, 1>(p, at, v, smem, total);
    x.next_pass();
    squares = total[0];
}

// Units: the graphs, then the shares; a team takes a (unit, tile).
template <int TT, typename XT, int VEC, int R>
__global__ void __launch_bounds__(Team<TT>::kThreads, team_ctas(TT)) norm_units(NormArgs p, int act, bool out_bf16) {
    using M = Team<TT>;
    extern __shared__ __align__(16) float s_all[];
    const int64_t id = static_cast<int64_t>(blockIdx.x) * M::kPerCta + M::index();
    const int64_t unit = id / p.p.tiles;
    const int tile = static_cast<int>(id - unit * p.p.tiles);
    if (unit >= p.graphs + p.p.shares) return;              // whole teams
    float *smem = s_all + M::index() * team_floats<1>(p.p.rows_at_once, p.p.cols);
    const Place<TT, VEC> at(p, tile);
    Tile<TT, XT, VEC, R> x;
    float mean[VEC], *squares;
    const int t = M::thread();
    if (unit < p.graphs) {
        bool bad;
        const RowRange r = graph_rows(p.offsets, unit, p.n, bad);
        if (bad && tile == 0 && t == 0) set_status(p.status, TFG_ERR_INDEX_RANGE);
        if (r.b - r.a > p.p.cap) return;                    // large: the shares'
        const int64_t out0 = unit * p.groups + at.group0;
        if (r.a == r.b) {                                   // an empty graph has no statistics: zeros
            for (int k = t; k < at.groups; k += TT) {
                if (p.mean) p.mean[out0 + k] = 0.f;
                if (p.rstd) p.rstd[out0 + k] = 0.f;
            }
            return;
        }
        x.load(p, at, r.a, r.b);
        statistics(p, at, x, r.a, r.b, smem, mean, squares);
        const float count = static_cast<float>((r.b - r.a) * p.c);
        float rstd[VEC];
#pragma unroll
        for (int q = 0; q < VEC; ++q) {
            rstd[q] = 1.f / sqrtf(squares[at.grp[q]] / count + p.eps);
            if (at.on && at.rl == 0 && (at.sub * VEC + q) % p.c == 0) {    // a group's first channel
                if (p.mean) p.mean[out0 + at.grp[q]] = mean[q];
                if (p.rstd) p.rstd[out0 + at.grp[q]] = rstd[q];
            }
        }
        apply_act(p, at, x, r.a, r.b, act, out_bf16, mean, rstd);
        return;
    }
    const int64_t share = unit - p.graphs;
#pragma unroll 1
    for (int slot = 0; slot < 2; ++slot) {
        const Piece piece = share_piece(p, share, slot);
        if (piece.a == piece.b) continue;
        x.load(p, at, piece.a, piece.b);
        statistics(p, at, x, piece.a, piece.b, smem, mean, squares);
#pragma unroll
        for (int q = 0; q < VEC; ++q)
            if (at.on && at.rl == 0 && (at.sub * VEC + q) % p.c == 0)
                p.part[(share * 2 + slot) * p.groups + at.group0 + at.grp[q]] = make_float2(mean[q], squares[at.grp[q]]);
        M::sync();                                          // before the next slot's sums
    }
}

// Joins the pieces of the large graph that begins in share blockIdx.x, a warp a group:
// the mean of the pieces' means, then their squares about it (the pooled-variance
// identity), each in a fixed order.
constexpr int kJoinWarps = 4;
__global__ void __launch_bounds__(kJoinWarps * 32) norm_join(NormArgs p) {
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
    auto values = [&](int64_t i) {                          // values of the piece in share i
        const int64_t a = i * p.p.share, b = a + p.p.share;
        return static_cast<float>(((b < r.b ? b : r.b) - (a > r.a ? a : r.a)) * p.c);
    };
    for (int k = blockIdx.y * kJoinWarps + warp; k < p.groups; k += gridDim.y * kJoinWarps) {
        auto part = [&](int64_t i) { return p.part[(i * 2 + (r.a > i * p.p.share ? 1 : 0)) * p.groups + k]; };
        float sum = 0.f;
        for (int64_t i = s + lane; i <= s1; i += 32) sum = fmaf(part(i).x, values(i), sum);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += lane_xor(sum, o);
        const float mean = sum / all;
        float squares = 0.f;
        for (int64_t i = s + lane; i <= s1; i += 32) {
            const float2 v = part(i);
            squares += fmaf((v.x - mean) * values(i), v.x - mean, v.y);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) squares += lane_xor(squares, o);
        const float rstd = 1.f / sqrtf(squares / all + p.eps);
        if (lane == 0) {
            p.joined[s * p.groups + k] = make_float2(mean, rstd);
            if (p.mean) p.mean[piece.graph * p.groups + k] = mean;
            if (p.rstd) p.rstd[piece.graph * p.groups + k] = rstd;
        }
    }
}

// The shares' large pieces once more: last share first, whose rows L2 still holds.
template <int TT, typename XT, int VEC, int R>
__global__ void __launch_bounds__(Team<TT>::kThreads, team_ctas(TT)) norm_apply(NormArgs p, int act, bool out_bf16) {
    using M = Team<TT>;
    const int64_t id = static_cast<int64_t>(blockIdx.x) * M::kPerCta + M::index();
    const int64_t back = id / p.p.tiles;
    const int tile = static_cast<int>(id - back * p.p.tiles);
    if (back >= p.p.shares) return;
    const int64_t share = p.p.shares - 1 - back;
    const Place<TT, VEC> at(p, tile);
#pragma unroll 1
    for (int slot = 0; slot < 2; ++slot) {
        const Piece piece = share_piece(p, share, slot);
        if (piece.a == piece.b) continue;
        Tile<TT, XT, VEC, R> x;
        x.load(p, at, piece.a, piece.b);
        float mean[VEC], rstd[VEC];
#pragma unroll
        for (int q = 0; q < VEC; ++q) {
            const float2 j = at.on ? __ldg(p.joined + piece.first_share * p.groups + at.group0 + at.grp[q]) : make_float2(0.f, 0.f);
            mean[q] = j.x;
            rstd[q] = j.y;
        }
        apply_act(p, at, x, piece.a, piece.b, act, out_bf16, mean, rstd);
    }
}

template <int TT, typename XT, int VEC>
cudaError_t launch_norm(const NormArgs &p, int act, bool out_bf16, cudaStream_t s) {
    using M = Team<TT>;
    constexpr int R = held_vectors(TT, VEC, false);
    const int smem = M::kPerCta * team_floats<1>(p.p.rows_at_once, p.p.cols) * static_cast<int>(sizeof(float));
    const int64_t units = (p.graphs + p.p.shares) * p.p.tiles;
    norm_units<TT, XT, VEC, R><<<static_cast<unsigned>((units + M::kPerCta - 1) / M::kPerCta), M::kThreads, smem, s>>>(p, act, out_bf16);
    cudaError_t err = cudaGetLastError();
    if (err != cudaSuccess || p.p.shares == 0) return err;
    const dim3 join(static_cast<unsigned>(p.p.shares), static_cast<unsigned>(min64((p.groups + kJoinWarps - 1) / kJoinWarps, 65535)));
    norm_join<<<join, kJoinWarps * 32, 0, s>>>(p);
    err = cudaGetLastError();
    if (err != cudaSuccess) return err;
    const int64_t again = p.p.shares * p.p.tiles;
    norm_apply<TT, XT, VEC, R><<<static_cast<unsigned>((again + M::kPerCta - 1) / M::kPerCta), M::kThreads, 0, s>>>(p, act, out_bf16);
    return cudaGetLastError();
}

template <typename XT, int VEC>
cudaError_t launch_team(const NormArgs &p, int act, bool out_bf16, cudaStream_t s) {
    if constexpr (VEC == 1) {
        if (p.p.team == 1024) return launch_norm<1024, XT, VEC>(p, act, out_bf16, s);
    }
    switch (p.p.team) {
        case 32: return launch_norm<32, XT, VEC>(p, act, out_bf16, s);
        case 128: return launch_norm<128, XT, VEC>(p, act, out_bf16, s);
        default: return launch_norm<256, XT, VEC>(p, act, out_bf16, s);
    }
}

}  // namespace

// Whether the teams of every type and alignment fit a grid.
bool group_norm_fits(int64_t n, int64_t graphs, int64_t f, int64_t groups) {
    const int64_t c = f / groups;
    for (const int elem : {4, 2}) {
        for (const bool aligned : {true, false}) {
            const NormPlan p = norm_plan(n, graphs, f, c, norm_vec(f, c, 16 / elem, aligned), elem, false);
            const NormPlan q = norm_plan(n, graphs, f, c, norm_vec(f, c, 4, aligned), elem, true);
            if ((graphs + p.shares) * p.tiles > 0x7fffffff || (graphs + q.shares) * q.tiles > 0x7fffffff) return false;
        }
    }
    return true;
}

// Bytes for any type and alignment of the inputs.
size_t group_norm_workspace_bytes(int64_t n, int64_t graphs, int64_t f, int64_t groups) {
    size_t most = 0;
    const int64_t c = f / groups;
    for (const int elem : {4, 2}) {
        for (const bool aligned : {true, false}) {
            const NormPlan p = norm_plan(n, graphs, f, c, norm_vec(f, c, 16 / elem, aligned), elem, false);
            const size_t bytes = size_t(p.shares) * 3 * size_t(groups) * sizeof(float2);
            if (bytes > most) most = bytes;
        }
    }
    return most;
}

cudaError_t launch_group_norm(const void *x, int x_dtype, const int64_t *offsets, int64_t n, int64_t graphs, int64_t f,
                              int64_t groups, const float *gamma, const float *beta, float eps, int act, void *out,
                              int out_dtype, float *mean, float *rstd, void *ws, int32_t *status, cudaStream_t s) {
    const cudaError_t err = cudaMemsetAsync(status, 0, sizeof(int32_t), s);
    if (err != cudaSuccess || graphs == 0) return err;
    const int elem = x_dtype == TFG_BF16 ? 2 : 4;
    const bool aligned = ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(out)) & 15) == 0;
    const int64_t c = f / groups;
    const int vec = norm_vec(f, c, 16 / elem, aligned);
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
    p.status = status;
    p.out = out;
    p.p = norm_plan(n, graphs, f, c, vec, elem, false);
    p.part = static_cast<float2 *>(ws);
    p.joined = p.part + p.p.shares * 2 * groups;
    const bool out_bf16 = out_dtype == TFG_BF16;
    if (x_dtype == TFG_BF16)
        return vec == 8 ? launch_team<uint16_t, 8>(p, act, out_bf16, s) : launch_team<uint16_t, 1>(p, act, out_bf16, s);
    return vec == 4 ? launch_team<float, 4>(p, act, out_bf16, s) : launch_team<float, 1>(p, act, out_bf16, s);
}

}  // namespace tfg
