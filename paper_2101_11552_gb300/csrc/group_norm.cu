// Group norm with an activation, forward (group_norm.cuh: the work split).
//
//   m = sum x / M, v = sum (x - m)^2 / M, r = 1 / sqrt(v + eps)    M = n_g * C values
//   y = gamma (x - m) r + beta, out = act(y)
//
// One pass over a team's rows gives mean and centred squares: a thread takes kDepth rows at
// a time, forms their mean and squares about it in registers, and merges them into its
// running (count, mean, squares) by the pooled-variance identity
//   delta = m_b - m_a, m = m_a + delta n_b / n, q = q_a + q_b + delta^2 n_a n_b / n,
// so a mean far from zero costs no precision; threads, and shares of a large graph, are
// joined by the same identity.
#include "group_norm.cuh"

namespace tfg {
namespace {

#ifndef TFG_NORM_DEPTH
#define TFG_NORM_DEPTH 8
#endif
constexpr int kDepth = TFG_NORM_DEPTH;            // rows in flight per thread

// This thread's count, means and centred squares.
template <int S>
struct Running {
    float n = 0.f, mean[S] = {}, squares[S] = {};
};

template <bool FULL, typename XT, int VEC, int S>
__device__ __forceinline__ void merge(Running<S> &r, const typename VecLoad<XT, VEC>::Raw (&raw)[kDepth], int rows) {
    constexpr int kPer = VEC / S;                           // values of a sum in a vector
    float m[S] = {}, sq[S] = {};
#pragma unroll
    for (int u = 0; u < kDepth; ++u) {
        if (!FULL && u >= rows) break;
        float v[VEC];
        VecLoad<XT, VEC>::widen(raw[u], v);
#pragma unroll
        for (int q = 0; q < VEC; ++q) m[q / kPer] += v[q];
    }
    const float n = static_cast<float>((FULL ? kDepth : rows) * kPer);
#pragma unroll
    for (int q = 0; q < S; ++q) m[q] = FULL ? m[q] * (1.f / (kDepth * kPer)) : m[q] / n;
#pragma unroll
    for (int u = 0; u < kDepth; ++u) {
        if (!FULL && u >= rows) break;
        float v[VEC];
        VecLoad<XT, VEC>::widen(raw[u], v);
#pragma unroll
        for (int q = 0; q < VEC; ++q) sq[q / kPer] = fmaf(v[q] - m[q / kPer], v[q] - m[q / kPer], sq[q / kPer]);
    }
    const float share = __fdividef(n, r.n + n);             // 1 for the first rows: exact
#pragma unroll
    for (int q = 0; q < S; ++q) {
        const float delta = m[q] - r.mean[q];
        r.mean[q] = fmaf(delta, share, r.mean[q]);
        r.squares[q] += fmaf(delta * delta, r.n * share, sq[q]);
    }
    r.n += n;
}

// Means and centred squares of rows [a, b), to every thread for its groups.
template <int TT, typename XT, int VEC, int S>
__device__ __forceinline__ void statistics(const NormArgs &p, const Place<TT, VEC, S> &at, int64_t a, int64_t b, float *smem,
                                           float (&mean)[S], float (&squares)[S]) {
    using V = VecLoad<XT, VEC>;
    Running<S> r;
    const int rows = at.rows(p, a, b);
    const XT *x = static_cast<const XT *>(p.x) + (a + at.rl) * p.f + at.c0;
    const int64_t step = p.p.rows_at_once * p.f;
    int i = 0;
#pragma unroll 1
    for (; i + kDepth <= rows; i += kDepth) {
        typename V::Raw raw[kDepth];
#pragma unroll
        for (int u = 0; u < kDepth; ++u) raw[u] = V::raw(x + u * step);
        x += kDepth * step;
        merge<true, XT, VEC, S>(r, raw, kDepth);
    }
    if (i < rows) {
        typename V::Raw raw[kDepth];
#pragma unroll
        for (int u = 0; u < kDepth; ++u)
            if (i + u < rows) raw[u] = V::raw(x + u * step);
        merge<false, XT, VEC, S>(r, raw, rows - i);
    }
    const float count = static_cast<float>((b - a) * p.c);
    float v[1][S];
#pragma unroll
    for (int q = 0; q < S; ++q) v[0][q] = r.n * r.mean[q];
    group_sums<TT, VEC, S, 1>(p, at, v, smem, 0);
#pragma unroll
    for (int q = 0; q < S; ++q) {
        mean[q] = v[0][q] / count;
        const float d = r.mean[q] - mean[q];
        v[0][q] = r.n > 0.f ? fmaf(d * d, r.n, r.squares[q]) : 0.f;
    }
    group_sums<TT, VEC, S, 1>(p, at, v, smem, 1);
#pragma unroll
    for (int q = 0; q < S; ++q) squares[q] = v[0][q];
}

template <int ACT, typename XT, typename OT, int VEC, int TT, int S>
__device__ __forceinline__ void apply(const NormArgs &p, const Place<TT, VEC, S> &at, int64_t a, int64_t b,
                                      const float (&m)[S], const float (&r)[S]) {
    using V = VecLoad<XT, VEC>;
    constexpr int kPer = VEC / S;
    const int rows = at.rows(p, a, b);
    if (rows == 0) return;
    const float *gamma = p.gamma, *beta = p.beta;
    float scale[VEC], shift[VEC];
#pragma unroll
    for (int q = 0; q < VEC; ++q) {
        scale[q] = gamma ? __ldg(gamma + at.c0 + q) * r[q / kPer] : r[q / kPer];
        shift[q] = beta ? __ldg(beta + at.c0 + q) : 0.f;
    }
    const int64_t first = (a + at.rl) * p.f + at.c0, step = p.p.rows_at_once * p.f;
    const XT *x = static_cast<const XT *>(p.x) + first;
    OT *o = static_cast<OT *>(p.out) + first;
#pragma unroll 1
    for (int i = 0; i < rows; i += kDepth) {
        typename V::Raw raw[kDepth];
#pragma unroll
        for (int u = 0; u < kDepth; ++u)
            if (i + u < rows) raw[u] = V::raw(x + u * step);
#pragma unroll
        for (int u = 0; u < kDepth; ++u) {
            if (i + u >= rows) break;
            float v[VEC];
            V::widen(raw[u], v);
#pragma unroll
            for (int q = 0; q < VEC; ++q) v[q] = activate<ACT>(fmaf(v[q] - m[q / kPer], scale[q], shift[q]));
            store_vec<VEC>(o + u * step, v);
        }
        x += kDepth * step;
        o += kDepth * step;
    }
}

template <typename XT, int VEC, int TT, int S>
__device__ __forceinline__ void apply_act(const NormArgs &p, const Place<TT, VEC, S> &at, int64_t a, int64_t b, int act,
                                          bool out_bf16, const float (&m)[S], const float (&r)[S]) {
    switch (act + (out_bf16 ? 4 : 0)) {
        case kActNone: return apply<kActNone, XT, float>(p, at, a, b, m, r);
        case kActRelu: return apply<kActRelu, XT, float>(p, at, a, b, m, r);
        case kActSilu: return apply<kActSilu, XT, float>(p, at, a, b, m, r);
        case kActGelu: return apply<kActGelu, XT, float>(p, at, a, b, m, r);
        case 4 + kActNone: return apply<kActNone, XT, uint16_t>(p, at, a, b, m, r);
        case 4 + kActRelu: return apply<kActRelu, XT, uint16_t>(p, at, a, b, m, r);
        case 4 + kActSilu: return apply<kActSilu, XT, uint16_t>(p, at, a, b, m, r);
        default: return apply<kActGelu, XT, uint16_t>(p, at, a, b, m, r);
    }
}

// Units: the graphs, then the two slots of every share; a team takes a (unit, tile).
template <int TT, typename XT, int VEC, int S>
__global__ void __launch_bounds__(Team<TT>::kThreads, team_ctas(TT, TFG_NORM_RESIDENT)) norm_units(NormArgs p, int act, bool out_bf16) {
    using M = Team<TT>;
    extern __shared__ __align__(16) float s_all[];
    if (p.status_all && blockIdx.x == gridDim.x - 1) return check_offsets(p);
    const uint32_t id = blockIdx.x * M::kPerCta + M::index();
    const int64_t unit = id / static_cast<uint32_t>(p.p.tiles);
    const int tile = static_cast<int>(id - static_cast<uint32_t>(unit) * p.p.tiles);
    if (unit >= p.graphs + 2 * p.p.shares) return;          // whole teams
    float *smem = s_all + M::index() * team_floats<1>(p.p, S);
    const Place<TT, VEC, S> at(p, tile);
    float mean[S], squares[S];
    const int t = M::thread();
    const int64_t slot = unit - p.graphs;                   // 2 * share + slot
    RowRange r;
    if (slot < 0) {
        bool bad;
        r = graph_rows(p.offsets, unit, p.n, bad);
        if (bad && tile == 0 && t == 0) set_status(p.status, TFG_ERR_INDEX_RANGE);
        if (r.b - r.a > p.p.most) return;                   // large: the shares'
    } else {
        const Piece piece = find_piece(p, slot >> 1, slot & 1);
        if (tile == 0 && t == 0) p.pieces[slot] = piece;
        if (piece.a == piece.b) return;
        r = {piece.a, piece.b};
    }
    const int64_t out0 = unit * p.groups + at.group0;
    if (r.a == r.b) {                                       // an empty graph has no statistics: zeros
        for (int k = t; k < at.groups; k += TT) {
            if (p.mean) p.mean[out0 + k] = 0.f;
            if (p.rstd) p.rstd[out0 + k] = 0.f;
        }
        return;
    }
    statistics<TT, XT>(p, at, r.a, r.b, smem, mean, squares);
    if (slot >= 0) {
#pragma unroll
        for (int q = 0; q < S; ++q)
            if (at.writes(p, q)) p.part[slot * p.groups + at.group0 + at.grp[q]] = make_float2(mean[q], squares[q]);
        return;
    }
    const float count = static_cast<float>((r.b - r.a) * p.c);
    float rstd[S];
#pragma unroll
    for (int q = 0; q < S; ++q) {
        rstd[q] = 1.f / sqrtf(squares[q] / count + p.eps);
        if (p.mean && at.writes(p, q)) {
            p.mean[out0 + at.grp[q]] = mean[q];
            p.rstd[out0 + at.grp[q]] = rstd[q];
        }
    }
    apply_act<XT>(p, at, r.a, r.b, act, out_bf16, mean, rstd);
}

// Joins the pieces of a large graph (rows r, from share s on) for group k, by a warp: the
// mean of the pieces' means, then their squares about it, each in a fixed order.
__device__ __forceinline__ float2 join(const NormArgs &p, const RowRange &r, int64_t s, int k) {
    const int lane = threadIdx.x & 31;
    const int64_t s1 = (r.b - 1) / p.p.share;
    const float all = static_cast<float>((r.b - r.a) * p.c);
    auto part = [&](int64_t i) { return p.part[slot_at(p, r.a, i) * p.groups + k]; };
    float sum = 0.f;
#pragma unroll 4
    for (int64_t i = s + lane; i <= s1; i += 32) sum = fmaf(part(i).x, piece_values(p, r, i), sum);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += lane_xor(sum, o);
    const float mean = sum / all;
    float squares = 0.f;
#pragma unroll 4
    for (int64_t i = s + lane; i <= s1; i += 32) {
        const float2 v = part(i);
        squares += fmaf((v.x - mean) * piece_values(p, r, i), v.x - mean, v.y);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) squares += lane_xor(squares, o);
    return make_float2(mean, 1.f / sqrtf(squares / all + p.eps));
}

// join_apart: the large graph that begins in share blockIdx.x, a warp a group.
constexpr int kJoinWarps = 4;
__global__ void __launch_bounds__(kJoinWarps * 32) norm_join(NormArgs p) {
    const int64_t s = blockIdx.x;
    Piece piece = p.pieces[s * 2];
    if (piece.a == piece.b || piece.first_share != s) piece = p.pieces[s * 2 + 1];
    if (piece.a == piece.b || piece.first_share != s) return;
    bool bad;
    const RowRange r = graph_rows(p.offsets, piece.graph, p.n, bad);
    for (int k = blockIdx.y * kJoinWarps + (threadIdx.x >> 5); k < p.groups; k += gridDim.y * kJoinWarps) {
        const float2 v = join(p, r, s, k);
        if ((threadIdx.x & 31) == 0) p.joined[s * p.groups + k] = v;
    }
}

// The pieces of large graphs once more, a CTA a (slot, tile), the last slot first.
template <int TT, typename XT, int VEC, int S>
__global__ void __launch_bounds__(TT, team_ctas(TT, TFG_NORM_RESIDENT)) norm_large(NormArgs p, int act, bool out_bf16) {
    extern __shared__ __align__(16) float s_all[];
    float2 *s_stat = reinterpret_cast<float2 *>(s_all);    // [tile's groups]
    const int64_t back = blockIdx.x / static_cast<uint32_t>(p.p.tiles);
    const int tile = static_cast<int>(blockIdx.x - static_cast<uint32_t>(back) * p.p.tiles);
    const Piece piece = p.pieces[2 * p.p.shares - 1 - back];
    if (piece.a == piece.b) return;
    const Place<TT, VEC, S> at(p, tile);
    joined_statistics<TT>(p, at, piece, s_stat, join);
    float mean[S], rstd[S];
#pragma unroll
    for (int q = 0; q < S; ++q) {
        const float2 v = s_stat[at.grp[q]];
        mean[q] = v.x;
        rstd[q] = v.y;
    }
    // the share in which the graph begins reports its statistics
    if (p.mean && piece.a < (piece.first_share + 1) * p.p.share) {
        const int64_t out0 = piece.graph * p.groups + at.group0;
#pragma unroll
        for (int q = 0; q < S; ++q) {
            if (!at.writes(p, q)) continue;
            p.mean[out0 + at.grp[q]] = mean[q];
            p.rstd[out0 + at.grp[q]] = rstd[q];
        }
    }
    apply_act<XT>(p, at, piece.a, piece.b, act, out_bf16, mean, rstd);
}

template <int TT, typename XT, int VEC, int S>
cudaError_t launch_units(const NormArgs &p, int act, bool out_bf16, cudaStream_t s) {
    using M = Team<TT>;
    const int smem = M::kPerCta * team_floats<1>(p.p, S) * static_cast<int>(sizeof(float));
    const int64_t teams = (p.graphs + 2 * p.p.shares) * p.p.tiles;
    const int64_t ctas = (teams + M::kPerCta - 1) / M::kPerCta + (p.status_all ? 1 : 0);
    norm_units<TT, XT, VEC, S><<<static_cast<unsigned>(ctas), M::kThreads, smem, s>>>(p, act, out_bf16);
    return cudaGetLastError();
}

template <int TT, typename XT, int VEC, int S>
cudaError_t launch_large(NormArgs p, int act, bool out_bf16, cudaStream_t s) {
    if (p.p.join_apart) {
        const dim3 grid(static_cast<unsigned>(p.p.shares), static_cast<unsigned>(min64((p.groups + kJoinWarps - 1) / kJoinWarps, 65535)));
        norm_join<<<grid, kJoinWarps * 32, 0, s>>>(p);
        const cudaError_t err = cudaGetLastError();
        if (err != cudaSuccess) return err;
    }
    p.p.rows_at_once = TT / p.p.row_vecs;
    const int smem = p.p.tile_groups * static_cast<int>(sizeof(float2));
    norm_large<TT, XT, VEC, S><<<static_cast<unsigned>(2 * p.p.shares * p.p.tiles), TT, smem, s>>>(p, act, out_bf16);
    return cudaGetLastError();
}

template <typename XT, int VEC, int S>
cudaError_t launch_team(const NormArgs &p, int act, bool out_bf16, cudaStream_t s) {
    const bool widest = VEC == 1 && p.p.team == 1024;
    cudaError_t err;
    if (widest) err = launch_units<VEC == 1 ? 1024 : 256, XT, VEC, S>(p, act, out_bf16, s);
    else if (p.p.team == 32) err = launch_units<32, XT, VEC, S>(p, act, out_bf16, s);
    else if (p.p.team == 128) err = launch_units<128, XT, VEC, S>(p, act, out_bf16, s);
    else err = launch_units<256, XT, VEC, S>(p, act, out_bf16, s);
    if (err != cudaSuccess || p.p.shares == 0) return err;
    return widest ? launch_large<VEC == 1 ? 1024 : 256, XT, VEC, S>(p, act, out_bf16, s)
                  : launch_large<kLargeTeam, XT, VEC, S>(p, act, out_bf16, s);
}

// S = 1 where a vector lies in one group.
template <typename XT>
cudaError_t launch_vec(const NormArgs &p, int act, bool out_bf16, cudaStream_t s) {
    if constexpr (sizeof(XT) == 2) {
        if (p.p.vec == 8) return launch_team<XT, 8, 1>(p, act, out_bf16, s);
    }
    if (p.p.vec == 1) return launch_team<XT, 1, 1>(p, act, out_bf16, s);
    return p.c % 4 == 0 ? launch_team<XT, 4, 1>(p, act, out_bf16, s) : launch_team<XT, 4, 4>(p, act, out_bf16, s);
}

}  // namespace

// Whether the teams of every type and alignment fit a grid.
bool group_norm_fits(int64_t n, int64_t graphs, int64_t f, int64_t groups) {
    const int64_t c = f / groups;
    for (const int vec : {4, 8, 1}) {
        const NormPlan p = norm_plan(n, graphs, f, c, norm_vec(f, c, vec, vec > 1));
        if ((graphs + 2 * p.shares) * p.tiles > 0x7fffffff) return false;
    }
    return true;
}

// Bytes for any type and alignment of the inputs.
size_t group_norm_workspace_bytes(int64_t n, int64_t graphs, int64_t f, int64_t groups) {
    size_t most = 0;
    const int64_t c = f / groups;
    for (const int vec : {4, 8, 1}) {
        const NormPlan p = norm_plan(n, graphs, f, c, norm_vec(f, c, vec, vec > 1));
        const size_t bytes = size_t(p.shares) * (2 * sizeof(Piece) + 3 * size_t(groups) * sizeof(float2));
        if (bytes > most) most = bytes;
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
    const bool aligned = ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(out)) & 15) == 0;
    const int64_t c = f / groups;
    const int vec = norm_vec(f, c, x_dtype == TFG_BF16 ? 8 : 4, aligned);
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
    p.p = norm_plan(n, graphs, f, c, vec);
    p.pieces = static_cast<Piece *>(ws);
    p.part = reinterpret_cast<float2 *>(p.pieces + 2 * p.p.shares);
    p.joined = p.part + p.p.shares * 2 * groups;
    const bool out_bf16 = out_dtype == TFG_BF16;
    return x_dtype == TFG_BF16 ? launch_vec<uint16_t>(p, act, out_bf16, s) : launch_vec<float>(p, act, out_bf16, s);
}

}  // namespace tfg
