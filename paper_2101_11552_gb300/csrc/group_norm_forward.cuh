// Group norm with an activation, forward: the kernels (group_norm.cuh: the work split).  A
// translation unit for each type of x compiles them.
//
//   m = sum x / M, v = sum (x - m)^2 / M, r = 1 / sqrt(v + eps)    M = n_g * C values
//   y = gamma (x - m) r + beta, out = act(y)
//
// The mean first, then the squares about it.  A sum of n values far from zero is off by a few
// u |m| and so is its mean, as its rounding to fp32 alone is, which h = (x - m) r would take for
// deviations: 1,000 everywhere in five rows of three channels is then h = 0.019, and with a
// spread of 0.01 about 1,000 the h of 800 values are off by up to 0.01.  So the deviations d from the mean as first found are summed too,
// m = that mean + rest with rest = sum d / M, and what is left is a few u of the deviations.  Shares
// of a large graph are joined by the pooled-variance identity, squares about the joint mean =
// squares of the parts + n (mean of the part - joint mean)^2, in the same two steps.  It costs 2
// instructions a value, 1 to 5 % of both directions (1,024 graphs of 110 rows 82.3 -> 85.1 us).
//
// What bounds it: issue slots and latency together, below memory.  1,024 graphs of 110 rows,
// F = 128 fp32, SiLU: 34 us (115 MB, 3.4 TB/s; 30 instructions a value, issue slots 47 % busy
// with 23 % of the warps that a multiprocessor can hold, as room for the largest graph is
// kept for each; and 4 us for a second kernel that finds no large graph).  Half as wide
// tiles, twice the warps: 34.5 us.  41 graphs of 232,965 rows, F = 128 bf16: 48 us (119 MB, 2.5
// TB/s: first pass 21, second read of x 20, the join between them).  300 ragged graphs of
// 19,717 rows, F = 123 fp32 (4-byte loads, GELU): 26 us.  4,096 single rows of 1,024 bf16 in 32
// groups: 17 us.  2,708 rows in one graph, F = 64: 10 us, two launches.
#pragma once

#include "group_norm.cuh"

namespace tfg {
namespace {

// The statistics of a thread's groups: means as -away + rest, squares of the deviations from that.
template <int S>
struct Moments {
    float away[S], rest[S], squares[S];
    __device__ __forceinline__ float mean(int q) const { return rest[q] - away[q]; }
};

// Squares of n values about m + rest, of those about m: rounding may take the difference below
// 0, and an infinity stays (rest^2 may be one too).
__device__ __forceinline__ float centred(float squares, float rest, float n) {
    const float less = fmaf(-rest * n, rest, squares);
    return less >= 0.f ? less : (less < 0.f ? 0.f : squares);
}

// What a first mean is taken relative to, one of the values, so that equal ones deviate by 0; not
// one whose differences from the others, summed, could leave the range of fp32 (2^96 times
// 2^31 values), or that is no number.
__device__ __forceinline__ float pivot_of(float v) { return fabsf(v) < 7.9e28f ? v : 0.f; }

// A thread's groups' first values in row `row`.
template <typename XT, int TT, int VEC, int S>
__device__ __forceinline__ void pivots(const NormArgs &p, const Place<TT, VEC, S> &at, int64_t row, float (&pivot)[S]) {
    const XT *x = static_cast<const XT *>(p.x) + row * p.f;
#pragma unroll
    for (int q = 0; q < S; ++q) {
        float w[1];
        VecLoad<XT, 1>::load(x + static_cast<int64_t>(at.group0 + at.grp[q]) * p.c, w);
        pivot[q] = pivot_of(w[0]);
    }
}

// Of the held rows, whose groups hold `values` values each.
template <int TT, typename XT, int VEC, int S>
__device__ __forceinline__ void statistics(const NormArgs &p, const Place<TT, VEC, S> &at, const Held<XT, VEC, TT> &held,
                                           const float (&pivot)[S], int rows, float values, float *smem, Moments<S> &m) {
    constexpr int kPer = VEC / S;                           // values of a sum in a vector
    const float per_value = 1.f / values;
    float sum[VEC] = {}, s[1][S] = {}, v[2][S] = {}, away[S];
#pragma unroll
    for (int q = 0; q < S; ++q) away[q] = -pivot[q];
#pragma unroll 4
    for (int i = 0; i < rows; ++i) {
        float w[VEC];
        held.widen(i, w);
        add_vec(w, away);
        add_vec(sum, w);
    }
#pragma unroll
    for (int q = 0; q < VEC; ++q) s[0][q / kPer] += sum[q];
    group_sums<TT, VEC, S, 1>(p, at, s, smem, 0);
#pragma unroll
    for (int q = 0; q < S; ++q) m.away[q] = -fmaf(s[0][q], per_value, pivot[q]);
    float squares[VEC] = {};
#pragma unroll
    for (int q = 0; q < VEC; ++q) sum[q] = 0.f;
#pragma unroll 4
    for (int i = 0; i < rows; ++i) {
        float w[VEC];
        held.widen(i, w);
        add_vec(w, m.away);
        add_vec(sum, w);
        fma_vec(squares, w, w, squares);
    }
#pragma unroll
    for (int q = 0; q < VEC; ++q) {
        v[0][q / kPer] += sum[q];
        v[1][q / kPer] += squares[q];
    }
    group_sums<TT, VEC, S, 2>(p, at, v, smem, 1);
#pragma unroll
    for (int q = 0; q < S; ++q) {
        m.rest[q] = v[0][q] * per_value;
        m.squares[q] = centred(v[1][q], m.rest[q], values);
    }
}

template <int ACT, typename OT, typename XT, int VEC, int TT, int S>
__device__ __forceinline__ void apply(const NormArgs &p, const Place<TT, VEC, S> &at, const Held<XT, VEC, TT> &held, int rows,
                                      int64_t a, const Moments<S> &m, const float (&r)[S]) {
    if (rows == 0) return;
    float scale[VEC], shift[VEC];
    channel_weights(p.gamma, at.c0, 1.f, scale);
    channel_weights(p.beta, at.c0, 0.f, shift);
    mul_vec(scale, r);
    float less[S];
#pragma unroll
    for (int q = 0; q < S; ++q) less[q] = -m.rest[q];
    fma_vec(shift, scale, less, shift);
    const int64_t step = p.p.rows_at_once * p.f;
    OT *o = static_cast<OT *>(p.out) + (a + at.rl) * p.f + at.c0;
#pragma unroll 4
    for (int i = 0; i < rows; ++i) {
        float v[VEC];
        held.widen(i, v);
        add_vec(v, m.away);
        fma_vec(v, v, scale, shift);
        activate<ACT>(v);
        store_vec<VEC>(o + i * step, v);
    }
}

template <typename XT, int VEC, int TT, int S>
__device__ __forceinline__ void apply_act(const NormArgs &p, const Place<TT, VEC, S> &at, const Held<XT, VEC, TT> &held,
                                          int rows, int64_t a, int act, bool out_bf16, const Moments<S> &m,
                                          const float (&r)[S]) {
    switch (act + (out_bf16 ? 4 : 0)) {
        case kActNone: return apply<kActNone, float>(p, at, held, rows, a, m, r);
        case kActRelu: return apply<kActRelu, float>(p, at, held, rows, a, m, r);
        case kActSilu: return apply<kActSilu, float>(p, at, held, rows, a, m, r);
        case kActGelu: return apply<kActGelu, float>(p, at, held, rows, a, m, r);
        case 4 + kActNone: return apply<kActNone, uint16_t>(p, at, held, rows, a, m, r);
        case 4 + kActRelu: return apply<kActRelu, uint16_t>(p, at, held, rows, a, m, r);
        case 4 + kActSilu: return apply<kActSilu, uint16_t>(p, at, held, rows, a, m, r);
        default: return apply<kActGelu, uint16_t>(p, at, held, rows, a, m, r);
    }
}

// Units: the graphs, then the shares with their two slots; a team takes a (unit, tile).
template <int TT, typename XT, int VEC, int S>
__global__ void __launch_bounds__(Team<TT>::kThreads, team_ctas(TT, kNormResident)) norm_units(NormArgs p, int act, bool out_bf16) {
    using M = Team<TT>;
    extern __shared__ __align__(16) char s_all[];
    if (p.status_all && blockIdx.x == gridDim.x - 1) return check_offsets(p);
    const uint32_t id = blockIdx.x * M::kPerCta + M::index();
    const int64_t unit = id / static_cast<uint32_t>(p.p.tiles);
    const int tile = static_cast<int>(id - static_cast<uint32_t>(unit) * p.p.tiles);
    if (unit >= p.graphs + p.p.shares) return;              // whole teams
    char *smem = s_all + M::index() * team_bytes(p.p, kForwardBuffers, S, VEC * sizeof(XT));
    const Held<XT, VEC, TT> held(smem + sum_floats(p.p, kForwardBuffers, S) * 4);
    const Place<TT, VEC, S> at(p, tile);
    const int t = M::thread();
    const int64_t share = unit - p.graphs;
    int64_t covered = 0;
#pragma unroll 1
    for (int slot = 0; slot < 2; ++slot) {
        RowRange r;
        if (share < 0) {
            bool bad;
            r = graph_rows(p.offsets, unit, p.n, bad);
            if (bad && tile == 0 && t == 0) set_status(p.status, TFG_ERR_INDEX_RANGE);
            if (r.b - r.a > p.p.most) return;               // large: the shares'
            if (r.a == r.b) {                               // an empty graph has no statistics: zeros
                for (int k = t; k < at.groups; k += TT) {
                    if (p.mean) p.mean[unit * p.groups + at.group0 + k] = 0.f;
                    if (p.rstd) p.rstd[unit * p.groups + at.group0 + k] = 0.f;
                }
                return;
            }
        } else {
            const Piece piece = find_piece(p, share, slot, covered);
            if (tile == 0 && t == 0) p.pieces[share * 2 + slot] = piece;
            if (piece.a == piece.b) continue;
            r = {piece.a, piece.b};
        }
        const int rows = at.rows(p, r.a, r.b);
        const float values = static_cast<float>((r.b - r.a) * p.c);
        held.copy(static_cast<const XT *>(p.x) + (r.a + at.rl) * p.f + at.c0, rows, p.p.rows_at_once * p.f);
        float pivot[S];
        pivots<XT>(p, at, r.a, pivot);
        copies_done();
        Moments<S> m;
        statistics(p, at, held, pivot, rows, values, reinterpret_cast<float *>(smem), m);
        if (share < 0) {
            float rstd[S];
#pragma unroll
            for (int q = 0; q < S; ++q) {
                rstd[q] = rsqrtf(fmaf(m.squares[q], 1.f / values, p.eps));
                if (p.mean && at.writes(p, q)) {
                    p.mean[unit * p.groups + at.group0 + at.grp[q]] = m.mean(q);
                    p.rstd[unit * p.groups + at.group0 + at.grp[q]] = rstd[q];
                }
            }
            return apply_act(p, at, held, rows, r.a, act, out_bf16, m, rstd);
        }
#pragma unroll
        for (int q = 0; q < S; ++q)
            if (at.writes(p, q))
                p.moments[(share * 2 + slot) * p.groups + at.group0 + at.grp[q]] = make_float4(m.away[q], m.rest[q], m.squares[q], values);
    }
}

// Joins the pieces of a large graph (rows r, from share s on) for group k: the mean of the
// pieces' means, relative to the first piece's, then what their distances from it sum up to and
// their squares about it, each in a fixed order.  Gives away, rest and r = 1 / sqrt(v + eps).
template <int TT>
__device__ __forceinline__ float4 join(const NormArgs &p, const JoinPlace<TT> &at, const RowRange &r, int64_t s, int k) {
    const Pieces<float4> pieces(p, p.moments, r, s, k);
    const float all = static_cast<float>((r.b - r.a) * p.c), pivot = pivot_of(pieces.first->x);
    float first[1] = {0.f}, v[2] = {0.f, 0.f};
    pieces.walk(at, [&](const float4 &w) { first[0] = fmaf(w.x - pivot, w.w, first[0]); });
    at.sums(first);
    const float away = pivot + first[0] / all;
    pieces.walk(at, [&](const float4 &w) {
        const float d = (away - w.x) + w.y;
        v[0] = fmaf(d, w.w, v[0]);
        v[1] += fmaf(d * w.w, d, w.z);
    });
    at.sums(v);
    const float rest = v[0] / all;
    return make_float4(away, rest, rsqrtf(centred(v[1], rest, all) / all + p.eps), 0.f);
}

__global__ void __launch_bounds__(kJoinThreads) norm_join(NormArgs p, int64_t per_cta) {
    join_graphs(p, per_cta, p.joined_moments, [&](const auto &at, const RowRange &r, int64_t s, int k) {
        return join(p, at, r, s, k);
    });
}

// The pieces of large graphs once more, a CTA a (share, tile), the last share first.
template <int TT, typename XT, int VEC, int S>
__global__ void __launch_bounds__(TT, team_ctas(TT, kNormResident)) norm_large(NormArgs p, int act, bool out_bf16) {
    extern __shared__ __align__(16) char s_all[];
    const Held<XT, VEC, TT> held(s_all);
    float4 *s_stat = reinterpret_cast<float4 *>(s_all + p.p.held * TT * VEC * sizeof(XT));   // [tile's groups]
    const uint32_t back = blockIdx.x / static_cast<uint32_t>(p.p.tiles);
    const int tile = static_cast<int>(blockIdx.x - back * p.p.tiles);
    const int64_t share = p.p.shares - 1 - back;
    if (no_piece(p, share)) return;
#pragma unroll 1
    for (int slot = 0; slot < 2; ++slot) {
        const Piece piece = p.pieces[share * 2 + slot];
        if (piece.a == piece.b) continue;
        const Place<TT, VEC, S> at(p, tile);
        const int rows = at.rows(p, piece.a, piece.b);
        held.copy(static_cast<const XT *>(p.x) + (piece.a + at.rl) * p.f + at.c0, rows, p.p.rows_at_once * p.f);
        float4 stat[S];
        joined_statistics<TT>(p, at, piece, p.joined_moments, s_stat, stat,
                              [&](const auto &place, const RowRange &r, int64_t s, int k) { return join(p, place, r, s, k); });
        copies_done();
        Moments<S> m;
        float rstd[S];
#pragma unroll
        for (int q = 0; q < S; ++q) {
            m.away[q] = stat[q].x;
            m.rest[q] = stat[q].y;
            rstd[q] = stat[q].z;
        }
        // the share in which the graph begins reports its statistics
        if (p.mean && piece.first_share == share) {
            const int64_t out0 = piece.graph * p.groups + at.group0;
#pragma unroll
            for (int q = 0; q < S; ++q) {
                if (!at.writes(p, q)) continue;
                p.mean[out0 + at.grp[q]] = m.mean(q);
                p.rstd[out0 + at.grp[q]] = rstd[q];
            }
        }
        apply_act(p, at, held, rows, piece.a, act, out_bf16, m, rstd);
    }
}

template <int TT, typename XT, int VEC, int S>
cudaError_t launch_units(const NormArgs &p, int act, bool out_bf16, cudaStream_t s) {
    using M = Team<TT>;
    const int smem = M::kPerCta * team_bytes(p.p, kForwardBuffers, S, VEC * sizeof(XT));
    const cudaError_t err = allow_shared(norm_units<TT, XT, VEC, S>, smem);
    if (err != cudaSuccess) return err;
    const int64_t teams = (p.graphs + p.p.shares) * p.p.tiles;
    const int64_t ctas = (teams + M::kPerCta - 1) / M::kPerCta + (p.status_all ? 1 : 0);
    norm_units<TT, XT, VEC, S><<<static_cast<unsigned>(ctas), M::kThreads, smem, s>>>(p, act, out_bf16);
    return cudaGetLastError();
}

template <int TT, typename XT, int VEC, int S>
cudaError_t launch_large(NormArgs p, int act, bool out_bf16, cudaStream_t s) {
    if (p.p.join_apart) {
        const JoinRange range = join_range(p.p, p.groups);
        norm_join<<<range.grid, kJoinThreads, 0, s>>>(p, range.per_cta);
        const cudaError_t launched = cudaGetLastError();
        if (launched != cudaSuccess) return launched;
    }
    set_rows_at_once(p.p, TT);
    p.p.held = static_cast<int>((p.p.share + p.p.rows_at_once - 1) / p.p.rows_at_once);
    const int smem = p.p.held * TT * VEC * static_cast<int>(sizeof(XT)) + p.p.tile_groups * static_cast<int>(sizeof(float4));
    const cudaError_t err = allow_shared(norm_large<TT, XT, VEC, S>, smem);
    if (err != cudaSuccess) return err;
    norm_large<TT, XT, VEC, S><<<static_cast<unsigned>(p.p.shares * p.p.tiles), TT, smem, s>>>(p, act, out_bf16);
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
}  // namespace tfg
