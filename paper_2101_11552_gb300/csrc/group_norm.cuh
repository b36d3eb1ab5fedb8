// Group norm with an activation over the graphs of a batch, channels last: what the
// forward (group_norm.cu) and the backward (group_norm_backward.cu) share.
//
// Graph g holds the rows node_offsets[g] .. node_offsets[g + 1] - 1 of x [N, F] (the
// reindexing trick of tf_geometric, Section 2.1.1, keeps a graph's nodes together), the
// F channels fall into groups of C, and statistics are taken over the n_g * C values of
// a (graph, group).
//
// Work split.  A team of threads (a warp, or a CTA) takes the rows of one graph and a
// tile of channels -- whole groups -- at once: every thread keeps the vectors of one
// column of the tile in registers, so that x is read from memory once although mean and
// centred squares are two passes.  A graph of more rows than a team holds ("large") is
// cut along a grid of row shares over all rows; the teams of its shares write partial
// statistics, a second kernel joins them in a fixed order, and a third one reads the
// shares again and applies them.  A share is no longer than what a team holds, so it
// meets at most two large graphs: one that covers its first row (slot 0) and one that
// begins behind it and runs past its end (slot 1).  Whether there are large graphs only
// the device knows; the host leaves the two later kernels out where all rows together fit
// a team.
#pragma once

#include <cuda_bf16.h>

#include "widen.cuh"

namespace tfg {
namespace {

constexpr int kActNone = TFG_ACT_NONE, kActRelu = TFG_ACT_RELU, kActSilu = TFG_ACT_SILU, kActGelu = TFG_ACT_GELU;

// Activations in fp32.  exp and erf are the CUDA math library's; the quotient of the
// sigmoid is __fdividef (2 ulp; 0 where the divisor passes 2^126, where y e^y is below
// 1e-36 anyway).  1 + erf leaves the gelu an absolute error of about |y| 2^-24 for
// negative y.
__device__ __forceinline__ float sigmoid_of(float y) { return __fdividef(1.f, 1.f + expf(-y)); }
template <int ACT>
__device__ __forceinline__ float activate(float y) {
    if constexpr (ACT == kActRelu) return y <= 0.f ? 0.f : y;      // a NaN stays
    else if constexpr (ACT == kActSilu) return __fdividef(y, 1.f + expf(-y));
    else if constexpr (ACT == kActGelu) return 0.5f * y * (1.f + erff(y * 0.70710678118654752f));
    else return y;
}
template <int ACT>
__device__ __forceinline__ float activation_slope(float y) {
    if constexpr (ACT == kActRelu) return y > 0.f ? 1.f : (y <= 0.f ? 0.f : y);
    else if constexpr (ACT == kActSilu) {
        const float p = sigmoid_of(y);
        return p * fmaf(y, 1.f - p, 1.f);
    } else if constexpr (ACT == kActGelu) {
        const float d = 0.39894228040143268f * expf(-0.5f * y * y);
        return fmaf(y, d, 0.5f * (1.f + erff(y * 0.70710678118654752f)));
    } else return 1.f;
}

// Geometry of a launch (see norm_plan).
struct NormPlan {
    int vec;              // values of a thread's vector
    int team;             // threads of a team
    int held;             // vectors a thread holds
    int row_vecs;         // vectors of a tile's row
    int cols;             // channels of a tile
    int tiles;
    int rows_at_once;     // rows a team reads at once
    int64_t cap;          // rows a team holds
    int64_t share;        // rows of a share, at most cap
    int64_t shares;       // 0: no graph can be large
};

constexpr int kNormTeamThreads = 128;             // threads of a CTA of warp teams
// Resident CTAs asked for: 128 registers a thread (64 in teams of 1,024).
constexpr int team_ctas(int team) { return team == 1024 ? 1 : (team == 256 ? 2 : 4); }

struct NormArgs {
    const void *x;
    const int64_t *offsets;
    int64_t n, graphs, f;
    int groups, c;                                // groups of c channels
    const float *gamma, *beta;
    float eps;
    float *mean, *rstd;                           // [graphs, groups]
    int32_t *status;
    void *out;
    const void *g;                                // backward: dL/dout
    float2 *part;                                 // [share][slot][group]
    float2 *joined;                               // [share of the graph's first row][group]
    const float *mean_in, *rstd_in;               // backward: the forward's statistics
    float2 *channel_part;                         // backward: [chain][F], sums for gamma and beta
    int64_t chains;                               // backward: teams a tile's units are dealt to
    NormPlan p;
};

// ---- rows of graphs and shares ------------------------------------------------------
struct RowRange {
    int64_t a, b;
};

// The rows of a graph, inside [0, n) whatever the offsets say; bad: they say otherwise.
__device__ __forceinline__ RowRange graph_rows(const int64_t *offsets, int64_t g, int64_t n, bool &bad) {
    const int64_t o0 = __ldg(offsets + g), o1 = __ldg(offsets + g + 1);
    bad = o0 < 0 || o1 < o0 || o1 > n;
    RowRange r;
    r.a = o0 < 0 ? 0 : (o0 > n ? n : o0);
    r.b = o1 < r.a ? r.a : (o1 > n ? n : o1);
    return r;
}

// Last graph that begins at or before row r, -1 if there is none; by the whole warp, 32
// probes a round.
__device__ __forceinline__ int64_t warp_graph_at(const int64_t *offsets, int64_t graphs, int64_t r) {
    const int lane = threadIdx.x & 31;
    int64_t lo = -1, hi = graphs - 1;
    while (lo < hi) {
        const int64_t step = (hi - lo + 31) / 32;
        const int64_t at = lo + (lane + 1) * step;
        const bool le = at <= hi && __ldg(offsets + at) <= r;
        const int c = __popc(lane_ballot(le));
        const int64_t top = lo + (c + 1) * step - 1;
        lo += c * step;
        hi = top < hi ? top : hi;
    }
    return lo;
}

// The piece of a large graph that share s holds in a slot; empty if there is none.
struct Piece {
    int64_t a, b;         // rows
    int64_t graph, first_share;
    bool begins;          // the graph's first row is here
};
__device__ __forceinline__ Piece share_piece(const NormArgs &a, int64_t s, int slot) {
    const int64_t r0 = s * a.p.share, r1 = min64(a.n, r0 + a.p.share);
    Piece p{0, 0, 0, 0, false};
    const int64_t g = warp_graph_at(a.offsets, a.graphs, slot == 0 ? r0 : r1 - 1);
    if (g < 0) return p;
    bool bad;
    const RowRange r = graph_rows(a.offsets, g, a.n, bad);
    if (r.b - r.a <= a.p.cap || r.b <= r0 || (slot == 1) != (r.a > r0)) return p;
    p.a = r.a > r0 ? r.a : r0;
    p.b = r.b < r1 ? r.b : r1;
    if (p.b < p.a) p.b = p.a;
    p.graph = g;
    p.first_share = r.a / a.p.share;
    p.begins = r.a >= r0;
    return p;
}

// ---- a team -------------------------------------------------------------------------
// TT threads: a warp of its own shared memory in a CTA of four, or a whole CTA.
template <int TT>
struct Team {
    static constexpr int kPerCta = TT == 32 ? kNormTeamThreads / 32 : 1;
    static constexpr int kThreads = TT * kPerCta;
    static __device__ __forceinline__ int index() { return TT == 32 ? threadIdx.x / 32 : 0; }
    static __device__ __forceinline__ int thread() { return TT == 32 ? threadIdx.x & 31 : threadIdx.x; }
    static __device__ __forceinline__ void sync() {
        if constexpr (TT == 32) __syncwarp();
        else __syncthreads();
    }
};

// Shared memory of a team: sums of the row lanes, of the channels, of the groups, each for
// NS sums.
template <int NS>
__host__ __device__ constexpr int team_floats(int rows_at_once, int cols) {
    return NS * (rows_at_once * cols + 2 * cols);
}

// Place of a thread in its team's tile.
template <int TT, int VEC>
struct Place {
    int sub, rl;          // vector of the row, row
    int64_t c0;           // first channel
    bool on;
    int groups, group0;   // whole groups of the tile
    int grp[VEC];         // the channels' groups, relative to the tile's first

    __device__ __forceinline__ Place(const NormArgs &a, int tile) {
        const int t = Team<TT>::thread();
        rl = t / a.p.row_vecs;
        sub = t - rl * a.p.row_vecs;
        c0 = static_cast<int64_t>(tile) * a.p.cols + sub * VEC;
        on = rl < a.p.rows_at_once && c0 < a.f;
        group0 = static_cast<int>(static_cast<int64_t>(tile) * a.p.cols / a.c);
        const int64_t left = a.f - static_cast<int64_t>(tile) * a.p.cols;
        groups = static_cast<int>(min64(a.p.cols, left) / a.c);
#pragma unroll
        for (int q = 0; q < VEC; ++q) grp[q] = on ? (sub * VEC + q) / a.c : 0;
    }
};

// Sums over the rows of the tile: v[s] holds this thread's sums of its channels, the
// returned array s the team's of every channel.  Collective over the team, which has to
// pass a barrier before the next sums overwrite these.
template <int TT, int VEC, int NS>
__device__ __forceinline__ void channel_sums(const NormArgs &a, const Place<TT, VEC> &at, const float (&v)[NS][VEC],
                                             float *smem, float *(&chan)[NS]) {
    using M = Team<TT>;
    const int t = M::thread();
    const int cols = a.p.cols, rows = a.p.rows_at_once;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        float *red = smem + s * (rows + 2) * cols;
        chan[s] = red + rows * cols;
        if (t < rows * a.p.row_vecs) {
#pragma unroll
            for (int q = 0; q < VEC; ++q) red[at.rl * cols + at.sub * VEC + q] = at.on ? v[s][q] : 0.f;
        }
    }
    M::sync();
    for (int i = t; i < cols; i += TT) {
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const float *red = smem + s * (rows + 2) * cols + i;
            float r = 0.f;
            for (int j = 0; j < rows; ++j) r += red[j * cols];
            chan[s][i] = r;
        }
    }
    M::sync();
}

// The same summed over the channels of every group: total[s][k] of the tile's group k.
template <int TT, int VEC, int NS>
__device__ __forceinline__ void group_sums(const NormArgs &a, const Place<TT, VEC> &at, const float (&v)[NS][VEC],
                                           float *smem, float *(&total)[NS]) {
    using M = Team<TT>;
    const int t = M::thread();
    float *chan[NS];
    channel_sums<TT, VEC, NS>(a, at, v, smem, chan);
    int width = 1;        // lanes of a group
    while (width < a.c && width < 32) width <<= 1;
    for (int k0 = 0; k0 < at.groups; k0 += TT / width) {
        const int k = k0 + t / width, l = t & (width - 1);
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            total[s] = chan[s] + a.p.cols;
            float r = 0.f;
            if (k < at.groups)
                for (int i = l; i < a.c; i += width) r += chan[s][k * a.c + i];
            for (int o = width >> 1; o > 0; o >>= 1) r += lane_xor(r, o);
            if (k < at.groups && l == 0) total[s][k] = r;
        }
    }
    M::sync();
}

// ---- host ---------------------------------------------------------------------------
int64_t gcd64(int64_t a, int64_t b) { return b == 0 ? a : gcd64(b, a % b); }

constexpr int64_t kNormCtasWanted = 912;          // six a multiprocessor

// Vectors that a thread holds of x, and in the backward of the gradient as well: what 128
// registers a thread (64 in teams of 1,024) have room for beside the sums.
constexpr int held_vectors(int team, int vec, bool backward) {
    if (vec > 1) return backward ? 8 : 12;
    return (backward ? 16 : 32) / (team == 1024 ? 2 : 1);
}

// Vectors of elem bytes where rows, pointers and groups allow them: a tile of whole groups
// and whole vectors must fit a team of 256.
int norm_vec(int64_t f, int64_t c, int vec, bool aligned) {
    return aligned && f % vec == 0 && c / gcd64(c, vec) <= 256 ? vec : 1;
}

// A tile is the fewest whole groups and whole vectors of 128 bytes or more; the smallest
// team that holds twice the mean graph takes it, and the tile is widened while that stays
// so.  Graphs no team holds are read in shares by the largest team.
NormPlan norm_plan(int64_t n, int64_t graphs, int64_t f, int64_t c, int vec, int elem, bool backward) {
    NormPlan p{};
    p.vec = vec;
    const int64_t unit = c / gcd64(c, vec);                     // vectors of the smallest tile
    const int64_t row = f / vec;
    const int64_t mean = graphs > 0 ? (n + graphs - 1) / graphs : 0;
    int64_t w = unit;
    while (w < row && w * vec * elem < 128) w += unit;
    const int teams[] = {32, 128, 256};
    auto holds = [&](int64_t vecs, int team) {
        return vecs <= team && held_vectors(team, vec, backward) * (team / vecs) >= 2 * mean;
    };
    p.team = 0;
    for (int t : teams) {
        if (holds(w, t)) {
            p.team = t;
            break;
        }
    }
    if (p.team) {
        while (w + unit <= row && holds(w + unit, p.team)) w += unit;
    } else {
        p.team = w <= 256 ? 256 : 1024;
        while (w + unit <= row && w + unit <= 64) w += unit;    // rows of up to 1 KB at once
    }
    p.held = held_vectors(p.team, vec, backward);
    p.row_vecs = static_cast<int>(w);
    p.cols = static_cast<int>(w * vec);
    p.tiles = static_cast<int>((f + p.cols - 1) / p.cols);
    p.rows_at_once = p.team / p.row_vecs;
    p.cap = int64_t(p.held) * p.rows_at_once;
    if (n <= p.cap) {
        p.share = p.cap;
        p.shares = 0;
        return p;
    }
    int64_t share = (n * p.tiles + kNormCtasWanted - 1) / kNormCtasWanted;
    share = (share + p.rows_at_once - 1) / p.rows_at_once * p.rows_at_once;
    p.share = share < p.cap ? share : p.cap;
    p.shares = (n + p.share - 1) / p.share;
    return p;
}

}  // namespace
}  // namespace tfg
