// Group norm with an activation over the graphs of a batch, channels last: what the
// forward (group_norm_forward.cuh) and the backward (group_norm_backward.cuh) share.
//
// Graph g holds the rows node_offsets[g] .. node_offsets[g + 1] - 1 of x [N, F] (the
// reindexing trick of tf_geometric, Section 2.1.1, keeps a graph's nodes together), the
// F channels fall into groups of C, and statistics are taken over the n_g * C values of
// a (graph, group).
//
// Work split.  A team of threads (a warp, or a CTA) takes a graph and a tile of channels,
// whole groups of them: the threads of a row take vectors side by side and step down the
// rows.  Each thread copies its vectors to shared memory of its own (cp.async: all of
// them in flight at once, no registers, no barrier), and the passes over them -- the sums,
// and the application of the statistics -- read them from there, so that x comes from
// memory once.  Held in registers, or read again from L2, there were too few bytes in
// flight (1,024 graphs of 110 rows, F = 128 fp32, forward: 82 and 27 us against 26 at that time).
//
// A graph of more rows than a team has room for ("large") is cut along a grid of row
// shares over all rows: teams of the first kernel write partial statistics of its pieces,
// and a second kernel joins them in a fixed order and applies them, last share first, as L2
// still holds rows of those (41 communities: of 60 MB forward it reads 17.5 from DRAM again, of
// 119 backward 67).  A share has no more rows than a team has room for, so it meets at most
// two large graphs: one that covers its first row (slot 0) and one that begins behind it
// and runs past its end (slot 1).  Whether there are large graphs only
// the device knows; the host leaves the second kernel out where all rows fit a team, and
// elsewhere it ends after one look at the slots.
#pragma once

#include "widen.cuh"

namespace tfg {
namespace {

constexpr int kActNone = TFG_ACT_NONE, kActRelu = TFG_ACT_RELU, kActSilu = TFG_ACT_SILU, kActGelu = TFG_ACT_GELU;

// Activations in fp32.  1 / (1 + 2^(-y log2 e)) by the hardware's exponential and reciprocal
// (ex2.approx and rcp.approx, 2 ulp and 1 ulp, without the steps that keep subnormal
// values): with the rounding of y log2 e the exponential is off by (2 + |y|) u relative,
// which counts |y| (1 - sigmoid) times at most, so the sigmoid is within 4 u of itself times
// max(|y|, 1).  Where 2^(...) passes 2^126 the sigmoid is 0 and y e^y below 1e-36.  The math
// library's expf and quotient cost 12 instructions more a value (110-row graphs, F = 128:
// the forward was bound by issue, 55 instructions a value).
__device__ __forceinline__ float exp2_of(float v) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
template <int VEC>
__device__ __forceinline__ void sigmoid_of(const float (&y)[VEC], float (&p)[VEC]) {
    const float minus_log2e[1] = {-1.44269504088896341f}, one[1] = {1.f};
#pragma unroll
    for (int q = 0; q < VEC; ++q) p[q] = y[q];
    mul_vec(p, minus_log2e);
#pragma unroll
    for (int q = 0; q < VEC; ++q) p[q] = exp2_of(p[q]);
    add_vec(p, one);
#pragma unroll
    for (int q = 0; q < VEC; ++q) asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(p[q]) : "f"(p[q]));
}
// 1 + erf leaves the gelu an absolute error of about |y| u for negative y.
__device__ __forceinline__ float normal_cdf(float y) { return fmaf(0.5f, erff(y * 0.70710678118654752f), 0.5f); }
template <int ACT, int VEC>
__device__ __forceinline__ void activate(float (&y)[VEC]) {
    if constexpr (ACT == kActRelu) {
#pragma unroll
        for (int q = 0; q < VEC; ++q) y[q] = y[q] <= 0.f ? 0.f : y[q];     // a NaN stays
    } else if constexpr (ACT == kActSilu) {
        float p[VEC];
        sigmoid_of(y, p);
        mul_vec(y, p);
    } else if constexpr (ACT == kActGelu) {
#pragma unroll
        for (int q = 0; q < VEC; ++q) y[q] *= normal_cdf(y[q]);
    }
}
// d times the slope at y
template <int ACT, int VEC>
__device__ __forceinline__ void times_slope(const float (&y)[VEC], float (&d)[VEC]) {
    if constexpr (ACT == kActRelu) {
#pragma unroll
        for (int q = 0; q < VEC; ++q) d[q] *= y[q] > 0.f ? 1.f : (y[q] <= 0.f ? 0.f : y[q]);
    } else if constexpr (ACT == kActSilu) {                 // p (1 + y (1 - p))
        const float one[1] = {1.f}, minus_one[1] = {-1.f};
        float p[VEC], r[VEC];
        sigmoid_of(y, p);
        fma_vec(r, p, minus_one, one);
        fma_vec(r, r, y, one);
        mul_vec(d, p);
        mul_vec(d, r);
    } else if constexpr (ACT == kActGelu) {
#pragma unroll
        for (int q = 0; q < VEC; ++q) {
            const float e = 0.39894228040143268f * exp2_of(y[q] * y[q] * -0.72134752044448170f);   // e^(-y^2 / 2)
            d[q] *= fmaf(y[q], e, normal_cdf(y[q]));
        }
    }
}

}  // namespace

// Geometry of a launch (see norm_plan).
struct NormPlan {
    int vec;              // values of a thread's vector
    int team;             // threads of a team
    int row_vecs;         // vectors of a tile's row
    int cols;             // channels of a tile
    int tiles;
    int rows_at_once;     // rows a team reads side by side
    int tile_groups;      // groups of a tile
    int lanes;            // vectors of a group (1 where a vector holds several groups)
    bool shuffles;        // groups and rows are powers of two of lanes: sums by lane exchanges
    int log_row, log_c, log_rows;   // then: logarithms of row_vecs, the channels of a group, rows_at_once
    uint32_t by_row, by_c, by_rows; // else: factors that divide by them (divisor_factor)
    int log_width;        // and the logarithm of the lanes that add up a group's channels
    int held;             // rows of a thread that its shared memory has room for
    int64_t most;         // rows of a graph that is not large
    int64_t share;        // rows of a share, at most that
    int64_t shares;       // 0: no graph can be large
    bool join_apart;      // there may be large graphs of so many shares that a kernel of its own joins them
};

// The rows of a large graph that share s holds in a slot, written by the first kernel.
struct alignas(16) Piece {
    int64_t a, b;         // rows, a == b: none
    int64_t graph;
    int64_t first_share;  // the share in which the graph begins
};

struct NormArgs {
    const void *x;
    const int64_t *offsets;
    int64_t n, graphs, f;
    int groups, c;                                // groups of c channels
    const float *gamma, *beta;
    float eps;
    float *mean, *rstd;                           // [graphs, groups]
    int32_t *status;      // null: checked by one CTA (status_all)
    int32_t *status_all;
    void *out;
    const void *g;                                // backward: dL/dout
    const float *mean_in, *rstd_in;               // backward: the forward's statistics
    Piece *pieces;                                // [share][slot]
    float4 *moments, *joined_moments;             // forward: [share][slot][group], [share of the graph's first row][group]
    float2 *part, *joined;                        // backward: the same of its two sums
    float2 *channel_part;                         // backward: [batches, then shares][F], sums for gamma and beta
    int64_t batches, batch;                       // backward: batches of so many graphs
    NormPlan p;
};

namespace {

// n / d = the upper half of n * factor, for n d < 2^32: factor = floor(2^32 / d) + 1 is off from 2^32 / d
// by at most 1, so the product by n < 2^32 / d, which no quotient's fraction 1 - 1/d can carry
// over.  Two instructions for the twenty of a division, several of which a team of few
// values felt.  0 stands for d = 1.
__host__ __device__ inline uint32_t divisor_factor(int d) {
    return d == 1 ? 0u : static_cast<uint32_t>((uint64_t(1) << 32) / static_cast<uint32_t>(d)) + 1u;
}
__device__ __forceinline__ int quotient(int n, uint32_t factor) {
    return factor ? static_cast<int>(__umulhi(static_cast<uint32_t>(n), factor)) : n;
}

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

// The status of all offsets, by one CTA: saves the launch that clears the word.
constexpr int64_t kStatusGraphs = 8192;
__device__ __forceinline__ void check_offsets(const NormArgs &p) {
    bool any = false;
    for (int64_t g = threadIdx.x; g < p.graphs; g += blockDim.x) {
        bool bad;
        graph_rows(p.offsets, g, p.n, bad);
        any |= bad;
    }
    const int all = __syncthreads_or(any);
    if (threadIdx.x == 0) *p.status_all = all ? TFG_ERR_INDEX_RANGE : TFG_OK;
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

// covered: the rows up to which slot 0's search has told what there is; slot 1 needs no search
// where that is the share's end.
__device__ __forceinline__ Piece find_piece(const NormArgs &a, int64_t s, int slot, int64_t &covered) {
    const int64_t r0 = s * a.p.share, r1 = min64(a.n, r0 + a.p.share);
    Piece p{0, 0, 0, 0};
    if (slot == 1 && covered >= r1) return p;
    const int64_t g = warp_graph_at(a.offsets, a.graphs, slot == 0 ? r0 : r1 - 1);
    covered = r0;
    if (g < 0) return p;
    bool bad;
    const RowRange r = graph_rows(a.offsets, g, a.n, bad);
    covered = r.b;
    if (r.b - r.a <= a.p.most || r.b <= r0 || (slot == 1) != (r.a > r0)) return p;
    p.a = r.a > r0 ? r.a : r0;
    p.b = r.b < r1 ? r.b : r1;
    if (p.b < p.a) p.b = p.a;
    p.graph = g;
    p.first_share = r.a / a.p.share;
    return p;
}

// ---- a team -------------------------------------------------------------------------
// TT threads: a warp in a CTA of four, each with shared memory of its own, or a whole CTA.
constexpr int kWarpTeams = 4;
// Resident threads asked for: 64 registers a thread forward, 80 backward (64 in teams of
// 1,024).  Forward 1,024 against 768: 4,096 single rows 17 / 19 us; backward 768 against 512
// and 1,024: 41 communities, both directions, 134 / 139 / 134 us, 900 graphs of 111 rows, F = 75
// fp32, 101 / 108 / 100, 20,000 of 3 rows 124 / 128 / 125 (1,024 graphs of 110 rows 84 / 81 / 85).
constexpr int kNormResident = 1024, kBackResident = 768;
constexpr int team_ctas(int team, int threads) { return team == 1024 ? 1 : threads / (team == 256 ? 256 : 128); }
template <int TT>
struct Team {
    static constexpr int kPerCta = TT == 32 ? kWarpTeams : 1;
    static constexpr int kThreads = TT * kPerCta;
    static constexpr int kWarps = TT / 32;
    static __device__ __forceinline__ int index() { return TT == 32 ? threadIdx.x / 32 : 0; }
    static __device__ __forceinline__ int thread() { return TT == 32 ? threadIdx.x & 31 : threadIdx.x; }
    static __device__ __forceinline__ void sync() {
        if constexpr (TT == 32) __syncwarp();
        else __syncthreads();
    }
};

// Place of a thread in its team's tile.  S: sums a thread keeps per quantity, one where
// its vector lies in one group, else one a channel.
template <int TT, int VEC, int S>
struct Place {
    int sub, rl;          // vector of the row, row
    int64_t c0;           // first channel
    bool on;
    int group0;           // first group of the tile
    int groups;           // whole groups of the tile
    int grp[S];           // the groups of the sums, relative to the tile's first

    __device__ __forceinline__ Place(const NormArgs &a, int tile) {
        const int t = Team<TT>::thread();
        rl = a.p.shuffles ? t >> a.p.log_row : quotient(t, a.p.by_row);
        sub = t - rl * a.p.row_vecs;
        c0 = static_cast<int64_t>(tile) * a.p.cols + sub * VEC;
        on = rl < a.p.rows_at_once && c0 < a.f;
        group0 = tile * a.p.tile_groups;
        groups = min(a.p.tile_groups, a.groups - group0);
#pragma unroll
        for (int q = 0; q < S; ++q) {
            const int c = sub * VEC + q;
            grp[q] = on ? (a.p.shuffles ? c >> a.p.log_c : quotient(c, a.p.by_c)) : 0;
        }
    }
    // rows of [a, b) that this thread visits: a + rl, a + rl + rows_at_once, ...
    __device__ __forceinline__ int rows(const NormArgs &p, int64_t a, int64_t b) const {
        const int left = static_cast<int>(b - a) - rl;
        const int up = left + p.p.rows_at_once - 1;
        return on && left > 0 ? (p.p.shuffles ? up >> p.p.log_rows : quotient(up, p.p.by_rows)) : 0;
    }
    // whether sum q is the one that writes its group's statistics
    __device__ __forceinline__ bool writes(const NormArgs &a, int q) const {
        return on && rl == 0 && sub * VEC + q == grp[q] * a.c;
    }
};

// Floats of shared memory that a team's sums take: the buffers of the exchange (one for a
// quantity; two calls after one another take their own), or per-channel sums of two.
constexpr int kForwardBuffers = 3, kBackBuffers = 4;       // one quantity, then two; two and two
__host__ __device__ inline int sum_floats(const NormPlan &p, int buffers, int sums) {
    return p.shuffles ? (p.team > 32 ? buffers * sums * p.team : 0) : 2 * (p.rows_at_once + 2) * p.cols;
}

// Bytes of shared memory of a team: sums and held rows.
__host__ __device__ inline int team_bytes(const NormPlan &p, int buffers, int sums, int row_bytes) {
    return (sum_floats(p, buffers, sums) * 4 + p.held * p.team * row_bytes + 15) / 16 * 16;
}

// A thread's rows in shared memory, one vector each; the team's threads side by side.
template <typename T, int VEC, int TT>
struct Held {
    static constexpr int kBytes = VEC * static_cast<int>(sizeof(T));
    T *at;

    __device__ __forceinline__ explicit Held(void *team_part) : at(static_cast<T *>(team_part) + Team<TT>::thread() * VEC) {}
    __device__ __forceinline__ void copy(const T *from, int rows, int64_t step) const {
#pragma unroll 4
        for (int i = 0; i < rows; ++i) copy_async<kBytes>(at + i * TT * VEC, from + i * step);
    }
    __device__ __forceinline__ void widen(int i, float (&v)[VEC]) const {
        VecLoad<T, VEC>::widen(load_plain<T, VEC>(at + i * TT * VEC), v);
    }
};

// Sums of v[s][q] over the rows and the channels of each group of the tile, to every thread
// for its own groups.  Collective over the team.  By lane exchanges and one barrier where
// group and row are powers of two (through buffer and those behind it, others than the last
// call's, so that this call's barrier separates that one's reads from the writes after it),
// else through per-channel sums in shared memory.
template <int TT, int VEC, int S, int NS>
__device__ __forceinline__ void group_sums(const NormArgs &a, const Place<TT, VEC, S> &at, float (&v)[NS][S], float *smem,
                                           int buffer) {
    using M = Team<TT>;
    const int t = M::thread();
    if (a.p.shuffles) {
        if (S > 1) {                                        // channels of a group in this vector
#pragma unroll
            for (int o = 1; o < S; o <<= 1) {
                if (o >= a.c) break;
#pragma unroll
                for (int s = 0; s < NS; ++s) {
                    float w[S];
#pragma unroll
                    for (int q = 0; q < S; ++q) w[q] = v[s][q] + v[s][q ^ o];
#pragma unroll
                    for (int q = 0; q < S; ++q) v[s][q] = w[q];
                }
            }
        }
        const int in_group = a.p.lanes < 32 ? a.p.lanes : 32, in_row = a.p.row_vecs < 32 ? a.p.row_vecs : 32;
        for (int o = 1; o < in_group; o <<= 1)
#pragma unroll
            for (int s = 0; s < NS; ++s)
#pragma unroll
                for (int q = 0; q < S; ++q) v[s][q] += lane_xor(v[s][q], o);
        for (int o = in_row; o < 32; o <<= 1)
#pragma unroll
            for (int s = 0; s < NS; ++s)
#pragma unroll
                for (int q = 0; q < S; ++q) v[s][q] += lane_xor(v[s][q], o);
        if constexpr (TT > 32) {
            const int lane = t & 31, warp = t >> 5;
            float *to = smem + buffer * S * TT;
#pragma unroll
            for (int s = 0; s < NS; ++s)
#pragma unroll
                for (int q = 0; q < S; ++q) to[(s * S + q) * TT + t] = v[s][q];
            M::sync();
            // warps that hold other rows of this warp's columns, or other columns of its group
            const int log_wide = max(0, a.p.log_row - 5);
            const int wide = (1 << log_wide) - 1, span = a.p.lanes > 32 ? a.p.lanes / 32 : 1;
#pragma unroll
            for (int s = 0; s < NS; ++s)
#pragma unroll
                for (int q = 0; q < S; ++q) {
                    const float *from = to + (s * S + q) * TT + lane;
                    float r = 0.f;
                    if (wide == 0) {                        // a warp holds whole rows
#pragma unroll
                        for (int w = 0; w < M::kWarps; ++w) r += from[w * 32];
                    } else {
                        const int mine = warp & wide & ~(span - 1);
                        for (int w = 0; w < M::kWarps; ++w)
                            if ((w & wide & ~(span - 1)) == mine) r += from[w * 32];
                    }
                    v[s][q] = r;
                }
        }
        return;
    }
    const int cols = a.p.cols, rows = a.p.rows_at_once;
    M::sync();                                              // the last sums have been read
    if (t < rows * a.p.row_vecs) {
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            float *red = smem + s * (rows + 2) * cols + at.rl * cols + at.sub * VEC;
#pragma unroll
            for (int q = 0; q < VEC; ++q) red[q] = S == 1 ? (q == 0 ? v[s][0] : 0.f) : v[s][S == 1 ? 0 : q];
        }
    }
    M::sync();
    for (int i = t; i < cols; i += TT) {
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const float *red = smem + s * (rows + 2) * cols + i;
            float r = 0.f;
            for (int j = 0; j < rows; ++j) r += red[j * cols];
            smem[s * (rows + 2) * cols + rows * cols + i] = r;
        }
    }
    M::sync();
    const int width = 1 << a.p.log_width;                   // lanes of a group
    for (int k0 = 0; k0 < at.groups; k0 += TT >> a.p.log_width) {
        const int k = k0 + (t >> a.p.log_width), l = t & (width - 1);
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            float *chan = smem + s * (rows + 2) * cols + rows * cols;
            float r = 0.f;
            if (k < at.groups)
                for (int i = l; i < a.c; i += width) r += chan[k * a.c + i];
            for (int o = width >> 1; o > 0; o >>= 1) r += lane_xor(r, o);
            if (k < at.groups && l == 0) chan[cols + k] = r;
        }
    }
    M::sync();
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int q = 0; q < S; ++q) v[s][q] = smem[s * (rows + 2) * cols + (rows + 1) * cols + at.grp[q]];
}

// gamma or beta of a thread's channels (aligned like the vectors of x), or their default.
template <int VEC>
__device__ __forceinline__ void channel_weights(const float *w, int64_t c0, float none, float (&v)[VEC]) {
    if (w) {
        RowVec<float, VEC> r;
        r.load(w + c0);
        r.widen(v);
    } else {
#pragma unroll
        for (int q = 0; q < VEC; ++q) v[q] = none;
    }
}

// ---- the second kernel ---------------------------------------------------------------
constexpr int kLargeTeam = 256;                   // its teams, but for tiles of 1,024 threads

// Whether a share has no piece: both slots in one round trip, as many shares have none.
__device__ __forceinline__ bool no_piece(const NormArgs &p, int64_t share) {
    const longlong2 a = *reinterpret_cast<const longlong2 *>(p.pieces + share * 2);
    const longlong2 b = *reinterpret_cast<const longlong2 *>(p.pieces + share * 2 + 1);
    return a.x == a.y && b.x == b.y;
}

// ---- joins of the pieces of a large graph ----------------------------------------------
// By a warp or a CTA of TT threads: 2^log_groups groups side by side, whose parts of a piece lie side by
// side too, and the other threads take pieces in turn.  (A warp a group, its lanes on pieces, read
// 16 bytes of every line: 112,640 rows, one graph of 101,000 and 1,024 small ones, F = 128 fp32 in
// 32 groups, forward 129 us against 57.)
template <int TT>
__device__ __forceinline__ float *join_buffer() {            // for two sums: with kNormRoom, four CTAs of 256 a multiprocessor
    __shared__ float s_sum[2 * TT];
    return s_sum;
}
template <int TT>
struct JoinPlace {
    int log_groups, k, lane, lanes;
    __device__ __forceinline__ explicit JoinPlace(int groups) {
        log_groups = 0;
        while ((1 << log_groups) < groups && (1 << log_groups) < TT) ++log_groups;
        const int t = TT == 32 ? threadIdx.x & 31 : threadIdx.x;
        k = t & ((1 << log_groups) - 1);
        lane = t >> log_groups;
        lanes = TT >> log_groups;
    }
    // Sums over the threads of a group, in a fixed order, to each of them.  Collective.
    template <int N>
    __device__ __forceinline__ void sums(float (&v)[N]) const {
#pragma unroll
        for (int i = 0; i < N; ++i)
            for (int o = 1 << log_groups; o < 32; o <<= 1) v[i] += lane_xor(v[i], o);
        if constexpr (TT > 32) {
            static_assert(N <= 2, "the buffer's sums");
            float *s_sum = join_buffer<TT>();
            const int wide = max(32, 1 << log_groups);
#pragma unroll
            for (int i = 0; i < N; ++i) s_sum[i * TT + threadIdx.x] = v[i];
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i) {
                v[i] = 0.f;
                for (int t = k; t < TT; t += wide) v[i] += s_sum[i * TT + t];
            }
            __syncthreads();
        }
    }
};

// The parts of a large graph's pieces for one group: its rows r begin in share s, there in slot 1
// if behind the share's first row, and go on in slot 0 of the shares behind it.
template <typename Part>
struct Pieces {
    const Part *first, *rest;                               // piece j > 0 at rest + j * stride
    int stride, last;

    __device__ __forceinline__ Pieces(const NormArgs &p, const Part *parts, const RowRange &r, int64_t s, int k) {
        stride = 2 * p.groups;
        rest = parts + s * stride + k;
        first = rest + (r.a > s * p.p.share ? p.groups : 0);
        last = static_cast<int>((r.b - 1) / p.p.share - s);
    }
    // use(part) for those of this thread, read four at a time, the last ones too (behind the end: read, not used)
    template <int TT, typename Use>
    __device__ __forceinline__ void walk(const JoinPlace<TT> &at, Use use) const {
        for (int j0 = at.lane; j0 <= last; j0 += 4 * at.lanes) {
            Part v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int j = min(j0 + u * at.lanes, last);
                v[u] = j == 0 ? *first : rest[static_cast<int64_t>(j) * stride];
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (j0 + u * at.lanes <= last) use(v[u]);
        }
    }
};

// Graphs of few pieces are joined by warps, kJoinGroups groups each: 16 rounds of their four
// lanes a group at most, and no barrier; the others by whole CTAs.
constexpr int kJoinFew = 64, kJoinGroups = 8;

// Joined statistics of this thread's groups of a piece's graph: what a kernel of its own
// joined, or join(place, rows, first share, group) of this CTA, through s_stat[group].
// Collective over the CTA.
template <int TT, typename At, int S, typename Stat, typename Join>
__device__ __forceinline__ void joined_statistics(const NormArgs &p, const At &at, const Piece &piece, const Stat *joined,
                                                  Stat *s_stat, Stat (&stat)[S], Join join) {
    if (p.p.join_apart) {
#pragma unroll
        for (int q = 0; q < S; ++q)
            stat[q] = at.on ? __ldg(joined + piece.first_share * p.groups + at.group0 + at.grp[q]) : Stat{};
        return;
    }
    bool bad;
    const RowRange r = graph_rows(p.offsets, piece.graph, p.n, bad);
    auto groups_of = [&](const auto &place, int k0, int step) {
        for (; k0 < at.groups; k0 += step) {
            const int k = k0 + place.k;
            const Stat v = join(place, r, piece.first_share, at.group0 + min(k, at.groups - 1));
            if (place.lane == 0 && k < min(at.groups, k0 + (1 << place.log_groups))) s_stat[k] = v;
        }
    };
    __syncthreads();                                        // the last statistics have been read
    if (r.b - r.a <= kJoinFew * p.p.share) {
        groups_of(JoinPlace<32>(min(at.groups, kJoinGroups)), (threadIdx.x >> 5) * kJoinGroups, TT / 32 * kJoinGroups);
    } else {
        const JoinPlace<TT> place(at.groups);
        groups_of(place, 0, 1 << place.log_groups);
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < S; ++q) stat[q] = s_stat[at.grp[q]];
}

// join_apart: a CTA takes a range of shares and kJoinGroups groups and finds the shares in which
// large graphs begin (one at most in each: such a graph has more rows than a share).  Its warps
// join those of few pieces, a graph each, and then all of them together the long ones.  Four
// CTAs a multiprocessor whatever the number of shares.
constexpr int kJoinThreads = 512, kJoinCtas = 608;
struct JoinRange {
    int64_t per_cta;      // shares
    dim3 grid;
};
inline JoinRange join_range(const NormPlan &p, int groups) {
    const int64_t y = min64((groups + kJoinGroups - 1) / kJoinGroups, 65535);
    const int64_t per = (p.shares * y + kJoinCtas - 1) / kJoinCtas;
    return {per, dim3(static_cast<unsigned>((p.shares + per - 1) / per), static_cast<unsigned>(y))};
}

template <typename Stat, typename Join>
__device__ __forceinline__ void join_graphs(const NormArgs &p, int64_t per_cta, Stat *joined, Join join) {
    __shared__ int64_t s_share[kJoinThreads], s_graph[kJoinThreads];
    __shared__ int s_count;
    const int64_t from = static_cast<int64_t>(blockIdx.x) * per_cta, to = min64(p.p.shares, from + per_cta);
    auto one = [&](const auto &place, int64_t s, const RowRange &r) {
        for (int k0 = blockIdx.y * kJoinGroups; k0 < p.groups; k0 += gridDim.y * kJoinGroups) {
            const int k = k0 + place.k;
            const Stat v = join(place, r, s, min(k, p.groups - 1));
            if (place.lane == 0 && k < min(p.groups, k0 + kJoinGroups)) joined[s * p.groups + k] = v;
        }
    };
    for (int64_t s0 = from; s0 < to; s0 += kJoinThreads) {
        if (threadIdx.x == 0) s_count = 0;
        __syncthreads();
        const int64_t mine = s0 + threadIdx.x;
        if (mine < to) {
#pragma unroll
            for (int slot = 0; slot < 2; ++slot) {
                const Piece piece = p.pieces[mine * 2 + slot];
                if (piece.a == piece.b || piece.first_share != mine) continue;
                const int at = atomicAdd(&s_count, 1);      // in any order: each is joined by itself
                if (at < kJoinThreads) {
                    s_share[at] = mine;
                    s_graph[at] = piece.graph;
                }
            }
        }
        __syncthreads();
        const int count = min(s_count, kJoinThreads);
        bool bad;
        for (int i = threadIdx.x >> 5; i < count; i += kJoinThreads / 32) {
            const RowRange r = graph_rows(p.offsets, s_graph[i], p.n, bad);
            if (r.b - r.a <= kJoinFew * p.p.share) one(JoinPlace<32>(min(p.groups, kJoinGroups)), s_share[i], r);
        }
        for (int i = 0; i < count; ++i) {
            const RowRange r = graph_rows(p.offsets, s_graph[i], p.n, bad);
            if (r.b - r.a > kJoinFew * p.p.share) one(JoinPlace<kJoinThreads>(min(p.groups, kJoinGroups)), s_share[i], r);
        }
        __syncthreads();
    }
}

// ---- host ---------------------------------------------------------------------------
int64_t gcd64(int64_t a, int64_t b) { return b == 0 ? a : gcd64(b, a % b); }
bool power_of_two(int64_t v) { return v > 0 && (v & (v - 1)) == 0; }

void set_rows_at_once(NormPlan &p, int team) {
    p.rows_at_once = team / p.row_vecs;
    p.log_rows = 0;
    p.by_rows = divisor_factor(p.rows_at_once);
    while ((1 << p.log_rows) < p.rows_at_once) ++p.log_rows;
}

// The longest vector, of at most `widest` values, that rows, pointers and groups allow: 8
// values only where they lie in one group (sums of 8 channels a thread spill), 4 where a
// tile of whole groups and whole vectors fits a team of 256.
int norm_vec(int64_t f, int64_t c, int widest, bool aligned) {
    if (widest == 8 && aligned && c % 8 == 0) return 8;
    return widest >= 4 && aligned && f % 4 == 0 && c / gcd64(c, 4) <= 256 ? 4 : 1;
}

// Vectors of a mean graph to a thread: 16 against 8 and 32, 1,024 graphs of 110 rows 84 / 86 /
// 126 us (both directions).
// Single values (odd widths): 32 to a thread against 16, as the fixed work of a team counts for
// more; 900 graphs of 111 rows, F = 75 fp32: 101 / 108 us, 21 of 83 rows, F = 58: 21.7 / 20.0.
constexpr int kVectorsAThread = 16, kValuesAThread = 32;
// Shares of all rows, of every tile: two for each CTA of 256 threads that is resident.  1,216
// against 608 and 2,432: 41 communities 134 / 134 / 142 us, 1,024 graphs of 110 rows 84 / 83 / 91.
constexpr int64_t kShareTeams = 1216;
// Shared memory of a CTA: four on a multiprocessor.  55 KB against 40 and 74: 1,024 graphs
// of 110 rows 84 / 145 / 92 us (40 KB have no room for the larger ones), 41 communities 134 / 150 /
// 131; 74 KB hold all 900 graphs of 111 rows of an odd width: 101 / 110 / 80.
constexpr int kNormRoom = 55 * 1024;
// Bytes a thread that kNormResident threads leave unused.  20,000 graphs of 3 rows on average, F =
// 35 fp32, both directions: 124 us against 196 with room for 8 rows, 4,096 single rows 17.1 / 17.9.
constexpr int kFreeShared = 216, kFewRows = 64;
constexpr int kNormSharedMost = 96 * 1024;        // allowed to every launch: room, a row's rounding, statistics

// Large graphs are joined by the second kernel itself, which saves a launch, as long as that costs
// little even where one graph has almost all rows: up to so many parts (a piece's sums for one
// group) read by a CTA, and by all of them.  Forward + backward in place / by a kernel of its
// own, one graph of 90 % of the rows among small ones, F = 128 fp32:
//   100 shares of 32 groups (20,000 rows)      14 + 17 /  17 + 20 us
//   385 shares of 32 groups (20,000)           25 + 27 /  20 + 25      12,320 parts a CTA
//   510 shares of 32 groups (112,640)          57 + 70 /  44 + 63      8 to 12 million in all
//   2,013 shares of 32 groups (249,576)       243 + 584 / 94 + 181
//   1,212 shares of one group (112,640)        42 + 72 /  41 + 80
//   4,051 shares of one group (109,376)        94 + 163 / 50 + 174
// A batch without large graphs pays 3 + 2 us of 29 + 50 for the kernel (112,131 rows in 1,024 graphs).
constexpr int64_t kPartsInPlace = 12288, kReadsInPlace = 12 << 20;

// operands: arrays whose rows are held; row_bytes: of the vectors held per row and thread.
// Tiles are whole groups and whole vectors: 32 vectors of a row, fewer (128 bytes at least)
// as long as a team has no room for twice the mean graph.  The team: kVectorsAThread
// vectors (kValuesAThread single values) of a mean graph to a thread, or 256 threads on
// shares of large ones.
NormPlan norm_plan(int64_t n, int64_t graphs, int64_t f, int64_t c, int vec, int operands, int row_bytes) {
    NormPlan p{};
    p.vec = vec;
    const int64_t unit = c / gcd64(c, vec);                     // vectors of the smallest tile
    const int64_t row = f / vec;
    const int64_t mean = graphs > 0 ? (n + graphs - 1) / graphs : 0;
    const int sums = c % vec == 0 ? 1 : vec;
    p.lanes = static_cast<int>(c > vec ? unit : 1);
    p.shuffles = power_of_two(c);                               // c a multiple or a divisor of vec then
    const int64_t least = (128 * operands + row_bytes - 1) / row_bytes;   // vectors of 128 bytes of one operand
    auto fits = [&](int64_t vecs) { return 2 * mean * vecs * row_bytes <= kNormRoom; };
    int64_t w = unit;
    if (p.shuffles) {
        while (w < row && w < 32) w <<= 1;
        int64_t narrow = w;
        while (narrow > unit && narrow / 2 >= least && !fits(narrow)) narrow >>= 1;
        if (fits(narrow)) w = narrow;
    } else {
        const int64_t most = fits(w < least ? least : w) ? 32 : 64;         // large graphs: whole rows at best
        while (w + unit <= row && w + unit <= most && (w < least || most == 64 || fits(w + unit))) w += unit;
    }
    p.row_vecs = static_cast<int>(w);
    p.cols = static_cast<int>(w * vec);
    p.tile_groups = static_cast<int>(p.cols / c);
    while ((1 << p.log_row) < p.row_vecs) ++p.log_row;
    while ((1 << p.log_c) < c) ++p.log_c;
    p.by_row = divisor_factor(p.row_vecs);
    p.by_c = divisor_factor(static_cast<int>(c));
    p.log_width = p.log_c < 5 ? p.log_c : 5;
    p.tiles = static_cast<int>((f + p.cols - 1) / p.cols);
    const int64_t per = vec == 1 ? kValuesAThread : kVectorsAThread;
    const int64_t t = (mean * w + per - 1) / per;
    p.team = t <= 32 && w <= 32 ? 32 : (t <= 128 && w <= 128 ? 128 : 256);
    if (w > 256) p.team = 1024;
    set_rows_at_once(p, p.team);
    const int per_cta = p.team == 32 ? kWarpTeams : 1;
    const int64_t room = (kNormRoom / per_cta - sum_floats(p, operands == 1 ? kForwardBuffers : kBackBuffers, sums) * 4) / (int64_t(p.team) * row_bytes);
    // Twice the mean graph, and of kFewRows what costs no resident team: graphs of a few rows are
    // seldom equal, and those that do not fit cost a share each.
    const int64_t few_rows = (kFewRows + p.rows_at_once - 1) / p.rows_at_once, unused = kFreeShared / row_bytes;
    int64_t wanted = (2 * mean + p.rows_at_once - 1) / p.rows_at_once;
    const int64_t least_rows = few_rows < unused ? few_rows : unused;
    if (wanted < least_rows) wanted = least_rows;
    p.held = static_cast<int>(wanted < room ? wanted : room);
    if (p.held < 1) p.held = 1;
    p.most = int64_t(p.held) * p.rows_at_once;
    // a share: an equal part of all rows for every resident team, if a team has room for it
    p.share = (n * p.tiles + kShareTeams - 1) / kShareTeams;
    const int64_t few = int64_t(p.rows_at_once) * 4;
    if (p.share < few) p.share = few;
    if (p.share > p.most || 2 * mean <= p.most) p.share = p.most;
    p.shares = n <= p.most ? 0 : (n + p.share - 1) / p.share;
    // One graph may hold almost all rows, whatever the mean: every CTA of the second kernel would
    // read all pieces' parts of its tile.
    const int64_t parts = p.shares * (f / c);
    p.join_apart = (parts >= 2048 && mean > 8 * p.share) || p.shares * p.tile_groups > kPartsInPlace || parts * p.shares > kReadsInPlace;
    return p;
}

// Launches of up to 48 KB, static shared memory with it, need no permission.  The limit is
// the same for every launch, so that no call lowers it under another's.
template <typename Kernel>
cudaError_t allow_shared(Kernel *kernel, int bytes) {
    return bytes <= 32 * 1024 ? cudaSuccess
                              : cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kNormSharedMost);
}

}  // namespace
}  // namespace tfg
