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
// A CTA takes the rows b, b + CTAs, ... (a row for each of its teams), keeps the sums of its columns
// for gamma and beta in registers and writes them once; a second kernel adds the CTAs' in order.
// The next rows are on their way to shared memory while a row is worked on.  Rows of whole 16 bytes come by
// bulk copies, one for an array; others value by value, each thread's own.
//
// What bounds it: memory.  131,072 rows of 1,024, an fp32 stream and bf16 gradients: 293 us (1.88 GB, 6.4 TB/s).  Copies of
// 16 bytes a lane in place of the bulk ones took 401 to 425 us however the rows were split, rows held in registers 599
// (182 of them a thread left 8 warps on a multiprocessor).  8,192 rows of 8,192 bf16: 93 us (5.8 TB/s), 16 values a
// thread; with 32 values and two CTAs a multiprocessor 115.  19,717 rows of 123 fp32 (4-byte copies) 10.4 us.  The
// second kernel 4 to 8 us.
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
    bool bulk;                // every row of every array is whole 16 bytes
    int ctas;
};

// CTAs of the first kernel: as many as fit, with four rows for each team where there are enough.
int back_ctas(int64_t n, int teams, int resident);
cudaError_t join_columns(const float *part, int ctas, int64_t f, float *gamma, float *beta, cudaStream_t s);

namespace {

// The three sums of a row: d, d (s - m), s - m.
template <int VEC>
__device__ __forceinline__ void row_terms(const float (&s)[VEC], const float (&g)[VEC], const float (&w)[VEC], float m,
                                          float (&sum)[3]) {
    const float away[1] = {-m};
    float c[VEC], d[VEC];
#pragma unroll
    for (int q = 0; q < VEC; ++q) c[q] = s[q], d[q] = g[q];
    add_vec(c, away);
    mul_vec(d, w);
    float t[3][VEC];
#pragma unroll
    for (int q = 0; q < VEC; ++q) t[0][q] = d[q], t[2][q] = c[q];
#pragma unroll
    for (int q = 0; q < VEC; ++q) t[1][q] = d[q];
    mul_vec(t[1], c);
#pragma unroll
    for (int k = 0; k < 3; ++k) {
#pragma unroll
        for (int o = VEC / 2; o > 0; o >>= 1)
#pragma unroll
            for (int q = 0; q < o; ++q) t[k][q] += t[k][q + o];
        sum[k] += t[k][0];
    }
}

// What the sums make of a row: h = (s - m) r - e and
// grad_s = r d + (s - m) slope + shift, slope = -r^2 mean(d h), shift = r (e mean(d h) - mean d).
struct RowMeans {
    float e, slope, shift;
    __device__ __forceinline__ RowMeans(const float (&sum)[3], float r, float per) {
        const float d = sum[0] * per;
        e = sum[2] * per * r;
        const float dh = fmaf(-e, d, sum[1] * r * per);
        slope = -r * r * dh;
        shift = r * fmaf(e, dh, -d);
    }
};

// grad_s of VEC values into o (which holds grad_sum), h into s.
template <int VEC>
__device__ __forceinline__ void row_gradient(float (&s)[VEC], const float (&g)[VEC], const float (&w)[VEC], float m, float r,
                                             const RowMeans &a, float (&o)[VEC]) {
    const float away[1] = {-m}, by[1] = {r}, less[1] = {-a.e}, slope[1] = {a.slope}, shift[1] = {a.shift};
    float d[VEC];
#pragma unroll
    for (int q = 0; q < VEC; ++q) d[q] = g[q];
    mul_vec(d, w);
    add_vec(s, away);
    add_vec(o, shift);
    fma_vec(o, s, slope, o);
    fma_vec(o, d, by, o);
    fma_vec(s, s, by, less);
}

template <typename ST, typename GT, typename DT, int VEC, int TT, int NV>
struct BackTeam {
    static constexpr bool kBulk = VEC > 1;
    static constexpr int kTeams = TT < 256 ? 256 / TT : 1, kThreads = TT * kTeams;
    static constexpr int kUnits = TT < 32 ? kThreads / 32 : kTeams;      // of threads that one copy serves: a warp, or a team
    static constexpr int kUnitRows = kTeams / kUnits;
    static constexpr int kHeld = VEC * NV;                               // values a thread
    static constexpr int kS = kThreads * kHeld * sizeof(ST), kG = kThreads * kHeld * sizeof(GT), kD = kThreads * kHeld * sizeof(DT);
    static constexpr int kStageBytes = (kS + kG + kD + 15) / 16 * 16;
    // up to 16 values a thread are kept in registers from the sums to the gradient, more are read again
    static constexpr bool kKeeps = kHeld <= 16;
    static constexpr int kKept = kKeeps ? NV : 1;
    // CTAs of a multiprocessor by their registers: 512 threads of 128, 768 of 80 where few values are held;
    // rows on their way: as many as those leave room for
    static constexpr int kWant = (kHeld <= 8 ? 768 : 512) / kThreads;
    static constexpr int kRoom = 216 * 1024 / kWant / kStageBytes;
    static constexpr int kStages = kRoom < 1 ? 1 : (kRoom < 4 ? kRoom : 4);
    static constexpr int kShared = kStages * kStageBytes;
    static constexpr int kFit = 220 * 1024 / (kShared + 3 * 1024);
    static constexpr int kCtas = kFit < 1 ? 1 : (kFit < kWant ? kFit : kWant);
};

// Values t, t + TT, ... of a row to slots `step` values apart.  There are no asynchronous copies of two bytes: those are
// loaded all at once and then stored (4,096 rows of 4,095 bf16 103 us; one after the other each waits for memory: 165).
template <int NV, int TT, typename T>
__device__ __forceinline__ void copy_values(char *to, int step, const T *row, int t, int cols) {
    if constexpr (sizeof(T) == 2) {
        T v[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = t + i * TT < cols ? row[t + i * TT] : T(0);
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (t + i * TT < cols) reinterpret_cast<T *>(to)[i * step] = v[i];
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (t + i * TT < cols) copy_async<sizeof(T)>(to + i * step * sizeof(T), row + t + i * TT);
    }
}

template <typename T, int VEC>
__device__ __forceinline__ void widen_shared(const T *p, float (&v)[VEC]) {
    VecLoad<T, VEC>::widen(load_plain<T, VEC>(p), v);
}

template <typename ST, typename GT, typename DT, int VEC, int TT, int NV>
__global__ void __launch_bounds__(BackTeam<ST, GT, DT, VEC, TT, NV>::kThreads, BackTeam<ST, GT, DT, VEC, TT, NV>::kCtas)
    row_norm_back(RowBackArgs p) {
    using B = BackTeam<ST, GT, DT, VEC, TT, NV>;
    constexpr int kTeams = B::kTeams, kStages = B::kStages, kWarps = TT > 32 ? TT / 32 : 1;
    extern __shared__ __align__(128) char s_rows[];
    __shared__ float s_sum[2][kTeams][3 * kWarps];
    __shared__ uint64_t s_full[kStages][B::kUnits];
    const int t = threadIdx.x % TT, team = threadIdx.x / TT;
    const int unit = TT < 32 ? threadIdx.x / 32 : team, unit_row = TT < 32 ? (threadIdx.x & 31) / TT : 0;
    const int cols = static_cast<int>(p.f);
    const float per = 1.f / static_cast<float>(p.f);
    const int64_t first = static_cast<int64_t>(blockIdx.x) * kTeams + team, step = static_cast<int64_t>(gridDim.x) * kTeams;
    // rows of the CTA: exchanges are by whole warps, so all teams go through all rounds
    const int64_t rounds = (p.n - static_cast<int64_t>(blockIdx.x) * kTeams + step - 1) / step;

    // where a thread finds its vectors in a stage: the unit's rows one after the other, or slots of its own
    const int at0 = B::kBulk ? unit * B::kUnitRows * TT * B::kHeld + unit_row * cols + t * VEC : threadIdx.x;
    constexpr int kAtStep = B::kBulk ? TT * VEC : B::kThreads;

    const auto copy = [&](int64_t round) {
        if constexpr (B::kBulk) {
            const bool leader = TT < 32 ? (threadIdx.x & 31) == 0 : t == 0;
            const int64_t row = first + round * step;        // the leader's is the first of its unit
            if (leader && row < p.n && round < rounds) {
                const int stage = static_cast<int>(round % kStages);
                char *to = s_rows + stage * B::kStageBytes;
                const int at = unit * B::kUnitRows * TT * B::kHeld;
                const uint32_t values = static_cast<uint32_t>(min64(p.n - row, B::kUnitRows)) * cols;
                uint64_t *bar = &s_full[stage][unit];
                arrive_expecting(bar, values * static_cast<uint32_t>(sizeof(ST) + sizeof(GT) + (p.skip ? sizeof(DT) : 0)));
                bulk_copy(to + at * sizeof(ST), static_cast<const ST *>(p.s) + row * p.f, values * sizeof(ST), bar);
                bulk_copy(to + B::kS + at * sizeof(GT), static_cast<const GT *>(p.g) + row * p.f, values * sizeof(GT), bar);
                if (p.skip)
                    bulk_copy(to + B::kS + B::kG + at * sizeof(DT), static_cast<const DT *>(p.skip) + row * p.f, values * sizeof(DT), bar);
            }
        } else {
            const int64_t row = first + round * step;
            if (row < p.n && round < rounds) {
                char *to = s_rows + static_cast<int>(round % kStages) * B::kStageBytes;
                copy_values<NV, TT>(to + at0 * sizeof(ST), kAtStep, static_cast<const ST *>(p.s) + row * p.f, t, cols);
                copy_values<NV, TT>(to + B::kS + at0 * sizeof(GT), kAtStep, static_cast<const GT *>(p.g) + row * p.f, t, cols);
                if (p.skip)
                    copy_values<NV, TT>(to + B::kS + B::kG + at0 * sizeof(DT), kAtStep, static_cast<const DT *>(p.skip) + row * p.f, t, cols);
            }
            copies_commit();
        }
    };
    if constexpr (B::kBulk) {
        if (threadIdx.x == 0) {
            for (int k = 0; k < kStages; ++k)
                for (int u = 0; u < B::kUnits; ++u) arrivals_init(&s_full[k][u], 1);
            arrivals_ready();
        }
        __syncthreads();
    }
    float gg[NV][VEC] = {}, gb[NV][VEC] = {}, w[B::kKept][VEC];
    if constexpr (B::kKeeps) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if ((t + i * TT) * VEC < cols) row_weights(p.gamma, (t + i * TT) * VEC, 1.f, w[i]);
    }
#pragma unroll
    for (int k = 0; k < (B::kBulk ? kStages : kStages - 1); ++k) copy(k);
    float m = 0.f, r = 0.f;
    if (first < p.n) {
        m = __ldg(p.mean + first);
        r = __ldg(p.rstd + first);
    }
#pragma unroll 1
    for (int64_t round = 0; round < rounds; ++round) {
        const int64_t row = first + round * step;
        const bool live = row < p.n;
        float next_m = 0.f, next_r = 0.f;
        if (row + step < p.n) {
            next_m = __ldg(p.mean + row + step);
            next_r = __ldg(p.rstd + row + step);
        }
        if constexpr (B::kBulk) {
            // a row that does not arrive becomes NaN
            if (live && !phase_done(&s_full[round % kStages][unit], static_cast<uint32_t>(round / kStages) & 1u)) r = NAN;
        } else {
            copy(round + kStages - 1);
            copies_wait<kStages - 1>();
        }
        const char *stage = s_rows + static_cast<int>(round % kStages) * B::kStageBytes;
        const ST *s_at = reinterpret_cast<const ST *>(stage) + at0;
        const GT *g_at = reinterpret_cast<const GT *>(stage + B::kS) + at0;
        const DT *d_at = reinterpret_cast<const DT *>(stage + B::kS + B::kG) + at0;
        float sum[3] = {0.f, 0.f, 0.f};
        float s[B::kKept][VEC], g[B::kKept][VEC];
        if (live) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (t + i * TT) * VEC, k = i % B::kKept;
                if (c < cols) {
                    widen_shared<ST, VEC>(s_at + i * kAtStep, s[k]);
                    widen_shared<GT, VEC>(g_at + i * kAtStep, g[k]);
                    if (!B::kKeeps) row_weights(p.gamma, c, 1.f, w[k]);
                    row_terms<VEC>(s[k], g[k], w[k], m, sum);
                }
            }
        }
        team_sums<TT, kTeams, 3>(sum, s_sum[round & 1][team]);
        const RowMeans a(sum, r, per);
        if (live) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (t + i * TT) * VEC, k = i % B::kKept;
                if (c < cols) {
                    float o[VEC];
                    if (!B::kKeeps) {
                        widen_shared<ST, VEC>(s_at + i * kAtStep, s[k]);
                        widen_shared<GT, VEC>(g_at + i * kAtStep, g[k]);
                        row_weights(p.gamma, c, 1.f, w[k]);
                    }
                    if (p.skip) {
                        widen_shared<DT, VEC>(d_at + i * kAtStep, o);
                    } else {
#pragma unroll
                        for (int q = 0; q < VEC; ++q) o[q] = 0.f;
                    }
                    row_gradient<VEC>(s[k], g[k], w[k], m, r, a, o);
                    fma_vec(gg[i], g[k], s[k], gg[i]);
                    add_vec(gb[i], g[k]);
                    store_vec<VEC>(static_cast<DT *>(p.grad_s) + row * p.f + c, o);
                }
            }
        }
        if constexpr (B::kBulk) {                            // the unit has read the stage: its next row
            if constexpr (TT <= 32) __syncwarp();
            else team_barrier<TT, kTeams>();
            copy(round + kStages);
        }
        m = next_m;
        r = next_r;
    }
    if (!p.part) return;
    // the teams' sums: those of a warp by exchanges, then one warp after the other
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
        constexpr int kCols = TT * NV * VEC, kLanes = TT < 32 ? TT : 32;
        static_assert(2 * kCols * 4 <= B::kShared, "the rows' shared memory, when they are done");
        float *s_cols = reinterpret_cast<float *>(s_rows);
        __syncthreads();
#pragma unroll
        for (int o = TT; o < 32; o <<= 1)
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int q = 0; q < VEC; ++q) {
                    gg[i][q] += lane_xor(gg[i][q], o);
                    gb[i][q] += lane_xor(gb[i][q], o);
                }
        constexpr int kPer = TT < 32 ? 32 : TT;              // threads that add at a time
        for (int j = 0; j < B::kThreads / kPer; ++j) {
            if (static_cast<int>(threadIdx.x) / kPer == j && (threadIdx.x & 31) < kLanes) {
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
        for (int c = threadIdx.x; c < cols; c += B::kThreads) {
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
        row_terms<VEC>(s, g, w, m, part);
#pragma unroll
        for (int k = 0; k < 3; ++k) sum[k] += part[k];
    }
    team_sums<1024, 1, 3>(sum, s_sum);
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
        row_gradient<VEC>(s, g, w, m, r, a, o);
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

// Threads and vectors by the width.  Up to 1,024 columns a warp takes a row, with up to 32 values a thread, and no barrier
// is needed (128 threads with 8 values: 40 warp instructions a value, bound by what a row costs besides its values); wider
// rows have 16 values a thread, so that they stay in registers between the sums and the gradient.  Narrow rows share a
// warp, 8 values a thread (250,000 rows of 128 bf16 64 us, with 32 threads each, half of them idle, 107).
template <typename ST, typename GT, typename DT, int VEC, int TT, int NV>
cudaError_t launch_back_team(const RowBackArgs &p, cudaStream_t s) {
    using B = BackTeam<ST, GT, DT, VEC, TT, NV>;
    auto *kernel = row_norm_back<ST, GT, DT, VEC, TT, NV>;
    if constexpr (B::kShared > 32 * 1024) {   // with the static part above the 48 KB every launch may use
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, B::kShared);
        if (e != cudaSuccess) return e;
    }
    RowBackArgs q = p;
    q.ctas = back_ctas(p.n, B::kTeams, B::kCtas);
    kernel<<<q.ctas, B::kThreads, B::kShared, s>>>(q);
    const cudaError_t e = cudaGetLastError();
    return e != cudaSuccess || !p.part ? e : join_columns(q.part, q.ctas, q.f, q.grad_gamma, q.grad_beta, s);
}
template <typename ST, typename GT, typename DT, int VEC>
cudaError_t launch_back_vec(const RowBackArgs &p, cudaStream_t s) {
    if constexpr (VEC > 1) {
        constexpr int kN = 8 / VEC;                          // vectors of 8 values
        if (p.f <= 32) return launch_back_team<ST, GT, DT, VEC, 4, kN>(p, s);
        if (p.f <= 64) return launch_back_team<ST, GT, DT, VEC, 8, kN>(p, s);
        if (p.f <= 128) return launch_back_team<ST, GT, DT, VEC, 16, kN>(p, s);
        if (p.f <= 256) return launch_back_team<ST, GT, DT, VEC, 32, kN>(p, s);
        if (p.f <= 512) return launch_back_team<ST, GT, DT, VEC, 32, 2 * kN>(p, s);
        if (p.f <= 1024) return launch_back_team<ST, GT, DT, VEC, 32, 4 * kN>(p, s);
        if (p.f <= 2048) return launch_back_team<ST, GT, DT, VEC, 128, 2 * kN>(p, s);
        if (p.f <= 4096) return launch_back_team<ST, GT, DT, VEC, 256, 2 * kN>(p, s);
        if (p.f <= 8192) return launch_back_team<ST, GT, DT, VEC, 512, 2 * kN>(p, s);
        if (p.f <= 16384) return launch_back_team<ST, GT, DT, VEC, 512, 4 * kN>(p, s);
    } else {
        if (p.f <= 32) return launch_back_team<ST, GT, DT, 1, 8, 4>(p, s);
        if (p.f <= 128) return launch_back_team<ST, GT, DT, 1, 32, 4>(p, s);
        if (p.f <= 512) return launch_back_team<ST, GT, DT, 1, 32, 16>(p, s);
        if (p.f <= 1024) return launch_back_team<ST, GT, DT, 1, 64, 16>(p, s);
        if (p.f <= 2048) return launch_back_team<ST, GT, DT, 1, 128, 16>(p, s);
        if (p.f <= 4096) return launch_back_team<ST, GT, DT, 1, 256, 16>(p, s);
    }
    row_norm_back_long<ST, GT, DT, VEC><<<static_cast<unsigned>(p.n), 1024, 0, s>>>(p);
    if (p.part) {
        const int ctas = back_ctas(p.n, 1, 2);
        long_columns<ST, GT><<<dim3(static_cast<unsigned>((p.f + 255) / 256), ctas), 256, 0, s>>>(p);
        const cudaError_t e = cudaGetLastError();
        return e != cudaSuccess ? e : join_columns(p.part, ctas, p.f, p.grad_gamma, p.grad_beta, s);
    }
    return cudaGetLastError();
}

// Vectors of 16 bytes of the widest type: of fp32 vectors of 32 bytes, lanes side by side would meet on banks.
template <typename ST, typename GT, typename DT>
cudaError_t launch_back_types(const RowBackArgs &p, cudaStream_t s) {
    constexpr int kVec = sizeof(ST) + sizeof(GT) + sizeof(DT) == 6 ? 8 : 4;
    return p.bulk ? launch_back_vec<ST, GT, DT, kVec>(p, s) : launch_back_vec<ST, GT, DT, 1>(p, s);
}

template <typename ST, typename GT>
cudaError_t launch_row_back(const RowBackArgs &p, cudaStream_t s) {
    return p.out_dtype == TFG_BF16 ? launch_back_types<ST, GT, uint16_t>(p, s) : launch_back_types<ST, GT, float>(p, s);
}

}  // namespace
}  // namespace tfg
