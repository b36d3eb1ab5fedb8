// Distillation from a teacher's top logits: the loss of each row and the gradient of the
// student's logits.
//
//   p = softmax over the row's K given teacher logits t / tau, entries that are padding left out
//   q = softmax over all V classes of the student's logits s / tau
//   loss = w tau^2 sum_k p_k (log p_k - log q_{id_k}),  dloss/ds = w tau (q - p)
//
// A team of threads, a warp or a CTA, takes a row.  The first pass keeps a running maximum m and
// the sum of e^((s - m) / tau), the second writes the gradient from them; the terms at the teacher's classes are
// written over it.  q is formed from s - m, which is exact or nearly so, and loss terms from
// (s - m) / tau - log(sum), so logits that share a large offset lose nothing.
#include "widen.cuh"

namespace tfg {
namespace {

struct DistilArgs {
    const void *logits;
    int64_t n, v;
    const void *ids;
    bool id32;
    const void *teacher;
    bool teacher_bf16;
    int k;
    int64_t padding;
    float tau, scale;         // scale = log2(e) / tau
    const float *weight;      // [n] or null: 1
    float *loss;              // [n]
    float2 *stats;            // [n] (m, sum) or null; of the backward: read
    const float *grad_loss;   // backward: [n]
    void *grad;               // [n][v] or null
    int32_t *status;
    int32_t *status_all;      // or null: written whole by the CTA behind the rows'
};

constexpr int kRowThreads = 512, kDistilThreads = 256;       // a CTA for a row; teams of a warp
constexpr int kWarpClasses = 2048, kWarpTop = 128;           // rows that a warp takes
constexpr int kInFlight = 4;                                 // vectors that a thread loads before it uses them

template <int TT>
__device__ __forceinline__ void team_sync() {
    if constexpr (TT == 32) __syncwarp();
    else __syncthreads();
}
template <int TT, typename F>
__device__ __forceinline__ float team_fold(float v, float *scratch, F fold) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fold(v, lane_xor(v, o));
    if constexpr (TT > 32) {
        __syncthreads();                                     // the last fold's have been read
        if ((threadIdx.x & 31) == 0) scratch[threadIdx.x / 32] = v;
        __syncthreads();
        v = scratch[0];
#pragma unroll
        for (int w = 1; w < TT / 32; ++w) v = fold(v, scratch[w]);
    }
    return v;
}
struct Add { __device__ __forceinline__ float operator()(float a, float b) const { return a + b; } };
struct Larger { __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); } };

__device__ __forceinline__ float finite_or_zero(float m) { return m == -INFINITY ? 0.f : m; }

// m and the sum of 2^((s - m) scale) over the values seen.
struct Running {
    float m = -INFINITY, sum = 0.f;
    template <int VEC>
    __device__ __forceinline__ void add(const float (&s)[VEC], float scale) {
        float most = s[0];
#pragma unroll
        for (int q = 1; q < VEC; ++q) most = fmaxf(most, s[q]);
        if (most > m) {
            sum *= exp2_of((m - most) * scale);              // 0 at first
            m = most;
        }
        const float away[1] = {-finite_or_zero(m)}, by[1] = {scale};
        float e[VEC];
#pragma unroll
        for (int q = 0; q < VEC; ++q) e[q] = s[q];
        add_vec(e, away);
        mul_vec(e, by);
#pragma unroll
        for (int q = 0; q < VEC; ++q) e[q] = exp2_of(e[q]);
#pragma unroll
        for (int o = VEC / 2; o > 0; o >>= 1)
#pragma unroll
            for (int q = 0; q < o; ++q) e[q] += e[q + o];
        sum += e[0];
    }
};

// A row of v values that begins anywhere: values up to the first 16-byte boundary and behind
// the last one by themselves, vectors between.  VEC = 1 has values alone.
template <typename XT, int VEC>
struct RowSpan {
    const XT *row;
    int head, loose;          // values before the vectors, values outside them
    int64_t vecs, v;
    __device__ __forceinline__ RowSpan(const XT *r, int64_t n) : row(r), head(0), loose(0), vecs(n), v(n) {
        if constexpr (VEC > 1) {
            const int off = static_cast<int>(reinterpret_cast<uintptr_t>(r) / sizeof(XT) % VEC);
            head = static_cast<int>(min64(n, off ? VEC - off : 0));
            vecs = (n - head) / VEC;
            loose = static_cast<int>(n - vecs * VEC);
        }
    }
    __device__ __forceinline__ int64_t loose_at(int i) const { return i < head ? i : vecs * VEC + i; }
};

// The teacher's side of a row, in the team's shared memory: classes (-1: padding) and p.
struct Top {
    int *ids;
    float *p;
    float log_sum, most;      // of the teacher's softmax
    bool any;
};

template <int TT>
__device__ __forceinline__ void load_top(const DistilArgs &a, int64_t row, int t, float *scratch, bool report, Top &top) {
    float most = -INFINITY;
    bool bad = false;
    for (int i = t; i < a.k; i += TT) {
        const int64_t at = row * a.k + i;
        const int64_t id = a.id32 ? static_cast<int64_t>(__ldg(static_cast<const int32_t *>(a.ids) + at))
                                  : __ldg(static_cast<const int64_t *>(a.ids) + at);
        const bool in = id >= 0 && id < a.v && id != a.padding;
        bad |= !in && id != a.padding;
        float l[1];
        if (a.teacher_bf16) VecLoad<uint16_t, 1>::load(static_cast<const uint16_t *>(a.teacher) + at, l);
        else VecLoad<float, 1>::load(static_cast<const float *>(a.teacher) + at, l);
        top.ids[i] = in ? static_cast<int>(id) : -1;
        top.p[i] = in ? l[0] : -INFINITY;
        if (in) most = l[0] != l[0] ? INFINITY : fmaxf(most, l[0]);      // a NaN reaches the sum
    }
    if (bad && report) set_status(a.status, TFG_ERR_INDEX_RANGE);
    most = team_fold<TT>(most, scratch, Larger{});
    top.any = most != -INFINITY;
    top.most = most;
    float sum = 0.f;
    if (top.any)
        for (int i = t; i < a.k; i += TT) {
            const float e = top.ids[i] < 0 ? 0.f : exp2_of((top.p[i] - most) * a.scale);
            sum += e;
        }
    sum = team_fold<TT>(sum, scratch, Add{});
    top.log_sum = logf(sum);
}

// p in place of the teacher's logits; the terms of the loss.
template <int TT, typename XT>
__device__ __forceinline__ float top_terms(const DistilArgs &a, const XT *row, int t, float *scratch, float m, float log_sum,
                                           Top &top) {
    float terms = 0.f;
    const float per_tau = 1.f / a.tau;
    for (int i = t; i < a.k; i += TT) {
        if (top.ids[i] < 0) continue;
        const float log_p = fmaf(top.p[i] - top.most, per_tau, -top.log_sum), p = expf(log_p);
        top.p[i] = p;
        if (row && p != 0.f) {
            float s[1];
            VecLoad<XT, 1>::load(row + top.ids[i], s);
            terms = fmaf(p, log_p - fmaf(s[0] - m, per_tau, -log_sum), terms);
        }
    }
    return row ? team_fold<TT>(terms, scratch, Add{}) : 0.f;
}

// grad = f (q - p) of a row.
template <int TT, typename XT, int VEC>
__device__ __forceinline__ void write_gradient(const DistilArgs &a, const RowSpan<XT, VEC> &r, XT *out, int t, float m,
                                               float sum, float f, const Top &top) {
    const float away[1] = {-finite_or_zero(m)}, by[1] = {a.scale}, times[1] = {f / sum};
    for (int64_t i0 = t; i0 < r.vecs; i0 += kInFlight * TT) {
        RowVec<XT, VEC> raw[kInFlight];
#pragma unroll
        for (int j = 0; j < kInFlight; ++j)
            if (i0 + j * TT < r.vecs) raw[j].load(r.row + r.head + (i0 + j * TT) * VEC);
#pragma unroll
        for (int j = 0; j < kInFlight; ++j)
            if (i0 + j * TT < r.vecs) {
                float e[VEC];
                raw[j].widen(e);
                add_vec(e, away);
                mul_vec(e, by);
#pragma unroll
                for (int q = 0; q < VEC; ++q) e[q] = exp2_of(e[q]);
                mul_vec(e, times);
                store_vec<VEC>(out + r.head + (i0 + j * TT) * VEC, e);
            }
    }
    if (t < r.loose) {
        float e[1];
        VecLoad<XT, 1>::load(r.row + r.loose_at(t), e);
        e[0] = exp2_of((e[0] + away[0]) * a.scale) * times[0];
        store_vec<1>(out + r.loose_at(t), e);
    }
    team_sync<TT>();
    // a class that is listed more than once has the sum of its p, and every listing writes it
    for (int i = t; i < a.k; i += TT) {
        const int id = top.ids[i];
        if (id < 0) continue;
        float p = 0.f, e[1];
        for (int j = 0; j < a.k; ++j) p += top.ids[j] == id ? top.p[j] : 0.f;
        VecLoad<XT, 1>::load(r.row + id, e);
        e[0] = fmaf(exp2_of((e[0] + away[0]) * a.scale), times[0], -f * p);
        store_vec<1>(out + id, e);
    }
}

template <int TT, typename XT, int VEC>
__device__ __forceinline__ void zero_row(const RowSpan<XT, VEC> &r, XT *out, int t) {
    const float z[VEC] = {}, z1[1] = {0.f};
    for (int64_t i = t; i < r.vecs; i += TT) store_vec<VEC>(out + r.head + i * VEC, z);
    if (t < r.loose) store_vec<1>(out + r.loose_at(t), z1);
}

__device__ __forceinline__ void check_ids(const DistilArgs &a) {
    bool any = false;
    for (int64_t i = threadIdx.x; i < a.n * a.k; i += blockDim.x) {
        const int64_t id = a.id32 ? static_cast<int64_t>(__ldg(static_cast<const int32_t *>(a.ids) + i))
                                  : __ldg(static_cast<const int64_t *>(a.ids) + i);
        any |= (id < 0 || id >= a.v) && id != a.padding;
    }
    const int all = __syncthreads_or(any);
    if (threadIdx.x == 0) *a.status_all = all ? TFG_ERR_INDEX_RANGE : TFG_OK;
}

// BACK: the backward from the forward's statistics; else the loss, and with a.grad the gradient.
template <typename XT, int VEC, int TT, bool BACK>
__global__ void __launch_bounds__(TT == 32 ? kDistilThreads : TT) distil_rows(DistilArgs a) {
    constexpr int kTeams = TT == 32 ? kDistilThreads / 32 : 1;
    extern __shared__ __align__(16) char s_top[];
    __shared__ float s_fold[TT / 32];
    if (a.status_all && blockIdx.x == gridDim.x - 1) return check_ids(a);
    const int t = threadIdx.x % TT, team = threadIdx.x / TT;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * kTeams + team;
    if (row >= a.n) return;                                  // whole teams
    Top top;
    top.ids = reinterpret_cast<int *>(s_top) + team * 2 * a.k;
    top.p = reinterpret_cast<float *>(top.ids + a.k);
    const RowSpan<XT, VEC> r(static_cast<const XT *>(a.logits) + row * a.v, a.v);
    XT *out = a.grad ? static_cast<XT *>(a.grad) + row * a.v : nullptr;
    float f = a.weight ? __ldg(a.weight + row) : 1.f;
    load_top<TT>(a, row, t, s_fold, !BACK && !a.status_all, top);
    if (f == 0.f || !top.any) {                              // a row that counts for nothing is not read
        if (!BACK && t == 0) {
            a.loss[row] = 0.f;
            if (a.stats) a.stats[row] = make_float2(0.f, 1.f);
        }
        if (out) zero_row<TT>(r, out, t);
        return;
    }
    float m, sum;
    if constexpr (BACK) {
        const float2 s = a.stats[row];
        m = s.x;
        sum = s.y;
        f *= __ldg(a.grad_loss + row);
        top_terms<TT, XT>(a, nullptr, t, s_fold, m, 0.f, top);
        team_sync<TT>();
    } else {
        Running run;
        for (int64_t i0 = t; i0 < r.vecs; i0 += kInFlight * TT) {
            RowVec<XT, VEC> raw[kInFlight];
#pragma unroll
            for (int j = 0; j < kInFlight; ++j)
                if (i0 + j * TT < r.vecs) raw[j].load(r.row + r.head + (i0 + j * TT) * VEC);
#pragma unroll
            for (int j = 0; j < kInFlight; ++j)
                if (i0 + j * TT < r.vecs) {
                    float s[VEC];
                    raw[j].widen(s);
                    run.add(s, a.scale);
                }
        }
        if (t < r.loose) {
            float s[1];
            VecLoad<XT, 1>::load(r.row + r.loose_at(t), s);
            run.add(s, a.scale);
        }
        m = team_fold<TT>(run.m, s_fold, Larger{});
        sum = team_fold<TT>(run.sum * exp2_of((finite_or_zero(run.m) - finite_or_zero(m)) * a.scale), s_fold, Add{});
        const float terms = top_terms<TT, XT>(a, r.row, t, s_fold, m, logf(sum), top);
        if (t == 0) {
            a.loss[row] = f * a.tau * a.tau * terms;
            if (a.stats) a.stats[row] = make_float2(m, sum);
        }
        if (!out) return;
        team_sync<TT>();
    }
    write_gradient<TT>(a, r, out, t, m, sum, f * a.tau, top);
}

template <typename XT, int VEC, bool BACK>
cudaError_t launch_team(const DistilArgs &a, cudaStream_t s) {
    const int extra = a.status_all ? 1 : 0;
    const size_t top = 8 * size_t(a.k);
    if (a.v <= kWarpClasses && a.k <= kWarpTop) {
        constexpr int kTeams = kDistilThreads / 32;
        const unsigned grid = static_cast<unsigned>((a.n + kTeams - 1) / kTeams + extra);
        distil_rows<XT, VEC, 32, BACK><<<grid, kDistilThreads, kTeams * top, s>>>(a);
    } else {
        distil_rows<XT, VEC, kRowThreads, BACK><<<static_cast<unsigned>(a.n + extra), kRowThreads, top, s>>>(a);
    }
    return cudaGetLastError();
}

constexpr int64_t kOneCheckerIds = 16384;

template <bool BACK>
cudaError_t launch_distil(DistilArgs &a, int dtype, int32_t *status, cudaStream_t s) {
    if (!BACK) {
        a.status = status;
        if (a.n * a.k <= kOneCheckerIds) {
            a.status_all = status;
        } else {
            const cudaError_t e = cudaMemsetAsync(status, 0, sizeof(int32_t), s);
            if (e != cudaSuccess) return e;
        }
    }
    if (a.n == 0 && !a.status_all) return cudaSuccess;
    // rows of both arrays reach their 16-byte boundaries together
    const bool vectors = !a.grad || (reinterpret_cast<uintptr_t>(a.grad) - reinterpret_cast<uintptr_t>(a.logits)) % 16 == 0;
    if (dtype == TFG_BF16) return vectors ? launch_team<uint16_t, 8, BACK>(a, s) : launch_team<uint16_t, 1, BACK>(a, s);
    return vectors ? launch_team<float, 4, BACK>(a, s) : launch_team<float, 1, BACK>(a, s);
}

}  // namespace

cudaError_t launch_distillation(const void *logits, int dtype, int64_t n, int64_t v, const void *ids, bool id32,
                                const void *teacher, int teacher_dtype, int k, int64_t padding, float tau, const float *weight,
                                float *loss, float *stats, void *grad, int32_t *status, cudaStream_t s) {
    DistilArgs a{logits, n, v, ids, id32, teacher, teacher_dtype == TFG_BF16, k, padding, tau,
                 static_cast<float>(1.4426950408889634 / tau), weight, loss, reinterpret_cast<float2 *>(stats), nullptr, grad,
                 nullptr, nullptr};
    return launch_distil<false>(a, dtype, status, s);
}

cudaError_t launch_distillation_backward(const void *logits, int dtype, int64_t n, int64_t v, const void *ids, bool id32,
                                         const void *teacher, int teacher_dtype, int k, int64_t padding, float tau,
                                         const float *weight, const float *stats, const float *grad_loss, void *grad,
                                         cudaStream_t s) {
    DistilArgs a{logits, n, v, ids, id32, teacher, teacher_dtype == TFG_BF16, k, padding, tau,
                 static_cast<float>(1.4426950408889634 / tau), weight, nullptr,
                 reinterpret_cast<float2 *>(const_cast<float *>(stats)), grad_loss, grad, nullptr, nullptr};
    return launch_distil<true>(a, dtype, nullptr, s);
}

}  // namespace tfg
