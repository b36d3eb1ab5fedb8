// Distillation from a teacher's top logits: the loss of each row and the gradient of the
// student's logits.
//
//   p = softmax over the row's K given teacher logits t / tau, entries that are padding left out
//   q = softmax over all V classes of the student's logits s / tau
//   loss = w tau^2 sum_k p_k (log p_k - log q_{id_k}),  dloss/ds = w tau (q - p)
//
// A team of threads, 8, a warp or a CTA, takes a row.  The first pass keeps a running maximum m and
// the sum of e^((s - m) / tau), the second writes the gradient from them; the terms at the teacher's classes are
// written over it.  q is formed from s - m, which is exact or nearly so, and loss terms from
// (s - m) / tau - log(sum), so logits that share a large offset lose nothing.
//
// With the gradient a row of up to 222 KB is held in shared memory, by bulk copies that the first pass follows, and read
// from memory once; the loss alone follows copies through a ring of six chunks.
//
// What bounds it: memory, and the exponentials beside it (two a value with the gradient, 16 a clock on a
// multiprocessor).  16,384 x 50,000 bf16 with gradient, a tenth masked: 541 us (3.1 GB, 5.8 TB/s; the exponentials take
// 319), read twice from L2 and memory 662.  4,096 x 131,072 bf16, the loss alone: 180 us (6.0 TB/s; plain loads, four
// vectors in flight a thread, 195).  2,500 x 49,999 fp32: loss 82 us (6.1 TB/s; plain loads 105), backward 154 (6.5 TB/s).
// 2,708 x 41 fp32, a warp a row: 8 us, latency.
#include <type_traits>

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
// Rows that a warp takes.  12,000 rows of 4,000 bf16: loss 26 us, with 128 threads a row 35; both 46, 50.  Of fp32, twice the
// bytes: loss 41 and 40, both 89 and 64, as the second read no longer comes from L2.
constexpr int kWarpBytes = 8192, kWarpTop = 128;
// Rows that part of a warp takes, where there are so many that warps would take turns: 200,000 rows of 41 fp32 45 us, a warp
// each 156; 9,000 rows take the same by either.
constexpr int kSmallTeam = 8, kSmallClasses = 128, kSmallTop = 32;
constexpr int kInFlight = 4;                                 // vectors that a thread loads before it uses them
// Rows held in shared memory, and the threads of a CTA that takes one: so many that rows of the size, and the
// threads, fill a multiprocessor (from 112 KB on one row at a time).  Longer rows are read twice.  They come in
// copies of kChunkBytes, each with a barrier, so that the first pass begins with the first of them; the loss alone
// needs no more than kRing of them at a time.
constexpr int kHold128 = 16 * 1024, kHold256 = 52 * 1024, kHoldMost = 222 * 1024;
constexpr int kChunkBytes = 16 * 1024, kChunks = (kHoldMost + kChunkBytes - 1) / kChunkBytes, kRing = 6;

// What a kernel makes of a row: the loss alone, the gradient from the forward's statistics, or both; with
// the row held, or chunks of it.
constexpr int kLoss = 0, kBack = 1, kBoth = 2, kBothHeld = 3, kLossRing = 4;

template <int TT>
__device__ __forceinline__ void team_sync() {
    if constexpr (TT <= 32) __syncwarp();
    else __syncthreads();
}
template <int TT, typename F>
__device__ __forceinline__ float team_fold(float v, float *scratch, F fold) {
#pragma unroll
    for (int o = (TT < 32 ? TT : 32) / 2; o > 0; o >>= 1) v = fold(v, lane_xor(v, o));
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
    __device__ __forceinline__ void add(const float (&s)[VEC], float most, float scale) {
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
        if constexpr (VEC == 8) {                            // pairs by packed additions
            float2 p = add2(make_float2(e[0], e[1]), make_float2(e[4], e[5])), q = add2(make_float2(e[2], e[3]), make_float2(e[6], e[7]));
            p = add2(p, q);
            sum += p.x + p.y;
        } else if constexpr (VEC == 4) {
            const float2 p = add2(make_float2(e[0], e[1]), make_float2(e[2], e[3]));
            sum += p.x + p.y;
        } else {
            sum += e[0];
        }
    }
    // VEC values as they lie in memory; the largest of bf16 values two at a time.
    template <typename XT, int VEC>
    __device__ __forceinline__ void add_raw(const typename VecLoad<XT, VEC>::Raw &raw, float scale) {
        float s[VEC], most;
        VecLoad<XT, VEC>::widen(raw, s);
        if constexpr (sizeof(XT) == 2 && VEC == 8) {
            const auto pair = [](uint32_t w) { return *reinterpret_cast<const __nv_bfloat162 *>(&w); };
            const __nv_bfloat162 p = __hmax2(__hmax2(pair(raw.x), pair(raw.y)), __hmax2(pair(raw.z), pair(raw.w)));
            most = fmaxf(__low2float(p), __high2float(p));
        } else {
            most = s[0];
#pragma unroll
            for (int q = 1; q < VEC; ++q) most = fmaxf(most, s[q]);
        }
        add(s, most, scale);
    }
};

// A row of v values that begins anywhere: values up to the first 16-byte boundary and behind
// the last one by themselves, vectors between.
template <typename XT, int VEC>
struct RowSpan {
    const XT *row;
    int head, loose;          // values before the vectors, values outside them
    int64_t vecs, v;
    __device__ __forceinline__ RowSpan(const XT *r, int64_t n) : row(r), v(n) {
        const int off = static_cast<int>(reinterpret_cast<uintptr_t>(r) / sizeof(XT) % VEC);
        head = static_cast<int>(min64(n, off ? VEC - off : 0));
        vecs = (n - head) / VEC;
        loose = static_cast<int>(n - vecs * VEC);
    }
    __device__ __forceinline__ int64_t loose_at(int i) const { return i < head ? i : vecs * VEC + i; }
};

// Vectors i, i + TT, ... of a row, all in flight.
template <int TT, typename XT, int VEC>
__device__ __forceinline__ void load_vectors(const RowSpan<XT, VEC> &r, int64_t i, RowVec<XT, VEC> (&raw)[kInFlight]) {
#pragma unroll
    for (int j = 0; j < kInFlight; ++j)
        if (i + j * TT < r.vecs) raw[j].load(r.row + r.head + (i + j * TT) * VEC);
}

// The vectors of a row in shared memory, in chunks: chunk c in slot c % SLOTS.
template <typename XT, int VEC, int SLOTS>
struct HeldRow {
    static constexpr int kVecs = kChunkBytes / 16;           // of a chunk
    char *data;
    uint64_t *bars;
    __device__ __forceinline__ int chunks(const RowSpan<XT, VEC> &r) const { return static_cast<int>((r.vecs + kVecs - 1) / kVecs); }
    __device__ __forceinline__ void copy(const RowSpan<XT, VEC> &r, int chunk) const {
        const int slot = chunk % SLOTS;
        const int64_t first = static_cast<int64_t>(chunk) * kVecs;
        const uint32_t bytes = static_cast<uint32_t>(min64(kVecs, r.vecs - first)) * 16;
        arrive_expecting(&bars[slot], bytes);
        bulk_copy(data + slot * kChunkBytes, r.row + r.head + first * VEC, bytes, &bars[slot]);
    }
    // false: the chunk did not arrive
    __device__ __forceinline__ bool wait(int chunk) const {
        return phase_done(&bars[chunk % SLOTS], static_cast<uint32_t>(chunk / SLOTS) & 1u);
    }
    __device__ __forceinline__ typename VecLoad<XT, VEC>::Raw raw(int64_t i) const {
        return load_plain<XT, VEC>(reinterpret_cast<const XT *>(data) + i * VEC);
    }
    __device__ __forceinline__ void widen(int64_t i, float (&v)[VEC]) const {
        VecLoad<XT, VEC>::widen(raw(i), v);
    }
    __device__ __forceinline__ float value(const RowSpan<XT, VEC> &r, int64_t c) const {
        float v[1];
        const int64_t i = c - r.head;
        if (i >= 0 && i < r.vecs * VEC) VecLoad<XT, 1>::widen(load_plain<XT, 1>(reinterpret_cast<const XT *>(data) + i), v);
        else VecLoad<XT, 1>::load(r.row + c, v);
        return v[0];
    }
};
struct NotHeld {
    template <typename R>
    __device__ __forceinline__ float value(const R &r, int64_t c) const {
        float v[1];
        using XT = typename std::remove_const<typename std::remove_pointer<decltype(r.row)>::type>::type;
        VecLoad<XT, 1>::load(r.row + c, v);
        return v[0];
    }
};

// The teacher's side of a row, in the team's shared memory: classes (-1: padding) and p.
struct Top {
    int *ids;
    float *p;
    int k;                    // entries
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
template <int TT, bool TERMS, typename Span, typename Held>
__device__ __forceinline__ float top_terms(const DistilArgs &a, const Span &r, const Held &held, int t, float *scratch, float m,
                                           float log_sum, Top &top) {
    float terms = 0.f;
    const float per_tau = 1.f / a.tau;
    for (int i = t; i < top.k; i += TT) {
        if (top.ids[i] < 0) continue;
        const float log_p = fmaf(top.p[i] - top.most, per_tau, -top.log_sum), p = expf(log_p);
        top.p[i] = p;
        if (TERMS && p != 0.f) terms = fmaf(p, log_p - fmaf(held.value(r, top.ids[i]) - m, per_tau, -log_sum), terms);
    }
    return TERMS ? team_fold<TT>(terms, scratch, Add{}) : 0.f;
}

// f q of VEC logits in e.
template <int VEC>
__device__ __forceinline__ void scaled_q(float (&e)[VEC], float away, float scale, float times) {
    const float less[1] = {away}, by[1] = {scale}, f[1] = {times};
    add_vec(e, less);
    mul_vec(e, by);
#pragma unroll
    for (int q = 0; q < VEC; ++q) e[q] = exp2_of(e[q]);
    mul_vec(e, f);
}

// grad = f (q - p) of a row.  APART: the gradient's rows reach their 16-byte boundaries elsewhere than the logits', and are
// written value by value, so that the row is read in vectors and held all the same (4,096 x 50,001 bf16 loss and gradient 218 us, on
// the logits' boundaries 156, with values alone read too 600).
template <int TT, bool HELD, bool APART, typename XT, int VEC, typename Held>
__device__ __forceinline__ void write_gradient(const DistilArgs &a, const RowSpan<XT, VEC> &r, const Held &held, XT *out, int t,
                                               float m, float sum, float f, const Top &top) {
    const float away = -finite_or_zero(m), times = f / sum;
    XT *body = out + r.head;
    if constexpr (APART && HELD) {
#pragma unroll 4
        for (int64_t i = t; i < r.v; i += TT) {
            float e[1] = {held.value(r, i)};
            scaled_q(e, away, a.scale, times);
            store_vec<1>(out + i, e);
        }
    } else if constexpr (APART) {
        constexpr int kFew = 8;                              // values that a thread loads before it uses them
        for (int64_t i0 = t; i0 < r.v; i0 += kFew * TT) {
            float e[kFew][1];
#pragma unroll
            for (int j = 0; j < kFew; ++j) e[j][0] = i0 + j * TT < r.v ? held.value(r, i0 + j * TT) : 0.f;
#pragma unroll
            for (int j = 0; j < kFew; ++j)
                if (i0 + j * TT < r.v) {
                    scaled_q(e[j], away, a.scale, times);
                    store_vec<1>(out + i0 + j * TT, e[j]);
                }
        }
    } else if constexpr (HELD) {
#pragma unroll 4
        for (int64_t i = t; i < r.vecs; i += TT) {
            float e[VEC];
            held.widen(i, e);
            scaled_q(e, away, a.scale, times);
            store_vec<VEC>(body + i * VEC, e);
        }
    } else {
        for (int64_t i0 = t; i0 < r.vecs; i0 += kInFlight * TT) {
            RowVec<XT, VEC> raw[kInFlight];
            load_vectors<TT>(r, i0, raw);
#pragma unroll
            for (int j = 0; j < kInFlight; ++j)
                if (i0 + j * TT < r.vecs) {
                    float e[VEC];
                    raw[j].widen(e);
                    scaled_q(e, away, a.scale, times);
                    store_vec<VEC>(body + (i0 + j * TT) * VEC, e);
                }
        }
    }
    for (int i = t; i < (APART ? 0 : r.loose); i += TT) {
        float e[1];
        VecLoad<XT, 1>::load(r.row + r.loose_at(i), e);
        scaled_q(e, away, a.scale, times);
        store_vec<1>(out + r.loose_at(i), e);
    }
    team_sync<TT>();
    // a class that is listed more than once has the sum of its p, and every listing writes it
    for (int i = t; i < top.k; i += TT) {
        const int id = top.ids[i];
        if (id < 0) continue;
        float p = 0.f, e[1] = {held.value(r, id)};
        for (int j = 0; j < top.k; ++j) p += top.ids[j] == id ? top.p[j] : 0.f;
        e[0] = fmaf(exp2_of((e[0] + away) * a.scale), times, -f * p);
        store_vec<1>(out + id, e);
    }
}

template <int TT, bool APART, typename XT, int VEC>
__device__ __forceinline__ void zero_row(const RowSpan<XT, VEC> &r, XT *out, int t) {
    const float z[VEC] = {}, z1[1] = {0.f};
    if constexpr (APART) {
        for (int64_t i = t; i < r.v; i += TT) store_vec<1>(out + i, z1);
        return;
    }
    for (int64_t i = t; i < r.vecs; i += TT) store_vec<VEC>(out + r.head + i * VEC, z);
    for (int i = t; i < r.loose; i += TT) store_vec<1>(out + r.loose_at(i), z1);
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

template <typename XT, int VEC, int TT, int MODE, bool APART>
__global__ void __launch_bounds__(TT <= 32 ? kDistilThreads : TT) distil_rows(DistilArgs a) {
    constexpr int kTeams = TT <= 32 ? kDistilThreads / TT : 1;
    constexpr bool kHeld = MODE == kBothHeld, kCopies = kHeld || MODE == kLossRing;
    constexpr int kSlots = kHeld ? kChunks : kRing;
    extern __shared__ __align__(128) char s_row[];
    __shared__ float s_fold[TT > 32 ? TT / 32 : 1];
    __shared__ uint64_t s_full[kCopies ? kSlots : 1];
    if (a.status_all && blockIdx.x == gridDim.x - 1) return check_ids(a);
    const int t = threadIdx.x % TT, team = threadIdx.x / TT;
    // Teams of whole warps may leave; smaller ones go through all exchanges, without entries and values.
    constexpr bool kWhole = TT >= 32;
    const int64_t row0 = static_cast<int64_t>(blockIdx.x) * kTeams + team;
    const bool mine = row0 < a.n;
    if (kWhole && !mine) return;
    const int64_t row = mine ? row0 : a.n - 1;
    RowSpan<XT, VEC> r(static_cast<const XT *>(a.logits) + row * a.v, a.v);
    XT *out = a.grad && mine ? static_cast<XT *>(a.grad) + row * a.v : nullptr;
    float f = !mine ? 0.f : (a.weight ? __ldg(a.weight + row) : 1.f);
    const HeldRow<XT, VEC, kSlots> copies{s_row, s_full};
    const int chunks = kCopies ? copies.chunks(r) : 0;
    if constexpr (kCopies) {
        if (f != 0.f && t == 0) {
            for (int c = 0; c < kSlots; ++c) arrivals_init(&s_full[c], 1);
            arrivals_ready();
            for (int c = 0; c < kSlots && c < chunks; ++c) copies.copy(r, c);
        }
    }
    const auto held = [&] {
        if constexpr (kHeld) return copies;
        else return NotHeld{};
    }();
    const int64_t copied = kHeld ? r.vecs * 16 : (kCopies ? min64(r.vecs * 16, kRing * kChunkBytes) : 0);
    Top top;
    top.ids = reinterpret_cast<int *>(s_row + copied) + team * 2 * a.k;
    top.p = reinterpret_cast<float *>(top.ids + a.k);
    top.k = a.k;
    // the first vectors are on their way while the teacher's side is looked at
    constexpr bool kStreams = MODE == kLoss || MODE == kBoth;
    RowVec<XT, VEC> raw[kInFlight];
    if constexpr (kStreams) {
        if (f != 0.f) load_vectors<TT>(r, t, raw);
    }
    load_top<TT>(a, row, t, s_fold, MODE != kBack && !a.status_all, top);   // with barriers, behind those of the copies
    if (f == 0.f || !top.any) {                              // a row that counts for nothing
        if (MODE != kBack && t == 0 && mine) {
            a.loss[row] = 0.f;
            if (a.stats) a.stats[row] = make_float2(0.f, 1.f);
        }
        if (out) zero_row<TT, APART>(r, out, t);
        if constexpr (kCopies) {                             // copies under way end in this CTA's memory
            if (f != 0.f)
                for (int c = 0; c < kSlots && c < chunks; ++c) copies.wait(c);
        }
        if constexpr (kWhole) return;
        out = nullptr;
        r.v = r.vecs = r.loose = top.k = 0;                  // no value of the row is read or written below
        f = 0.f;
    }
    float m, sum;
    if constexpr (MODE == kBack) {
        const float2 s = a.stats[row];
        m = s.x;
        sum = s.y;
        f *= __ldg(a.grad_loss + row);
        top_terms<TT, false>(a, r, held, t, s_fold, m, 0.f, top);
        team_sync<TT>();
    } else {
        Running run;
        if constexpr (kCopies) {
            constexpr int kVecs = HeldRow<XT, VEC, kSlots>::kVecs;
            static_assert(kVecs % TT == 0 || TT == 32, "a chunk is whole vectors of every thread");
            bool there = true;
            int64_t at = t;                                  // in the row
            for (int c = 0; c < chunks; ++c) {
                there = copies.wait(c) && there;
                const int slot = c % kSlots * kVecs;
#pragma unroll
                for (int j = 0; j < kVecs / TT; ++j, at += TT)
                    if (at < r.vecs) run.template add_raw<XT, VEC>(copies.raw(slot + t + j * TT), a.scale);
                if (!kHeld && c + kSlots < chunks) {         // its slot is free for another
                    __syncthreads();
                    if (t == 0) copies.copy(r, c + kSlots);
                }
            }
            if (!there) run.sum = NAN;                       // a row that does not arrive
        } else {
            for (int64_t i0 = t; i0 < r.vecs; i0 += kInFlight * TT) {
                if (i0 != t) load_vectors<TT>(r, i0, raw);
#pragma unroll
                for (int j = 0; j < kInFlight; ++j)
                    if (i0 + j * TT < r.vecs) run.template add_raw<XT, VEC>(raw[j].r, a.scale);
            }
        }
        for (int i = t; i < r.loose; i += TT) {
            float s[1];
            VecLoad<XT, 1>::load(r.row + r.loose_at(i), s);
            run.add(s, s[0], a.scale);
        }
        m = team_fold<TT>(run.m, s_fold, Larger{});
        sum = team_fold<TT>(run.sum * exp2_of((finite_or_zero(run.m) - finite_or_zero(m)) * a.scale), s_fold, Add{});
        const float terms = top_terms<TT, true>(a, r, held, t, s_fold, m, logf(sum), top);
        if (t == 0 && (kWhole || top.k > 0)) {
            a.loss[row] = f * a.tau * a.tau * terms;
            if (a.stats) a.stats[row] = make_float2(m, sum);
        }
        if (MODE == kLoss || MODE == kLossRing) return;
        team_sync<TT>();
    }
    if constexpr (MODE != kLoss && MODE != kLossRing) write_gradient<TT, kHeld, APART>(a, r, held, out, t, m, sum, f * a.tau, top);
}

template <typename XT, int VEC, int TT, int MODE, bool APART>
cudaError_t launch_rows(const DistilArgs &a, size_t shared, cudaStream_t s) {
    auto *kernel = distil_rows<XT, VEC, TT, MODE, APART>;
    if constexpr (MODE == kBothHeld || MODE == kLossRing) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kHoldMost);
        if (e != cudaSuccess) return e;
    }
    constexpr int kTeams = TT <= 32 ? kDistilThreads / TT : 1;
    const unsigned grid = static_cast<unsigned>((a.n + kTeams - 1) / kTeams + (a.status_all ? 1 : 0));
    kernel<<<grid, TT <= 32 ? kDistilThreads : TT, shared, s>>>(a);
    return cudaGetLastError();
}

// The team goes by the rows' size and number, and the vectors by where the logits lie, so that a loss has the same bits with and
// without its gradient, wherever that lies.
template <typename XT, int VEC, int MODE, bool APART>
cudaError_t launch_team(const DistilArgs &a, cudaStream_t s) {
    const size_t top = 8 * size_t(a.k);
    if (a.v <= kSmallClasses && a.k <= kSmallTop && a.n > 64 * sm_count())
        return launch_rows<XT, VEC, kSmallTeam, MODE, APART>(a, kDistilThreads / kSmallTeam * top, s);
    if (a.v * static_cast<int64_t>(sizeof(XT)) <= kWarpBytes && a.k <= kWarpTop) return launch_rows<XT, VEC, 32, MODE, APART>(a, kDistilThreads / 32 * top, s);
    constexpr int kMode = MODE == kBoth ? kBothHeld : (MODE == kLoss ? kLossRing : kBack);
    const size_t values = size_t(a.v) * sizeof(XT), row = values + top, ring = size_t(kRing) * kChunkBytes;
    const size_t shared = kMode == kBothHeld ? row : (kMode == kBack ? top : top + (values < ring ? values : ring));
    if (row <= kHold128) return launch_rows<XT, VEC, 128, kMode, APART>(a, shared, s);
    if (row <= kHold256) return launch_rows<XT, VEC, 256, kMode, APART>(a, shared, s);
    if constexpr (kMode == kBothHeld) {
        if (row > kHoldMost) return launch_rows<XT, VEC, kRowThreads, MODE, APART>(a, top, s);
    }
    return launch_rows<XT, VEC, kRowThreads, kMode, APART>(a, shared, s);
}

template <typename XT, int VEC>
cudaError_t launch_mode(const DistilArgs &a, bool back, cudaStream_t s) {
    if (!back && !a.grad) return launch_team<XT, VEC, kLoss, false>(a, s);
    const bool apart = (reinterpret_cast<uintptr_t>(a.grad) - reinterpret_cast<uintptr_t>(a.logits)) % 16 != 0;
    if (back) return apart ? launch_team<XT, VEC, kBack, true>(a, s) : launch_team<XT, VEC, kBack, false>(a, s);
    return apart ? launch_team<XT, VEC, kBoth, true>(a, s) : launch_team<XT, VEC, kBoth, false>(a, s);
}

constexpr int64_t kOneCheckerIds = 16384;

cudaError_t launch_distil(DistilArgs &a, int dtype, bool back, int32_t *status, cudaStream_t s) {
    if (!back) {
        a.status = status;
        if (a.n * a.k <= kOneCheckerIds) {
            a.status_all = status;
        } else {
            const cudaError_t e = cudaMemsetAsync(status, 0, sizeof(int32_t), s);
            if (e != cudaSuccess) return e;
        }
    }
    if (a.n == 0 && !a.status_all) return cudaSuccess;
    return dtype == TFG_BF16 ? launch_mode<uint16_t, 8>(a, back, s) : launch_mode<float, 4>(a, back, s);
}

}  // namespace

cudaError_t launch_distillation(const void *logits, int dtype, int64_t n, int64_t v, const void *ids, bool id32,
                                const void *teacher, int teacher_dtype, int k, int64_t padding, float tau, const float *weight,
                                float *loss, float *stats, void *grad, int32_t *status, cudaStream_t s) {
    DistilArgs a{logits, n, v, ids, id32, teacher, teacher_dtype == TFG_BF16, k, padding, tau,
                 static_cast<float>(1.4426950408889634 / tau), weight, loss, reinterpret_cast<float2 *>(stats), nullptr, grad,
                 nullptr, nullptr};
    return launch_distil(a, dtype, false, status, s);
}

cudaError_t launch_distillation_backward(const void *logits, int dtype, int64_t n, int64_t v, const void *ids, bool id32,
                                         const void *teacher, int teacher_dtype, int k, int64_t padding, float tau,
                                         const float *weight, const float *stats, const float *grad_loss, void *grad,
                                         cudaStream_t s) {
    DistilArgs a{logits, n, v, ids, id32, teacher, teacher_dtype == TFG_BF16, k, padding, tau,
                 static_cast<float>(1.4426950408889634 / tau), weight, nullptr,
                 reinterpret_cast<float2 *>(const_cast<float *>(stats)), grad_loss, grad, nullptr, nullptr};
    return launch_distil(a, dtype, true, nullptr, s);
}

}  // namespace tfg
