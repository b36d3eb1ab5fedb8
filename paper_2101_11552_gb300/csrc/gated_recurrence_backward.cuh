// Gated linear recurrence, backward: the kernel (gated_recurrence.cuh: the method).  A translation unit for
// each type of the inputs compiles it.
//
//   l_t = g_t + a_{t+1} l_{t+1} (behind a sequence's last row: dL/dfinal)
//   sigmoid gate: dL/dz = l (v_{t-1} - x) a (1 - a), dL/dx = l (1 - a)
//   exp gate:     dL/dz = l v_{t-1} a,              dL/dx = l
//   dL/dinitial = a l of the sequence's first row
//
// The adjoint is a recurrence of the same form from the last row to the first, so tiles are
// worked on from the last to the first.  What passes from row t to t - 1 is c = a_t l_t.  The states v
// are made again, in fp32 as the forward had them, from the state that entered the tile, which the forward
// keeps: one value for 128 rows in place of a read of all states, and no rounding of a
// state stored in bf16 reaches a gradient.
#pragma once

#include "gated_recurrence.cuh"

namespace tfg {
namespace {

// A tile's inputs value by value; the decays take the gates' place, in slots wide enough for it.
template <typename XT, typename GT>
struct BackwardSlots {
    using T = ScanTile<XT, 1>;
    using Gate = Slots<XT, 1, T::kEach, kScanThreads, T::kLane, T::kRow>;
    using Decay = Slots<float, 1, T::kEach, kScanThreads>;
    using In = Slots<XT, 1, T::kEach, kScanThreads>;
    using Grad = Slots<GT, 1, T::kEach, kScanThreads>;
    static constexpr int kBytes = Decay::kAll + In::kAll + Grad::kAll;
    Gate z;
    Decay d;
    In x;
    Grad g;
    __device__ __forceinline__ explicit BackwardSlots(char *stage)
        : z(stage), d(stage), x(stage + Decay::kAll), g(stage + Decay::kAll + In::kAll) {}
    __device__ __forceinline__ void copy(const ScanArgs &p, const Job &job, TileRows &rows) const {
        const int lane = threadIdx.x % T::kAcross, group = threadIdx.x / T::kAcross;
        const int64_t tile = p.tiles - 1 - job.order, r0 = tile * kTileRows + group * T::kEach;
        const int64_t c = static_cast<int64_t>(job.strip) * T::kWide + lane;
        const int left = c < p.f ? static_cast<int>(min64(p.n - r0, T::kEach)) : 0;
        const XT *zp = static_cast<const XT *>(p.gate) + r0 * p.gate_ld + c, *xp = static_cast<const XT *>(p.x) + r0 * p.x_ld + c;
        const GT *gp = static_cast<const GT *>(p.g) + r0 * p.f + c;
#pragma unroll
        for (int j = 0; j < T::kEach; ++j)
            if (j < left) {
                z.copy(j, zp + j * p.gate_ld);
                x.copy(j, xp + j * p.x_ld);
                if (p.g) g.copy(j, gp + j * p.f);
            }
        if (p.linked) copy_plan(p, tile, rows);
    }
};
// A tile's inputs by tensor copies; the decays take the gates' place.
template <typename XT, typename GT, int VEC>
struct BackwardTile {
    using T = ScanTile<XT, VEC>;
    using Decay = Slots<float, VEC, T::kEach, kScanThreads>;
    using In = TileRow<XT, T>;
    using Grad = TileRow<GT, T>;
    static constexpr int kBytes = Decay::kAll + In::kBytes + Grad::kBytes;
    char *stage;
    Decay d;
    In x;
    Grad g;
    __device__ __forceinline__ explicit BackwardTile(char *s) : stage(s), d(s), x(s + Decay::kAll), g(s + Decay::kAll + In::kBytes) {}
    __device__ __forceinline__ void copy(const ScanArgs &p, const ScanMaps &maps, const Job &job, TileRows &rows, uint64_t *bar) const {
        if (threadIdx.x != 0) return;
        arrive_expecting(bar, 2 * In::kBytes + (p.g ? Grad::kBytes : 0) + (p.linked ? static_cast<uint32_t>(sizeof(TileRows)) : 0u));
        const int64_t tile = p.tiles - 1 - job.order;
        const int c = job.strip * T::kWide, r = static_cast<int>(tile) * kTileRows;
        tile_copy(stage, &maps.gate, c, r, bar);
        tile_copy(stage + Decay::kAll, &maps.x, c, r, bar);
        if (p.g) tile_copy(stage + Decay::kAll + In::kBytes, &maps.g, c, r, bar);
        if (p.linked) bulk_copy(&rows, p.plan + tile, sizeof(TileRows), bar);
    }
    __device__ __forceinline__ void prefetch(const ScanArgs &p, const ScanMaps &maps, const Job &job) const {
        const int c = job.strip * T::kWide, r = static_cast<int>(p.tiles - 1 - job.order) * kTileRows;
        tile_prefetch(&maps.gate, c, r);
        tile_prefetch(&maps.x, c, r);
        if (p.g) tile_prefetch(&maps.g, c, r);
    }
};
template <typename XT, typename GT, int VEC> struct BackwardStageOf { using Type = BackwardTile<XT, GT, VEC>; };
template <typename XT, typename GT> struct BackwardStageOf<XT, GT, 1> { using Type = BackwardSlots<XT, GT>; };
template <typename XT, typename GT, int VEC> using BackwardStage = typename BackwardStageOf<XT, GT, VEC>::Type;

// CTAs of a multiprocessor, by shared memory: 75 KB where all is bf16 but the decay.
template <typename XT, typename GT, int VEC>
constexpr int kBackwardCtas = BackwardStage<XT, GT, VEC>::kBytes > 64 * 1024 ? 2 : 3;

// What leaves the thread's rows upward when nothing enters them, from the last row to the first (exponential gates: the
// decays of the rows up to one, which sigmoid gates have at hand, may pass fp32).
template <bool PLAIN, int FORM, int EACH, int VEC, typename Grad, typename Decay>
__device__ __forceinline__ void compose_up(const ScanArgs &p, const Grad &g, const Decay &d, const float *grad_final,
                                           const int32_t *seq, int64_t c, uint32_t begin, uint32_t end, uint32_t in,
                                           float (&w)[VEC]) {
#pragma unroll
    for (int q = 0; q < VEC; ++q) w[q] = 0.f;
#pragma unroll
    for (int j = EACH - 1; j >= 0; --j) {
        if (!PLAIN && !((in >> j) & 1u)) continue;
        if (!PLAIN && ((end >> j) & 1u)) state_or_zero(grad_final, seq[j], p.f, c, w);
        float v[VEC], dj[VEC];
        g.widen(j, v);
        d.widen(j, dj);
        add_vec(w, v);
        decay<FORM>(w, dj);
        if (!PLAIN && ((begin >> j) & 1u)) {
#pragma unroll
            for (int q = 0; q < VEC; ++q) w[q] = 0.f;
        }
    }
}

// Both maps of the thread's rows: (a, b) of the states, (a, w) of the adjoint.
template <bool PLAIN, int FORM, int KIND, int VEC, int EACH, typename Gate, typename In, typename Decay, typename Grad>
__device__ __forceinline__ void compose_both(const ScanArgs &p, const Gate &z, const In &x, const Decay &d, const Grad &g,
                                             const float *initial, const float *grad_final, const int32_t *seq, int64_t c,
                                             uint32_t begin, uint32_t end, uint32_t in, float (&a)[VEC],
                                             float (&b)[VEC], float (&w)[VEC]) {
    if constexpr (KIND == TFG_GATE_EXP) {
        compose_down<PLAIN, FORM, KIND, VEC, EACH>(p, z, x, d, NoGrad{}, initial, grad_final, seq, c, begin, end, in, a, b, w);
        compose_up<PLAIN, FORM, EACH>(p, g, d, grad_final, seq, c, begin, end, in, w);
    } else {
        compose_down<PLAIN, FORM, KIND, VEC, EACH>(p, z, x, d, g, initial, grad_final, seq, c, begin, end, in, a, b, w);
    }
}

// How dL/dz hangs on l in a row that v enters: sigmoid (x - v) a (1 - a), with the sign turned round; exp v a.
template <int KIND, int FORM, int VEC>
__device__ __forceinline__ void gate_slope(const float (&v)[VEC], const float (&r)[VEC], const float (&x)[VEC], float (&s)[VEC]) {
    if constexpr (KIND == TFG_GATE_EXP) {
        whole_part(r, s);
        add_vec(s, r);
        mul_vec(s, v);
    } else {
        const float minus[1] = {-1.f};
        float t[VEC];
        if constexpr (FORM == kLess) {                       // (v - x) d (1 + d), d = a - 1
            fma_vec(t, r, r, r);
            fma_vec(s, x, minus, v);
        } else {
            float h[VEC];
            whole_part(r, h);
            one_less(r, h, t);
            add_vec(h, r);
            mul_vec(t, h);
            fma_vec(s, v, minus, x);
        }
        mul_vec(s, t);
    }
}

// dL/dz of a row in place of its slope, dL/dx, and a l in place of l.
template <int KIND, int FORM, int VEC>
__device__ __forceinline__ void row_gradient(float (&l)[VEC], const float (&r)[VEC], float (&gz)[VEC], float (&gx)[VEC]) {
#pragma unroll
    for (int q = 0; q < VEC; ++q) gx[q] = l[q];
    if constexpr (KIND == TFG_GATE_EXP) {
        mul_vec(gz, l);
    } else {
        const float minus[1] = {-1.f};
        mul_vec(gx, minus);
        mul_vec(gz, gx);
        if constexpr (FORM == kLess) {
            mul_vec(gx, r);
        } else {
            float less[VEC];                                 // a - 1
            whole_part(r, less);
            add_vec(less, minus);
            add_vec(less, r);
            mul_vec(gx, less);
        }
    }
    decay<FORM>(l, r);
}

// The gradients of the thread's rows from the state v that enters them and what enters their last, w: the slopes down
// the rows, then the adjoint up them.
template <bool PLAIN, int FORM, int KIND, typename XT, int EACH, int VEC, typename In, typename Grad, typename Decay>
__device__ __forceinline__ void write_gradients(const ScanArgs &p, const In &x, const Grad &g, const Decay &d,
                                                const int32_t *seq, XT *gate, XT *input, int64_t c, uint32_t begin, uint32_t end,
                                                uint32_t in, float (&v)[VEC], float (&w)[VEC]) {
    float slope[EACH][VEC];
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
        if (!PLAIN && ((begin >> j) & 1u)) state_or_zero(p.initial, seq[j], p.f, c, v);
        float xv[VEC], dj[VEC];
        x.widen(j, xv);
        d.widen(j, dj);
        gate_slope<KIND, FORM>(v, dj, xv, slope[j]);
        if (j + 1 < EACH) advance<KIND, FORM>(v, dj, xv);
    }
#pragma unroll
    for (int j = EACH - 1; j >= 0; --j) {
        if (!PLAIN && !((in >> j) & 1u)) continue;
        if (!PLAIN && ((end >> j) & 1u)) state_or_zero(p.grad_final, seq[j], p.f, c, w);
        float gx[VEC], dj[VEC];
        g.widen(j, gx);
        add_vec(w, gx);                                      // l
        d.widen(j, dj);
        row_gradient<KIND, FORM>(w, dj, slope[j], gx);
        store_vec<VEC>(gate + j * p.grad_gate_ld, slope[j]);
        store_vec<VEC>(input + j * p.grad_x_ld, gx);
        if (!PLAIN && ((begin >> j) & 1u)) {
            if (p.grad_initial) store_vec<VEC>(p.grad_initial + seq[j] * p.f + c, w);
#pragma unroll
            for (int q = 0; q < VEC; ++q) w[q] = 0.f;
        }
    }
}

template <typename XT, typename GT, int VEC, int KIND>
__global__ void __launch_bounds__(kScanThreads, kBackwardCtas<XT, GT, VEC>)
    scan_backward(ScanArgs p, const __grid_constant__ ScanMaps maps) {
    using T = ScanTile<XT, VEC>;
    using Stage = BackwardStage<XT, GT, VEC>;
    extern __shared__ __align__(128) char s_stage[];
    __shared__ TileRows rows;
    __shared__ uint64_t s_full;
    __shared__ __align__(16) float s_a[kScanWarps][T::kWide], s_b[kScanWarps][T::kWide];      // of the states
    __shared__ __align__(16) float s_u[kScanWarps][T::kWide], s_w[kScanWarps][T::kWide];      // of the adjoint
    __shared__ float2 s_part[kScanThreads / T::kWide][T::kWide];
    __shared__ float s_carry[T::kWide];
    __shared__ uint32_t s_next;
    __shared__ int s_from;
    if (!p.status_all) cudaGridDependencySynchronize();
    if (static_cast<int>(blockIdx.x) < p.checkers) return check_sequences(p, p.grad_final, p.grad_initial);
    const int lane = threadIdx.x % T::kAcross, group = threadIdx.x / T::kAcross, warp = threadIdx.x / 32;
    const Stage in_stage(s_stage);
    Jobs jobs(p, &s_next);
    if (VEC > 1 && threadIdx.x == 0) {
        arrivals_init(&s_full, 1);
        arrivals_ready();
    }
    if (!p.g) {                                              // nothing is copied there
#pragma unroll
        for (int j = 0; j < T::kEach; ++j) in_stage.g.zero(j);
    }
    uint32_t number, parity = 0;
#pragma unroll 1
    while (jobs.next(p, number)) {
        const Job job(p, number);
        if constexpr (VEC > 1) {
            in_stage.copy(p, maps, job, rows, &s_full);
            uint32_t then;
            if (threadIdx.x == 0 && jobs.later(p, number, then)) in_stage.prefetch(p, maps, Job(p, then));
        } else {
            in_stage.copy(p, job, rows);
        }
        const int64_t tile = p.tiles - 1 - job.order, r0 = tile * kTileRows;
        const int64_t c0 = static_cast<int64_t>(job.strip) * T::kWide, c = c0 + lane * VEC;
        const bool on = c < p.f, column = static_cast<int>(threadIdx.x) < T::kWide;
        if (p.linked && warp == 0) {
            const int from = cut_before<true>(p, job.order);
            if (threadIdx.x == 0) s_from = from;
        }
        const int sc = static_cast<int>(threadIdx.x) - T::kWide;                     // threads of the next columns: states
        float state = 0.f;
        if (sc >= 0 && sc < T::kWide && c0 + sc < p.f) state = __ldg(p.entered + tile * p.f + c0 + sc);
        if (!p.linked) find_rows(p, rows);
        if constexpr (VEC > 1) {
            if (!phase_done(&s_full, parity)) set_status(p.status, TFG_ERR_TIMEOUT);
            parity ^= 1u;
        } else {
            copies_done();
            if (p.linked) __syncthreads();                       // the plan is there
        }
        const uint32_t begin = row_bits<T::kEach>(rows.begin, group), end = row_bits<T::kEach>(rows.end, group),
                       in = row_bits<T::kEach>(rows.in, group), begin_warps = warps_word(rows.begin_warps),
                       cut_warps = warps_word(rows.cut_warps);
        const bool plain = (begin | end) == 0u && in == (1u << T::kEach) - 1u;
        const int32_t *seq = rows.seq + group * T::kEach;
        if (!plain && on) prefetch_states<T::kEach>(p.initial, begin, seq, p.f, c);
        if (!plain && on) prefetch_states<T::kEach>(p.grad_final, end, seq, p.f, c);

        // the thread's maps: of the state down its rows, of the adjoint up
        float a[VEC], b[VEC], u[VEC], w[VEC];
        const auto z = [&] {
            if constexpr (VEC > 1) return HeldGate<XT, T>(s_stage);
            else return in_stage.z;
        }();
        if (VEC > 1) __syncthreads();                            // the gates are held: the decays lie otherwise
        bool small = false;
        if constexpr (KIND == TFG_GATE_SIGMOID) small = small_gates<T>(z, plain && on);
        const auto compose = [&](auto is_plain, auto form) {
            compose_both<decltype(is_plain)::value, decltype(form)::value, KIND, VEC, T::kEach>(
                p, z, in_stage.x, in_stage.d, in_stage.g, on ? p.initial : nullptr, on ? p.grad_final : nullptr, seq, c, begin, end, in,
                a, b, w);
        };
        if (!plain || small) compose(No{}, Form<kEither>{});
        else compose(Yes{}, Form<KIND == TFG_GATE_EXP ? kEither : kLess>{});
#pragma unroll
        for (int q = 0; q < VEC; ++q) u[q] = a[q];
        bool cut = begin != 0u, cut_up = (begin | end) != 0u;
        scan_groups<T, KIND, false>(a, b, cut, warp, lane, s_a, s_b);
        scan_groups<T, KIND, true>(u, w, cut_up, warp, lane, s_u, s_w);
        __syncthreads();

        // threads of the first columns: up the warps; of the next: down them, from the state kept
        float tu = 1.f, tw = 0.f;
        if (column) {
#pragma unroll
            for (int i = kScanWarps - 1; i >= 0; --i) {
                const float gu = s_u[i][threadIdx.x], gw = s_w[i][threadIdx.x];
                s_u[i][threadIdx.x] = held_back<KIND>(tu);
                s_w[i][threadIdx.x] = tw;
                const bool fresh = (cut_warps >> warp_bit(i)) & 1u;
                tw = fresh ? gw : through<KIND>(gu, tw, gw);
                tu = fresh ? 0.f : tu * gu;
            }
        } else if (sc < T::kWide) {
#pragma unroll
            for (int i = 0; i < kScanWarps; ++i) {
                const float ga = s_a[i][sc], gb = s_b[i][sc];
                s_b[i][sc] = state;
                state = (begin_warps >> warp_bit(i)) & 1u ? gb : through<KIND>(ga, state, gb);
            }
        }
        const bool wants = (rows.in[kTileRows / 32 - 1] & ~rows.end[kTileRows / 32 - 1]) >> 31;
        const float carry = enter_tile<T::kWide, KIND>(p, job.order, c0, tu, tw, cut_warps != 0u, wants, s_from, s_part);
        jobs.ask(p);
        if (column) s_carry[threadIdx.x] = carry;
        __syncthreads();

        float v[VEC], l[VEC];
        const bool far = cut_warps >> warp_bit(warp) >> 1 != 0u;                     // a warp behind this one is cut
#pragma unroll
        for (int q = 0; q < VEC; ++q) {
            const int i = lane * VEC + q;
            v[q] = s_b[warp][i];
            l[q] = far ? s_w[warp][i] : through<KIND>(s_u[warp][i], s_carry[i], s_w[warp][i]);
        }
        enter_group<T, KIND, false>(a, b, cut, v);
        enter_group<T, KIND, true>(u, w, cut_up, l);
        if (on) {                                            // no way round the loop's end: the warp is whole at its barrier
            const int64_t row = r0 + group * T::kEach;
            XT *gate = static_cast<XT *>(p.grad_gate) + row * p.grad_gate_ld + c, *input = static_cast<XT *>(p.grad_x) + row * p.grad_x_ld + c;
            // not folded into every row's address ahead of the walks, which spilled 50 registers (bf16 80: 315 us, so 285)
            asm volatile("" : "+l"(gate), "+l"(input));
            const auto write = [&](auto is_plain, auto form) {
                write_gradients<decltype(is_plain)::value, decltype(form)::value, KIND, XT, T::kEach>(
                    p, in_stage.x, in_stage.g, in_stage.d, seq, gate, input, c, begin, end, in, v, l);
            };
            if (!plain || small) write(No{}, Form<kEither>{});
            else write(Yes{}, Form<KIND == TFG_GATE_EXP ? kEither : kLess>{});
        }
        __syncwarp();
    }
}

template <typename XT, typename GT, int VEC, int KIND>
cudaError_t launch_backward(const ScanArgs &p, const ScanMaps &maps, cudaStream_t s) {
    return launch_tiles(scan_backward<XT, GT, VEC, KIND>, p, maps, kBackwardCtas<XT, GT, VEC>, BackwardStage<XT, GT, VEC>::kBytes, s);
}
template <typename XT, typename GT, int VEC>
cudaError_t launch_backward_kind(const ScanArgs &p, const ScanMaps &maps, int kind, cudaStream_t s) {
    return kind == TFG_GATE_SIGMOID ? launch_backward<XT, GT, VEC, TFG_GATE_SIGMOID>(p, maps, s)
                                    : launch_backward<XT, GT, VEC, TFG_GATE_EXP>(p, maps, s);
}
template <typename XT, int VEC>
cudaError_t launch_backward_grad(const ScanArgs &p, const ScanMaps &maps, int kind, cudaStream_t s) {
    return p.out_bf16 ? launch_backward_kind<XT, uint16_t, VEC>(p, maps, kind, s) : launch_backward_kind<XT, float, VEC>(p, maps, kind, s);
}

}  // namespace
}  // namespace tfg
