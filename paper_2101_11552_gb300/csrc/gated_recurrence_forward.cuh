// Gated linear recurrence, forward: the kernel (gated_recurrence.cuh: the method).  A translation unit
// for each type of the inputs compiles it.
#pragma once

#include "gated_recurrence.cuh"

namespace tfg {
namespace {

// A tile's inputs value by value; the decays take the gates' place, in slots wide enough for it.
template <typename XT>
struct ForwardSlots {
    using T = ScanTile<XT, 1>;
    using Gate = Slots<XT, 1, T::kEach, kScanThreads, T::kLane, T::kRow>;
    using Decay = Slots<float, 1, T::kEach, kScanThreads>;
    using In = Slots<XT, 1, T::kEach, kScanThreads>;
    static constexpr int kBytes = Decay::kAll + In::kAll;
    Gate z;
    Decay d;
    In x;
    __device__ __forceinline__ explicit ForwardSlots(char *stage) : z(stage), d(stage), x(stage + Decay::kAll) {}
    __device__ __forceinline__ void copy(const ScanArgs &p, const Job &job, TileRows &rows) const {
        const int lane = threadIdx.x % T::kAcross, group = threadIdx.x / T::kAcross;
        const int64_t c = static_cast<int64_t>(job.strip) * T::kWide + lane, r0 = job.order * kTileRows + group * T::kEach;
        const int left = c < p.f ? static_cast<int>(min64(p.n - r0, T::kEach)) : 0;
        const XT *zp = static_cast<const XT *>(p.gate) + r0 * p.gate_ld + c, *xp = static_cast<const XT *>(p.x) + r0 * p.x_ld + c;
#pragma unroll
        for (int j = 0; j < T::kEach; ++j)
            if (j < left) {
                z.copy(j, zp + j * p.gate_ld);
                x.copy(j, xp + j * p.x_ld);
            }
        if (p.linked) copy_plan(p, job.order, rows);
    }
};
// A tile's inputs by tensor copies; the decays take the gates' place.
template <typename XT, int VEC>
struct ForwardTile {
    using T = ScanTile<XT, VEC>;
    using Decay = Slots<float, VEC, T::kEach, kScanThreads>;
    using In = TileRow<XT, T>;
    static constexpr int kBytes = Decay::kAll + In::kBytes;
    char *stage;
    Decay d;
    In x;
    __device__ __forceinline__ explicit ForwardTile(char *s) : stage(s), d(s), x(s + Decay::kAll) {}
    __device__ __forceinline__ void copy(const ScanArgs &p, const ScanMaps &maps, const Job &job, TileRows &rows, uint64_t *bar) const {
        if (threadIdx.x != 0) return;
        arrive_expecting(bar, 2 * In::kBytes + (p.linked ? static_cast<uint32_t>(sizeof(TileRows)) : 0u));
        const int c = job.strip * T::kWide, r = static_cast<int>(job.order) * kTileRows;
        tile_copy(stage, &maps.gate, c, r, bar);
        tile_copy(stage + Decay::kAll, &maps.x, c, r, bar);
        if (p.linked) bulk_copy(&rows, p.plan + job.order, sizeof(TileRows), bar);
    }
    __device__ __forceinline__ void prefetch(const ScanMaps &maps, const Job &job) const {
        const int c = job.strip * T::kWide, r = static_cast<int>(job.order) * kTileRows;
        tile_prefetch(&maps.gate, c, r);
        tile_prefetch(&maps.x, c, r);
    }
};
template <typename XT, int VEC> struct ForwardStageOf { using Type = ForwardTile<XT, VEC>; };
template <typename XT> struct ForwardStageOf<XT, 1> { using Type = ForwardSlots<XT>; };
template <typename XT, int VEC> using ForwardStage = typename ForwardStageOf<XT, VEC>::Type;

// CTAs of a multiprocessor: as many as their shared memory allows (55 and 39 KB), 64 registers a thread.
constexpr int kForwardCtas = 4;

// The rows again, from the state v that enters the thread's first.
template <bool PLAIN, int FORM, int KIND, int EACH, typename OT, int VEC, typename In, typename Decay>
__device__ __forceinline__ void write_rows(const ScanArgs &p, const In &x, const Decay &d, const int32_t *seq, int64_t c,
                                           uint32_t begin, uint32_t end, uint32_t in, OT *out, float (&v)[VEC]) {
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
        if (!PLAIN && !((in >> j) & 1u)) continue;
        if (!PLAIN && ((begin >> j) & 1u)) state_or_zero(p.initial, seq[j], p.f, c, v);
        float w[VEC], dj[VEC];
        x.widen(j, w);
        d.widen(j, dj);
        advance<KIND, FORM>(v, dj, w);
        store_vec<VEC>(out + j * p.f, v);
        if (!PLAIN && ((end >> j) & 1u) && p.final_state) store_vec<VEC>(p.final_state + seq[j] * p.f + c, v);
    }
}

template <typename XT, typename OT, int VEC, int KIND>
__global__ void __launch_bounds__(kScanThreads, kForwardCtas)
    scan_forward(ScanArgs p, const __grid_constant__ ScanMaps maps) {
    using T = ScanTile<XT, VEC>;
    using Stage = ForwardStage<XT, VEC>;
    extern __shared__ __align__(128) char s_stage[];
    __shared__ TileRows rows;
    __shared__ uint64_t s_full;
    __shared__ __align__(16) float s_a[kScanWarps][T::kWide], s_b[kScanWarps][T::kWide];
    __shared__ float2 s_part[kScanThreads / T::kWide][T::kWide];
    __shared__ float s_state[T::kWide];
    __shared__ uint32_t s_next;
    __shared__ int s_from;
    if (!p.status_all) cudaGridDependencySynchronize();
    if (static_cast<int>(blockIdx.x) < p.checkers) return check_sequences(p, p.initial, p.final_state);
    const int lane = threadIdx.x % T::kAcross, group = threadIdx.x / T::kAcross, warp = threadIdx.x / 32;
    const Stage in_stage(s_stage);
    Jobs jobs(p, &s_next);
    if (VEC > 1 && threadIdx.x == 0) {
        arrivals_init(&s_full, 1);
        arrivals_ready();
    }
    uint32_t number, parity = 0;
#pragma unroll 1
    while (jobs.next(p, number)) {
        const Job job(p, number);
        if constexpr (VEC > 1) {
            in_stage.copy(p, maps, job, rows, &s_full);
            uint32_t then;
            if (threadIdx.x == 0 && jobs.later(p, number, then)) in_stage.prefetch(maps, Job(p, then));
        } else {
            in_stage.copy(p, job, rows);
        }
        const int64_t r0 = job.order * kTileRows, c0 = static_cast<int64_t>(job.strip) * T::kWide, c = c0 + lane * VEC;
        const bool on = c < p.f;
        if (p.linked && warp == 0) {
            const int from = cut_before<false>(p, job.order);
            if (threadIdx.x == 0) s_from = from;
        }
        if (!p.linked) find_rows(p, rows);
        if constexpr (VEC > 1) {
            if (!phase_done(&s_full, parity)) set_status(p.status, TFG_ERR_TIMEOUT);
            parity ^= 1u;
        } else {
            copies_done();
            if (p.linked) __syncthreads();                       // the plan is there
        }
        const uint32_t begin = row_bits<T::kEach>(rows.begin, group), end = row_bits<T::kEach>(rows.end, group),
                       in = row_bits<T::kEach>(rows.in, group), begin_warps = warps_word(rows.begin_warps);
        const bool plain = (begin | end) == 0u && in == (1u << T::kEach) - 1u;
        const int32_t *seq = rows.seq + group * T::kEach;
        if (!plain && on) prefetch_states<T::kEach>(p.initial, begin, seq, p.f, c);

        float a[VEC], b[VEC];
        const auto z = [&] {
            if constexpr (VEC > 1) return HeldGate<XT, T>(s_stage);
            else return in_stage.z;
        }();
        if (VEC > 1) __syncthreads();                            // the gates are held: the decays lie otherwise
        float none[VEC];
        bool small = false;
        if constexpr (KIND == TFG_GATE_SIGMOID) small = small_gates<T>(z, plain && on);
        const auto compose = [&](auto is_plain, auto form) {
            compose_down<decltype(is_plain)::value, decltype(form)::value, KIND, VEC, T::kEach>(
                p, z, in_stage.x, in_stage.d, NoGrad{}, on ? p.initial : nullptr, nullptr, seq, c, begin, end, in, a, b, none);
        };
        if (!plain || small) compose(No{}, Form<kEither>{});
        else compose(Yes{}, Form<KIND == TFG_GATE_EXP ? kEither : kLess>{});
        bool cut = begin != 0u;
        scan_groups<T, KIND, false>(a, b, cut, warp, lane, s_a, s_b);
        __syncthreads();

        // down the warps, a thread for each channel: what stands before each, and the tile's map
        const int64_t mc = c0 + threadIdx.x;
        const bool column = static_cast<int>(threadIdx.x) < T::kWide;
        float ta = 1.f, tb = 0.f;
        if (column) {
#pragma unroll
            for (int w = 0; w < kScanWarps; ++w) {
                const float wa = s_a[w][threadIdx.x], wb = s_b[w][threadIdx.x];
                s_a[w][threadIdx.x] = held_back<KIND>(ta);
                s_b[w][threadIdx.x] = tb;
                const bool fresh = (begin_warps >> warp_bit(w)) & 1u;
                tb = fresh ? wb : through<KIND>(wa, tb, wb);     // not 0 times what may be an infinity
                ta = fresh ? 0.f : ta * wa;
            }
        }
        const bool wants = (rows.in[0] & ~rows.begin[0] & 1u) != 0u;
        const float state = enter_tile<T::kWide, KIND>(p, job.order, c0, ta, tb, begin_warps != 0u, wants, s_from, s_part);
        jobs.ask(p);
        if (column) s_state[threadIdx.x] = state;
        if (column && mc < p.f && p.entering) p.entering[job.order * p.f + mc] = state;
        __syncthreads();

        float v[VEC];
        const bool far = (begin_warps & ((1u << warp_bit(warp)) - 1u)) != 0u;
#pragma unroll
        for (int q = 0; q < VEC; ++q) {
            const int i = lane * VEC + q;
            v[q] = far ? s_b[warp][i] : through<KIND>(s_a[warp][i], s_state[i], s_b[warp][i]);
        }
        enter_group<T, KIND, false>(a, b, cut, v);
        if (on) {                                            // no way round the loop's end: the warp is whole at its barrier
            OT *out = static_cast<OT *>(p.out) + (r0 + group * T::kEach) * p.f + c;
            const auto write = [&](auto is_plain, auto form) {
                write_rows<decltype(is_plain)::value, decltype(form)::value, KIND, T::kEach>(p, in_stage.x, in_stage.d, seq, c, begin, end,
                                                                                             in, out, v);
            };
            if (!plain || small) write(No{}, Form<kEither>{});
            else write(Yes{}, Form<KIND == TFG_GATE_EXP ? kEither : kLess>{});
        }
        __syncwarp();
    }
}

template <typename XT, typename OT, int VEC, int KIND>
cudaError_t launch_forward(const ScanArgs &p, const ScanMaps &maps, cudaStream_t s) {
    return launch_tiles(scan_forward<XT, OT, VEC, KIND>, p, maps, kForwardCtas, ForwardStage<XT, VEC>::kBytes, s);
}
template <typename XT, int VEC>
cudaError_t launch_forward_kind(const ScanArgs &p, const ScanMaps &maps, int kind, cudaStream_t s) {
    if (kind == TFG_GATE_SIGMOID)
        return p.out_bf16 ? launch_forward<XT, uint16_t, VEC, TFG_GATE_SIGMOID>(p, maps, s) : launch_forward<XT, float, VEC, TFG_GATE_SIGMOID>(p, maps, s);
    return p.out_bf16 ? launch_forward<XT, uint16_t, VEC, TFG_GATE_EXP>(p, maps, s) : launch_forward<XT, float, VEC, TFG_GATE_EXP>(p, maps, s);
}

}  // namespace
}  // namespace tfg
