// Gated linear recurrence, backward (gated_recurrence.cuh: the method).
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
#include "gated_recurrence.cuh"

namespace tfg {
namespace {

template <typename XT, typename GT, int VEC>
struct BackwardStage {
    using T = ScanTile<VEC>;
    using In = Slots<XT, VEC, T::kEach, kScanThreads>;
    using Grad = Slots<GT, VEC, T::kEach, kScanThreads>;
    static constexpr int kBytes = 2 * In::kAll + Grad::kAll;
    In z, x;
    Grad g;
    __device__ __forceinline__ explicit BackwardStage(char *stage) : z(stage), x(stage + In::kAll), g(stage + 2 * In::kAll) {}
    __device__ __forceinline__ void copy(const ScanArgs &p, const Job &job, TileRows &rows) const {
        const int lane = threadIdx.x % T::kAcross, group = threadIdx.x / T::kAcross;
        const int64_t tile = p.tiles - 1 - job.order, r0 = tile * kTileRows + group * T::kEach;
        const int64_t c = static_cast<int64_t>(job.strip) * T::kWide + lane * VEC;
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

constexpr int kBackwardCtas = 2;          // of a multiprocessor: 128 registers a thread

template <typename XT, typename GT, int VEC, int KIND>
__global__ void __launch_bounds__(kScanThreads, kBackwardCtas) scan_backward(ScanArgs p) {
    using T = ScanTile<VEC>;
    using Stage = BackwardStage<XT, GT, VEC>;
    extern __shared__ __align__(16) char s_stage[];
    __shared__ TileRows rows;
    __shared__ float s_a[kScanWarps][T::kWide], s_b[kScanWarps][T::kWide];      // of the states
    __shared__ float s_u[kScanWarps][T::kWide], s_w[kScanWarps][T::kWide];      // of the adjoint
    __shared__ float2 s_part[kScanThreads / T::kWide][T::kWide];
    __shared__ float s_carry[T::kWide];
    __shared__ uint32_t s_next;
    __shared__ int s_from;
    if (static_cast<int>(blockIdx.x) < p.checkers) return check_sequences(p, p.grad_final, p.grad_initial);
    const int lane = threadIdx.x % T::kAcross, group = threadIdx.x / T::kAcross, warp = threadIdx.x / 32;
    const Job job = next_job(p, &s_next);
    const Stage in_stage(s_stage);
    in_stage.copy(p, job, rows);
    const int64_t tile = p.tiles - 1 - job.order, r0 = tile * kTileRows;
    const int64_t c0 = static_cast<int64_t>(job.strip) * T::kWide, c = c0 + lane * VEC;
    if (p.linked && warp == 0) {
        const int from = cut_before(p, job.order, kAnyBegin | kAnyEnd, true);
        if (threadIdx.x == 0) s_from = from;
    }
    const bool on = c < p.f;
    const bool column = static_cast<int>(threadIdx.x) < T::kWide;
    const int sc = static_cast<int>(threadIdx.x) - T::kWide;                 // threads of the next columns: states
    float state = 0.f;
    if (sc >= 0 && sc < T::kWide && c0 + sc < p.f) state = __ldg(p.entered + tile * p.f + c0 + sc);
    copies_done();
    if (p.linked) __syncthreads();                       // the plan is there
    else find_rows(p, rows);
    const uint32_t begin = row_bits<T::kEach>(rows.begin, group), end = row_bits<T::kEach>(rows.end, group),
                   in = row_bits<T::kEach>(rows.in, group);
    const float *initial = on ? p.initial : nullptr, *grad_final = on ? p.grad_final : nullptr;

    // the thread's maps: of the state down its rows, of the adjoint up
    float d[T::kEach][VEC], a[VEC], b[VEC], u[VEC], w[VEC];
#pragma unroll
    for (int q = 0; q < VEC; ++q) a[q] = u[q] = 1.f, b[q] = w[q] = 0.f;
#pragma unroll
    for (int j = 0; j < T::kEach; ++j) {
        float v[VEC];
        in_stage.z.widen(j, v);
        decay_less_one<KIND>(v, d[j]);
        if (!((in >> j) & 1u)) continue;
        if ((begin >> j) & 1u) {
#pragma unroll
            for (int q = 0; q < VEC; ++q) a[q] = 0.f;
            state_or_zero(initial, rows.seq[group * T::kEach + j], p.f, c, b);
        }
        in_stage.x.widen(j, v);
        fma_vec(a, d[j], a, a);
        fma_vec(b, d[j], b, b);
        add_input<KIND>(b, d[j], v);
    }
    uint32_t cut = begin;
    scan_groups<VEC, false>(a, b, cut, warp, lane, s_a, s_b);
#pragma unroll
    for (int j = T::kEach - 1; j >= 0; --j) {
        if (!((in >> j) & 1u)) continue;
        if ((end >> j) & 1u) {
#pragma unroll
            for (int q = 0; q < VEC; ++q) u[q] = 0.f;
            state_or_zero(grad_final, rows.seq[group * T::kEach + j], p.f, c, w);
        }
        if (p.g) {
            float v[VEC];
            in_stage.g.widen(j, v);
            add_vec(w, v);
        }
        fma_vec(u, d[j], u, u);
        fma_vec(w, d[j], w, w);
        if ((begin >> j) & 1u) {
#pragma unroll
            for (int q = 0; q < VEC; ++q) u[q] = w[q] = 0.f;
        }
    }
    uint32_t cut_up = begin | end;
    scan_groups<VEC, true>(u, w, cut_up, warp, lane, s_u, s_w);
    __syncthreads();

    // threads of the first columns: up the warps; of the next: down them, from the state kept
    float tu = 1.f, tw = 0.f;
    if (column) {
#pragma unroll
        for (int i = kScanWarps - 1; i >= 0; --i) {
            const float gu = s_u[i][threadIdx.x], gw = s_w[i][threadIdx.x];
            s_u[i][threadIdx.x] = tu;
            s_w[i][threadIdx.x] = tw;
            const bool fresh = (row_bits<kWarpRows>(rows.begin, i) | row_bits<kWarpRows>(rows.end, i)) != 0u;
            tw = fresh ? gw : fmaf(gu, tw, gw);
            tu = fresh ? 0.f : tu * gu;
        }
    } else if (sc < T::kWide) {
#pragma unroll
        for (int i = 0; i < kScanWarps; ++i) {
            const float ga = s_a[i][sc], gb = s_b[i][sc];
            s_b[i][sc] = state;
            state = row_bits<kWarpRows>(rows.begin, i) != 0u ? gb : fmaf(ga, state, gb);
        }
    }
    const bool wants = row_bit(rows.in, kTileRows - 1) && !row_bit(rows.end, kTileRows - 1);
    const float carry = enter_tile<T::kWide>(p, job.order, c0, tu, tw, any_from(rows.begin, 0) || any_from(rows.end, 0),
                                             wants, s_from, s_part);
    if (column) s_carry[threadIdx.x] = carry;
    __syncthreads();

    if (on) {
        float before[T::kEach][VEC], v[VEC];
        const int after = (warp + 1) * kWarpRows;
        const bool far = after < kTileRows && (any_from(rows.begin, after) || any_from(rows.end, after));
#pragma unroll
        for (int q = 0; q < VEC; ++q) {
            const int i = lane * VEC + q;
            v[q] = cut ? b[q] : fmaf(a[q], s_b[warp][i], b[q]);
            const float c_in = far ? s_w[warp][i] : fmaf(s_u[warp][i], s_carry[i], s_w[warp][i]);
            w[q] = cut_up ? w[q] : fmaf(u[q], c_in, w[q]);
        }
#pragma unroll
        for (int j = 0; j < T::kEach; ++j) {
            if ((begin >> j) & 1u) state_or_zero(initial, rows.seq[group * T::kEach + j], p.f, c, v);
            float xv[VEC];
            in_stage.x.widen(j, xv);
#pragma unroll
            for (int q = 0; q < VEC; ++q) before[j][q] = v[q];
            fma_vec(v, d[j], v, v);
            add_input<KIND>(v, d[j], xv);
        }
#pragma unroll
        for (int j = T::kEach - 1; j >= 0; --j) {
            if (!((in >> j) & 1u)) continue;
            const int row = group * T::kEach + j;
            if ((end >> j) & 1u) state_or_zero(grad_final, rows.seq[row], p.f, c, w);
            float gz[VEC], gx[VEC];
            if (p.g) {
                in_stage.g.widen(j, gx);
                add_vec(w, gx);                          // l
            }
            in_stage.x.widen(j, gx);
#pragma unroll
            for (int q = 0; q < VEC; ++q) {
                const float less = -d[j][q];             // 1 - a
                if constexpr (KIND == TFG_GATE_SIGMOID) {
                    gz[q] = w[q] * (before[j][q] - gx[q]) * fmaf(less, d[j][q], less);
                    gx[q] = w[q] * less;
                } else {
                    gz[q] = w[q] * (before[j][q] * (1.f + d[j][q]));
                    gx[q] = w[q];
                }
            }
            store_vec<VEC>(static_cast<XT *>(p.grad_gate) + (r0 + row) * p.grad_gate_ld + c, gz);
            store_vec<VEC>(static_cast<XT *>(p.grad_x) + (r0 + row) * p.grad_x_ld + c, gx);
            fma_vec(w, d[j], w, w);
            if ((begin >> j) & 1u) {
                if (p.grad_initial) store_vec<VEC>(p.grad_initial + rows.seq[row] * p.f + c, w);
#pragma unroll
                for (int q = 0; q < VEC; ++q) w[q] = 0.f;
            }
        }
    }
}

template <typename XT, typename GT, int VEC, int KIND>
cudaError_t launch_backward(const ScanArgs &p, cudaStream_t s) {
    constexpr int kShared = BackwardStage<XT, GT, VEC>::kBytes;
    if constexpr (kShared > 32 * 1024) {   // with the static part above the 48 KB every launch may use
        const cudaError_t e =
            cudaFuncSetAttribute(scan_backward<XT, GT, VEC, KIND>, cudaFuncAttributeMaxDynamicSharedMemorySize, kShared);
        if (e != cudaSuccess) return e;
    }
    scan_backward<XT, GT, VEC, KIND><<<static_cast<unsigned>(p.checkers + p.tiles * p.strips), kScanThreads, kShared, s>>>(p);
    return cudaGetLastError();
}
template <typename XT, typename GT, int VEC>
cudaError_t launch_kind(const ScanArgs &p, int kind, cudaStream_t s) {
    return kind == TFG_GATE_SIGMOID ? launch_backward<XT, GT, VEC, TFG_GATE_SIGMOID>(p, s)
                                    : launch_backward<XT, GT, VEC, TFG_GATE_EXP>(p, s);
}
template <typename XT, int VEC>
cudaError_t launch_grad(const ScanArgs &p, int kind, cudaStream_t s) {
    return p.out_bf16 ? launch_kind<XT, uint16_t, VEC>(p, kind, s) : launch_kind<XT, float, VEC>(p, kind, s);
}

}  // namespace

cudaError_t launch_gated_recurrence_backward(const void *gate, int64_t gate_ld, const void *x, int64_t x_ld, int dtype,
                                             const int64_t *offsets, int64_t n, int64_t seqs, int64_t f, int kind,
                                             const float *initial, const float *entered, const void *g, int g_dtype,
                                             const float *grad_final, void *grad_gate, int64_t grad_gate_ld, void *grad_x,
                                             int64_t grad_x_ld, float *grad_initial, void *ws, int32_t *status,
                                             cudaStream_t s) {
    ScanArgs p{};
    p.gate = gate, p.gate_ld = gate_ld, p.x = x, p.x_ld = x_ld, p.offsets = offsets, p.n = n, p.seqs = seqs, p.f = f;
    p.initial = initial, p.entered = entered, p.g = g, p.out_bf16 = g_dtype == TFG_BF16, p.grad_final = grad_final;
    p.grad_gate = grad_gate, p.grad_gate_ld = grad_gate_ld, p.grad_x = grad_x, p.grad_x_ld = grad_x_ld;
    p.grad_initial = grad_initial;
    const bool vectors = scan_vectors(p, dtype, true);
    scan_geometry(p, dtype, vectors, ws, status);
    cudaError_t e = scan_plan(p, ws, s);
    if (e != cudaSuccess || p.checkers + p.tiles * p.strips == 0) return e;
    if (dtype == TFG_BF16) return vectors ? launch_grad<uint16_t, 8>(p, kind, s) : launch_grad<uint16_t, 1>(p, kind, s);
    return vectors ? launch_grad<float, 4>(p, kind, s) : launch_grad<float, 1>(p, kind, s);
}

}  // namespace tfg
