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

// VEC values of dL/dout, zeros without.
template <int VEC>
struct GradVec {
    float v[VEC];
    __device__ __forceinline__ void load(const ScanArgs &p, int64_t at) {
        if (p.out_bf16) VecLoad<uint16_t, VEC>::load(static_cast<const uint16_t *>(p.g) + at, v);
        else VecLoad<float, VEC>::load(static_cast<const float *>(p.g) + at, v);
    }
};

template <typename XT, int VEC, int KIND>
__global__ void __launch_bounds__(kScanThreads) scan_backward(ScanArgs p) {
    using T = ScanTile<VEC>;
    __shared__ TileRows rows;
    __shared__ __align__(16) float s_a[T::kTall][T::kWide], s_b[T::kTall][T::kWide];      // of the states
    __shared__ __align__(16) float s_u[T::kTall][T::kWide], s_w[T::kTall][T::kWide];      // of the adjoint
    __shared__ float s_carry[T::kWide];
    __shared__ uint32_t s_next;
    __shared__ int s_from;
    if (static_cast<int>(blockIdx.x) < p.checkers) return check_sequences(p, p.grad_final, p.grad_initial);
    int strip;
    const int64_t order = next_tile(p, strip, &s_next), tile = p.tiles - 1 - order, r0 = tile * kTileRows;
    const int lane = threadIdx.x % T::kAcross, group = threadIdx.x / T::kAcross;
    const int64_t c0 = static_cast<int64_t>(strip) * T::kWide, c = c0 + lane * VEC;
    const bool on = c < p.f;

    RowVec<XT, VEC> z[T::kEach], x[T::kEach];
    GradVec<VEC> g[T::kEach];
#pragma unroll
    for (int j = 0; j < T::kEach; ++j) {
        const int64_t r = r0 + group * T::kEach + j;
        z[j] = x[j] = RowVec<XT, VEC>{};
        g[j] = GradVec<VEC>{};
        if (on && r < p.n) {
            z[j].load(static_cast<const XT *>(p.gate) + r * p.gate_ld + c);
            x[j].load(static_cast<const XT *>(p.x) + r * p.x_ld + c);
            if (p.g) g[j].load(p, r * p.f + c);
        }
    }
    find_rows(p, r0, rows);
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
        z[j].widen(v);
        decay_less_one<KIND>(v, d[j]);
        if (!((in >> j) & 1u)) continue;
        if ((begin >> j) & 1u) {
#pragma unroll
            for (int q = 0; q < VEC; ++q) a[q] = 0.f;
            state_or_zero(initial, rows.seq[group * T::kEach + j], p.f, c, b);
        }
        x[j].widen(v);
        fma_vec(a, d[j], a, a);
        fma_vec(b, d[j], b, b);
        add_input<KIND>(b, d[j], v);
    }
#pragma unroll
    for (int j = T::kEach - 1; j >= 0; --j) {
        if (!((in >> j) & 1u)) continue;
        if ((end >> j) & 1u) {
#pragma unroll
            for (int q = 0; q < VEC; ++q) u[q] = 0.f;
            state_or_zero(grad_final, rows.seq[group * T::kEach + j], p.f, c, w);
        }
        add_vec(w, g[j].v);
        fma_vec(u, d[j], u, u);
        fma_vec(w, d[j], w, w);
        if ((begin >> j) & 1u) {
#pragma unroll
            for (int q = 0; q < VEC; ++q) u[q] = w[q] = 0.f;
        }
    }
#pragma unroll
    for (int q = 0; q < VEC; ++q) {
        const int i = lane * VEC + q;
        s_a[group][i] = a[q];
        s_b[group][i] = b[q];
        s_u[group][i] = u[q];
        s_w[group][i] = w[q];
    }
    __syncthreads();

    // threads of the first columns: up the tile; of the next: down it, from the state kept
    const int64_t mc = c0 + threadIdx.x;
    const bool column = static_cast<int>(threadIdx.x) < T::kWide, mine = column && mc < p.f;
    float tu = 1.f, tw = 0.f;
    if (column) {
#pragma unroll
        for (int i = T::kTall - 1; i >= 0; --i) {
            const float gu = s_u[i][threadIdx.x], gw = s_w[i][threadIdx.x];
            s_u[i][threadIdx.x] = tu;
            s_w[i][threadIdx.x] = tw;
            const bool fresh = (row_bits<T::kEach>(rows.begin, i) | row_bits<T::kEach>(rows.end, i)) != 0u;
            tw = fresh ? gw : fmaf(gu, tw, gw);
            tu = fresh ? 0.f : tu * gu;
        }
    } else if (static_cast<int>(threadIdx.x) < 2 * T::kWide) {
        const int i = threadIdx.x - T::kWide;
        float state = c0 + i < p.f ? __ldg(p.entered + tile * p.f + c0 + i) : 0.f;
#pragma unroll
        for (int k = 0; k < T::kTall; ++k) {
            const float ga = s_a[k][i], gb = s_b[k][i];
            s_b[k][i] = state;
            state = row_bits<T::kEach>(rows.begin, k) != 0u ? gb : fmaf(ga, state, gb);
        }
    }
    const bool wants = row_bit(rows.in, kTileRows - 1) && !row_bit(rows.end, kTileRows - 1);
    const float carry = enter_tile(p, order, strip, mc, mine, tu, tw, any_from(rows.begin, 0) || any_from(rows.end, 0), wants,
                                   &s_from);
    if (column) s_carry[threadIdx.x] = carry;
    __syncthreads();
    if (!on) return;

    float before[T::kEach][VEC], v[VEC];
    const int after = (group + 1) * T::kEach;
    const bool cut = after < kTileRows && (any_from(rows.begin, after) || any_from(rows.end, after));
#pragma unroll
    for (int q = 0; q < VEC; ++q) {
        const int i = lane * VEC + q;
        v[q] = s_b[group][i];
        w[q] = cut ? s_w[group][i] : fmaf(s_u[group][i], s_carry[i], s_w[group][i]);
    }
#pragma unroll
    for (int j = 0; j < T::kEach; ++j) {
        if ((begin >> j) & 1u) state_or_zero(initial, rows.seq[group * T::kEach + j], p.f, c, v);
        float xv[VEC];
        x[j].widen(xv);
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
        add_vec(w, g[j].v);                                  // l
        float gz[VEC], gx[VEC];
        x[j].widen(gx);
#pragma unroll
        for (int q = 0; q < VEC; ++q) {
            const float less = -d[j][q];                     // 1 - a
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

template <typename XT, int VEC>
cudaError_t launch_kind(const ScanArgs &p, int kind, cudaStream_t s) {
    const unsigned grid = static_cast<unsigned>(p.checkers + p.tiles * p.strips);
    if (kind == TFG_GATE_SIGMOID) scan_backward<XT, VEC, TFG_GATE_SIGMOID><<<grid, kScanThreads, 0, s>>>(p);
    else scan_backward<XT, VEC, TFG_GATE_EXP><<<grid, kScanThreads, 0, s>>>(p);
    return cudaGetLastError();
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
    cudaError_t e = scan_clear(p, ws, s);
    if (e != cudaSuccess || p.checkers + p.tiles * p.strips == 0) return e;
    if (dtype == TFG_BF16) return vectors ? launch_kind<uint16_t, 8>(p, kind, s) : launch_kind<uint16_t, 1>(p, kind, s);
    return vectors ? launch_kind<float, 4>(p, kind, s) : launch_kind<float, 1>(p, kind, s);
}

}  // namespace tfg
