// Gated linear recurrence, forward, and the host side of both directions
// (gated_recurrence.cuh: the method).
#include "gated_recurrence.cuh"

namespace tfg {
namespace {

template <typename XT, int VEC, int KIND>
__global__ void __launch_bounds__(kScanThreads) scan_forward(ScanArgs p) {
    using T = ScanTile<VEC>;
    __shared__ TileRows rows;
    __shared__ __align__(16) float s_a[T::kTall][T::kWide], s_b[T::kTall][T::kWide];
    __shared__ float s_state[T::kWide];
    __shared__ uint32_t s_next;
    __shared__ int s_from;
    if (static_cast<int>(blockIdx.x) < p.checkers) return check_sequences(p, p.initial, p.final_state);
    int strip;
    const int64_t tile = next_tile(p, strip, &s_next), r0 = tile * kTileRows;
    const int lane = threadIdx.x % T::kAcross, group = threadIdx.x / T::kAcross;
    const int64_t c0 = static_cast<int64_t>(strip) * T::kWide, c = c0 + lane * VEC;
    const bool on = c < p.f;

    RowVec<XT, VEC> z[T::kEach], x[T::kEach];
#pragma unroll
    for (int j = 0; j < T::kEach; ++j) {
        const int64_t r = r0 + group * T::kEach + j;
        z[j] = x[j] = RowVec<XT, VEC>{};
        if (on && r < p.n) {
            z[j].load(static_cast<const XT *>(p.gate) + r * p.gate_ld + c);
            x[j].load(static_cast<const XT *>(p.x) + r * p.x_ld + c);
        }
    }
    find_rows(p, r0, rows);
    const uint32_t begin = row_bits<T::kEach>(rows.begin, group), end = row_bits<T::kEach>(rows.end, group),
                   in = row_bits<T::kEach>(rows.in, group);

    // the thread's map
    float d[T::kEach][VEC], a[VEC], b[VEC];
#pragma unroll
    for (int q = 0; q < VEC; ++q) a[q] = 1.f, b[q] = 0.f;
#pragma unroll
    for (int j = 0; j < T::kEach; ++j) {
        float v[VEC];
        z[j].widen(v);
        decay_less_one<KIND>(v, d[j]);
        if (!((in >> j) & 1u)) continue;
        if ((begin >> j) & 1u) {
#pragma unroll
            for (int q = 0; q < VEC; ++q) a[q] = 0.f;
            state_or_zero(on ? p.initial : nullptr, rows.seq[group * T::kEach + j], p.f, c, b);
        }
        x[j].widen(v);
        fma_vec(a, d[j], a, a);
        fma_vec(b, d[j], b, b);
        add_input<KIND>(b, d[j], v);
    }
#pragma unroll
    for (int q = 0; q < VEC; ++q) {
        s_a[group][lane * VEC + q] = a[q];
        s_b[group][lane * VEC + q] = b[q];
    }
    __syncthreads();

    // down the tile, a thread for each channel: what stands before each group, and the tile's map
    const int64_t mc = c0 + threadIdx.x;
    const bool column = static_cast<int>(threadIdx.x) < T::kWide, mine = column && mc < p.f;
    float ta = 1.f, tb = 0.f;
    if (column) {
#pragma unroll
        for (int g = 0; g < T::kTall; ++g) {
            const float ga = s_a[g][threadIdx.x], gb = s_b[g][threadIdx.x];
            s_a[g][threadIdx.x] = ta;
            s_b[g][threadIdx.x] = tb;
            const bool fresh = row_bits<T::kEach>(rows.begin, g) != 0u;
            tb = fresh ? gb : fmaf(ga, tb, gb);              // not 0 times what may be an infinity
            ta = fresh ? 0.f : ta * ga;
        }
    }
    const bool wants = row_bit(rows.in, 0) && !row_bit(rows.begin, 0);
    const float state = enter_tile(p, tile, strip, mc, mine, ta, tb, any_from(rows.begin, 0), wants, &s_from);
    if (column) s_state[threadIdx.x] = state;
    if (mine && p.entering) p.entering[tile * p.f + mc] = state;
    __syncthreads();
    if (!on) return;

    // the rows again, from the state that enters the thread's first
    float v[VEC];
    const bool cut = any_before(rows.begin, group * T::kEach);
#pragma unroll
    for (int q = 0; q < VEC; ++q) {
        const int i = lane * VEC + q;
        v[q] = cut ? s_b[group][i] : fmaf(s_a[group][i], s_state[i], s_b[group][i]);
    }
#pragma unroll
    for (int j = 0; j < T::kEach; ++j) {
        if (!((in >> j) & 1u)) continue;
        const int row = group * T::kEach + j;
        if ((begin >> j) & 1u) state_or_zero(p.initial, rows.seq[row], p.f, c, v);
        float w[VEC];
        x[j].widen(w);
        fma_vec(v, d[j], v, v);
        add_input<KIND>(v, d[j], w);
        if (p.out_bf16) store_vec<VEC>(static_cast<uint16_t *>(p.out) + (r0 + row) * p.f + c, v);
        else store_vec<VEC>(static_cast<float *>(p.out) + (r0 + row) * p.f + c, v);
        if (((end >> j) & 1u) && p.final_state) store_vec<VEC>(p.final_state + rows.seq[row] * p.f + c, v);
    }
}

__global__ void __launch_bounds__(256) clear_words(uint4 *words, int64_t n, int32_t *status) {
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (i < n) words[i] = make_uint4(0u, 0u, 0u, 0u);
    if (i == 0) *status = TFG_OK;
}

constexpr int64_t kOneChecker = 8192;     // sequences that one CTA looks at

}  // namespace

bool scan_vectors(const ScanArgs &p, int dtype, bool backward) {
    const int vec = dtype == TFG_BF16 ? 8 : 4, size = dtype == TFG_BF16 ? 2 : 4;
    const auto at = [](const void *q, int bytes) { return reinterpret_cast<uintptr_t>(q) % bytes == 0; };
    if (p.f % vec || p.gate_ld % vec || p.x_ld % vec || !at(p.gate, 16) || !at(p.x, 16) || !at(p.initial, 16)) return false;
    const int wide = p.out_bf16 ? vec * 2 : 16;              // bytes of a vector of out or its gradient
    if (!backward) return at(p.out, wide) && at(p.final_state, 16);
    return at(p.g, wide) && at(p.grad_final, 16) && at(p.grad_initial, 16) && p.grad_gate_ld % vec == 0 &&
           p.grad_x_ld % vec == 0 && at(p.grad_gate, vec * size) && at(p.grad_x, vec * size) && at(p.entered, 16);
}

void scan_geometry(ScanArgs &p, int dtype, bool vectors, void *ws, int32_t *status) {
    const int wide = !vectors ? ScanTile<1>::kWide : (dtype == TFG_BF16 ? ScanTile<8>::kWide : ScanTile<4>::kWide);
    p.tiles = (p.n + kTileRows - 1) / kTileRows;
    p.windows = (p.tiles + kWindow - 1) / kWindow;
    p.strips = static_cast<int>((p.f + wide - 1) / wide);
    p.linked = p.tiles > 1;
    const bool whole = !p.linked && p.seqs <= kOneChecker;
    p.checkers = whole ? 1 : static_cast<int>(min64((p.seqs + kScanThreads - 1) / kScanThreads, 8 * sm_count()));
    p.status = status;
    p.status_all = whole ? status : nullptr;
    if (p.linked) {
        const ScanSpace space(p.n, p.f);
        char *w = static_cast<char *>(ws);
        p.next = reinterpret_cast<uint32_t *>(w);
        p.ready = p.next + 4;
        p.passed = p.ready + p.strips * p.tiles;
        p.maps = reinterpret_cast<float2 *>(w + space.maps);
        p.states = reinterpret_cast<float *>(w + space.states);
    }
}

cudaError_t scan_clear(const ScanArgs &p, void *ws, cudaStream_t s) {
    if (p.status_all) return cudaSuccess;
    const int64_t words = p.linked ? static_cast<int64_t>(ScanSpace(p.n, p.f).clear / 16) : 0;
    clear_words<<<static_cast<unsigned>(words / 256 + 1), 256, 0, s>>>(static_cast<uint4 *>(ws), words, p.status);
    return cudaGetLastError();
}

size_t gated_recurrence_workspace_bytes(int64_t n, int64_t f) { return ScanSpace(n, f).bytes; }

namespace {

template <typename XT, int VEC>
cudaError_t launch_kind(const ScanArgs &p, int kind, cudaStream_t s) {
    const unsigned grid = static_cast<unsigned>(p.checkers + p.tiles * p.strips);
    if (kind == TFG_GATE_SIGMOID) scan_forward<XT, VEC, TFG_GATE_SIGMOID><<<grid, kScanThreads, 0, s>>>(p);
    else scan_forward<XT, VEC, TFG_GATE_EXP><<<grid, kScanThreads, 0, s>>>(p);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_gated_recurrence(const void *gate, int64_t gate_ld, const void *x, int64_t x_ld, int dtype,
                                    const int64_t *offsets, int64_t n, int64_t seqs, int64_t f, int kind,
                                    const float *initial, void *out, int out_dtype, float *final_state, float *entering,
                                    void *ws, int32_t *status, cudaStream_t s) {
    ScanArgs p{};
    p.gate = gate, p.gate_ld = gate_ld, p.x = x, p.x_ld = x_ld, p.offsets = offsets, p.n = n, p.seqs = seqs, p.f = f;
    p.initial = initial, p.out = out, p.out_bf16 = out_dtype == TFG_BF16, p.final_state = final_state, p.entering = entering;
    const bool vectors = scan_vectors(p, dtype, false);
    scan_geometry(p, dtype, vectors, ws, status);
    cudaError_t e = scan_clear(p, ws, s);
    if (e != cudaSuccess || p.checkers + p.tiles * p.strips == 0) return e;
    if (dtype == TFG_BF16) return vectors ? launch_kind<uint16_t, 8>(p, kind, s) : launch_kind<uint16_t, 1>(p, kind, s);
    return vectors ? launch_kind<float, 4>(p, kind, s) : launch_kind<float, 1>(p, kind, s);
}

}  // namespace tfg
