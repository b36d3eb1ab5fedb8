// Gated linear recurrence, forward, and the host side of both directions
// (gated_recurrence.cuh: the method).
#include "gated_recurrence.cuh"

namespace tfg {
namespace {

template <typename XT, int VEC>
struct ForwardStage {
    using T = ScanTile<VEC>;
    using In = Slots<XT, VEC, T::kEach, kScanThreads>;
    static constexpr int kBytes = 2 * In::kAll;
    In z, x;
    __device__ __forceinline__ explicit ForwardStage(char *stage) : z(stage), x(stage + In::kAll) {}
    __device__ __forceinline__ void copy(const ScanArgs &p, const Job &job, TileRows &rows) const {
        const int lane = threadIdx.x % T::kAcross, group = threadIdx.x / T::kAcross;
        const int64_t c = static_cast<int64_t>(job.strip) * T::kWide + lane * VEC, r0 = job.order * kTileRows + group * T::kEach;
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

// CTAs of a multiprocessor: registers for 64 (two values a word) and 32 channels a tile.
template <int VEC>
constexpr int kForwardCtas = VEC == 8 ? 3 : 4;

template <typename XT, int VEC, int KIND>
__global__ void __launch_bounds__(kScanThreads, kForwardCtas<VEC>) scan_forward(ScanArgs p) {
    using T = ScanTile<VEC>;
    using Stage = ForwardStage<XT, VEC>;
    extern __shared__ __align__(16) char s_stage[];
    __shared__ TileRows rows;
    __shared__ float s_a[kScanWarps][T::kWide], s_b[kScanWarps][T::kWide];
    __shared__ float2 s_part[kScanThreads / T::kWide][T::kWide];
    __shared__ float s_state[T::kWide];
    __shared__ uint32_t s_next;
    __shared__ int s_from;
    if (static_cast<int>(blockIdx.x) < p.checkers) return check_sequences(p, p.initial, p.final_state);
    const int lane = threadIdx.x % T::kAcross, group = threadIdx.x / T::kAcross, warp = threadIdx.x / 32;
    const Job job = next_job(p, &s_next);
    const Stage in_stage(s_stage);
    in_stage.copy(p, job, rows);
    const int64_t r0 = job.order * kTileRows, c0 = static_cast<int64_t>(job.strip) * T::kWide, c = c0 + lane * VEC;
    if (p.linked && warp == 0) {
        const int from = cut_before(p, job.order, kAnyBegin, false);
        if (threadIdx.x == 0) s_from = from;
    }
    const bool on = c < p.f;
    copies_done();
    if (p.linked) __syncthreads();                       // the plan is there
    else find_rows(p, rows);
    const uint32_t begin = row_bits<T::kEach>(rows.begin, group), end = row_bits<T::kEach>(rows.end, group),
                   in = row_bits<T::kEach>(rows.in, group);

    // the thread's map
    float d[T::kEach][VEC], a[VEC], b[VEC];
#pragma unroll
    for (int q = 0; q < VEC; ++q) a[q] = 1.f, b[q] = 0.f;
#pragma unroll
    for (int j = 0; j < T::kEach; ++j) {
        float v[VEC];
        in_stage.z.widen(j, v);
        decay_less_one<KIND>(v, d[j]);
        if (!((in >> j) & 1u)) continue;
        if ((begin >> j) & 1u) {
#pragma unroll
            for (int q = 0; q < VEC; ++q) a[q] = 0.f;
            state_or_zero(on ? p.initial : nullptr, rows.seq[group * T::kEach + j], p.f, c, b);
        }
        in_stage.x.widen(j, v);
        fma_vec(a, d[j], a, a);
        fma_vec(b, d[j], b, b);
        add_input<KIND>(b, d[j], v);
    }
    uint32_t cut = begin;
    scan_groups<VEC, false>(a, b, cut, warp, lane, s_a, s_b);
    __syncthreads();

    // down the warps, a thread for each channel: what stands before each, and the tile's map
    const int64_t mc = c0 + threadIdx.x;
    const bool column = static_cast<int>(threadIdx.x) < T::kWide;
    float ta = 1.f, tb = 0.f;
    if (column) {
#pragma unroll
        for (int w = 0; w < kScanWarps; ++w) {
            const float wa = s_a[w][threadIdx.x], wb = s_b[w][threadIdx.x];
            s_a[w][threadIdx.x] = ta;
            s_b[w][threadIdx.x] = tb;
            const bool fresh = row_bits<kWarpRows>(rows.begin, w) != 0u;
            tb = fresh ? wb : fmaf(wa, tb, wb);          // not 0 times what may be an infinity
            ta = fresh ? 0.f : ta * wa;
        }
    }
    const bool wants = row_bit(rows.in, 0) && !row_bit(rows.begin, 0);
    const float state = enter_tile<T::kWide>(p, job.order, c0, ta, tb, any_from(rows.begin, 0), wants, s_from, s_part);
    if (column) s_state[threadIdx.x] = state;
    if (column && mc < p.f && p.entering) p.entering[job.order * p.f + mc] = state;
    __syncthreads();

    // the rows again, from the state that enters the thread's first
    if (on) {
        float v[VEC];
        const bool far = any_before(rows.begin, warp * kWarpRows);
#pragma unroll
        for (int q = 0; q < VEC; ++q) {
            const int i = lane * VEC + q;
            v[q] = far ? s_b[warp][i] : fmaf(s_a[warp][i], s_state[i], s_b[warp][i]);
            v[q] = cut ? b[q] : fmaf(a[q], v[q], b[q]);
        }
#pragma unroll
        for (int j = 0; j < T::kEach; ++j) {
            if (!((in >> j) & 1u)) continue;
            const int row = group * T::kEach + j;
            if ((begin >> j) & 1u) state_or_zero(p.initial, rows.seq[row], p.f, c, v);
            float w[VEC];
            in_stage.x.widen(j, w);
            fma_vec(v, d[j], v, v);
            add_input<KIND>(v, d[j], w);
            if (p.out_bf16) store_vec<VEC>(static_cast<uint16_t *>(p.out) + (r0 + row) * p.f + c, v);
            else store_vec<VEC>(static_cast<float *>(p.out) + (r0 + row) * p.f + c, v);
            if (((end >> j) & 1u) && p.final_state) store_vec<VEC>(p.final_state + rows.seq[row] * p.f + c, v);
        }
    }
}

// Clears the counter, sets maps and states to what is not there yet, and describes the rows of every
// tile, a warp for each.
__global__ void __launch_bounds__(256) scan_plan_kernel(ScanArgs p, uint4 *words, int64_t n, TileRows *plan) {
    const int64_t threads = static_cast<int64_t>(gridDim.x) * 256, id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (id == 0) *p.status = TFG_OK;
    if (!p.linked) return;
    for (int64_t i = id; i < n; i += threads) words[i] = i ? make_uint4(~0u, ~0u, ~0u, ~0u) : make_uint4(0u, 0u, 0u, 0u);
    for (int64_t tile = id / 32; tile < p.tiles; tile += threads / 32) {
        const int64_t r0 = tile * kTileRows;
        TileRows &t = plan[tile];
        const int lo = static_cast<int>(warp_graph_at(p.offsets, p.seqs, r0));
        const int hi = static_cast<int>(warp_graph_at(p.offsets, p.seqs, min64(r0 + kTileRows, p.n) - 1));
        uint32_t any = 0;
#pragma unroll
        for (int w = 0; w < kTileRows / 32; ++w) any |= describe_row(p, r0 + w * 32 + (threadIdx.x & 31), lo, hi, w, t);
        if ((threadIdx.x & 31) == 0) t.any = any;
    }
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
        p.maps = reinterpret_cast<uint64_t *>(w + ScanSpace::kMaps);
        p.states = reinterpret_cast<uint32_t *>(w + space.states);
        p.plan = reinterpret_cast<const TileRows *>(w + space.plan);
    }
}

cudaError_t scan_plan(const ScanArgs &p, void *ws, cudaStream_t s) {
    if (p.status_all) return cudaSuccess;
    const ScanSpace space(p.n, p.f);
    const int64_t words = static_cast<int64_t>(space.plan / 16);
    const int64_t ctas = min64(words / 256 + 1 + p.tiles / 8, 8 * static_cast<int64_t>(sm_count()));
    scan_plan_kernel<<<static_cast<unsigned>(ctas), 256, 0, s>>>(
        p, static_cast<uint4 *>(ws), words, reinterpret_cast<TileRows *>(static_cast<char *>(ws) + space.plan));
    return cudaGetLastError();
}

size_t gated_recurrence_workspace_bytes(int64_t n, int64_t f) { return ScanSpace(n, f).bytes; }

namespace {

template <typename XT, int VEC, int KIND>
cudaError_t launch_forward(const ScanArgs &p, cudaStream_t s) {
    constexpr int kShared = ForwardStage<XT, VEC>::kBytes;
    static_assert(kShared <= 32 * 1024, "with the static part below the 48 KB every launch may use");
    scan_forward<XT, VEC, KIND><<<static_cast<unsigned>(p.checkers + p.tiles * p.strips), kScanThreads, kShared, s>>>(p);
    return cudaGetLastError();
}
template <typename XT, int VEC>
cudaError_t launch_kind(const ScanArgs &p, int kind, cudaStream_t s) {
    return kind == TFG_GATE_SIGMOID ? launch_forward<XT, VEC, TFG_GATE_SIGMOID>(p, s) : launch_forward<XT, VEC, TFG_GATE_EXP>(p, s);
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
    cudaError_t e = scan_plan(p, ws, s);
    if (e != cudaSuccess || p.checkers + p.tiles * p.strips == 0) return e;
    if (dtype == TFG_BF16) return vectors ? launch_kind<uint16_t, 8>(p, kind, s) : launch_kind<uint16_t, 1>(p, kind, s);
    return vectors ? launch_kind<float, 4>(p, kind, s) : launch_kind<float, 1>(p, kind, s);
}

}  // namespace tfg
