// Gated linear recurrence: the host side of both directions, and the kernel that describes the rows
// (gated_recurrence.cuh: the method; gated_recurrence_forward.cuh, gated_recurrence_backward.cuh: the kernels).
#include <mutex>

#include "gated_recurrence.cuh"

namespace tfg {
namespace {

// Clears the counter, sets maps and states to what is not there yet, and describes the rows of every
// tile, a warp for each 32.
__global__ void __launch_bounds__(256) scan_plan_kernel(ScanArgs p, uint4 *words, int64_t n, TileRows *plan) {
    cudaTriggerProgrammaticLaunchCompletion();               // the tiles' kernel may be set up; it waits for this one's end
    // CTAs of their own: beside the rest the two offsets cost every CTA a trip to memory (1,024 molecules 107 -> 110 us)
    if (static_cast<int>(blockIdx.x) < p.clear_ctas) return clear_outside(p, blockIdx.x * 8 + threadIdx.x / 32, p.clear_ctas * 8);
    const int64_t threads = static_cast<int64_t>(gridDim.x - p.clear_ctas) * 256,
                  id = static_cast<int64_t>(blockIdx.x - p.clear_ctas) * 256 + threadIdx.x;
    if (id == 0) *p.status = TFG_OK;
    if (!p.linked) return;
    for (int64_t i = id; i < n; i += threads) words[i] = i ? make_uint4(~0u, ~0u, ~0u, ~0u) : make_uint4(0u, 0u, 0u, 0u);
    constexpr int kWords = kTileRows / 32;
    for (int64_t word = id / 32; word < p.tiles * kWords; word += threads / 32) {
        const int64_t tile = word / kWords, r0 = word * 32, last = min64(r0 + 32, p.n) - 1;
        const int lo = static_cast<int>(warp_graph_at(p.offsets, p.seqs, r0 < p.n ? r0 : last));
        const int hi = static_cast<int>(warp_graph_at(p.offsets, p.seqs, last));
        describe_row(p, r0 + (threadIdx.x & 31), lo, hi, static_cast<int>(word % kWords), plan[tile]);
    }
}

constexpr int64_t kOneChecker = 8192;     // sequences that one CTA looks at

int scan_vector(const ScanArgs &p, int dtype, bool backward) {
    const int size = dtype == TFG_BF16 ? 2 : 4;
    const auto at = [](const void *q, int bytes) { return reinterpret_cast<uintptr_t>(q) % bytes == 0; };
    const auto fits = [&](int vec) {
        if (p.f % vec || p.gate_ld % vec || p.x_ld % vec || !at(p.gate, 16) || !at(p.x, 16) || !at(p.initial, 16)) return false;
        if (p.gate_ld * size >= int64_t(1) << 40 || p.x_ld * size >= int64_t(1) << 40) return false;   // strides that a map can have
        const int wide = p.out_bf16 ? vec * 2 : 16;          // bytes of a vector of out or its gradient
        if (!backward) return at(p.out, wide) && at(p.final_state, 16);
        const int rows = p.out_bf16 ? 2 : 4;                 // dL/dout comes by copies of whole 16 bytes
        return at(p.g, 16) && p.f * rows % 16 == 0 && at(p.grad_final, 16) && at(p.grad_initial, 16) && p.grad_gate_ld % vec == 0 &&
               p.grad_x_ld % vec == 0 && at(p.grad_gate, 16) && at(p.grad_x, 16);
    };
    return fits(16 / size) ? 4 : 1;
}

// Channels of a tile.
int tile_channels(int dtype, int vec) {
    if (vec == 1) return ScanTile<float, 1>::kWide;
    return dtype == TFG_BF16 ? ScanTile<uint16_t, 4>::kWide : ScanTile<float, 4>::kWide;
}

// The rows of up to two outputs that become zeros outside all sequences.
void clear_rows(ScanArgs &p, int size, void *a, int64_t a_ld, void *b, int64_t b_ld) {
    p.clear[0] = static_cast<char *>(a), p.clear[1] = static_cast<char *>(b);
    p.clear_ld[0] = a_ld * size, p.clear_ld[1] = b_ld * size, p.clear_width = p.f * size;
    const uint64_t all = reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b) | p.clear_ld[0] | p.clear_ld[1] | p.clear_width;
    p.clear_unit = all % 16 == 0 ? 16 : size;
    p.clear_ctas = sm_count();
}

void scan_geometry(ScanArgs &p, int dtype, int vec, void *ws, int32_t *status) {
    const int wide = tile_channels(dtype, vec);
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

using EncodeTiledFn = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                   const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                   CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's encoder of tensor maps, looked up through the runtime (the library links no libcuda).
EncodeTiledFn encode_tiled() {
    static std::once_flag once;
    static EncodeTiledFn fn = nullptr;
    std::call_once(once, [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult q{};
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeTiledFn>(f);
    });
    return fn;
}

// Rows of f values, ld apart, in tiles of kTileRows by `wide` channels.
bool row_map(CUtensorMap &map, const void *rows, bool bf16, int64_t n, int64_t f, int64_t ld, int wide) {
    const EncodeTiledFn encode = encode_tiled();
    if (!encode) return false;
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(f), static_cast<cuuint64_t>(n)};
    const cuuint64_t stride[1] = {static_cast<cuuint64_t>(ld) * (bf16 ? 2 : 4)};
    const cuuint32_t box[2] = {static_cast<cuuint32_t>(wide), kTileRows}, step[2] = {1, 1};
    return encode(&map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, const_cast<void *>(rows), dims,
                  stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool scan_maps(const ScanArgs &p, int dtype, bool backward, ScanMaps &maps) {
    const bool bf16 = dtype == TFG_BF16;
    const int wide = tile_channels(dtype, 4);
    return row_map(maps.gate, p.gate, bf16, p.n, p.f, p.gate_ld, wide) && row_map(maps.x, p.x, bf16, p.n, p.f, p.x_ld, wide) &&
           (!backward || !p.g || row_map(maps.g, p.g, p.out_bf16, p.n, p.f, p.f, wide));
}

cudaError_t scan_plan(const ScanArgs &p, void *ws, cudaStream_t s) {
    if (p.status_all) return cudaSuccess;
    const ScanSpace space(p.n, p.f);
    const int64_t words = static_cast<int64_t>(space.plan / 16);
    const int64_t ctas = min64(words / 256 + 1 + p.tiles * (kTileRows / 32) / 8, 8 * static_cast<int64_t>(sm_count()));
    scan_plan_kernel<<<static_cast<unsigned>(ctas + p.clear_ctas), 256, 0, s>>>(
        p, static_cast<uint4 *>(ws), words, reinterpret_cast<TileRows *>(static_cast<char *>(ws) + space.plan));
    return cudaGetLastError();
}

}  // namespace

size_t gated_recurrence_workspace_bytes(int64_t n, int64_t f) { return ScanSpace(n, f).bytes; }

cudaError_t launch_scan_forward_f32(const ScanArgs &p, const ScanMaps &maps, int vec, int kind, cudaStream_t s);
cudaError_t launch_scan_forward_bf16(const ScanArgs &p, const ScanMaps &maps, int vec, int kind, cudaStream_t s);
cudaError_t launch_scan_backward_f32(const ScanArgs &p, const ScanMaps &maps, int vec, int kind, cudaStream_t s);
cudaError_t launch_scan_backward_bf16(const ScanArgs &p, const ScanMaps &maps, int vec, int kind, cudaStream_t s);

cudaError_t launch_gated_recurrence(const void *gate, int64_t gate_ld, const void *x, int64_t x_ld, int dtype,
                                    const int64_t *offsets, int64_t n, int64_t seqs, int64_t f, int kind, bool zeroes,
                                    const float *initial, void *out, int out_dtype, float *final_state, float *entering,
                                    void *ws, int32_t *status, cudaStream_t s) {
    ScanArgs p{};
    p.gate = gate, p.gate_ld = gate_ld, p.x = x, p.x_ld = x_ld, p.offsets = offsets, p.n = n, p.seqs = seqs, p.f = f;
    p.initial = initial, p.out = out, p.out_bf16 = out_dtype == TFG_BF16, p.final_state = final_state, p.entering = entering;
    if (zeroes) clear_rows(p, out_dtype == TFG_BF16 ? 2 : 4, out, f, nullptr, 0);
    const int vec = scan_vector(p, dtype, false);
    scan_geometry(p, dtype, vec, ws, status);
    const cudaError_t e = scan_plan(p, ws, s);
    if (e != cudaSuccess || p.checkers + p.tiles * p.strips == 0) return e;
    ScanMaps maps;
    if (vec > 1 && p.tiles > 0 && !scan_maps(p, dtype, false, maps)) return cudaErrorNotSupported;
    return dtype == TFG_BF16 ? launch_scan_forward_bf16(p, maps, vec, kind, s) : launch_scan_forward_f32(p, maps, vec, kind, s);
}

cudaError_t launch_gated_recurrence_backward(const void *gate, int64_t gate_ld, const void *x, int64_t x_ld, int dtype,
                                             const int64_t *offsets, int64_t n, int64_t seqs, int64_t f, int kind, bool zeroes,
                                             const float *initial, const float *entered, const void *g, int g_dtype,
                                             const float *grad_final, void *grad_gate, int64_t grad_gate_ld, void *grad_x,
                                             int64_t grad_x_ld, float *grad_initial, void *ws, int32_t *status,
                                             cudaStream_t s) {
    ScanArgs p{};
    p.gate = gate, p.gate_ld = gate_ld, p.x = x, p.x_ld = x_ld, p.offsets = offsets, p.n = n, p.seqs = seqs, p.f = f;
    p.initial = initial, p.entered = entered, p.g = g, p.out_bf16 = g_dtype == TFG_BF16, p.grad_final = grad_final;
    p.grad_gate = grad_gate, p.grad_gate_ld = grad_gate_ld, p.grad_x = grad_x, p.grad_x_ld = grad_x_ld;
    p.grad_initial = grad_initial;
    if (zeroes) clear_rows(p, dtype == TFG_BF16 ? 2 : 4, grad_gate, grad_gate_ld, grad_x, grad_x_ld);
    const int vec = scan_vector(p, dtype, true);
    scan_geometry(p, dtype, vec, ws, status);
    const cudaError_t e = scan_plan(p, ws, s);
    if (e != cudaSuccess || p.checkers + p.tiles * p.strips == 0) return e;
    ScanMaps maps;
    if (vec > 1 && p.tiles > 0 && !scan_maps(p, dtype, true, maps)) return cudaErrorNotSupported;
    return dtype == TFG_BF16 ? launch_scan_backward_bf16(p, maps, vec, kind, s) : launch_scan_backward_f32(p, maps, vec, kind, s);
}

}  // namespace tfg
