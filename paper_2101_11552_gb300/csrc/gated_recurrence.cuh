// Gated linear recurrence along the rows of each sequence of a batch: what the forward
// (gated_recurrence.cu) and the backward (gated_recurrence_backward.cu) share.
//
//   v_t = a_t v_{t-1} + b_t, channel by channel, rows node_offsets[s] .. node_offsets[s + 1] - 1
//   sigmoid gate: a = 1 / (1 + e^-z), b = (1 - a) x;   exp gate: a = e^z, b = x
//
// A row is an affine map of the state, and maps compose: (A, B) then (a, b) is (a A, a B + b).
// A CTA takes a tile of 128 rows by 32 or 64 channels and holds its gates and inputs in
// registers; each thread composes the maps of its few rows, the threads' maps are composed
// down the tile in shared memory, the tile's map is published, the state that enters the tile
// is found from what the tiles before it published, and a second walk over the registers makes the
// outputs.  So the inputs come from memory once, however long a sequence is.  A row that begins
// a sequence forgets what comes before it, so tiles need not know sequences.
//
// The entering state.  Tiles stand in windows of 32.  A tile composes the maps of those before it
// in its window, and the last one of a window publishes the state that enters the next.  A tile
// behind the beginning of a sequence in its window needs no more than that.  What is composed
// and in which order depends on nothing but the sizes and offsets, so results are bitwise
// reproducible; with states passed on from tile to tile a batch of 1,000 tiles would take as
// many trips through L2.  Tiles are handed out in order by a counter: a tile waits only for
// tiles that are already running.
//
// Precision.  1 - a is formed directly and the state advances as v - (1 - a) v + b: a gate near 1 keeps
// its distance from 1 to a few u, where a rounded a would change a memory of 1,000 steps by
// 1,000 u.  All in fp32.
#pragma once

#include "widen.cuh"

namespace tfg {

constexpr int kTileRows = TFG_RECURRENCE_TILE_ROWS;
constexpr int kScanThreads = 256;
constexpr int kWindow = 32;               // tiles of a window, one for each lane that waits

struct ScanArgs {
    const void *gate, *x;
    int64_t gate_ld, x_ld;                // from row to row, in values
    const int64_t *offsets;
    int64_t n, seqs, f;
    const float *initial;                 // [seqs][f] or null: zeros
    void *out;
    bool out_bf16;
    float *final_state;                   // [seqs][f] or null
    float *entering;                      // [tiles][f]: states that enter the tiles; or null
    const float *entered;                 // backward: the same
    const void *g;                        // backward: dL/dout or null
    const float *grad_final;              // backward: dL/dfinal or null
    void *grad_gate, *grad_x;
    int64_t grad_gate_ld, grad_x_ld;
    float *grad_initial;                  // or null
    int64_t tiles;
    int strips;                           // of channels
    bool linked;                          // there are tiles to wait for
    int checkers;                         // CTAs in front that look at the sequences
    uint32_t *next;                       // the counter that hands out tiles
    uint32_t *ready;                      // [strip][tile in order of work]: kMapReady, kMapFresh
    uint32_t *passed;                     // [strip][window]: the state that enters it is there
    float2 *maps;                         // [tile in order of work][f]
    float *states;                        // [window][f]
    int64_t windows;
    int32_t *status;
    int32_t *status_all;                  // or null: written whole by the one checker
};

// Bytes of a call that links tiles: [counter, flags] cleared beforehand, maps, states.
struct ScanSpace {
    size_t clear, maps, states, bytes;
    __host__ ScanSpace(int64_t n, int64_t f) {
        const int64_t tiles = (n + kTileRows - 1) / kTileRows, windows = (tiles + kWindow - 1) / kWindow;
        const int64_t strips = (f + 31) / 32;                // of the narrowest tiles
        if (tiles <= 1) {
            clear = maps = states = bytes = 0;
            return;
        }
        clear = (sizeof(uint32_t) * size_t(4 + strips * (tiles + windows)) + 15) / 16 * 16;
        maps = clear;
        states = maps + sizeof(float2) * size_t(tiles * f);
        bytes = (states + sizeof(float) * size_t(windows * f) + 15) / 16 * 16;
    }
};

bool scan_vectors(const ScanArgs &p, int dtype, bool backward);
void scan_geometry(ScanArgs &p, int dtype, bool vectors, void *ws, int32_t *status);
cudaError_t scan_clear(const ScanArgs &p, void *ws, cudaStream_t s);

namespace {

constexpr uint32_t kMapReady = 1, kMapFresh = 2;             // fresh: nothing before the tile reaches behind it
constexpr int kWaitLimit = 1 << 22;                          // looks at a flag, some seconds

__device__ __forceinline__ uint32_t ld_acquire(const uint32_t *p) {
    uint32_t v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ void st_release(uint32_t *p, uint32_t v) {
    asm volatile("st.release.gpu.global.u32 [%0], %1;" ::"l"(p), "r"(v) : "memory");
}
// The flag once it is set; after too many looks the status tells and the wait ends.
__device__ __forceinline__ uint32_t wait_for(const uint32_t *flag, int32_t *status) {
    for (int i = 0; i < kWaitLimit; ++i) {
        const uint32_t v = ld_acquire(flag);
        if (v) return v;
        __nanosleep(20);
    }
    set_status(status, TFG_ERR_TIMEOUT);
    return kMapReady;
}

// ---- gates ----------------------------------------------------------------------------
// expm1(z) for |z| <= 0.35: z + z^2 q(z), q of degree 4 through the Chebyshev points of that
// interval; within 1.5 u of itself over all fp32 values there.
__device__ __forceinline__ float expm1_near(float z) {
    float q = 0.0013934534508734941f;
    q = fmaf(q, z, 0.008363769389688969f);
    q = fmaf(q, z, 0.04166645556688309f);
    q = fmaf(q, z, 0.16666573286056519f);
    q = fmaf(q, z, 0.5f);
    return fmaf(z * z, q, z);
}

// a - 1 of VEC gates.  Sigmoid: -1 / (1 + 2^(z log2 e)), within (|z| + 4) u of itself.  Exp:
// further from 0 than 0.35, 2^(z log2 e) - 1.
template <int KIND, int VEC>
__device__ __forceinline__ void decay_less_one(const float (&z)[VEC], float (&d)[VEC]) {
    const float log2e[1] = {1.44269504088896341f};
#pragma unroll
    for (int q = 0; q < VEC; ++q) d[q] = z[q];
    mul_vec(d, log2e);
#pragma unroll
    for (int q = 0; q < VEC; ++q) d[q] = exp2_of(d[q]);
    if constexpr (KIND == TFG_GATE_SIGMOID) {
        const float one[1] = {1.f};
        add_vec(d, one);
#pragma unroll
        for (int q = 0; q < VEC; ++q) asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(d[q]) : "f"(-d[q]));
    } else {
        const float minus_one[1] = {-1.f};
        add_vec(d, minus_one);
#pragma unroll
        for (int q = 0; q < VEC; ++q) d[q] = fabsf(z[q]) <= 0.35f ? expm1_near(z[q]) : d[q];
    }
}

// b of a row added to a state, d = a - 1.
template <int KIND, int VEC>
__device__ __forceinline__ void add_input(float (&v)[VEC], const float (&d)[VEC], const float (&x)[VEC]) {
    if constexpr (KIND == TFG_GATE_SIGMOID) {
#pragma unroll
        for (int q = 0; q < VEC; ++q) v[q] = fmaf(-d[q], x[q], v[q]);
    } else {
        add_vec(v, x);
    }
}

// ---- the rows of a tile ----------------------------------------------------------------
struct TileRows {
    int32_t seq[kTileRows];               // of the rows inside sequences
    uint32_t begin[kTileRows / 32];       // bits: the row begins its sequence,
    uint32_t end[kTileRows / 32];         // ends it,
    uint32_t in[kTileRows / 32];          // lies inside one
    int lo, hi;
};

template <int PER>
__device__ __forceinline__ uint32_t row_bits(const uint32_t *bits, int group) {
    return (bits[group * PER / 32] >> (group * PER % 32)) & ((1u << PER) - 1u);
}
// Whether a bit is set before, or from, row r on.
__device__ __forceinline__ bool any_before(const uint32_t *bits, int r) {
    bool any = false;
#pragma unroll
    for (int i = 0; i < kTileRows / 32; ++i) {
        const int left = r - i * 32;
        any |= left > 0 && (bits[i] & (left >= 32 ? kAllLanes : (1u << left) - 1u)) != 0u;
    }
    return any;
}
__device__ __forceinline__ bool any_from(const uint32_t *bits, int r) {
    bool any = false;
#pragma unroll
    for (int i = 0; i < kTileRows / 32; ++i) {
        const int skip = r - i * 32;
        any |= skip < 32 && (skip <= 0 ? bits[i] : bits[i] >> skip) != 0u;
    }
    return any;
}
__device__ __forceinline__ bool row_bit(const uint32_t *bits, int r) { return (bits[r / 32] >> (r % 32)) & 1u; }

// Whole CTA; ends with a barrier.  Whatever the offsets say, seq lies in [0, seqs).
__device__ __forceinline__ void find_rows(const ScanArgs &p, int64_t r0, TileRows &t) {
    const int tid = threadIdx.x;
    if (tid < 64) {
        const int64_t last = min64(r0 + kTileRows, p.n) - 1;
        const int64_t s = warp_graph_at(p.offsets, p.seqs, tid < 32 ? r0 : last);
        if ((tid & 31) == 0) (tid < 32 ? t.lo : t.hi) = static_cast<int>(s);
    }
    __syncthreads();
    if (tid < kTileRows) {
        const int64_t r = r0 + tid;
        int lo = t.lo, hi = t.hi;
        while (lo < hi) {
            const int mid = lo + (hi - lo + 1) / 2;
            if (__ldg(p.offsets + mid) <= r) lo = mid;
            else hi = mid - 1;
        }
        bool begins = false, ends = false, in = false;
        if (lo >= 0 && r < p.n) {
            const int64_t a = __ldg(p.offsets + lo), b = __ldg(p.offsets + lo + 1);
            in = a <= r && r < b;
            begins = in && a == r;
            ends = in && b == r + 1;
        }
        t.seq[tid] = lo < 0 ? 0 : lo;
        const uint32_t bb = lane_ballot(begins), eb = lane_ballot(ends), ib = lane_ballot(in);
        if ((tid & 31) == 0) {
            t.begin[tid / 32] = bb;
            t.end[tid / 32] = eb;
            t.in[tid / 32] = ib;
        }
    }
    __syncthreads();
}

// The sequences by themselves: offsets that decrease or leave [0, n], and what an empty
// sequence hands on: to = from (zeros without).
__device__ __forceinline__ void check_sequences(const ScanArgs &p, const float *from, float *to) {
    const int lane = threadIdx.x & 31;
    bool any = false;
    const int64_t step = static_cast<int64_t>(p.checkers) * kScanThreads;
    for (int64_t s0 = static_cast<int64_t>(blockIdx.x) * kScanThreads + threadIdx.x - lane; s0 < p.seqs; s0 += step) {
        const int64_t s = s0 + lane;
        bool empty = false;
        if (s < p.seqs) {
            const int64_t a = __ldg(p.offsets + s), b = __ldg(p.offsets + s + 1);
            any |= a < 0 || b < a || b > p.n;
            empty = b <= a;
        }
        if (!to) continue;
        uint32_t left = lane_ballot(empty);
        for (; left; left &= left - 1) {
            const int64_t at = (s0 + __ffs(left) - 1) * p.f;
            for (int64_t c = lane; c < p.f; c += 32) to[at + c] = from ? __ldg(from + at + c) : 0.f;
        }
    }
    const int all = __syncthreads_or(any);
    if (threadIdx.x != 0) return;
    if (p.status_all) *p.status_all = all ? TFG_ERR_INDEX_RANGE : TFG_OK;
    else if (all) set_status(p.status, TFG_ERR_INDEX_RANGE);
}

// ---- a tile ------------------------------------------------------------------------------
template <int VEC>
struct ScanTile {
    static constexpr int kAcross = VEC == 1 ? 32 : 8;        // threads side by side in a row
    static constexpr int kTall = kScanThreads / kAcross;     // threads down the rows
    static constexpr int kEach = kTileRows / kTall;          // rows of a thread
    static constexpr int kWide = kAcross * VEC;              // channels
};

// The state that enters the order-th tile of a strip, for the channel c of each of the first
// `wide` threads, from the maps (a, b) of the tiles before.  Whole CTA.  fresh: nothing that
// enters the tile leaves it.  wants: the tile's first row (in order of work) goes on from
// the tile before.
__device__ __forceinline__ float enter_tile(const ScanArgs &p, int64_t order, int strip, int64_t c, bool mine, float a, float b,
                                            bool fresh, bool wants, int *s_from) {
    if (!p.linked) return 0.f;
    const int64_t window = order / kWindow;
    const int place = static_cast<int>(order - window * kWindow);
    if (mine) __stcg(p.maps + order * p.f + c, make_float2(a, b));
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        st_release(p.ready + strip * p.tiles + order, fresh ? kMapFresh : kMapReady);
    }
    float state = 0.f;
    wants = wants && order > 0;
    if (wants) {
        if (threadIdx.x < 32) {
            uint32_t flag = 0;
            if (static_cast<int>(threadIdx.x) < place) flag = wait_for(p.ready + strip * p.tiles + order - place + threadIdx.x, p.status);
            const uint32_t cut = lane_ballot(flag == kMapFresh);
            if (threadIdx.x == 0) *s_from = 31 - __clz(static_cast<int>(cut));
        }
        __syncthreads();
        const int from = *s_from;
        float ma = from < 0 ? 1.f : 0.f, mb = 0.f;
        if (mine) {
            const float2 *maps = p.maps + (order - place) * p.f + c;
            if (from >= 0) mb = __ldcg(maps + from * p.f).y;
#pragma unroll 8
            for (int i = from + 1; i < place; ++i) {
                const float2 m = __ldcg(maps + i * p.f);
                mb = fmaf(m.x, mb, m.y);
                ma *= m.x;
            }
        }
        state = mb;
        if (from < 0 && window > 0) {
            if (threadIdx.x == 0) wait_for(p.passed + strip * p.windows + window, p.status);
            __syncthreads();
            if (mine) state = fmaf(ma, __ldcg(p.states + window * p.f + c), mb);
        }
    }
    if (place == kWindow - 1 && order + 1 < p.tiles) {
        if (mine) __stcg(p.states + (window + 1) * p.f + c, fresh ? b : fmaf(a, state, b));
        __syncthreads();
        if (threadIdx.x == 0) {
            __threadfence();
            st_release(p.passed + strip * p.windows + window + 1, kMapReady);
        }
    }
    return state;
}

// The tile of this CTA in order of work, and its strip.
__device__ __forceinline__ int64_t next_tile(const ScanArgs &p, int &strip, uint32_t *s_next) {
    int64_t job = static_cast<int64_t>(blockIdx.x) - p.checkers;
    if (p.linked) {
        if (threadIdx.x == 0) *s_next = atomicAdd(p.next, 1u);
        __syncthreads();
        job = *s_next;
    }
    const int64_t order = job / p.strips;
    strip = static_cast<int>(job - order * p.strips);
    return order;
}

template <int VEC>
__device__ __forceinline__ void state_or_zero(const float *states, int64_t seq, int64_t f, int64_t c, float (&v)[VEC]) {
    if (states) {
        VecLoad<float, VEC>::load(states + seq * f + c, v);
    } else {
#pragma unroll
        for (int q = 0; q < VEC; ++q) v[q] = 0.f;
    }
}

}  // namespace
}  // namespace tfg
