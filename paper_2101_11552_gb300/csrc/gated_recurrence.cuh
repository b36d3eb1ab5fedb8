// Gated linear recurrence along the rows of each sequence of a batch: what the forward
// (gated_recurrence_forward.cuh) and the backward (gated_recurrence_backward.cuh) share.
//
//   v_t = a_t v_{t-1} + b_t, channel by channel, rows node_offsets[s] .. node_offsets[s + 1] - 1
//   sigmoid gate: a = 1 / (1 + e^-z), b = (1 - a) x;   exp gate: a = e^z, b = x
//
// A row is an affine map of the state, and maps compose: (A, B) then (a, b) is (a A, a B + b).
// A CTA takes tiles of 128 rows by 32 or 64 channels into shared memory (one tensor copy for an array; value by value
// where rows are not whole 16 bytes).  Each thread composes the maps of its few rows, the threads' maps are composed down
// the tile, the tile's map is published, the state that enters the tile is found from what the tiles before it
// published, and a second walk over the tile makes the outputs.  So the inputs come from memory once, however long a
// sequence is.  A row that begins a sequence forgets what comes before it, so tiles need not know sequences.
//
// The entering state.  Tiles stand in windows of 32.  A tile composes the maps of those before it in its window, and the
// last one of a window publishes the state that enters the next.  A tile behind the beginning of a sequence in its window
// needs no more than that.  What is composed and in which order depends on nothing but the sizes and offsets, so results
// are bitwise reproducible; with states passed on from tile to tile a batch of 1,000 tiles would take as many trips
// through L2.  A map and a state are each one word, all ones until they are published, so a reader looks at the value
// itself: no flag, no fence, one trip.  Tiles are handed out in order by a counter: a tile waits only for tiles that are
// already running.  It publishes before it waits, and asks for its next tile when its own waiting is over: CTAs that held
// a second tile while the first waited made a convoy of it (1,024 molecules forward: 213 us, where one tile at a
// time took 42).
//
// The decay of a composed map.  Sigmoid gates: the product of the a, at most 1.  Exponential gates: the square root of the
// product, e^(sum of z / 2) of a thread's rows, at most the largest number.  Gates above 0 grow, and the product of 100 rows may pass
// what fp32 holds where the states do not: a state of 0 stays 0 and one of 1e-30 comes back to ordinary size, where an
// infinite product makes NaN of the one and an infinity of the other; and a product below 2^-126 is not lost before a large
// state meets it.  (The logarithm in its place, an exponential for each map applied: 204 us where the root took 196, one
// sequence of 131,072 x 256 in both directions.)  A gate alone whose exponential passes fp32, from 88.8 on, is an infinity.
//
// Precision.  A decay near 1 is held as a - 1, formed directly, and the state advances as v + (a - 1) v + b: a gate near 1 keeps
// its distance from 1 to a few u, where a rounded a would change a memory of 1,000 steps by 1,000 u.  A decay near 0 is held as a: a
// large state cut down to what is left of it, and the gate's own gradient, which has a as a factor, keep their digits, where
// 1 + (a - 1) is a multiple of 2^-25.  One word holds either.  All in fp32.
//
// What bounds it: instructions and latency, with memory at 60 % of its rate.  131,072 rows of 1,024 bf16: forward 182 us
// (805 MB, 4.4 TB/s, 26 warp instructions for 32 values, half of them a tile's fixed work; of 220 us at an earlier step 168
// were left without the waits for other tiles), backward 284 us (1.34 GB, 4.7 TB/s, 36 instructions).  One sequence of
// 131,072 x 256, bf16 to fp32: 70 and 111 us.  1,024 molecules, 112,640 x 128 fp32: 39 and 59 us, and 4 us each for the
// plan.  Of a tile's 18,000 cycles forward 5,000 go by before its inputs are there and 7,000 before the state that enters
// is; tiles asked for in L2 a round ahead of their copies: 4 % of the kernel (185 us forward without, where 179 with).  128 threads a tile
// with twice the rows each take a third fewer instructions and are slower (209 and 459 us for the first, too few warps),
// 8 channels a thread 200 and 353, copies of 16 bytes a lane 220 and 383.
#pragma once

#include <type_traits>

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
    char *clear[2];                       // outputs whose rows outside all sequences become zeros, or null
    int64_t clear_ld[2];                  // their strides
    int64_t clear_width;                  // and a row's width, in bytes
    int clear_unit;                       // 16 where all of that is, else a value's size
    int clear_ctas;                       // of the plan's kernel: in front, for this alone
    int checkers;                         // CTAs in front that look at the sequences
    const struct TileRows *plan;          // of each tile, where tiles are linked
    uint32_t *next;                       // the counter that hands out tiles
    uint64_t *maps;                       // [tile in order of work][f]: (a, b), or kNoMap
    uint32_t *states;                     // [window][f]: what enters it, or kNoState
    int64_t windows;
    int32_t *status;
    int32_t *status_all;                  // or null: written whole by the one checker
};

// The rows of a tile: what the walk down a tile has to know of sequences.
struct alignas(16) TileRows {
    int32_t seq[kTileRows];               // of the rows inside sequences
    uint32_t begin[kTileRows / 32];       // bits: the row begins its sequence,
    uint32_t end[kTileRows / 32];         // ends it,
    uint32_t in[kTileRows / 32];          // lies inside one
    int32_t lo, hi;                       // of the first and the last row
    uint8_t begin_warps[kTileRows / 32];  // two bits each: a row of the even, the odd warp begins a sequence,
    uint8_t cut_warps[kTileRows / 32];    // begins or ends one
};

// Bytes of a call that links tiles: counter, maps and states (ones beforehand), plan.
struct ScanSpace {
    size_t states, plan, bytes;
    static constexpr size_t kMaps = 16;
    __host__ ScanSpace(int64_t n, int64_t f) {
        const int64_t tiles = (n + kTileRows - 1) / kTileRows, windows = (tiles + kWindow - 1) / kWindow;
        if (tiles <= 1) {
            states = plan = bytes = 0;
            return;
        }
        states = kMaps + sizeof(uint64_t) * size_t(tiles * f);
        plan = (states + sizeof(uint32_t) * size_t(windows * f) + 15) / 16 * 16;
        bytes = plan + sizeof(TileRows) * size_t(tiles);
    }
};

// Tensor maps of gate, x and dL/dout, for tiles of a vector width above 1.
struct ScanMaps {
    CUtensorMap gate, x, g;
};

// CTAs of a launch, with at most `resident` on a multiprocessor.
inline unsigned scan_ctas(const ScanArgs &p, int resident) {
    const int64_t jobs = p.tiles * p.strips;
    return static_cast<unsigned>(p.checkers + (p.linked ? min64(jobs, static_cast<int64_t>(resident) * sm_count()) : jobs));
}

// Launches a kernel of tiles so that it is set up while the plan is made; it begins with a wait for the plan.
template <typename Kernel>
cudaError_t launch_tiles(Kernel *kernel, const ScanArgs &p, const ScanMaps &maps, int resident, int shared, cudaStream_t s) {
    if (shared > 32 * 1024) {   // with the static part above the 48 KB every launch may use
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, shared);
        if (e != cudaSuccess) return e;
    }
    cudaLaunchAttribute early{};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t config{};
    config.gridDim = dim3(scan_ctas(p, resident));
    config.blockDim = dim3(kScanThreads);
    config.dynamicSmemBytes = static_cast<size_t>(shared);
    config.stream = s;
    config.attrs = &early;
    config.numAttrs = p.status_all ? 0 : 1;                  // no plan is made where one CTA checks all
    return cudaLaunchKernelEx(&config, kernel, p, maps);
}

namespace {

constexpr uint64_t kNoMap = ~uint64_t(0);
constexpr uint32_t kNoState = ~uint32_t(0);
#ifndef TFG_WAIT_LOOKS
#define TFG_WAIT_LOOKS (1 << 21)
#endif
constexpr int kWaitLimit = TFG_WAIT_LOOKS;                   // looks at a word after the first, a second or more

// Words that other CTAs write while the kernel runs.
__device__ __forceinline__ uint64_t ld_word(const uint64_t *p) {
    uint64_t v;
    asm volatile("ld.relaxed.gpu.global.b64 %0, [%1];" : "=l"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t ld_word(const uint32_t *p) {
    uint32_t v;
    asm volatile("ld.relaxed.gpu.global.b32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ void st_word(uint64_t *p, uint64_t v) {
    asm volatile("st.relaxed.gpu.global.b64 [%0], %1;" ::"l"(p), "l"(v) : "memory");
}
__device__ __forceinline__ void st_word(uint32_t *p, uint32_t v) {
    asm volatile("st.relaxed.gpu.global.b32 [%0], %1;" ::"l"(p), "r"(v) : "memory");
}
// A NaN of all ones is another NaN of those that a reader may meet.
__device__ __forceinline__ uint64_t map_word(float a, float b) {
    const uint64_t w = static_cast<uint64_t>(__float_as_uint(b)) << 32 | __float_as_uint(a);
    return w == kNoMap ? w & 0x7fffffff7fffffffull : w;
}
__device__ __forceinline__ uint32_t state_word(float v) {
    const uint32_t w = __float_as_uint(v);
    return w == kNoState ? w & 0x7fffffffu : w;
}
// The word once it is there; after too many looks the status tells and the wait ends.
template <typename W>
__device__ __forceinline__ W wait_for(const W *p, W none, int32_t *status) {
    for (int i = 0; i < kWaitLimit; ++i) {
        const W v = ld_word(p);
        if (v != none) return v;
    }
    set_status(status, TFG_ERR_TIMEOUT);
    return none;
}

// ---- gates ----------------------------------------------------------------------------
// How the decays of a thread's rows are held.  kLess: a - 1, for sigmoid gates that are all above kSmallGate.  kEither: a - 1
// near 1, with the sign bit set and never 0, else a, with it clear.
constexpr int kLess = 0, kEither = 1;
template <int FORM> using Form = std::integral_constant<int, FORM>;
using Yes = std::true_type;
using No = std::false_type;
// a = 2^-8.  a - 1 is within 2 u, which is up to 512 u of such an a; below it kEither has a few u.  Words of either kind take twice the
// instructions to apply, and a tile that takes longer holds up those behind it: 131,072 x 1,024 bf16 with gates of mean
// 2.5 and deviation 1.8, both directions, 472 us with words of either kind below 2^-9, 475 below 2^-8, 517 below 2^-7, 632 below 2^-6 and
// 621 with no others.  Rows with a gate as small take the code of rows that begin and end sequences: a copy of their own (536 us with no
// others) makes a kernel that is slower wherever the copy is not taken, by the instructions' cache (481 us; 130,000 x 512 in 4,000
// sequences 406, so 380; 1,024 molecules fp32 106, so 103).
constexpr float kSmallGate = -5.55f;

// expm1(z) + `more` for |z| <= 0.35: z (1 + z q(z)), q of degree 4 through the Chebyshev points of
// the interval; within 2 u of itself over all normal fp32 values there.
template <int VEC>
__device__ __forceinline__ void expm1_near(const float (&z)[VEC], float more, float (&d)[VEC]) {
    const float c[6] = {0.0013934534508734941f, 0.008363769389688969f, 0.04166645556688309f, 0.16666573286056519f, 0.5f, 1.f};
    const float last[1] = {more};
#pragma unroll
    for (int q = 0; q < VEC; ++q) d[q] = c[0];
#pragma unroll
    for (int k = 1; k < 6; ++k) {
        const float ck[1] = {c[k]};
        fma_vec(d, d, z, ck);
    }
    fma_vec(d, d, z, last);
}

// The words of VEC gates; beside them 1 - a of sigmoid gates held as kEither.  Sigmoid: with t = z log2 e, 1 / (1 + 2^t) is
// 1 - a and 2^t times it a, each within (2 |z| + 10) u of itself.  Exp: a = 2^t within (2 |z| + 4) u, or a - 1 from -0.35 to 0.
template <int KIND, int FORM, int VEC>
__device__ __forceinline__ void decay_words(const float (&z)[VEC], float (&r)[VEC], float (&less)[VEC]) {
    const float log2e[1] = {1.44269504088896341f};
    float e[VEC];
#pragma unroll
    for (int q = 0; q < VEC; ++q) e[q] = z[q];
    mul_vec(e, log2e);
    if constexpr (KIND == TFG_GATE_EXP) {
        float near[VEC];
        expm1_near(z, -1.1754943508222875e-38f, near);       // never 0, so that the sign tells
#pragma unroll
        for (int q = 0; q < VEC; ++q) {
            // the bits of -0.35 and what lies between it and -0, as whole numbers
            r[q] = __float_as_int(z[q]) <= __float_as_int(-0.35f) ? near[q] : exp2_of(e[q]);
        }
    } else {
        const float one[1] = {FORM == kLess ? -1.f : 1.f};   // kLess: -1 / (1 + 2^t)
#pragma unroll
        for (int q = 0; q < VEC; ++q) less[q] = e[q] = exp2_of(e[q]);
        fma_vec(less, less, one, one);
#pragma unroll
        for (int q = 0; q < VEC; ++q) asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(less[q]) : "f"(less[q]));
        if constexpr (FORM == kLess) {
#pragma unroll
            for (int q = 0; q < VEC; ++q) r[q] = less[q];
        } else {
            const float minus[1] = {-1.f}, tiny[1] = {-1.1754943508222875e-38f};
            mul_vec(e, less);
            fma_vec(r, less, minus, tiny);
#pragma unroll
            for (int q = 0; q < VEC; ++q) r[q] = z[q] < 0.f ? e[q] : r[q];
        }
    }
}

// kEither: 1 where a word is a - 1, 0 where it is a.
template <int VEC>
__device__ __forceinline__ void whole_part(const float (&r)[VEC], float (&h)[VEC]) {
#pragma unroll
    for (int q = 0; q < VEC; ++q) asm("mul.rn.sat.f32 %0, %1, %2;" : "=f"(h[q]) : "f"(r[q]), "f"(-1.7014118346046923e38f));
}
// a v.
template <int FORM, int VEC>
__device__ __forceinline__ void decay(float (&v)[VEC], const float (&r)[VEC]) {
    if constexpr (FORM == kLess) {
        fma_vec(v, r, v, v);
    } else {
        float h[VEC];
        whole_part(r, h);
        mul_vec(h, v);
        fma_vec(v, r, v, h);
    }
}
// 1 - a of words of either kind.
template <int VEC>
__device__ __forceinline__ void one_less(const float (&r)[VEC], const float (&h)[VEC], float (&less)[VEC]) {
    const float one[1] = {1.f}, minus[1] = {-1.f};
    fma_vec(less, h, minus, one);
    fma_vec(less, r, minus, less);
}
// a v + b of a row, from its word.
template <int KIND, int FORM, int VEC>
__device__ __forceinline__ void advance(float (&v)[VEC], const float (&r)[VEC], const float (&x)[VEC]) {
    float h[VEC];
    if constexpr (FORM == kLess) {                           // v + (a - 1) (v - x)
        const float minus[1] = {-1.f};
        fma_vec(h, x, minus, v);
        fma_vec(v, r, h, v);
    } else {
        whole_part(r, h);
        if constexpr (KIND == TFG_GATE_SIGMOID) {
            float less[VEC];
            one_less(r, h, less);
            mul_vec(h, v);
            fma_vec(h, r, v, h);
            fma_vec(v, less, x, h);
        } else {
            fma_vec(h, h, v, x);
            fma_vec(v, r, v, h);
        }
    }
}

// ---- composed maps -----------------------------------------------------------------------
// The decay of the rows of two maps, one after the other: of sigmoid gates the product of the a, of exponential gates its root.
constexpr float kMostDecay = 3.402823466e38f;
template <int KIND>
__device__ __forceinline__ float held_back(float a) {
    return KIND == TFG_GATE_EXP ? fminf(a, kMostDecay) : a;
}
// What the map (a, b) makes of v.  Exponential gates: v a is between v and v a^2, so nothing is lost on the way.  A product
// held back to 2^256 makes an infinity of every v from 2^-128 on, as it should.  A gate that is NaN, or too large
// for fp32, is NaN or an infinity in b too.
template <int KIND>
__device__ __forceinline__ float through(float a, float v, float b) {
    return KIND == TFG_GATE_EXP ? fmaf(v * a, a, b) : fmaf(a, v, b);
}

// ---- the rows of a tile ----------------------------------------------------------------
template <int PER>
__device__ __forceinline__ uint32_t row_bits(const uint32_t *bits, int group) {
    return (bits[group * PER / 32] >> (group * PER % 32)) & ((1u << PER) - 1u);
}
// The bits of begin_warps and cut_warps as one word, and a warp's place in it.
__device__ __forceinline__ uint32_t warps_word(const uint8_t (&w)[kTileRows / 32]) {
    static_assert(kTileRows / 32 == 4, "four bytes");
    return *reinterpret_cast<const uint32_t *>(w);
}
__host__ __device__ constexpr int warp_bit(int warp) { return warp / 2 * 8 + warp % 2; }

// Row r of a tile whose sequences lie in [lo, hi], by a warp for its 32 rows: word is the tile's
// word of bits that they fill.  Whatever the offsets say, seq lies in [0, seqs).
__device__ __forceinline__ void describe_row(const ScanArgs &p, int64_t r, int lo, int hi, int word, TileRows &t) {
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
    const int lane = threadIdx.x & 31;
    t.seq[word * 32 + lane] = lo < 0 ? 0 : lo;
    const uint32_t bb = lane_ballot(begins), eb = lane_ballot(ends), ib = lane_ballot(in);
    if (lane == 0) {
        t.begin[word] = bb;
        t.end[word] = eb;
        t.in[word] = ib;
        t.begin_warps[word] = static_cast<uint8_t>(((bb & 0xffffu) ? 1 : 0) | ((bb >> 16) ? 2 : 0));
        t.cut_warps[word] = static_cast<uint8_t>((((bb | eb) & 0xffffu) ? 1 : 0) | (((bb | eb) >> 16) ? 2 : 0));
    }
}

// The rows of the one tile of a call by a whole CTA; ends with a barrier.
__device__ __forceinline__ void find_rows(const ScanArgs &p, TileRows &t) {
    const int tid = threadIdx.x;
    if (tid < 64) {
        const int64_t s = warp_graph_at(p.offsets, p.seqs, tid < 32 ? 0 : p.n - 1);
        if ((tid & 31) == 0) (tid < 32 ? t.lo : t.hi) = static_cast<int>(s);
    }
    __syncthreads();
    if (tid < kTileRows) describe_row(p, tid, t.lo, t.hi, tid / 32, t);
    __syncthreads();
}

// Zeros in the rows before the first sequence and behind the last, a warp a row.
__device__ __forceinline__ void clear_outside(const ScanArgs &p, int64_t warp, int64_t warps) {
    if (!p.clear[0]) return;
    const auto inside = [&](int64_t r) { return r < 0 ? 0 : min64(r, p.n); };
    const int64_t lo = p.seqs ? inside(__ldg(p.offsets)) : 0, hi = p.seqs ? inside(__ldg(p.offsets + p.seqs)) : 0;
    for (int64_t i = warp; i < lo + p.n - hi; i += warps) {
        const int64_t row = i < lo ? i : hi + i - lo;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (!p.clear[k]) continue;
            char *at = p.clear[k] + row * p.clear_ld[k];
            for (int64_t b = (threadIdx.x & 31) * p.clear_unit; b < p.clear_width; b += 32 * p.clear_unit) {
                if (p.clear_unit == 16) *reinterpret_cast<uint4 *>(at + b) = make_uint4(0u, 0u, 0u, 0u);
                else if (p.clear_unit == 4) *reinterpret_cast<uint32_t *>(at + b) = 0u;
                else *reinterpret_cast<uint16_t *>(at + b) = 0;
            }
        }
    }
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
    if (p.status_all) clear_outside(p, threadIdx.x / 32, kScanThreads / 32);         // no plan is made
    const int all = __syncthreads_or(any);
    if (threadIdx.x != 0) return;
    if (p.status_all) *p.status_all = all ? TFG_ERR_INDEX_RANGE : TFG_OK;
    else if (all) set_status(p.status, TFG_ERR_INDEX_RANGE);
}

// ---- a tile ------------------------------------------------------------------------------
constexpr int kScanWarps = kScanThreads / 32;
constexpr int kWarpRows = kTileRows / kScanWarps;            // rows of a warp

// VEC values a thread, kAcross threads side by side in a row, kEach rows of a thread.  Tiles of bf16 have 64
// channels in vectors of 4, so that a warp has two groups of rows and exchanges little between them (8 threads of 8
// channels, four groups: 200 us for 131,072 x 1,024 forward, with 4 channels 184); of fp32 32 channels, as 64 would
// leave room for three CTAs on a multiprocessor in place of four (1,024 molecules 118 us, so 109).
template <typename XT, int N>
struct ScanTile {
    static constexpr int VEC = N;
    static constexpr int kLane = VEC * 4, kRow = kLane * kScanThreads;                         // of fp32 slots
    static constexpr int kAcross = VEC == 1 ? 32 : (sizeof(XT) == 2 ? 16 : 8);
    static constexpr int kEach = kTileRows * kAcross / kScanThreads;
    static constexpr int kWide = kAcross * VEC;              // channels
};

// The plan of a tile, with the copies of its inputs.
__device__ __forceinline__ void copy_plan(const ScanArgs &p, int64_t tile, TileRows &to) {
    static_assert(sizeof(TileRows) % 16 == 0 && sizeof(TileRows) / 16 <= kScanThreads, "one copy a thread");
    if (threadIdx.x < sizeof(TileRows) / 16)
        copy_async<16>(reinterpret_cast<char *>(&to) + threadIdx.x * 16,
                       reinterpret_cast<const char *>(p.plan + tile) + threadIdx.x * 16);
}

// A thread's vectors of a tile that lies in shared memory row by row.
template <typename T, typename Tile>
struct TileRow {
    static constexpr int VEC = Tile::VEC, kBytes = kTileRows * Tile::kWide * static_cast<int>(sizeof(T));
    T *at;
    __device__ __forceinline__ explicit TileRow(char *tile)
        : at(reinterpret_cast<T *>(tile) + threadIdx.x / Tile::kAcross * Tile::kEach * Tile::kWide + threadIdx.x % Tile::kAcross * VEC) {}
    __device__ __forceinline__ void widen(int j, float (&v)[VEC]) const {
        VecLoad<T, VEC>::widen(load_plain<T, VEC>(at + j * Tile::kWide), v);
    }
    __device__ __forceinline__ void zero(int j) const {
#pragma unroll
        for (int q = 0; q < VEC; ++q) at[j * Tile::kWide + q] = T(0);
    }
};
// The gates of a thread, taken from their tile before the decays are written over it.
template <typename T, typename Tile>
struct HeldGate {
    static constexpr int VEC = Tile::VEC;
    typename VecLoad<T, VEC>::Raw r[Tile::kEach];
    __device__ __forceinline__ explicit HeldGate(char *tile) {
        const TileRow<T, Tile> from(tile);
#pragma unroll
        for (int j = 0; j < Tile::kEach; ++j) r[j] = load_plain<T, VEC>(from.at + j * Tile::kWide);
    }
    __device__ __forceinline__ void widen(int j, float (&v)[VEC]) const { VecLoad<T, VEC>::widen(r[j], v); }
    // Whether a gate lies below kSmallGate; a NaN does not.
    __device__ __forceinline__ bool any_small() const {
        float least = INFINITY;
        if constexpr (sizeof(T) == 2) {
            const auto pair = [](uint32_t w) { return *reinterpret_cast<const __nv_bfloat162 *>(&w); };
            __nv_bfloat162 m = pair(r[0].x);
#pragma unroll
            for (int j = 0; j < Tile::kEach; ++j) m = __hmin2(m, __hmin2(pair(r[j].x), pair(r[j].y)));
            least = fminf(__low2float(m), __high2float(m));
        } else {
#pragma unroll
            for (int j = 0; j < Tile::kEach; ++j) least = fminf(least, fminf(fminf(r[j].x, r[j].y), fminf(r[j].z, r[j].w)));
        }
        return least < kSmallGate;
    }
};

// Whether the rows of a thread, all of one sequence (plain), have a sigmoid gate below kSmallGate in one of the tile's channels: the
// same for all threads of the rows, and no matter what other rows hold.  By whole warps.
template <typename Tile, typename Gate>
__device__ __forceinline__ bool small_gates(const Gate &z, bool mine) {
    bool small;
    if constexpr (Tile::VEC > 1) {
        small = z.any_small();
    } else {
        float least = INFINITY, v[1];
#pragma unroll
        for (int j = 0; j < Tile::kEach; ++j) {
            z.widen(j, v);
            least = fminf(least, v[0]);
        }
        small = least < kSmallGate;
    }
    constexpr uint32_t kRows = Tile::kAcross == 32 ? ~0u : (1u << (Tile::kAcross & 31)) - 1u;
    return (lane_ballot(mine && small) >> ((threadIdx.x & 31) / Tile::kAcross * Tile::kAcross) & kRows) != 0u;
}

// A job: a tile in order of work, and a strip of channels.
struct Job {
    int64_t order;
    int strip;
    __device__ __forceinline__ Job(const ScanArgs &p, uint32_t job) {
        const uint32_t o = job / static_cast<uint32_t>(p.strips);
        order = o;
        strip = static_cast<int>(job - o * p.strips);
    }
};

// The jobs of a CTA, one after the other.  ask: once the CTA waits for no other tile; next: by the whole CTA,
// with a barrier (s_next and what the last job left in shared memory are free behind it).
struct Jobs {
    uint32_t *s_next;
    uint32_t count, asked;
    __device__ __forceinline__ Jobs(const ScanArgs &p, uint32_t *s)
        : s_next(s), count(static_cast<uint32_t>(p.tiles * p.strips)), asked(blockIdx.x - p.checkers) {
        if (p.linked) ask(p);
    }
    __device__ __forceinline__ void ask(const ScanArgs &p) {
        if (threadIdx.x == 0) asked = p.linked ? atomicAdd(p.next, 1u) : count;
    }
    // A job that some CTA takes about when this one is done, to be asked for in L2; false behind the last.
    __device__ __forceinline__ bool later(const ScanArgs &p, uint32_t job, uint32_t &then) const {
        then = job + (gridDim.x - p.checkers);
        return then < count;
    }
    __device__ __forceinline__ bool next(const ScanArgs &p, uint32_t &job) {
        if (threadIdx.x == 0) *s_next = asked;               // the last one was read many barriers ago
        before_copies();
        __syncthreads();
        job = *s_next;
        return job < count;
    }
};

// The last tile before this one in its window, in order of work, that lets nothing through, by its place
// in the window, -1 if there is none; by a whole warp.
template <bool UP>
__device__ __forceinline__ int cut_before(const ScanArgs &p, int64_t order) {
    const int place = static_cast<int>(order % kWindow), lane = threadIdx.x & 31;
    uint32_t cut = 0;
    if (lane < place) {
        const int64_t other = order - place + lane;
        const TileRows &t = p.plan[UP ? p.tiles - 1 - other : other];
        cut = __ldg(reinterpret_cast<const uint32_t *>(UP ? t.cut_warps : t.begin_warps));
    }
    return 31 - __clz(static_cast<int>(lane_ballot(cut != 0u)));
}

// The state of a sequence, zeros without states.
template <int VEC>
__device__ __forceinline__ void state_or_zero(const float *states, int64_t seq, int64_t f, int64_t c, float (&v)[VEC]) {
    if (states) {
        VecLoad<float, VEC>::load(states + seq * f + c, v);
    } else {
#pragma unroll
        for (int q = 0; q < VEC; ++q) v[q] = 0.f;
    }
}

// States that the rows of a thread begin or end with, on their way to L1 all at once: row by row each would be
// waited for by itself.
template <int EACH>
__device__ __forceinline__ void prefetch_states(const float *states, uint32_t which, const int32_t *seq, int64_t f, int64_t c) {
    if (!states) return;
#pragma unroll
    for (int j = 0; j < EACH; ++j)
        if ((which >> j) & 1u) asm volatile("prefetch.global.L1 [%0];" ::"l"(states + seq[j] * f + c));
}

// Maps of a warp's groups of rows, composed across the lanes from where values enter (the first
// row; UP: the last): on return (a, b) is the map of the groups up to this one, `fresh` whether
// one of them cuts off what enters; the last group leaves the whole warp's map.
template <typename Tile, int KIND, bool UP, int VEC>
__device__ __forceinline__ void scan_groups(float (&a)[VEC], float (&b)[VEC], bool &fresh, int warp, int lane,
                                            float (*s_a)[Tile::kWide], float (*s_b)[Tile::kWide]) {
    constexpr int kAcross = Tile::kAcross;
    const int l = threadIdx.x & 31;
#pragma unroll
    for (int o = kAcross; o < 32; o <<= 1) {
        const int from = (UP ? l + o : l - o) & 31;          // the neighbour nearer to where values enter
        const bool has = UP ? l + o < 32 : l >= o, joins = has && !fresh;
        const uint32_t other = lane_ballot(fresh) >> from & 1u;
#pragma unroll
        for (int q = 0; q < VEC; ++q) {
            const float pa = lane_get(a[q], from), pb = lane_get(b[q], from);
            if (joins) {
                b[q] = through<KIND>(a[q], pb, b[q]);
                a[q] = held_back<KIND>(a[q] * pa);           // not looked at behind a cut
            }
        }
        fresh = fresh || (has && other);
    }
    if (UP ? l < kAcross : l >= 32 - kAcross) {
        if constexpr (VEC % 4 == 0) {
#pragma unroll
            for (int q = 0; q < VEC; q += 4) {
                *reinterpret_cast<float4 *>(&s_a[warp][lane * VEC + q]) = make_float4(a[q], a[q + 1], a[q + 2], a[q + 3]);
                *reinterpret_cast<float4 *>(&s_b[warp][lane * VEC + q]) = make_float4(b[q], b[q + 1], b[q + 2], b[q + 3]);
            }
        } else {
#pragma unroll
            for (int q = 0; q < VEC; ++q) {
                s_a[warp][lane * VEC + q] = a[q];
                s_b[warp][lane * VEC + q] = b[q];
            }
        }
    }
}

// What enters the thread's rows, into v: at the warp's first group what enters the warp (v), else what leaves
// the group before, by the map (a, b) up to it.  By whole warps.
template <typename Tile, int KIND, bool UP, int VEC>
__device__ __forceinline__ void enter_group(const float (&a)[VEC], const float (&b)[VEC], bool fresh, float (&v)[VEC]) {
    constexpr int kAcross = Tile::kAcross;
    if constexpr (kAcross < 32) {
        const int l = threadIdx.x & 31, from = (UP ? l + kAcross : l - kAcross) & 31;
        const bool has = UP ? l + kAcross < 32 : l >= kAcross;
#pragma unroll
        for (int q = 0; q < VEC; ++q) {
            const float leaves = lane_get(fresh ? b[q] : through<KIND>(a[q], v[q], b[q]), from);
            if (has) v[q] = leaves;
        }
    }
}

// No adjoint beside the states' map.
struct NoGrad {};

// The thread's rows as one map, and the word of each row's decay into d, which may lie where z does.  PLAIN: the rows
// lie in a sequence that neither begins nor ends there.  With gradients g (sigmoid gates): w is what leaves the rows upward when
// nothing enters them, the sum of g_j times the decays of the rows up to j, and one of grad_final behind a sequence's end; its
// own decay is a.
template <bool PLAIN, int FORM, int KIND, int VEC, int EACH, typename Gate, typename In, typename Decay, typename Grad>
__device__ __forceinline__ void compose_down(const ScanArgs &p, const Gate &z, const In &x, const Decay &d, const Grad &g,
                                             const float *initial, const float *grad_final, const int32_t *seq, int64_t c,
                                             uint32_t begin, uint32_t end, uint32_t in, float (&a)[VEC],
                                             float (&b)[VEC], float (&w)[VEC]) {
    const float half[1] = {0.5f};
    constexpr bool kAdjoint = !std::is_same<Grad, NoGrad>::value;
    bool open = true;
#pragma unroll
    for (int q = 0; q < VEC; ++q) a[q] = KIND == TFG_GATE_EXP ? 0.f : 1.f, b[q] = w[q] = 0.f;
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
        float v[VEC], dj[VEC], zj[VEC], less[VEC];
        z.widen(j, zj);
        decay_words<KIND, FORM>(zj, dj, less);
        d.put(j, dj);
        if (!PLAIN && !((in >> j) & 1u)) continue;
        if (!PLAIN && ((begin >> j) & 1u)) {
#pragma unroll
            for (int q = 0; q < VEC; ++q) a[q] = 0.f;
            state_or_zero(initial, seq[j], p.f, c, b);
            open = false;
        }
        x.widen(j, v);
        if constexpr (KIND == TFG_GATE_EXP) {
            fma_vec(a, zj, half, a);
            advance<KIND, kEither>(b, dj, v);
        } else if constexpr (FORM == kEither) {
            decay<kEither>(b, dj);
            fma_vec(b, less, v, b);
            decay<kEither>(a, dj);
        } else {
            advance<KIND, kLess>(b, dj, v);
            decay<kLess>(a, dj);
        }
        if constexpr (kAdjoint) {
            if (PLAIN || open) {
                g.widen(j, v);
                fma_vec(w, a, v, w);
                if (!PLAIN && ((end >> j) & 1u)) {
                    state_or_zero(grad_final, seq[j], p.f, c, v);
                    fma_vec(w, a, v, w);
                    open = false;
                }
            }
        }
    }
    if constexpr (KIND == TFG_GATE_EXP) {
        // near 1 within u / 2 of itself, as one root stands for all groups of rows that a state passes
        const float log2e[1] = {1.44269504088896341f};
        float near[VEC], far[VEC];
        expm1_near(a, 1.f, near);
#pragma unroll
        for (int q = 0; q < VEC; ++q) far[q] = a[q];
        mul_vec(far, log2e);
#pragma unroll
        for (int q = 0; q < VEC; ++q) a[q] = fabsf(a[q]) <= 0.35f ? near[q] : fminf(exp2_of(far[q]), kMostDecay);
    }
}

// The state that enters the order-th tile, for the channel of each of the first WIDE threads, from
// the maps of the tiles before; (a, b) is the map of the tile for that channel.  Whole CTA.  fresh: nothing that
// enters the tile leaves it.  wants: the tile's first row (in order of work) goes on from
// the tile before.  from: cut_before.  The maps are looked at by all threads, a part of the
// window each, and the parts joined in shared memory.
template <int WIDE, int KIND>
__device__ __forceinline__ float enter_tile(const ScanArgs &p, int64_t order, int64_t c0, float a, float b, bool fresh,
                                            bool wants, int from, float2 (*s_part)[WIDE]) {
    constexpr int kParts = kScanThreads / WIDE, kMaps = kWindow / kParts;
    if (!p.linked) return 0.f;
    const int64_t window = order / kWindow;
    const int place = static_cast<int>(order - window * kWindow);
    const int channel = threadIdx.x % WIDE, part = threadIdx.x / WIDE;
    const int64_t c = c0 + channel;
    const bool mine = part == 0 && c < p.f;
    if (mine) st_word(p.maps + order * p.f + c, map_word(held_back<KIND>(a), b));
    float state = 0.f;
    if (wants && order > 0) {
        const int first = from < 0 ? 0 : from, begin = part * kMaps;
        uint32_t entered = 0;                                // in flight beside the maps
        if (mine && from < 0 && window > 0) entered = ld_word(p.states + window * p.f + c);
        if (c < p.f && begin + kMaps > first && begin < place) {
            const uint64_t *maps = p.maps + (order - place + begin) * p.f + c;
            uint64_t word[kMaps];
#pragma unroll
            for (int i = 0; i < kMaps; ++i)
                word[i] = begin + i >= first && begin + i < place ? ld_word(maps + i * p.f) : 0;
            float ma = 1.f, mb = 0.f;
#pragma unroll
            for (int i = 0; i < kMaps; ++i) {
                if (begin + i < first || begin + i >= place) continue;
                if (word[i] == kNoMap) word[i] = wait_for(maps + i * p.f, kNoMap, p.status);
                const float wa = __uint_as_float(static_cast<uint32_t>(word[i])), wb = __uint_as_float(static_cast<uint32_t>(word[i] >> 32));
                mb = begin + i == from ? wb : through<KIND>(wa, mb, wb);
                ma *= wa;
            }
            s_part[part][channel] = make_float2(held_back<KIND>(ma), mb);
        }
        if (entered == kNoState) entered = wait_for(p.states + window * p.f + c, kNoState, p.status);
        state = __uint_as_float(entered);
        __syncwarp();                                        // lanes waited for words of their own, or for none
        __syncthreads();
        if (mine) {
#pragma unroll
            for (int i = 0; i < kParts; ++i) {
                if ((i + 1) * kMaps <= first || i * kMaps >= place) continue;
                const float2 m = s_part[i][channel];
                state = i * kMaps <= from ? m.y : through<KIND>(m.x, state, m.y);   // the part with `from` begins anew
            }
        }
    }
    if (mine && place == kWindow - 1 && order + 1 < p.tiles)
        st_word(p.states + (window + 1) * p.f + c, state_word(fresh ? b : through<KIND>(held_back<KIND>(a), state, b)));
    return state;
}

}  // namespace
}  // namespace tfg
