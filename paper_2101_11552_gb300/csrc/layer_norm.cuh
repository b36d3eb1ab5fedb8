// Layer norm of rows: what the forward (layer_norm.cu) and the backward
// (layer_norm_backward.cu) share.
//
// A team of TT threads, part of a warp, a warp, or a CTA, takes a row; thread t holds the
// vectors t, t + TT, ... of it.
#pragma once

#include "widen.cuh"

namespace tfg {
namespace {

// A barrier of a team of TT threads: the whole CTA's, or one of its own where a CTA has several teams.
template <int TT, int TEAMS>
__device__ __forceinline__ void team_barrier() {
    if constexpr (TEAMS == 1) __syncthreads();
    else asm volatile("bar.sync %0, %1;" ::"r"(static_cast<int>(threadIdx.x) / TT + 1), "n"(TT) : "memory");
}

// Adds v[s] over the TT threads of a team, to all of them, in a fixed order.  scratch: of a team of several
// warps, NS * TT / 32 floats that no other call uses before the team's next barrier.
template <int TT, int TEAMS, int NS>
__device__ __forceinline__ void team_sums(float (&v)[NS], float *scratch) {
#pragma unroll
    for (int o = (TT < 32 ? TT : 32) >> 1; o > 0; o >>= 1)
#pragma unroll
        for (int s = 0; s < NS; ++s) v[s] += lane_xor(v[s], o);
    if constexpr (TT > 32) {
        constexpr int kWarps = TT / 32;
        if ((threadIdx.x & 31) == 0)
#pragma unroll
            for (int s = 0; s < NS; ++s) scratch[s * kWarps + threadIdx.x % TT / 32] = v[s];
        team_barrier<TT, TEAMS>();
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            v[s] = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) v[s] += scratch[s * kWarps + w];
        }
    }
}

// VEC values of an array that the kernel may also write (the residual stream in place): no
// loads through the read-only path.  p aligned to the vector, 32 bytes for eight fp32 values.
template <int VEC>
__device__ __forceinline__ void load_row(const float *p, float (&v)[VEC]) {
    if constexpr (VEC == 8) {
        asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
                     : "l"(p)
                     : "memory");
    } else {
        VecLoad<float, VEC>::widen(load_plain<float, VEC>(p), v);
    }
}
template <int VEC>
__device__ __forceinline__ void load_row(const uint16_t *p, float (&v)[VEC]) {
    VecLoad<uint16_t, VEC>::widen(load_plain<uint16_t, VEC>(p), v);
}

// gamma or beta of VEC channels, `none` without them; 16-byte aligned where VEC is more than one.
template <int VEC>
__device__ __forceinline__ void row_weights(const float *w, int64_t c, float none, float (&v)[VEC]) {
    if (!w) {
#pragma unroll
        for (int q = 0; q < VEC; ++q) v[q] = none;
    } else {
        VecLoad<float, VEC>::load(w + c, v);
    }
}

template <int VEC>
__device__ __forceinline__ void store_row(void *out, bool bf16, int64_t at, const float (&v)[VEC]) {
    if (bf16) store_vec<VEC>(static_cast<uint16_t *>(out) + at, v);
    else store_vec<VEC>(static_cast<float *>(out) + at, v);
}

}  // namespace

// Whether vectors of vec values of an array lie on their boundary in every row.
inline bool vec_fits(const void *p, int dtype, int64_t f, int vec) {
    return f % vec == 0 && reinterpret_cast<uintptr_t>(p) % (vec * (dtype == TFG_BF16 ? 2 : 4)) == 0;
}
// gamma and beta are read in 16-byte halves.
inline bool weights_fit(const float *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

}  // namespace tfg
