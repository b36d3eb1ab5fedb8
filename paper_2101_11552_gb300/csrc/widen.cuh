// Rows read and fp32 results stored in either storage type, shared by the operators whose outputs
// may be fp32 or bf16 (embedding lookup, group norm, clipped gradients).
#pragma once

#include <cuda_bf16.h>

#include "common.cuh"

namespace tfg {

// Two fp32 values rounded to nearest even, packed as the two bf16 halves of a word.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&p);
}

// VEC values of a row as they lie in memory, and widened: VecLoad with its eight fp32 values
// as two 16-byte loads, for rows that are 16-byte but not 32-byte aligned.
template <typename TT, int VEC> struct RowVec;
template <> struct RowVec<float, 8> {
    float4 a, b;
    __device__ __forceinline__ void load(const float *p) {
        a = __ldg(reinterpret_cast<const float4 *>(p));
        b = __ldg(reinterpret_cast<const float4 *>(p) + 1);
    }
    __device__ __forceinline__ void widen(float (&v)[8]) const {
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
};
template <typename TT, int VEC> struct RowVec {
    typename VecLoad<TT, VEC>::Raw r;
    __device__ __forceinline__ void load(const TT *p) { r = VecLoad<TT, VEC>::raw(p); }
    __device__ __forceinline__ void widen(float (&v)[VEC]) const { VecLoad<TT, VEC>::widen(r, v); }
};

// Arithmetic on VEC values, two to an instruction where VEC is even (packed fp32: each half
// is the ordinary correctly rounded operation).  b and c may be shared by several values:
// value q takes element q / (VEC / N).
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 ra, rb, rd;\n\tmov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %5};\n\t"
        "add.rn.f32x2 rd, ra, rb;\n\tmov.b64 {%0, %1}, rd;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 ra, rb, rd;\n\tmov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %5};\n\t"
        "mul.rn.f32x2 rd, ra, rb;\n\tmov.b64 {%0, %1}, rd;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
template <int VEC, int N>
__device__ __forceinline__ float2 pair_of(const float (&v)[N], int q) {
    return make_float2(v[q / (VEC / N)], v[(q + 1) / (VEC / N)]);
}
template <int VEC, int N>
__device__ __forceinline__ void add_vec(float (&a)[VEC], const float (&b)[N]) {       // a + b
    if constexpr (VEC % 2 == 0) {
#pragma unroll
        for (int q = 0; q < VEC; q += 2) {
            const float2 r = add2(make_float2(a[q], a[q + 1]), pair_of<VEC>(b, q));
            a[q] = r.x;
            a[q + 1] = r.y;
        }
    } else {
#pragma unroll
        for (int q = 0; q < VEC; ++q) a[q] += b[q / (VEC / N)];
    }
}
template <int VEC, int N>
__device__ __forceinline__ void mul_vec(float (&a)[VEC], const float (&b)[N]) {       // a b
    if constexpr (VEC % 2 == 0) {
#pragma unroll
        for (int q = 0; q < VEC; q += 2) {
            const float2 r = mul2(make_float2(a[q], a[q + 1]), pair_of<VEC>(b, q));
            a[q] = r.x;
            a[q + 1] = r.y;
        }
    } else {
#pragma unroll
        for (int q = 0; q < VEC; ++q) a[q] *= b[q / (VEC / N)];
    }
}
template <int VEC, int N, int M>
__device__ __forceinline__ void fma_vec(float (&d)[VEC], const float (&a)[VEC], const float (&b)[N], const float (&c)[M]) {   // a b + c
    if constexpr (VEC % 2 == 0) {
#pragma unroll
        for (int q = 0; q < VEC; q += 2) {
            const float2 r = fma2(make_float2(a[q], a[q + 1]), pair_of<VEC>(b, q), pair_of<VEC>(c, q));
            d[q] = r.x;
            d[q + 1] = r.y;
        }
    } else {
#pragma unroll
        for (int q = 0; q < VEC; ++q) d[q] = fmaf(a[q], b[q / (VEC / N)], c[q / (VEC / M)]);
    }
}

// A vector by plain loads: from shared memory, or from memory that the kernel also writes.
template <typename T, int VEC>
__device__ __forceinline__ typename VecLoad<T, VEC>::Raw load_plain(const T *p) {
    if constexpr (VEC == 1) {
        if constexpr (sizeof(T) == 2) return static_cast<uint32_t>(*p) << 16;
        else return *p;
    } else {
        return *reinterpret_cast<const typename VecLoad<T, VEC>::Raw *>(p);
    }
}

// Copies of 4, 8 or 16 bytes to shared memory that go on while the thread does; one bf16
// value is too short for one and is copied at once.
template <int BYTES>
__device__ __forceinline__ void copy_async(void *shared, const void *global) {
    if constexpr (BYTES == 2) {
        *static_cast<uint16_t *>(shared) = __ldg(static_cast<const uint16_t *>(global));
    } else {
        const uint32_t to = static_cast<uint32_t>(__cvta_generic_to_shared(shared));
        if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(global) : "memory");
        else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(global), "n"(BYTES) : "memory");
    }
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// VEC values to p (fp32, or bf16 bits), p aligned to the vector it is stored as: 16 bytes,
// or 8 for four bf16 values.  The one rounding of a bf16 result is here.
// Eight fp32 values go out as one 32-byte store where p allows it: as two, every lane's half
// sectors go to L2 by themselves.
template <int VEC>
__device__ __forceinline__ void store_vec(float *p, const float (&v)[VEC]) {
    if constexpr (VEC == 8) {
        if (reinterpret_cast<uintptr_t>(p) % 32 == 0) {
            asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(v[0]), "f"(v[1]), "f"(v[2]),
                         "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
                         : "memory");
            return;
        }
    }
    if constexpr (VEC % 4 == 0) {
#pragma unroll
        for (int q = 0; q < VEC; q += 4)
            *reinterpret_cast<float4 *>(p + q) = make_float4(v[q], v[q + 1], v[q + 2], v[q + 3]);
    } else {
#pragma unroll
        for (int q = 0; q < VEC; ++q) p[q] = v[q];
    }
}
template <int VEC>
__device__ __forceinline__ void store_vec(uint16_t *p, const float (&v)[VEC]) {
    if constexpr (VEC == 8) {
        *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]),
                                                   pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    } else if constexpr (VEC == 4) {
        *reinterpret_cast<uint2 *>(p) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
    } else {
#pragma unroll
        for (int q = 0; q < VEC; ++q) p[q] = static_cast<uint16_t>(pack_bf16(v[q], 0.f));
    }
}

}  // namespace tfg
