// The norm over all gradients of a model, and gradients clipped by it.
//
//   norm = sqrt(sum over tensors t, values i of t_i^2)
//   out  = t * clip_norm / max(norm, clip_norm)
//
// Training a model on top of the aggregations ends each step with it (the gradient of
// every layer is an output of the backward calls).  Two launches: partial sums of
// squares, one per CTA; then every CTA of the second adds the partials in the same fixed
// order and scales its share.  Both walk chunks of kChunk values across all tensors, so
// that a model of many small tensors costs no more launches than one large tensor.
//
// Precision.  A thread adds 32 squares in fp32 and carries the sums of those in two
// floats (the rounding error of every addition is kept), so long gradients lose nothing;
// squares that leave the range of fp32 (values above 1e15 or all below 1e-13 or so) are
// taken again in fp64.  The partials, the root and the factor are fp64, and the factor is
// rounded once to fp32, with a power of two split off where it is below the normal numbers.
//
// What bounds it: memory.  1,000 million bf16 values: the sums 285 us (7.0 TB/s), the scaling
// 620 us (4.0 GB read and written, 6.5 TB/s), 905 us in all; the second read is what the
// definition costs beyond a read and a write (590 us), as the factor is known last.  85 million
// of mixed types 94 us: the second pass goes backwards, but finds little of the first in L2 (it
// reads 156 of its 170 MB from DRAM).  100,000 values in six tensors 8.3 us: two launches.
#include "widen.cuh"

namespace tfg {
namespace {

constexpr int kNormThreads = 256;
constexpr int kPerThread = 64;                    // values of a chunk that a thread sums
constexpr int kChunk = kNormThreads * kPerThread;
constexpr int kNormCtas = 1216;                   // eight a multiprocessor: partials of one launch
// Tensors of a launch, passed as 1 or 16 KB of parameters.
constexpr int kListSmall = 32, kListLarge = 512;

// The tensors of one launch, passed by value: nothing is copied to the device and a
// captured launch keeps its list.  first[t] is the first chunk of tensor t.
template <int CAP>
struct TensorList {
    const void *in[CAP];
    void *out[CAP];
    int64_t size[CAP];
    int64_t first[CAP + 1];
    uint8_t bf16[CAP];
    int count;
};

// The tensor of a chunk: the last one that begins at or before it.
template <int CAP>
__device__ __forceinline__ int tensor_of(const TensorList<CAP> &list, int64_t chunk, int from) {
    int lo = from, hi = list.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (list.first[mid] <= chunk) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// ---- sums of squares --------------------------------------------------------------
struct SquareSum {
    float hi = 0.f, lo = 0.f;                     // sum = hi + lo
    double wide = 0.0;                            // what left the range of fp32

    __device__ __forceinline__ void add(float s) {
        const float t = hi + s;                   // two-sum: t + e == hi + s
        const float b = t - hi;
        lo += (hi - (t - b)) + (s - b);
        hi = t;
    }
    __device__ __forceinline__ double total() const { return static_cast<double>(hi) + lo + wide; }
};

// Squares of a thread's values of one chunk.  In range: the sum is below 2^100 and either
// large enough that squares lost below 2^-149 do not count, or of zeros alone.
template <int N>
__device__ __forceinline__ void add_squares(SquareSum &acc, const float (&v)[N]) {
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < N; ++i) s[i & 3] = fmaf(v[i], v[i], s[i & 3]);
    const float sum = (s[0] + s[1]) + (s[2] + s[3]);
    if (sum > 8.3e-25f && sum < 1.2e30f) {        // 2^-80, 2^100
        acc.add(sum);
        return;
    }
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) most = fmaxf(most, fabsf(v[i]));
    if (most == 0.f && sum == 0.f) return;        // zeros (a NaN makes the sum a NaN)
    double w = 0.0;
#pragma unroll
    for (int i = 0; i < N; ++i) w += static_cast<double>(v[i]) * v[i];
    acc.wide += w;
}

template <typename T, int VEC>
__device__ __forceinline__ void square_chunk(SquareSum &acc, const T *p, int64_t left) {
    constexpr int kLoads = 32 / VEC;              // half a thread's values at a time
#pragma unroll
    for (int h = 0; h < kPerThread / 32; ++h) {
        typename VecLoad<T, VEC>::Raw raw[kLoads];
        const int64_t base = static_cast<int64_t>(h) * 32 * kNormThreads;
        if (base >= left) break;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int64_t at = base + (static_cast<int64_t>(i) * kNormThreads + threadIdx.x) * VEC;
            raw[i] = VecLoad<T, VEC>::zero();
            if (at + VEC <= left) raw[i] = VecLoad<T, VEC>::raw(p + at);
        }
        float v[32];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            float w[VEC];
            VecLoad<T, VEC>::widen(raw[i], w);
#pragma unroll
            for (int q = 0; q < VEC; ++q) v[i * VEC + q] = w[q];
        }
        add_squares<32>(acc, v);
    }
    if (VEC > 1 && left < kChunk && left % VEC != 0 && static_cast<int64_t>(threadIdx.x) < left % VEC) {
        float v[1];
        VecLoad<T, 1>::load(p + left / VEC * VEC + threadIdx.x, v);
        add_squares<1>(acc, v);
    }
}

// Sum over the CTA in a fixed order; thread 0 has it.
__device__ __forceinline__ double cta_sum(double v, double *s_warp) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += lane_xor(v, o);
    if (lane == 0) s_warp[warp] = v;
    __syncthreads();
    double t = 0.0;
    if (threadIdx.x == 0)
        for (int w = 0; w < kNormThreads / 32; ++w) t += s_warp[w];
    __syncthreads();
    return t;
}

template <int CAP>
__global__ void __launch_bounds__(kNormThreads)
sum_squares(const __grid_constant__ TensorList<CAP> list, double *__restrict__ partial) {
    __shared__ double s_warp[kNormThreads / 32];
    SquareSum acc;
    const int64_t chunks = list.first[list.count];
    int t = 0;
    for (int64_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        t = tensor_of(list, c, t);
        const int64_t at = (c - list.first[t]) * kChunk;
        const int64_t left = min64(kChunk, list.size[t] - at);
        const bool aligned = reinterpret_cast<uintptr_t>(list.in[t]) % 16 == 0;
        if (list.bf16[t]) {
            const uint16_t *p = static_cast<const uint16_t *>(list.in[t]) + at;
            if (aligned) square_chunk<uint16_t, 8>(acc, p, left);
            else square_chunk<uint16_t, 1>(acc, p, left);
        } else {
            const float *p = static_cast<const float *>(list.in[t]) + at;
            if (aligned) square_chunk<float, 4>(acc, p, left);
            else square_chunk<float, 1>(acc, p, left);
        }
    }
    const double sum = cta_sum(acc.total(), s_warp);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

// Sum of all partials, the same in every CTA.
__device__ __forceinline__ double add_partials(const double *__restrict__ partial, int n, double *s_warp) {
    double v = 0.0;
    for (int i = threadIdx.x; i < n; i += kNormThreads) v += __ldg(partial + i);
    return cta_sum(v, s_warp);
}

__global__ void __launch_bounds__(kNormThreads)
write_norm(const double *__restrict__ partial, int n, float *__restrict__ norm) {
    __shared__ double s_warp[kNormThreads / 32];
    const double sum = add_partials(partial, n, s_warp);
    if (threadIdx.x == 0) *norm = static_cast<float>(sqrt(sum));
}

// ---- scaling ----------------------------------------------------------------------
// Plain loads: out may be the tensor itself, and then what is read is written here.
// Stores that leave L2 first, so that what the pass has yet to read may stay.
template <int VEC>
__device__ __forceinline__ void store_stream(float *p, const float (&v)[VEC]) {
    if constexpr (VEC == 4) __stcs(reinterpret_cast<float4 *>(p), make_float4(v[0], v[1], v[2], v[3]));
    else store_vec<VEC>(p, v);
}
template <int VEC>
__device__ __forceinline__ void store_stream(uint16_t *p, const float (&v)[VEC]) {
    if constexpr (VEC == 8)
        __stcs(reinterpret_cast<uint4 *>(p), make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]),
                                                        pack_bf16(v[6], v[7])));
    else store_vec<VEC>(p, v);
}

// The factor as lift * f.  One below fp32's normal numbers (clip_norm 1e-3, norm 1e36) would keep
// a few bits there: lift is 2^-126 then, else 1.  v * lift is exact wherever the result is
// a normal number, as only a v above 1 has one.  (Products in fp64 behind a branch: 905 -> 915 us
// for 1,000 million values, in a loop of their own 969, by registers.)
struct Factor {
    float lift, f;
    __device__ __forceinline__ float of(float v) const { return v * lift * f; }
};

template <typename T, int VEC>
__device__ __forceinline__ void scale_chunk(const T *p, T *o, int64_t left, const Factor &factor) {
    constexpr int kLoads = 32 / VEC;
#pragma unroll
    for (int h = 0; h < kPerThread / 32; ++h) {
        typename VecLoad<T, VEC>::Raw raw[kLoads];
        const int64_t base = static_cast<int64_t>(h) * 32 * kNormThreads;
        if (base >= left) break;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int64_t at = base + (static_cast<int64_t>(i) * kNormThreads + threadIdx.x) * VEC;
            raw[i] = VecLoad<T, VEC>::zero();
            if (at + VEC <= left) raw[i] = load_plain<T, VEC>(p + at);
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int64_t at = base + (static_cast<int64_t>(i) * kNormThreads + threadIdx.x) * VEC;
            if (at + VEC > left) continue;
            float v[VEC];
            VecLoad<T, VEC>::widen(raw[i], v);
#pragma unroll
            for (int q = 0; q < VEC; ++q) v[q] = factor.of(v[q]);
            store_stream<VEC>(o + at, v);
        }
    }
    if (VEC > 1 && left < kChunk && static_cast<int64_t>(threadIdx.x) < left % VEC) {
        const int64_t at = left / VEC * VEC + threadIdx.x;
        float v[1];
        VecLoad<T, 1>::widen(load_plain<T, 1>(p + at), v);
        v[0] = factor.of(v[0]);
        store_vec<1>(o + at, v);
    }
}

// norm: written by the first CTA where it is not null (the first of several launches).
template <int CAP>
__global__ void __launch_bounds__(kNormThreads)
scale_by_norm(const __grid_constant__ TensorList<CAP> list, const double *__restrict__ partial, int n, float clip,
              float *__restrict__ norm) {
    __shared__ double s_warp[kNormThreads / 32];
    __shared__ Factor s_factor;
    const double sum = add_partials(partial, n, s_warp);
    if (threadIdx.x == 0) {
        const double root = sqrt(sum);
        const float rounded = static_cast<float>(root);
        if (norm && blockIdx.x == 0) *norm = rounded;
        // a norm that is no finite number leaves nothing to keep: NaN everywhere
        Factor factor{1.f, isfinite(rounded) ? 1.f : __int_as_float(0x7fc00000)};
        if (isfinite(rounded) && root > clip) {
            const double quotient = clip / root;
            if (quotient < 0x1p-126) factor.lift = 0x1p-126f;
            factor.f = static_cast<float>(quotient < 0x1p-126 ? quotient * 0x1p126 : quotient);
        }
        s_factor = factor;
    }
    __syncthreads();
    const Factor factor = s_factor;
    const int64_t chunks = list.first[list.count];
    for (int64_t back = blockIdx.x; back < chunks; back += gridDim.x) {
        const int64_t c = chunks - 1 - back;      // the last chunks first: what L2 still holds
        const int t = tensor_of(list, c, 0);
        if (factor.lift * factor.f == 1.f && list.in[t] == list.out[t]) continue;      // in place and nothing to do
        const int64_t at = (c - list.first[t]) * kChunk;
        const int64_t left = min64(kChunk, list.size[t] - at);
        const bool aligned = (reinterpret_cast<uintptr_t>(list.in[t]) | reinterpret_cast<uintptr_t>(list.out[t])) % 16 == 0;
        if (list.bf16[t]) {
            const uint16_t *p = static_cast<const uint16_t *>(list.in[t]) + at;
            uint16_t *o = static_cast<uint16_t *>(list.out[t]) + at;
            if (aligned) scale_chunk<uint16_t, 8>(p, o, left, factor);
            else scale_chunk<uint16_t, 1>(p, o, left, factor);
        } else {
            const float *p = static_cast<const float *>(list.in[t]) + at;
            float *o = static_cast<float *>(list.out[t]) + at;
            if (aligned) scale_chunk<float, 4>(p, o, left, factor);
            else scale_chunk<float, 1>(p, o, left, factor);
        }
    }
}

int64_t chunks_of(int64_t size) { return (size + kChunk - 1) / kChunk; }
int ctas_for(int64_t chunks) { return static_cast<int>(min64(chunks, kNormCtas)); }

template <int CAP>
int64_t fill(TensorList<CAP> &list, int64_t from, int64_t to, const void *const *in, void *const *out,
             const int64_t *sizes, const int *dtypes) {
    int64_t chunk = 0;
    list.count = 0;
    for (int64_t t = from; t < to; ++t) {
        if (sizes[t] == 0) continue;              // no chunk: the search would not tell it from its neighbour
        const int i = list.count++;
        list.in[i] = in[t];
        list.out[i] = out ? out[t] : nullptr;
        list.size[i] = sizes[t];
        list.first[i] = chunk;
        list.bf16[i] = dtypes[t] == TFG_BF16;
        chunk += chunks_of(sizes[t]);
    }
    list.first[list.count] = chunk;
    return chunk;
}

template <int CAP>
cudaError_t squares_of(int64_t from, int64_t to, const void *const *in, const int64_t *sizes, const int *dtypes,
                       double *partial, int *ctas, cudaStream_t s) {
    TensorList<CAP> list;
    *ctas = ctas_for(fill(list, from, to, in, nullptr, sizes, dtypes));
    if (*ctas == 0) return cudaSuccess;
    sum_squares<CAP><<<*ctas, kNormThreads, 0, s>>>(list, partial);
    return cudaGetLastError();
}

template <int CAP>
cudaError_t scale_of(int64_t from, int64_t to, const void *const *in, void *const *out, const int64_t *sizes,
                     const int *dtypes, const double *partial, int n, float clip, float *norm, cudaStream_t s) {
    TensorList<CAP> list;
    const int ctas = ctas_for(fill(list, from, to, in, out, sizes, dtypes));
    if (ctas == 0 && !norm) return cudaSuccess;
    scale_by_norm<CAP><<<ctas > 0 ? ctas : 1, kNormThreads, 0, s>>>(list, partial, n, clip, norm);
    return cudaGetLastError();
}

}  // namespace

size_t global_norm_workspace_bytes(int64_t tensors) {
    const int64_t launches = (tensors + kListLarge - 1) / kListLarge;
    return sizeof(double) * kNormCtas * size_t(launches < 1 ? 1 : launches);
}

// outs null: the norm alone.
cudaError_t launch_global_norm(int64_t tensors, const void *const *in, const int64_t *sizes, const int *dtypes,
                               float clip, void *const *outs, float *norm, void *ws, cudaStream_t s) {
    double *partial = static_cast<double *>(ws);
    int n = 0;
    for (int64_t from = 0; from < tensors; from += kListLarge) {
        const int64_t to = min64(tensors, from + kListLarge);
        int ctas = 0;
        const cudaError_t err = to - from <= kListSmall
                                    ? squares_of<kListSmall>(from, to, in, sizes, dtypes, partial + n, &ctas, s)
                                    : squares_of<kListLarge>(from, to, in, sizes, dtypes, partial + n, &ctas, s);
        if (err != cudaSuccess) return err;
        n += ctas;
    }
    if (!outs) {
        write_norm<<<1, kNormThreads, 0, s>>>(partial, n, norm);
        return cudaGetLastError();
    }
    int64_t from = 0;
    do {
        const int64_t to = min64(tensors, from + kListLarge);
        float *first = from == 0 ? norm : nullptr;
        const cudaError_t err =
            to - from <= kListSmall
                ? scale_of<kListSmall>(from, to, in, outs, sizes, dtypes, partial, n, clip, first, s)
                : scale_of<kListLarge>(from, to, in, outs, sizes, dtypes, partial, n, clip, first, s);
        if (err != cudaSuccess) return err;
        from = to;
    } while (from < tensors);
    return cudaSuccess;
}

}  // namespace tfg
