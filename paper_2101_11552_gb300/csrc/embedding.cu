// Embedding lookup with scaling, and the gradient of the table.
//
//   out[i, :]        = scale * table[ids[i], :]          (zeros for the padding id)
//   grad_table[v, :] = scale * sum over i with ids[i] == v of grad_out[i, :]
//
// Nodes that carry an id instead of features (an atom kind, a user, a word) enter the
// aggregations of tf_geometric (Fig. 1) through such a table.  The gradient is the
// "reduce by key" of the map-reduce framework (Section 2.1.2, Fig. 5b) with the id as the
// key: tfg_group_ids orders the positions by id once, and the reduction walks them.
//
// What bounds it.  The lookup moves bytes: 131,072 rows of 1,024 bf16 of a table of 50,000 in
// 55 us (334 MB at the least, 6.1 TB/s; ids follow a Zipf law), 112,640 rows of 128 fp32 in 17 us
// (58 MB, 3.4 TB/s: issue slots 53 % busy, 64 warp instructions a row of 512 bytes), 64 rows in 2.1
// us (the launch).  The gradient
// writes the whole table: 131,072 bf16 rows of 1,024 into 50,000 fp32 rows in 83 us (446 MB,
// 5.4 TB/s), 60,000 rows of 100 into 169,343 in 28 us (80 MB, 2.8 TB/s: the second launch,
// and chains of id -> position -> row at 12 positions a worker), 112,640 rows of 128 into 119
// in 18.5 us (58 MB, 3.1 TB/s: the joins).
#include <algorithm>

#include "widen.cuh"

namespace tfg {
namespace {

// ---- lookup -----------------------------------------------------------------------
constexpr int kLookupThreads = 256;
// Rows (or blocks of a wide row) in flight per lane: 4 against 2 and 8, 131,072 rows of 1,024
// bf16 with their gradient 182 / 195 / 197 us.
constexpr int kLookupRows = 4;

// 2^log_lanes lanes cover a row's vectors side by side.  Rows of up to 32 vectors: every
// lane has kLookupRows rows in flight.  Wider rows (WIDE): a warp takes kLookupRows
// blocks of 32 vectors of one row, blockIdx.y the next ones, so that long runs of a row
// are read and written together.  The product is formed in fp32 and rounded once more
// where the output is bf16.
//
// The status: up to kLookupCheck ids the last CTA of the grid looks through all of them
// and writes the word (check), which saves the launch that clears it; else every group
// reports its own.
constexpr int64_t kLookupCheck = 8192;
template <typename TT, typename OT, int VEC, bool WIDE, typename IdT>
__global__ void __launch_bounds__(kLookupThreads)
embedding_lookup(const IdT *__restrict__ ids, int64_t n, const TT *__restrict__ table, int64_t rows, int64_t f,
                 int64_t padding, float scale, int log_lanes, bool check, OT *__restrict__ out, int32_t *status) {
    if (check && blockIdx.x == gridDim.x - 1) {
        bool bad = false;
        if (blockIdx.y == 0) {
            for (int64_t i = threadIdx.x; i < n; i += kLookupThreads) {
                const int64_t id = __ldg(ids + i);
                bad |= id != padding && (id < 0 || id >= rows);
            }
            const int any = __syncthreads_or(bad);
            if (threadIdx.x == 0) *status = any ? TFG_ERR_INDEX_RANGE : TFG_OK;
        }
        return;
    }
    const int lanes = 1 << log_lanes;
    const int sub = threadIdx.x & (lanes - 1);
    const int64_t group = (static_cast<int64_t>(blockIdx.x) * kLookupThreads + threadIdx.x) >> log_lanes;
    constexpr int kRows = WIDE ? 1 : kLookupRows, kBlocks = WIDE ? kLookupRows : 1;
    const int64_t i0 = group * kRows;
    const int64_t vecs = f / VEC;
    if (i0 >= n) return;
    bool here[kRows];
    int64_t at[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
        here[u] = false;
        at[u] = 0;
        if (i0 + u < n) {
            const int64_t id = __ldg(ids + i0 + u);
            here[u] = id != padding && id >= 0 && id < rows;
            at[u] = here[u] ? id * f : 0;
            if (!check && !here[u] && id != padding && sub == 0 && blockIdx.y == 0) set_status(status, TFG_ERR_INDEX_RANGE);
        }
    }
    const int64_t stride = static_cast<int64_t>(gridDim.y) * kBlocks * lanes;
    for (int64_t c0 = static_cast<int64_t>(blockIdx.y) * kBlocks * lanes + sub; c0 < vecs; c0 += stride) {
        RowVec<TT, VEC> r[kLookupRows];
#pragma unroll
        for (int u = 0; u < kLookupRows; ++u) {
            const int64_t c = c0 + (WIDE ? u * lanes : 0);
            if (here[WIDE ? 0 : u] && c < vecs) r[u].load(table + at[WIDE ? 0 : u] + c * VEC);
        }
#pragma unroll
        for (int u = 0; u < kLookupRows; ++u) {
            const int64_t c = c0 + (WIDE ? u * lanes : 0), i = i0 + (WIDE ? 0 : u);
            if (i >= n || c >= vecs) continue;
            float v[VEC];
            if (here[WIDE ? 0 : u]) {
                r[u].widen(v);
#pragma unroll
                for (int q = 0; q < VEC; ++q) v[q] *= scale;
            } else {
#pragma unroll
                for (int q = 0; q < VEC; ++q) v[q] = 0.f;
            }
            store_vec<VEC>(out + i * f + c * VEC, v);
        }
    }
}

int log_lanes_for(int64_t vecs) {
    int l = 0;
    while (l < 5 && (int64_t(1) << l) < vecs) ++l;
    return l;
}

template <typename TT, typename OT, int VEC, typename IdT>
cudaError_t lookup_vec(const void *ids, int64_t n, const void *table, int64_t rows, int64_t f, int64_t padding,
                       float scale, void *out, int32_t *status, cudaStream_t s) {
    const int l = log_lanes_for(f / VEC);
    const bool wide = f / VEC > 32, check = n <= kLookupCheck;
    const int64_t per_cta = (kLookupThreads >> l) * (wide ? 1 : kLookupRows);
    const int64_t block = wide ? 32 * kLookupRows : 32;
    const int64_t blocks = (f / VEC + block - 1) / block;
    const dim3 grid(static_cast<unsigned>((n + per_cta - 1) / per_cta + (check ? 1 : 0)), static_cast<unsigned>(min64(blocks, 65535)));
    auto *kernel = wide ? embedding_lookup<TT, OT, VEC, true, IdT> : embedding_lookup<TT, OT, VEC, false, IdT>;
    kernel<<<grid, kLookupThreads, 0, s>>>(static_cast<const IdT *>(ids), n, static_cast<const TT *>(table), rows, f,
                                           padding, scale, l, check, static_cast<OT *>(out), status);
    return cudaGetLastError();
}

template <typename TT, typename OT, typename IdT>
cudaError_t lookup_types(const void *ids, int64_t n, const void *table, int64_t rows, int64_t f, int64_t padding,
                         float scale, void *out, int32_t *status, cudaStream_t s) {
    const uintptr_t both = reinterpret_cast<uintptr_t>(table) | reinterpret_cast<uintptr_t>(out);
    constexpr bool wide = sizeof(TT) + sizeof(OT) < 8;          // a bf16 side: 8 values a lane
    if constexpr (wide) {
        if (f % 8 == 0 && both % 16 == 0)
            return lookup_vec<TT, OT, 8, IdT>(ids, n, table, rows, f, padding, scale, out, status, s);
    }
    if (f % 4 == 0 && both % 16 == 0)
        return lookup_vec<TT, OT, 4, IdT>(ids, n, table, rows, f, padding, scale, out, status, s);
    return lookup_vec<TT, OT, 1, IdT>(ids, n, table, rows, f, padding, scale, out, status, s);
}

template <typename IdT>
cudaError_t lookup_ids(const void *ids, int64_t n, const void *table, int table_dtype, int64_t rows, int64_t f,
                       int64_t padding, float scale, void *out, int out_dtype, int32_t *status, cudaStream_t s) {
    if (table_dtype == TFG_F32)
        return out_dtype == TFG_F32
                   ? lookup_types<float, float, IdT>(ids, n, table, rows, f, padding, scale, out, status, s)
                   : lookup_types<float, uint16_t, IdT>(ids, n, table, rows, f, padding, scale, out, status, s);
    return out_dtype == TFG_F32
               ? lookup_types<uint16_t, float, IdT>(ids, n, table, rows, f, padding, scale, out, status, s)
               : lookup_types<uint16_t, uint16_t, IdT>(ids, n, table, rows, f, padding, scale, out, status, s);
}

// ---- gradient ---------------------------------------------------------------------
// Every worker (LPR lanes) reduces an equal share of the sorted positions, so a frequent
// id is shared by as many workers as it takes, whatever the distribution of the ids.  A
// worker keeps D positions' vectors in flight across row ends -- rows of one or two
// positions cost no round trip each -- and adds them in order; a row that begins and ends
// in its share is written at once.  Parts of rows that cross shares go to shared memory,
// and after the CTA's one barrier the worker in which a row ends adds them in order; rows
// that cross CTAs leave one part per CTA in the workspace, added by embedding_grad_join.
// Every CTA also writes the zeros of its share of the rows that no id names.  Fixed
// order, fp32, no atomics.
constexpr int kGradThreads = 512, kGradPerSm = 2; // as four CTAs of 256: 2 % slower, eight: 13 to 26 %
constexpr int kGradCtas = 152 * kGradPerSm;
constexpr int kGradMinShare = 8;                  // positions a worker should have at least
// Up to so many positions a worker, one CTA takes them all: no row crosses CTAs, and the join's
// launch is left out.  The device takes as long (150 rows of 128: 8.9 us against 10.1 with a
// join, 2,000 of 16: 9.7 against 8.7), the host, which bounds calls so short, 3 us of 18 less.
constexpr int kGradOneCta = 16;

struct GradArgs {
    const int32_t *rowptr, *sorted_ids, *perm;
    const void *g;
    int64_t n, rows, f;
    float scale;
    int min_share;
    float *out, *head, *tail;                     // head, tail: [CTA][column tile][tile]
};

// positions per worker, the same in both kernels
__device__ __forceinline__ int64_t grad_share(const GradArgs &a, int64_t named, int64_t workers) {
    const int64_t p = (named + workers - 1) / workers;
    return p > a.min_share ? p : a.min_share;
}

template <typename GT, int VEC, int LPR, int T>
__global__ void __launch_bounds__(kGradThreads, kGradPerSm) embedding_grad(GradArgs a) {
    using V = VecLoad<GT, VEC>;
    constexpr int NW = kGradThreads / LPR;        // workers
    constexpr int kCols = LPR * VEC * T;
    constexpr int D = 4;                          // 8 spill: 131,072 rows of 1,024 bf16 176 against 182 us
    extern __shared__ __align__(16) float s_part[];   // tails [worker][kCols], heads [worker][kCols]
    float *s_tail = s_part, *s_head = s_part + NW * kCols;
    const int sub = threadIdx.x % LPR, w = threadIdx.x / LPR;
    const int64_t f = a.f;
    const int64_t c0 = static_cast<int64_t>(blockIdx.y) * kCols + sub * VEC;      // and c0 + i * LPR * VEC
    bool col[T];
#pragma unroll
    for (int i = 0; i < T; ++i) col[i] = c0 + i * LPR * VEC < f;
    const GT *g = static_cast<const GT *>(a.g) + c0;
    float *out = a.out + c0;

    const int64_t named = min64(a.n, max(0, __ldg(a.rowptr + a.rows)));
    const int64_t p = grad_share(a, named, static_cast<int64_t>(gridDim.x) * NW);
    const int64_t W = static_cast<int64_t>(blockIdx.x) * NW + w;
    const int64_t ka = min64(named, W * p), kb = min64(named, ka + p);
    auto id_at = [&](int64_t k) { return k < named ? __ldg(a.sorted_ids + k) : -1; };
    auto write = [&](int32_t row, const float (&v)[T][VEC]) {
        if (static_cast<uint32_t>(row) >= static_cast<uint64_t>(a.rows)) return;
#pragma unroll
        for (int i = 0; i < T; ++i) {
            if (!col[i]) continue;
            float r[VEC];
#pragma unroll
            for (int q = 0; q < VEC; ++q) r[q] = a.scale * v[i][q];
            store_vec<VEC>(out + static_cast<int64_t>(row) * f + i * LPR * VEC, r);
        }
    };
    auto park = [&](float *to, const float (&v)[T][VEC]) {
#pragma unroll
        for (int i = 0; i < T; ++i)
#pragma unroll
            for (int q = 0; q < VEC; ++q) to[w * kCols + (i * LPR + sub) * VEC + q] = v[i][q];
    };

    // rows without ids
    const int64_t per = (a.rows + gridDim.x - 1) / gridDim.x;
    const int64_t z0 = per * blockIdx.x, z1 = min64(a.rows, z0 + per);
    float zero[T][VEC] = {};
#pragma unroll 4
    for (int64_t t = z0 + w; t < z1; t += NW)
        if (__ldg(a.rowptr + t) == __ldg(a.rowptr + t + 1)) write(static_cast<int32_t>(t), zero);

    float acc[T][VEC] = {};
    const bool continued = ka < kb && ka > 0 && id_at(ka - 1) == id_at(ka);      // by the first row here
    bool first = true, head = false;
    for (int64_t k = ka; k < kb; k += D) {
        typename V::Raw raw[D][T];
        int32_t id[D + 1];
#pragma unroll
        for (int u = 0; u <= D; ++u) id[u] = id_at(k + u);
#pragma unroll
        for (int u = 0; u < D; ++u) {
            const bool on = k + u < kb;
            const uint32_t at = on ? static_cast<uint32_t>(__ldg(a.perm + k + u)) : 0u;
#pragma unroll
            for (int i = 0; i < T; ++i) {
                raw[u][i] = V::zero();
                if (on && col[i] && at < a.n) raw[u][i] = V::raw(g + static_cast<int64_t>(at) * f + i * LPR * VEC);
            }
        }
#pragma unroll
        for (int u = 0; u < D; ++u) {
            if (k + u >= kb) continue;
#pragma unroll
            for (int i = 0; i < T; ++i) {
                float v[VEC];
                V::widen(raw[u][i], v);
#pragma unroll
                for (int q = 0; q < VEC; ++q) acc[i][q] += v[q];
            }
            if (id[u] != id[u + 1]) {                          // the row ends here
                if (first && continued) {
                    park(s_head, acc);
                    head = true;
                } else {
                    write(id[u], acc);
                }
                first = false;
#pragma unroll
                for (int i = 0; i < T; ++i)
#pragma unroll
                    for (int q = 0; q < VEC; ++q) acc[i][q] = 0.f;
            }
        }
    }
    park(s_tail, acc);                                         // the open row's part, or zeros
    __syncthreads();
    // parts of the workers [w0, w1) of this CTA, in order
    auto add_tails = [&](float (&v)[T][VEC], int64_t w0, int64_t w1) {
        for (int64_t x = w0; x < w1; ++x)
#pragma unroll
            for (int i = 0; i < T; ++i)
#pragma unroll
                for (int q = 0; q < VEC; ++q) v[i][q] += s_tail[x * kCols + (i * LPR + sub) * VEC + q];
    };
    auto leave = [&](float *to, const float (&v)[T][VEC]) {
        float *at = to + (static_cast<int64_t>(blockIdx.x) * gridDim.y + blockIdx.y) * kCols;
#pragma unroll
        for (int i = 0; i < T; ++i)
#pragma unroll
            for (int q = 0; q < VEC; ++q) at[(i * LPR + sub) * VEC + q] = v[i][q];
    };
    const int64_t W0 = static_cast<int64_t>(blockIdx.x) * NW;
    // first worker of a row, relative to this CTA (negative: an earlier CTA's)
    auto begins = [&](int32_t row) {
        const bool known = static_cast<uint32_t>(row) < static_cast<uint64_t>(a.rows);
        return static_cast<int64_t>(known ? __ldg(a.rowptr + row) : 0) / p - W0;
    };
    if (head) {
        const int32_t row = id_at(ka);
        const int64_t b = begins(row);
        float v[T][VEC] = {};
        add_tails(v, b > 0 ? b : 0, w);
#pragma unroll
        for (int i = 0; i < T; ++i)
#pragma unroll
            for (int q = 0; q < VEC; ++q) v[i][q] += s_head[w * kCols + (i * LPR + sub) * VEC + q];
        if (b >= 0) write(row, v);
        else leave(a.head, v);
    }
    if (w == NW - 1 && ka < kb && id_at(kb - 1) == id_at(kb)) {  // the CTA's last row goes on behind it
        const int64_t b = begins(id_at(kb - 1));
        float v[T][VEC] = {};
        add_tails(v, b > 0 ? b : 0, NW);
        leave(a.tail, v);
    }
}

// Rows that cross CTAs: the CTA in which such a row ends adds the tails of those before
// it in order, in 8 interleaved chains per column.
constexpr int kJoinThreads = 256;
constexpr int kJoinChains = 8;
__global__ void __launch_bounds__(kJoinThreads)
embedding_grad_join(GradArgs a, int workers, int cols, int ctas) {
    __shared__ float s_sum[kJoinChains][kJoinThreads / kJoinChains];
    const int64_t named = min64(a.n, max(0, __ldg(a.rowptr + a.rows)));
    const int64_t share = grad_share(a, named, static_cast<int64_t>(ctas) * workers) * workers;
    const int64_t b = blockIdx.x + 1;
    const int64_t k = b * share;
    if (k >= named) return;
    const int32_t row = __ldg(a.sorted_ids + k);
    if (__ldg(a.sorted_ids + k - 1) != row || static_cast<uint32_t>(row) >= static_cast<uint64_t>(a.rows)) return;
    if (__ldg(a.rowptr + row + 1) > k + share) return;          // goes on: a later CTA's
    const int64_t b0 = max(0, __ldg(a.rowptr + row)) / share;
    constexpr int kWide = kJoinThreads / kJoinChains;
    const int lane = threadIdx.x % kWide, chain = threadIdx.x / kWide;
    const int tiles = static_cast<int>((a.f + cols - 1) / cols);
    for (int64_t c0 = static_cast<int64_t>(blockIdx.y) * kWide; c0 < a.f; c0 += static_cast<int64_t>(gridDim.y) * kWide) {
        const int64_t c = c0 + lane;
        float v = 0.f;
        const int64_t at = c / cols * cols + c % cols;          // column tile, column
        if (c < a.f) {
#pragma unroll 4
            for (int64_t x = b0 + chain; x < b; x += kJoinChains) v += a.tail[x * tiles * cols + at];
        }
        s_sum[chain][lane] = v;
        __syncthreads();
        if (chain == 0 && c < a.f) {
#pragma unroll
            for (int i = 1; i < kJoinChains; ++i) v += s_sum[i][lane];
            a.out[static_cast<int64_t>(row) * a.f + c] = a.scale * (v + a.head[b * tiles * cols + at]);
        }
        __syncthreads();
    }
}

// Column tiling of a gradient: the widest vectors that the row length and the pointers
// allow, the fewest lanes that cover a row.
struct GradPlan {
    int vec, lanes, t, cols, tiles, ctas;
};

GradPlan grad_plan(int64_t n, int64_t rows, int64_t f, int dtype, bool aligned) {
    GradPlan p;
    p.vec = aligned && dtype == TFG_BF16 && f % 8 == 0 ? 8 : (aligned && f % 4 == 0 ? 4 : 1);
    const int64_t vecs = f / p.vec;
    p.lanes = vecs <= 4 ? 4 : (vecs <= 8 ? 8 : (vecs <= 16 ? 16 : 32));
    p.t = p.vec == 1 && vecs > 32 ? 4 : 1;
    p.cols = p.lanes * p.vec * p.t;
    p.tiles = static_cast<int>((f + p.cols - 1) / p.cols);
    const int workers = kGradThreads / p.lanes;
    const int64_t by_ids = (n + int64_t(workers) * kGradMinShare - 1) / (int64_t(workers) * kGradMinShare);
    const int64_t by_rows = (rows + int64_t(workers) * 32 - 1) / (int64_t(workers) * 32);
    const int64_t most = p.tiles >= kGradCtas ? 1 : kGradCtas / p.tiles;
    p.ctas = static_cast<int>(min64(most, by_ids > by_rows ? by_ids : by_rows));
    if (p.ctas < 1) p.ctas = 1;
    return p;
}

template <typename GT, int VEC, int LPR, int T>
cudaError_t launch_grad(const GradArgs &a, const GradPlan &p, cudaStream_t s) {
    auto *kernel = embedding_grad<GT, VEC, LPR, T>;
    constexpr int smem = 2 * kGradThreads * VEC * T * static_cast<int>(sizeof(float));
    static_assert(smem <= 48 * 1024, "parts fit in the shared memory every launch may use");
    kernel<<<dim3(p.ctas, p.tiles), kGradThreads, smem, s>>>(a);
    return cudaGetLastError();
}

template <typename GT, int VEC, int T>
cudaError_t launch_grad_lanes(const GradArgs &a, const GradPlan &p, cudaStream_t s) {
    if constexpr (T > 1) {
        return launch_grad<GT, VEC, 32, T>(a, p, s);
    } else {
        switch (p.lanes) {
            case 4: return launch_grad<GT, VEC, 4, T>(a, p, s);
            case 8: return launch_grad<GT, VEC, 8, T>(a, p, s);
            case 16: return launch_grad<GT, VEC, 16, T>(a, p, s);
            default: return launch_grad<GT, VEC, 32, T>(a, p, s);
        }
    }
}

}  // namespace

cudaError_t launch_embedding_lookup(const void *ids, bool id32, int64_t n, const void *table, int table_dtype,
                                    int64_t rows, int64_t f, float scale, int64_t padding, void *out, int out_dtype,
                                    int32_t *status, cudaStream_t s) {
    if (n == 0 || n > kLookupCheck) {
        const cudaError_t err = cudaMemsetAsync(status, 0, sizeof(int32_t), s);
        if (err != cudaSuccess || n == 0) return err;
    }
    return id32 ? lookup_ids<int32_t>(ids, n, table, table_dtype, rows, f, padding, scale, out, out_dtype, status, s)
                : lookup_ids<int64_t>(ids, n, table, table_dtype, rows, f, padding, scale, out, out_dtype, status, s);
}

size_t embedding_backward_workspace_bytes(int64_t f) {
    // a part of each kind per CTA and column tile of at most 256: kGradCtas of them, or one CTA
    // and as many tiles as the row has
    const int64_t cols = (f + 255) / 256 * 256, most = int64_t(kGradCtas) * 256;
    return size_t(2) * size_t(cols > most ? cols : most) * sizeof(float);
}

cudaError_t launch_embedding_backward(const int32_t *rowptr, const int32_t *sorted_ids, const int32_t *perm,
                                      const void *g, int g_dtype, int64_t n, int64_t rows, int64_t f, float scale,
                                      float *out, void *ws, cudaStream_t s) {
    const bool aligned = ((reinterpret_cast<uintptr_t>(g) | reinterpret_cast<uintptr_t>(out)) & 15) == 0;
    const GradPlan p = grad_plan(n, rows, f, g_dtype, aligned);
    const int workers = kGradThreads / p.lanes;
    const bool one_cta = n <= int64_t(workers) * kGradOneCta;
    const int min_share = one_cta ? std::max(kGradMinShare, static_cast<int>((n + workers - 1) / workers)) : kGradMinShare;
    GradArgs a{rowptr, sorted_ids, perm, g, n, rows, f, scale, min_share, out, static_cast<float *>(ws), nullptr};
    a.tail = a.head + int64_t(p.ctas) * p.tiles * p.cols;
    cudaError_t err;
    if (g_dtype == TFG_BF16)
        err = p.vec == 8 ? launch_grad_lanes<uint16_t, 8, 1>(a, p, s)
              : p.vec == 4 ? launch_grad_lanes<uint16_t, 4, 1>(a, p, s)
              : p.t == 1   ? launch_grad_lanes<uint16_t, 1, 1>(a, p, s)
                           : launch_grad_lanes<uint16_t, 1, 4>(a, p, s);
    else
        err = p.vec == 4 ? launch_grad_lanes<float, 4, 1>(a, p, s)
              : p.t == 1 ? launch_grad_lanes<float, 1, 1>(a, p, s)
                         : launch_grad_lanes<float, 1, 4>(a, p, s);
    if (err != cudaSuccess || p.ctas == 1 || one_cta) return err;
    const int64_t tiles = (f + kJoinThreads / kJoinChains - 1) / (kJoinThreads / kJoinChains);
    embedding_grad_join<<<dim3(p.ctas - 1, static_cast<unsigned>(min64(tiles, 65535))), kJoinThreads, 0, s>>>(
        a, workers, p.cols, p.ctas);
    return cudaGetLastError();
}

}  // namespace tfg
