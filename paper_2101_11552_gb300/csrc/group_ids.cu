// Grouping of ids: the positions of a list of ids ordered by id, equal ids in their
// original order -- the "reduce by key" grouping of the graph map-reduce framework
// (tf_geometric Section 2.1.2, Fig. 5b) with a table row as the key.  The gradient of an
// embedding table is the reduction over these groups (embedding.cu).
//
// A stable least-significant-digit radix sort of (key, position) pairs, digits of at most
// 9 bits, in tiles of 2,048 pairs.  Positions that take part in nothing (the padding id,
// ids outside the table) get the key `rows`, behind every row.  A pass is
//   upsweep    a tile's digit counts -> cnt[digit][tile]
//   scan       exclusive sums over the tiles of each digit, and the digit's total
//              (only where there are more than kDirectTiles tiles: up to there the
//              downsweep adds the counts up itself, which saves a launch)
//   downsweep  ranks a tile's pairs, stages them in shared memory in digit order and
//              writes each digit's run with coalesced stores
// and the row boundaries are found by binary search in the sorted keys.  The status word
// is written by that last kernel from one flag per tile, so nothing has to be cleared.
// No kernel waits on another CTA.
#include "common.cuh"

namespace tfg {
namespace {

constexpr int kGroupThreads = 256;
constexpr int kGroupWarps = kGroupThreads / 32;
constexpr int kGroupItems = 8;
constexpr int kGroupTile = kGroupThreads * kGroupItems;
constexpr int kGroupBits = 9;                     // most bits of a digit
constexpr int kDirectTiles = 64;

struct GroupPlan {
    int passes, width, tiles;
};

GroupPlan group_plan(int64_t rows, int64_t n) {
    int bits = 1;
    while ((int64_t(1) << bits) < rows + 1) ++bits;
    const int passes = (bits + kGroupBits - 1) / kGroupBits;
    return {passes, (bits + passes - 1) / passes, ceil_div(n, kGroupTile)};
}

size_t round256(size_t b) { return (b + 255) & ~size_t(255); }

template <typename IdT>
__device__ __forceinline__ uint32_t group_key(IdT id, int64_t rows, int64_t padding, bool &bad) {
    const int64_t v = id;
    if (v == padding) return static_cast<uint32_t>(rows);
    if (v < 0 || v >= rows) {
        bad = true;
        return static_cast<uint32_t>(rows);
    }
    return static_cast<uint32_t>(v);
}

template <bool FIRST, typename IdT>
__global__ void __launch_bounds__(kGroupThreads)
group_upsweep(const IdT *__restrict__ ids, const uint32_t *__restrict__ keys, int64_t n, int64_t rows, int64_t padding,
              int shift, int width, int tiles, int32_t *__restrict__ cnt, int32_t *__restrict__ bad_tile) {
    __shared__ int32_t s_cnt[1 << kGroupBits];
    const int radix = 1 << width;
    for (int d = threadIdx.x; d < radix; d += kGroupThreads) s_cnt[d] = 0;
    __syncthreads();
    const int64_t base = static_cast<int64_t>(blockIdx.x) * kGroupTile;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < kGroupItems; ++i) {
        const int64_t at = base + i * kGroupThreads + threadIdx.x;
        if (at < n) {
            const uint32_t key = FIRST ? group_key(__ldg(ids + at), rows, padding, bad) : __ldg(keys + at);
            atomicAdd(&s_cnt[(key >> shift) & (radix - 1)], 1);
        }
    }
    const int any_bad = __syncthreads_or(bad);
    if (FIRST && threadIdx.x == 0) bad_tile[blockIdx.x] = any_bad;
    for (int d = threadIdx.x; d < radix; d += kGroupThreads)
        cnt[static_cast<int64_t>(d) * tiles + blockIdx.x] = s_cnt[d];
}

// One warp a digit: cnt[digit][tile] becomes the pairs of the digit in earlier tiles.
__global__ void __launch_bounds__(kGroupThreads)
group_scan(int32_t *__restrict__ cnt, int tiles, int radix, int32_t *__restrict__ total) {
    const int lane = threadIdx.x & 31;
    const int d = blockIdx.x * kGroupWarps + (threadIdx.x >> 5);
    if (d >= radix) return;                       // whole warps
    int32_t *row = cnt + static_cast<int64_t>(d) * tiles;
    int32_t run = 0;
    for (int t0 = 0; t0 < tiles; t0 += 32) {
        const int t = t0 + lane;
        const int32_t v = t < tiles ? row[t] : 0;
        int32_t incl = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int32_t y = lane_up(incl, o);
            if (lane >= o) incl += y;
        }
        if (t < tiles) row[t] = run + incl - v;
        run += lane_get(incl, 31);
    }
    if (lane == 0) total[d] = run;
}

// Exclusive sums over the threads of the CTA; every thread calls it.
__device__ __forceinline__ int32_t scan_threads(int32_t v, int32_t *s_warp) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int32_t incl = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int32_t y = lane_up(incl, o);
        if (lane >= o) incl += y;
    }
    if (lane == 31) s_warp[warp] = incl;
    __syncthreads();
    int32_t before = 0;
#pragma unroll
    for (int w = 0; w < kGroupWarps; ++w) before += w < warp ? s_warp[w] : 0;
    __syncthreads();
    return before + incl - v;
}

template <bool FIRST, bool DIRECT, typename IdT>
__global__ void __launch_bounds__(kGroupThreads)
group_downsweep(const IdT *__restrict__ ids, const uint32_t *__restrict__ key_in, const int32_t *__restrict__ pos_in,
                int64_t n, int64_t rows, int64_t padding, int shift, int width, int tiles,
                const int32_t *__restrict__ cnt, const int32_t *__restrict__ total, uint32_t *__restrict__ key_out,
                int32_t *__restrict__ pos_out) {
    __shared__ uint32_t s_key[kGroupTile];
    __shared__ int32_t s_pos[kGroupTile];
    __shared__ int32_t s_mine[kGroupWarps][1 << kGroupBits];
    __shared__ int32_t s_delta[1 << kGroupBits];
    __shared__ int32_t s_warp[kGroupWarps];
    const int radix = 1 << width;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t tile0 = static_cast<int64_t>(blockIdx.x) * kGroupTile;
    const int count = static_cast<int>(min64(kGroupTile, n - tile0));
    int32_t *mine = s_mine[warp];
    for (int d = lane; d < radix; d += 32) mine[d] = 0;
    // the warp's 256 pairs, in original order round by round
    uint32_t keys[kGroupItems];
    int32_t pos[kGroupItems], rank[kGroupItems];
    bool bad = false;
#pragma unroll
    for (int r = 0; r < kGroupItems; ++r) {
        const int64_t at = tile0 + warp * 32 * kGroupItems + r * 32 + lane;
        keys[r] = 0;
        pos[r] = 0;
        if (at < n) {
            keys[r] = FIRST ? group_key(__ldg(ids + at), rows, padding, bad) : __ldg(key_in + at);
            pos[r] = FIRST ? static_cast<int32_t>(at) : __ldg(pos_in + at);
        }
    }
    __syncwarp();
    // rank among the warp's earlier pairs of the digit: lanes with equal digits are found
    // with one ballot per bit, and the first of them advances the warp's counter
#pragma unroll
    for (int r = 0; r < kGroupItems; ++r) {
        const bool ok = warp * 32 * kGroupItems + r * 32 + lane < count;
        const uint32_t dig = (keys[r] >> shift) & (radix - 1);
        unsigned peers = lane_ballot(ok);
        for (int b = 0; b < width; ++b) {
            const bool set = (dig >> b) & 1u;
            const unsigned bal = lane_ballot(set);
            peers &= set ? bal : ~bal;
        }
        const int leader = ok ? __ffs(peers) - 1 : lane;
        int32_t base = 0;
        if (ok && lane == leader) {
            base = mine[dig];
            mine[dig] = base + __popc(peers);
        }
        base = lane_get(base, leader);
        rank[r] = base + __popc(peers & ((1u << lane) - 1u));
        __syncwarp();
    }
    __syncthreads();
    // per digit: the tile's first slot of it, and how far its run lies from there in the output
    int32_t slot0 = 0, out0 = 0;
    for (int d0 = 0; d0 < radix; d0 += kGroupThreads) {
        const int d = d0 + threadIdx.x;
        int32_t here = 0, all = 0, earlier = 0;
        if (d < radix) {
#pragma unroll
            for (int w = 0; w < kGroupWarps; ++w) {
                const int32_t c = s_mine[w][d];
                s_mine[w][d] = here;
                here += c;
            }
            const int32_t *row = cnt + static_cast<int64_t>(d) * tiles;
            if (DIRECT) {
#pragma unroll 8
                for (int t = 0; t < tiles; ++t) {
                    const int32_t c = __ldg(row + t);
                    all += c;
                    earlier += t < static_cast<int>(blockIdx.x) ? c : 0;
                }
            } else {
                earlier = __ldg(row + blockIdx.x);
                all = __ldg(total + d);
            }
        }
        const int32_t slot = slot0 + scan_threads(here, s_warp);
        const int32_t out = out0 + scan_threads(all, s_warp);
        if (d < radix) {
#pragma unroll
            for (int w = 0; w < kGroupWarps; ++w) s_mine[w][d] += slot;
            s_delta[d] = out + earlier - slot;
        }
        if (d0 + kGroupThreads < radix) {         // the next 256 digits begin where these end
            __shared__ int32_t s_end[2];
            if (threadIdx.x == kGroupThreads - 1) {
                s_end[0] = slot + here;
                s_end[1] = out + all;
            }
            __syncthreads();
            slot0 = s_end[0];
            out0 = s_end[1];
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kGroupItems; ++r) {
        if (warp * 32 * kGroupItems + r * 32 + lane < count) {
            const int slot = mine[(keys[r] >> shift) & (radix - 1)] + rank[r];
            s_key[slot] = keys[r];
            s_pos[slot] = pos[r];
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kGroupItems; ++i) {
        const int slot = i * kGroupThreads + threadIdx.x;
        if (slot < count) {
            const uint32_t key = s_key[slot];
            const int32_t at = s_delta[(key >> shift) & (radix - 1)] + slot;
            key_out[at] = key;
            pos_out[at] = s_pos[slot];
        }
    }
}

// rowptr[k] = first sorted position whose key is at least k, for k in [0, rows]; the first
// CTA also writes the status.
__global__ void __launch_bounds__(kGroupThreads)
group_bounds(const uint32_t *__restrict__ keys, int64_t n, int64_t rows, int32_t *__restrict__ rowptr,
             const int32_t *__restrict__ bad_tile, int tiles, int32_t *__restrict__ status) {
    const int64_t k = static_cast<int64_t>(blockIdx.x) * kGroupThreads + threadIdx.x;
    if (k <= rows) {
        int64_t lo = 0, hi = n;
        while (lo < hi) {
            const int64_t mid = (lo + hi) >> 1;
            if (static_cast<int64_t>(__ldg(keys + mid)) < k) lo = mid + 1;
            else hi = mid;
        }
        rowptr[k] = static_cast<int32_t>(lo);
    }
    if (blockIdx.x == 0) {
        bool bad = false;
        for (int t = threadIdx.x; t < tiles; t += kGroupThreads) bad |= __ldg(bad_tile + t) != 0;
        const int any_bad = __syncthreads_or(bad);
        if (threadIdx.x == 0) *status = any_bad ? TFG_ERR_INDEX_RANGE : TFG_OK;
    }
}

}  // namespace

size_t group_ids_workspace_bytes(int64_t rows, int64_t n) {
    if (n <= 0) return 256;
    const GroupPlan p = group_plan(rows, n);
    const size_t pairs = p.passes > 1 ? 2 * round256(sizeof(int32_t) * size_t(n)) : 0;
    const size_t spare = p.passes > 2 ? pairs : 0;
    return pairs + spare + round256(sizeof(int32_t) * size_t(p.tiles) * (size_t(1) << p.width)) +
           round256(sizeof(int32_t) << p.width) + round256(sizeof(int32_t) * size_t(p.tiles));
}

namespace {
template <typename IdT>
cudaError_t group_ids_impl(const IdT *ids, int64_t n, int64_t rows, int64_t padding, int32_t *rowptr,
                           int32_t *sorted_ids, int32_t *perm, void *ws, int32_t *status, cudaStream_t s) {
    const GroupPlan p = n > 0 ? group_plan(rows, n) : GroupPlan{0, 0, 0};
    const int32_t *bad = nullptr;
    if (n > 0) {
        char *w = static_cast<char *>(ws);
        auto take = [&w](size_t bytes) {
            char *at = w;
            w += round256(bytes);
            return at;
        };
        // odd and even passes write to buffers of their own, the last one to the caller's
        uint32_t *key_buf[2] = {nullptr, nullptr};
        int32_t *pos_buf[2] = {nullptr, nullptr};
        for (int b = 0; b < 2 && b < p.passes - 1; ++b) {
            key_buf[b] = reinterpret_cast<uint32_t *>(take(sizeof(int32_t) * size_t(n)));
            pos_buf[b] = reinterpret_cast<int32_t *>(take(sizeof(int32_t) * size_t(n)));
        }
        int32_t *cnt = reinterpret_cast<int32_t *>(take(sizeof(int32_t) * size_t(p.tiles) * (size_t(1) << p.width)));
        int32_t *total = reinterpret_cast<int32_t *>(take(sizeof(int32_t) << p.width));
        int32_t *bad_tile = reinterpret_cast<int32_t *>(take(sizeof(int32_t) * size_t(p.tiles)));
        bad = bad_tile;
        const bool direct = p.tiles <= kDirectTiles;
        const int radix = 1 << p.width;
        const uint32_t *key_in = nullptr;
        const int32_t *pos_in = nullptr;
        for (int pass = 0; pass < p.passes; ++pass) {
            const int shift = pass * p.width;
            const bool first = pass == 0, last = pass == p.passes - 1;
            uint32_t *key_out = last ? reinterpret_cast<uint32_t *>(sorted_ids) : key_buf[pass & 1];
            int32_t *pos_out = last ? perm : pos_buf[pass & 1];
            if (first)
                group_upsweep<true, IdT><<<p.tiles, kGroupThreads, 0, s>>>(ids, nullptr, n, rows, padding, shift, p.width,
                                                                           p.tiles, cnt, bad_tile);
            else
                group_upsweep<false, int32_t><<<p.tiles, kGroupThreads, 0, s>>>(nullptr, key_in, n, rows, padding, shift,
                                                                                p.width, p.tiles, cnt, bad_tile);
            if (!direct) group_scan<<<ceil_div(radix, kGroupWarps), kGroupThreads, 0, s>>>(cnt, p.tiles, radix, total);
            auto down = [&](auto *kernel, const auto *id) {
                kernel<<<p.tiles, kGroupThreads, 0, s>>>(id, key_in, pos_in, n, rows, padding, shift, p.width, p.tiles, cnt,
                                                         total, key_out, pos_out);
            };
            const int32_t *none = nullptr;
            if (first && direct) down(group_downsweep<true, true, IdT>, ids);
            else if (first) down(group_downsweep<true, false, IdT>, ids);
            else if (direct) down(group_downsweep<false, true, int32_t>, none);
            else down(group_downsweep<false, false, int32_t>, none);
            const cudaError_t err = cudaGetLastError();
            if (err != cudaSuccess) return err;
            key_in = key_out;
            pos_in = pos_out;
        }
    }
    group_bounds<<<ceil_div(rows + 1, kGroupThreads), kGroupThreads, 0, s>>>(
        reinterpret_cast<const uint32_t *>(sorted_ids), n, rows, rowptr, bad, p.tiles, status);
    return cudaGetLastError();
}
}  // namespace

cudaError_t launch_group_ids(const void *ids, bool id32, int64_t n, int64_t rows, int64_t padding, int32_t *rowptr,
                             int32_t *sorted_ids, int32_t *perm, void *ws, int32_t *status, cudaStream_t s) {
    return id32 ? group_ids_impl(static_cast<const int32_t *>(ids), n, rows, padding, rowptr, sorted_ids, perm, ws, status, s)
                : group_ids_impl(static_cast<const int64_t *>(ids), n, rows, padding, rowptr, sorted_ids, perm, ws, status, s);
}

}  // namespace tfg
