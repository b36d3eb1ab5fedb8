// Grouping of ids: the positions of a list of ids ordered by id, equal ids in their
// original order -- the "reduce by key" grouping of the graph map-reduce framework
// (tf_geometric Section 2.1.2, Fig. 5b) with a table row as the key.  The gradient of an
// embedding table is the reduction over these groups (embedding.cu).
//
// A stable least-significant-digit radix sort of (key, position) pairs, digits of at most
// 9 bits, in tiles of 2,048 pairs.  Positions that take part in nothing (the padding id,
// ids outside the table) get the key `rows`, behind every row.
//   upsweep    a tile's digit counts
//   scan       exclusive sums over the tiles of each digit, and the digit's total
//              (only where there are more than kDirectTiles tiles: up to there the
//              downsweep adds the counts up itself, which saves a launch; the counts
//              lie [tile][digit] then, a thread a digit, and [digit][tile] for the scan,
//              a warp a digit)
//   downsweep  ranks a tile's pairs, stages them in shared memory in digit order and
//              writes each digit's run with coalesced stores
// A list of one tile is sorted by one CTA in shared memory, all digits in one launch.
// The row boundaries are the places where the digits begin if there is one digit, else they
// are searched in the sorted keys, a thread a row, between the places where the last digit
// begins.  The status word is written with them from one flag per tile, so nothing has to
// be cleared.  No kernel waits on another CTA.
//
// What bounds it: launches and round trips, not bytes.  112,640 ids of 119 rows (one digit,
// two launches) 10.3 us, 60,000 of 169,343 (two digits of 9 bits, five launches) 20.6 us,
// 131,072 of 50,000 (two of 8) 24 us; the pairs alone would take under 1 us.  A downsweep's
// reading of the tile counts was half of its time until all of them were in flight (the
// last, incomplete round of an unrolled loop reads one by one: 70 -> 58 us for the sampled
// batch with its lookup and gradient, together with the boundaries between the digits'
// begins in place of searches of the whole list).  Counting the next digit with atomics in
// the downsweep instead of an upsweep of its own took as long, and longer where one id is
// frequent; all digits in one launch by a cluster of eight CTAs that write the pairs into
// one another's shared memory took 46 us against 24 (the scattered remote stores).
#include "common.cuh"

namespace tfg {
namespace {

constexpr int kGroupThreads = 512;                // a thread a digit; 256 took a second round of loads for 9 bits
constexpr int kGroupWarps = kGroupThreads / 32;
constexpr int kGroupItems = 4;
constexpr int kGroupTile = kGroupThreads * kGroupItems;
constexpr int kGroupBits = 9;                     // most bits of a digit
static_assert(kGroupThreads == 1 << kGroupBits, "every digit has a thread of its own");
constexpr int kDirectTiles = 64;                  // two rounds of 32 loads; the scan's launch costs 2 us

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
              int shift, int width, int tiles, bool direct, int32_t *__restrict__ cnt, int32_t *__restrict__ bad_tile) {
    __shared__ int32_t s_cnt[1 << kGroupBits];
    const int radix = 1 << width;
    s_cnt[threadIdx.x] = 0;
    __syncthreads();
    const int64_t base = static_cast<int64_t>(blockIdx.x) * kGroupTile + threadIdx.x;
    bool bad = false;
    uint32_t key[kGroupItems];
#pragma unroll
    for (int i = 0; i < kGroupItems; ++i) {
        const int64_t at = base + i * kGroupThreads;
        key[i] = 0;
        if (at < n) key[i] = FIRST ? group_key(__ldg(ids + at), rows, padding, bad) : __ldg(keys + at);
    }
#pragma unroll
    for (int i = 0; i < kGroupItems; ++i)
        if (base + i * kGroupThreads < n) atomicAdd(&s_cnt[(key[i] >> shift) & (radix - 1)], 1);
    const int any_bad = __syncthreads_or(bad);
    if (FIRST && threadIdx.x == 0) bad_tile[blockIdx.x] = any_bad;
    if (threadIdx.x < radix)
        cnt[direct ? static_cast<int64_t>(blockIdx.x) * radix + threadIdx.x
                   : static_cast<int64_t>(threadIdx.x) * tiles + blockIdx.x] = s_cnt[threadIdx.x];
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

// A tile's pairs in registers, warp by warp and round by round in original order.
struct TilePairs {
    uint32_t key[kGroupItems];
    int32_t pos[kGroupItems], rank[kGroupItems];
    static __device__ __forceinline__ int at(int r) {
        return (threadIdx.x >> 5) * 32 * kGroupItems + r * 32 + (threadIdx.x & 31);
    }

    // rank[r]: the warp's earlier pairs of the same digit; mine[digit]: the warp's pairs of
    // it.  Lanes with equal digits are found with one ballot per bit, and the first of them
    // advances the warp's counter.
    __device__ __forceinline__ void rank_digits(int count, int shift, int width, uint16_t *mine) {
        const int lane = threadIdx.x & 31;
        for (int d = lane; d < 1 << width; d += 32) mine[d] = 0;
        __syncwarp();
#pragma unroll
        for (int r = 0; r < kGroupItems; ++r) {
            const bool ok = at(r) < count;
            const uint32_t dig = (key[r] >> shift) & ((1u << width) - 1u);
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
                mine[dig] = static_cast<uint16_t>(base + __popc(peers));
            }
            base = lane_get(base, leader);
            rank[r] = base + __popc(peers & ((1u << lane) - 1u));
            __syncwarp();
        }
    }
};

using TileCounts = uint16_t[kGroupWarps][1 << kGroupBits];      // at most 2,048: 16 bits

// The tile's pairs of digit d.
__device__ __forceinline__ int32_t tile_count(const TileCounts &mine, int d) {
    int32_t here = 0;
#pragma unroll
    for (int w = 0; w < kGroupWarps; ++w) here += mine[w][d];
    return here;
}
// Turns the warps' counts of digit d into the slots where their pairs begin.
__device__ __forceinline__ void place_warps(TileCounts &mine, int d, int32_t slot) {
#pragma unroll
    for (int w = 0; w < kGroupWarps; ++w) {
        const int32_t c = mine[w][d];
        mine[w][d] = static_cast<uint16_t>(slot);
        slot += c;
    }
}

// The status word, by one CTA.
__device__ __forceinline__ void write_status(const int32_t *bad_tile, int tiles, int32_t *status) {
    bool bad = false;
    for (int t = threadIdx.x; t < tiles; t += kGroupThreads) bad |= bad_tile[t] != 0;
    const int any_bad = __syncthreads_or(bad);
    if (threadIdx.x == 0) *status = any_bad ? TFG_ERR_INDEX_RANGE : TFG_OK;
}

// What the last pass also writes: where each value of the last digit begins, and with one
// digit alone the row boundaries and the status.
struct GroupEnds {
    int32_t *begin, *rowptr;
    const int32_t *bad_tile;
    int32_t *status;
};

template <bool FIRST, bool DIRECT, typename IdT>
__global__ void __launch_bounds__(kGroupThreads)
group_downsweep(const IdT *__restrict__ ids, const uint32_t *__restrict__ key_in, const int32_t *__restrict__ pos_in,
                int64_t n, int64_t rows, int64_t padding, int shift, int width, int tiles,
                const int32_t *__restrict__ cnt, const int32_t *__restrict__ total, uint32_t *__restrict__ key_out,
                int32_t *__restrict__ pos_out, GroupEnds ends) {
    __shared__ uint32_t s_key[kGroupTile];
    __shared__ int32_t s_pos[kGroupTile];
    __shared__ TileCounts s_mine;
    __shared__ int32_t s_delta[1 << kGroupBits];
    __shared__ int32_t s_warp[kGroupWarps];
    const int radix = 1 << width, d = threadIdx.x;
    const int warp = threadIdx.x >> 5;
    const int64_t tile0 = static_cast<int64_t>(blockIdx.x) * kGroupTile;
    const int count = static_cast<int>(min64(kGroupTile, n - tile0));
    TilePairs t;
    bool bad = false;
#pragma unroll
    for (int r = 0; r < kGroupItems; ++r) {
        const int i = t.at(r);
        t.key[r] = 0;
        t.pos[r] = 0;
        if (i < count) {
            t.key[r] = FIRST ? group_key(__ldg(ids + tile0 + i), rows, padding, bad) : __ldg(key_in + tile0 + i);
            t.pos[r] = FIRST ? static_cast<int32_t>(tile0 + i) : __ldg(pos_in + tile0 + i);
        }
    }
    // this thread's digit: its pairs in all tiles and in earlier ones
    int32_t all = 0, earlier = 0;
    if (d < radix) {
        if (DIRECT) {
            for (int i0 = 0; i0 < tiles; i0 += 32) {       // 32 in flight, the last ones too
#pragma unroll
                for (int u = 0; u < 32; ++u) {
                    const int i = i0 + u;
                    const int32_t c = i < tiles ? __ldg(cnt + i * radix + d) : 0;
                    all += c;
                    earlier += i < static_cast<int>(blockIdx.x) ? c : 0;
                }
            }
        } else {
            earlier = __ldg(cnt + static_cast<int64_t>(d) * tiles + blockIdx.x);
            all = __ldg(total + d);
        }
    }
    t.rank_digits(count, shift, width, s_mine[warp]);
    __syncthreads();
    const int32_t here = d < radix ? tile_count(s_mine, d) : 0;
    const int32_t slot0 = scan_threads(here, s_warp), out0 = scan_threads(all, s_warp);
    if (d < radix) {
        place_warps(s_mine, d, slot0);
        s_delta[d] = out0 + earlier - slot0;      // from a slot of the tile to its place in the output
    }
    if (blockIdx.x == 0) {
        if (ends.begin && d < radix) ends.begin[d] = out0;
        if (ends.begin && d == 0) ends.begin[radix] = static_cast<int32_t>(n);
        if (ends.rowptr) {                        // one digit: it is the row
            if (d <= rows) ends.rowptr[d] = out0;
            write_status(ends.bad_tile, tiles, ends.status);
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kGroupItems; ++r) {
        if (t.at(r) < count) {
            const int slot = s_mine[warp][(t.key[r] >> shift) & (radix - 1)] + t.rank[r];
            s_key[slot] = t.key[r];
            s_pos[slot] = t.pos[r];
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

// First of n sorted keys that is at least k.
__device__ __forceinline__ int first_at(const uint32_t *keys, int n, int64_t k) {
    int a = 0, b = n;
    while (a < b) {
        const int mid = (a + b) >> 1;
        if (static_cast<int64_t>(keys[mid]) < k) a = mid + 1;
        else b = mid;
    }
    return a;
}

// One tile, all digits, and the boundaries of up to kTileRows rows.  With a launch of their own
// 250 ids take 8 us whatever the rows; here 8.3 us for 3,000 rows, 9.1 for 4,000, 12.6 for 8,000.
// The launch costs the host, which bounds calls so short, 3.5 us of 24.
constexpr int64_t kTileRows = 4096;
template <typename IdT>
__global__ void __launch_bounds__(kGroupThreads)
group_tile(const IdT *__restrict__ ids, int n, int64_t rows, int64_t padding, int passes, int width,
           int32_t *__restrict__ sorted_ids, int32_t *__restrict__ perm, int32_t *__restrict__ rowptr,
           int32_t *__restrict__ status) {
    __shared__ uint32_t s_key[kGroupTile];
    __shared__ int32_t s_pos[kGroupTile];
    __shared__ TileCounts s_mine;
    __shared__ int32_t s_warp[kGroupWarps];
    const int radix = 1 << width, d = threadIdx.x;
    const int warp = threadIdx.x >> 5;
    TilePairs t;
    bool bad = false;
#pragma unroll
    for (int r = 0; r < kGroupItems; ++r) {
        const int i = t.at(r);
        t.key[r] = i < n ? group_key(__ldg(ids + i), rows, padding, bad) : 0u;
        t.pos[r] = i;
    }
    const int any_bad = __syncthreads_or(bad);
    if (threadIdx.x == 0) *status = any_bad ? TFG_ERR_INDEX_RANGE : TFG_OK;
    for (int pass = 0; pass < passes; ++pass) {
        t.rank_digits(n, pass * width, width, s_mine[warp]);
        __syncthreads();
        const int32_t slot0 = scan_threads(d < radix ? tile_count(s_mine, d) : 0, s_warp);
        if (d < radix) place_warps(s_mine, d, slot0);
        if (passes == 1 && d <= rows) rowptr[d] = slot0;        // one digit: it is the row
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kGroupItems; ++r) {
            if (t.at(r) < n) {
                const int slot = s_mine[warp][(t.key[r] >> (pass * width)) & (radix - 1)] + t.rank[r];
                s_key[slot] = t.key[r];
                s_pos[slot] = t.pos[r];
            }
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kGroupItems; ++r) {
            if (t.at(r) < n) {
                t.key[r] = s_key[t.at(r)];
                t.pos[r] = s_pos[t.at(r)];
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int r = 0; r < kGroupItems; ++r) {
        if (t.at(r) < n) {
            sorted_ids[t.at(r)] = static_cast<int32_t>(t.key[r]);
            perm[t.at(r)] = t.pos[r];
        }
    }
    if (passes > 1 && rows < kTileRows)           // s_key holds the sorted keys
        for (int64_t k = threadIdx.x; k <= rows; k += kGroupThreads) rowptr[k] = first_at(s_key, n, k);
}

// First sorted position in [lo, hi] whose key is at least k, by the whole warp (hi if there
// is none before it): 32 probes a round.
__device__ __forceinline__ int64_t warp_first_at(const uint32_t *keys, int64_t lo, int64_t hi, int64_t k) {
    const int lane = threadIdx.x & 31;
    while (lo < hi) {
        const int64_t step = (hi - lo + 31) / 32;
        const int64_t p = lo + lane * step;                     // probes in [lo, hi)
        const bool less = p < hi && static_cast<int64_t>(__ldg(keys + p)) < k;
        const int c = __popc(lane_ballot(less));                // monotone: lanes 0 .. c - 1
        if (c == 0) return lo;
        const int64_t top = lo + c * step;
        lo = lo + (c - 1) * step + 1;
        hi = top < hi ? top : hi;
    }
    return lo;
}

// rowptr[k] = first sorted position whose key is at least k, for k in [0, rows], a thread a
// row: a CTA's rows lie between the places where their last digits begin (no begin: in the
// whole list), or more than a tile apart between the ends that two warps search.  What fits
// a tile is searched in shared memory.  The first CTA also writes the status.
__global__ void __launch_bounds__(kGroupThreads)
group_bounds(const uint32_t *__restrict__ keys, int64_t n, int64_t rows, const int32_t *__restrict__ begin, int shift,
             int32_t *__restrict__ rowptr, const int32_t *__restrict__ bad_tile, int tiles, int32_t *__restrict__ status) {
    __shared__ uint32_t s_key[kGroupTile];
    __shared__ int64_t s_end[2];
    const int64_t k0 = static_cast<int64_t>(blockIdx.x) * kGroupThreads, k1 = min64(rows, k0 + kGroupThreads - 1);
    const int64_t k = k0 + threadIdx.x;
    int64_t lo = 0, hi = n;
    if (begin) {
        lo = __ldg(begin + (k0 >> shift));
        hi = __ldg(begin + (k1 >> shift) + 1);
    }
    if (hi - lo > kGroupTile) {                                 // the same in all threads
        const int end = threadIdx.x >> 5;
        if (end < 2) {
            const int64_t at = warp_first_at(keys, lo, hi, end == 0 ? k0 : k1 + 1);
            if ((threadIdx.x & 31) == 0) s_end[end] = at;
        }
        __syncthreads();
        lo = s_end[0];
        hi = s_end[1];
    }
    const int64_t from = lo;
    const int count = static_cast<int>(hi - lo < kGroupTile ? hi - lo : kGroupTile);
    if (hi - lo <= kGroupTile) {
#pragma unroll
        for (int i = 0; i < kGroupItems; ++i) {
            const int at = i * kGroupThreads + threadIdx.x;
            if (at < count) s_key[at] = __ldg(keys + from + at);
        }
        __syncthreads();
        lo = from + first_at(s_key, count, k);
    } else {
        while (lo < hi) {
            const int64_t mid = (lo + hi) >> 1;
            if (static_cast<int64_t>(__ldg(keys + mid)) < k) lo = mid + 1;
            else hi = mid;
        }
    }
    if (k <= rows) rowptr[k] = static_cast<int32_t>(lo);
    if (blockIdx.x == 0 && tiles != 1) write_status(bad_tile, tiles, status);     // one tile: written with it
}

}  // namespace

size_t group_ids_workspace_bytes(int64_t rows, int64_t n) {
    const GroupPlan p = group_plan(rows, n);
    if (p.tiles <= 1) return 0;
    const size_t flags = round256(sizeof(int32_t) * size_t(p.tiles));
    const size_t pairs = 2 * round256(sizeof(int32_t) * size_t(n));
    const size_t counters = round256(sizeof(int32_t) * size_t(p.tiles) * (size_t(1) << p.width));
    const int buffers = p.passes > 2 ? 2 : p.passes - 1;
    return flags + buffers * pairs + counters + 2 * round256((sizeof(int32_t) << p.width) + sizeof(int32_t));
}

namespace {
template <typename IdT>
cudaError_t group_ids_impl(const IdT *ids, int64_t n, int64_t rows, int64_t padding, int32_t *rowptr,
                           int32_t *sorted_ids, int32_t *perm, void *ws, int32_t *status, cudaStream_t s) {
    const GroupPlan p = n > 0 ? group_plan(rows, n) : GroupPlan{0, 0, 0};
    int32_t *bad_tile = nullptr, *begin = nullptr;
    char *w = static_cast<char *>(ws);
    auto take = [&w](size_t bytes) {
        char *at = w;
        w += round256(bytes);
        return at;
    };
    if (p.tiles == 1) {
        group_tile<<<1, kGroupThreads, 0, s>>>(ids, static_cast<int>(n), rows, padding, p.passes, p.width, sorted_ids, perm,
                                               rowptr, status);
        const cudaError_t err = cudaGetLastError();
        if (err != cudaSuccess || p.passes == 1 || rows < kTileRows) return err;
    } else if (n > 0) {
        bad_tile = reinterpret_cast<int32_t *>(take(sizeof(int32_t) * size_t(p.tiles)));
        // odd and even passes write to buffers of their own, the last one to the caller's
        uint32_t *key_buf[2] = {nullptr, nullptr};
        int32_t *pos_buf[2] = {nullptr, nullptr};
        for (int b = 0; b < 2 && b < p.passes - 1; ++b) {
            key_buf[b] = reinterpret_cast<uint32_t *>(take(sizeof(int32_t) * size_t(n)));
            pos_buf[b] = reinterpret_cast<int32_t *>(take(sizeof(int32_t) * size_t(n)));
        }
        int32_t *cnt = reinterpret_cast<int32_t *>(take(sizeof(int32_t) * size_t(p.tiles) * (size_t(1) << p.width)));
        const size_t digits = (sizeof(int32_t) << p.width) + sizeof(int32_t);
        int32_t *total = reinterpret_cast<int32_t *>(take(digits));
        begin = reinterpret_cast<int32_t *>(take(digits));
        const bool direct = p.tiles <= kDirectTiles;
        const int radix = 1 << p.width;
        const uint32_t *key_in = nullptr;
        const int32_t *pos_in = nullptr, *none = nullptr;
        for (int pass = 0; pass < p.passes; ++pass) {
            const bool first = pass == 0, last = pass == p.passes - 1;
            const int shift = pass * p.width;
            uint32_t *key_out = last ? reinterpret_cast<uint32_t *>(sorted_ids) : key_buf[pass & 1];
            int32_t *pos_out = last ? perm : pos_buf[pass & 1];
            if (first)
                group_upsweep<true><<<p.tiles, kGroupThreads, 0, s>>>(ids, key_in, n, rows, padding, shift, p.width, p.tiles, direct,
                                                                      cnt, bad_tile);
            else
                group_upsweep<false><<<p.tiles, kGroupThreads, 0, s>>>(none, key_in, n, rows, padding, shift, p.width, p.tiles,
                                                                       direct, cnt, bad_tile);
            if (!direct) group_scan<<<ceil_div(radix, kGroupWarps), kGroupThreads, 0, s>>>(cnt, p.tiles, radix, total);
            const GroupEnds ends{last && !first ? begin : nullptr, last && first ? rowptr : nullptr, bad_tile, status};
            auto down = [&](auto *kernel, const auto *id) {
                kernel<<<p.tiles, kGroupThreads, 0, s>>>(id, key_in, pos_in, n, rows, padding, shift, p.width, p.tiles, cnt,
                                                         total, key_out, pos_out, ends);
            };
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
    if (p.tiles > 1 && p.passes == 1) return cudaSuccess;      // the last pass has written them
    group_bounds<<<ceil_div(rows + 1, kGroupThreads), kGroupThreads, 0, s>>>(
        reinterpret_cast<const uint32_t *>(sorted_ids), n, rows, begin, (p.passes - 1) * p.width, rowptr, bad_tile, p.tiles, status);
    return cudaGetLastError();
}
}  // namespace

cudaError_t launch_group_ids(const void *ids, bool id32, int64_t n, int64_t rows, int64_t padding, int32_t *rowptr,
                             int32_t *sorted_ids, int32_t *perm, void *ws, int32_t *status, cudaStream_t s) {
    return id32 ? group_ids_impl(static_cast<const int32_t *>(ids), n, rows, padding, rowptr, sorted_ids, perm, ws, status, s)
                : group_ids_impl(static_cast<const int64_t *>(ids), n, rows, padding, rowptr, sorted_ids, perm, ws, status, s);
}

}  // namespace tfg
