// Rows of a table by id, and the table's gradient.
//
//   out[i] = scale * table[ids[i]], zeros where ids[i] < 0
//   d_table[v] = scale * sum over ids[i] = v of d_out[i], the terms in a fixed order
//
// Bound by memory both ways: the lookup reads the rows it needs and writes one per id; the gradient reads every row of
// d_out once and writes every row of the table's gradient once.  For the gradient the ids are sorted (stably, so that a
// run of equal ids holds its rows in ascending order), the sorted list is cut into equal parts whatever the lengths of the
// runs, and runs that a cut divides are joined afterwards.  Sums are held in fp32 and rounded once.
#include <algorithm>
#include <type_traits>

#include "rows.cuh"

namespace emc2 {
namespace {

constexpr int kLookupUnroll = 4;

__device__ __forceinline__ float4 scaled(float4 f, float s) {
    return make_float4(f.x * s, f.y * s, f.z * s, f.w * s);
}

struct LookupArgs {
    const int32_t* ids;
    const void* table;
    void* out;
    float scale;
    int rows, type;
    FastDiv row;                // division by the units of a row
    uint32_t units;             // n rows of them
    int* status;
};

// A unit of 16 bytes per thread and step (of 8 where a row of 16-bit elements is no multiple of 16), kLookupUnroll of them
// requested before the first is stored.  The result passes the L2 cache by, which the table's rows need.  Bound by memory, by
// reads of short rows in any order: 1.2 million ids of 600,000 rows of 80 bf16 channels take 62 us, 4.7 TB/s of the ids,
// rows read once and result (92 us by vectors of four values whatever their size).
template <typename Unit>
__global__ void __launch_bounds__(kLookupThreads) lookup_kernel(LookupArgs a) {
    const uint32_t t0 = blockIdx.x * (kLookupThreads * kLookupUnroll) + threadIdx.x;
    Unit f[kLookupUnroll];
    bool bad = false;
#pragma unroll
    for (int u = 0; u < kLookupUnroll; ++u) {
        const uint32_t t = t0 + u * kLookupThreads;
        f[u] = Unit{};
        if (t >= a.units) continue;
        uint32_t i, v;
        a.row.divmod(t, i, v);
        const int id = __ldg(a.ids + i);
        bad |= id >= a.rows;
        if (id >= 0 && id < a.rows) f[u] = __ldg(static_cast<const Unit*>(a.table) + (size_t)id * a.row.d + v);
    }
#pragma unroll
    for (int u = 0; u < kLookupUnroll; ++u) {
        const uint32_t t = t0 + u * kLookupThreads;
        if (t >= a.units) continue;
        uint32_t* w = reinterpret_cast<uint32_t*>(&f[u]);
#pragma unroll
        for (int k = 0; k < (int)sizeof(Unit) / 4; ++k) {
            if (a.type == EMC2_F32) {
                w[k] = __float_as_uint(__uint_as_float(w[k]) * a.scale);
            } else {
                const float4 p = as_floats(make_uint2(w[k], 0u), a.type);
                w[k] = as_halves(p.x * a.scale, p.y * a.scale, a.type);
            }
        }
        __stcs(static_cast<Unit*>(a.out) + t, f[u]);
    }
    if (bad) atomicOr(a.status, kStatusBadRows);
}

// ---------------------------------------------------------------- the ids in ascending order, each with its place
// A stable radix sort, least significant digit first, of up to ten bits per pass (two passes for a million table rows, one
// for a thousand).  The key of an id is the id, or `rows` (behind all of them) where there is none.  Bound by latency: a
// tile's items are few loads per thread and three kernels a pass wait for one another (600,000 ids, two passes: 20 us for
// the counts, 12 for their sums, 32 for the moves, of 15 MB).
constexpr int kSortThreads = 256, kSortWarps = kSortThreads / 32;
constexpr int kSortRounds = 8;                         // of 32 items per warp
static_assert(kSortItems == kSortThreads * kSortRounds, "a tile is a CTA's");

struct SortArgs {
    const int32_t* ids;         // of the first pass, else null
    const uint32_t* keys_in;
    const uint32_t* vals_in;
    uint32_t* keys_out;
    uint32_t* vals_out;
    int* counts;                // [digits][stride], one per tile; the stride a multiple of 4
    int* totals;                // [digits]
    int* status;
    int n, rows, tiles, stride, shift, digits;
};

__device__ __forceinline__ uint32_t sort_key(const SortArgs& a, int i) {
    if (!a.ids) return a.keys_in[i];
    const int id = a.ids[i];
    return id >= 0 && id < a.rows ? (uint32_t)id : (uint32_t)a.rows;
}

// counts[d][tile]: items of the tile with digit d.
__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(SortArgs a) {
    await_predecessor();
    __shared__ int hist[kMaxDigits];
    for (int d = threadIdx.x; d < a.digits; d += kSortThreads) hist[d] = 0;
    __syncthreads();
    bool bad = false;
#pragma unroll
    for (int k = 0; k < kSortRounds; ++k) {
        const int i = blockIdx.x * kSortItems + k * kSortThreads + threadIdx.x;
        if (i >= a.n) continue;
        const uint32_t key = sort_key(a, i);
        bad |= a.ids && a.ids[i] >= a.rows;
        atomicAdd(&hist[key >> a.shift & (a.digits - 1)], 1);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < a.digits; d += kSortThreads) a.counts[(size_t)d * a.stride + blockIdx.x] = hist[d];
    if (bad) atomicOr(a.status, kStatusBadRows);
    release_successor();
}

// Exclusive prefix sums over every row of counts, a warp per digit and 128 tiles at a time, and the digits' totals.
__global__ void __launch_bounds__(kSortThreads) sort_scan_kernel(SortArgs a) {
    await_predecessor();
    const int d = blockIdx.x * kSortWarps + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (d >= a.digits) return;
    int4* row = reinterpret_cast<int4*>(a.counts + (size_t)d * a.stride);
    int run = 0;
    for (int t0 = 0; t0 < a.stride / 4; t0 += 32) {
        const int t = t0 + lane;
        int4 v = t < a.stride / 4 ? row[t] : make_int4(0, 0, 0, 0);
        if (4 * t + 3 >= a.tiles) {                                        // behind the last tile
            if (4 * t >= a.tiles) v.x = 0;
            if (4 * t + 1 >= a.tiles) v.y = 0;
            if (4 * t + 2 >= a.tiles) v.z = 0;
            v.w = 0;
        }
        const int sum = v.x + v.y + v.z + v.w;
        int inc = sum;
#pragma unroll
        for (int k = 1; k < 32; k <<= 1) {
            const int y = __shfl_up_sync(0xFFFFFFFFu, inc, k);
            if (lane >= k) inc += y;
        }
        const int x = run + inc - sum;
        if (t < a.stride / 4) row[t] = make_int4(x, x + v.x, x + v.x + v.y, x + v.x + v.y + v.z);
        run += __shfl_sync(0xFFFFFFFFu, inc, 31);
    }
    if (lane == 0) a.totals[d] = run;
    release_successor();
}

// Exclusive prefix sum of v[0 .. n) in shared memory, n <= kMaxDigits, by the whole CTA.
__device__ __forceinline__ void scan_digits(int* v, int n, int* warp_sums) {
    constexpr int kPer = kMaxDigits / kSortThreads;
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    int x[kPer], sum = 0;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        x[k] = t * kPer + k < n ? v[t * kPer + k] : 0;
        sum += x[k];
    }
    int inc = sum;
#pragma unroll
    for (int k = 1; k < 32; k <<= 1) {
        const int y = __shfl_up_sync(0xFFFFFFFFu, inc, k);
        if (lane >= k) inc += y;
    }
    if (lane == 31) warp_sums[warp] = inc;
    __syncthreads();
    int run = inc - sum;
    for (int w = 0; w < warp; ++w) run += warp_sums[w];
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        if (t * kPer + k < n) v[t * kPer + k] = run;
        run += x[k];
    }
    __syncthreads();
}

// Moves a tile's items to their places.  A warp takes 256 consecutive items in rounds of 32, so that "earlier in the list" is
// "earlier round, or lower lane": the rank among the warp's items of a digit is a running count plus a match over the lanes.
// The tile is put in order in shared memory first and leaves in runs.
__global__ void __launch_bounds__(kSortThreads, 4) sort_move_kernel(SortArgs a) {
    await_predecessor();
    __shared__ uint16_t wcnt[kSortWarps][kMaxDigits];  // items of a digit by warp, then those of the warps before
    __shared__ int first[kMaxDigits];                  // place of a digit's first item in the tile ...
    __shared__ int to[kMaxDigits];                     // ... and of it in the whole list, less that
    __shared__ int warp_sums[kSortWarps];
    __shared__ uint32_t keys[kSortItems], vals[kSortItems];
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5, tile0 = blockIdx.x * kSortItems;
    const uint32_t mask = a.digits - 1;
    // Requested before anything waits: the items, and the places of their digits (a column of `counts`).
    uint32_t key[kSortRounds], val[kSortRounds];
    uint16_t rank[kSortRounds];
#pragma unroll
    for (int k = 0; k < kSortRounds; ++k) {
        const int i = tile0 + warp * (32 * kSortRounds) + k * 32 + lane;
        key[k] = i < a.n ? sort_key(a, i) : 0xFFFFFFFFu;
        val[k] = a.ids || i >= a.n ? (uint32_t)i : a.vals_in[i];
    }
    int* place = reinterpret_cast<int*>(keys);          // until the keys come there
    for (int d = t; d < a.digits; d += kSortThreads) place[d] = a.counts[(size_t)d * a.stride + blockIdx.x];
    for (int d = t; d < a.digits; d += kSortThreads) {
#pragma unroll
        for (int w = 0; w < kSortWarps; ++w) wcnt[w][d] = 0;
        to[d] = a.totals[d];
    }
    __syncthreads();
    scan_digits(to, a.digits, warp_sums);              // items of smaller digits in the whole list
#pragma unroll
    for (int k = 0; k < kSortRounds; ++k) {
        const bool in = tile0 + warp * (32 * kSortRounds) + k * 32 + lane < a.n;
        const uint32_t d = key[k] >> a.shift & mask;
        const unsigned peers = __match_any_sync(0xFFFFFFFFu, in ? d : 0xFFFFFFFFu);
        const int before = in ? wcnt[warp][d] : 0;
        rank[k] = (uint16_t)(before + __popc(peers & ((1u << lane) - 1u)));
        __syncwarp();
        if (in && (peers & ((1u << lane) - 1u)) == 0) wcnt[warp][d] = (uint16_t)(before + __popc(peers));
        __syncwarp();
    }
    __syncthreads();
    for (int d = t; d < a.digits; d += kSortThreads) {
        int run = 0;
#pragma unroll
        for (int w = 0; w < kSortWarps; ++w) {
            const int c = wcnt[w][d];
            wcnt[w][d] = (uint16_t)run;
            run += c;
        }
        first[d] = run;
    }
    __syncthreads();
    scan_digits(first, a.digits, warp_sums);
    for (int d = t; d < a.digits; d += kSortThreads) to[d] += place[d] - first[d];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kSortRounds; ++k) {
        const int i = tile0 + warp * (32 * kSortRounds) + k * 32 + lane;
        if (i >= a.n) continue;
        const uint32_t d = key[k] >> a.shift & mask;
        const int at = first[d] + wcnt[warp][d] + rank[k];
        keys[at] = key[k];
        vals[at] = val[k];
    }
    __syncthreads();
    const int here = min(kSortItems, a.n - tile0);
    for (int i = t; i < here; i += kSortThreads) {
        const uint32_t k = keys[i];
        const int place = to[k >> a.shift & mask] + i;
        a.keys_out[place] = k;
        a.vals_out[place] = vals[i];
    }
    release_successor();
}

// First place in [lo, hi) of the ascending keys whose key is at least k; hi if there is none.
__device__ __forceinline__ int lower_place(const uint32_t* keys, int lo, int hi, uint32_t k) {
    while (lo < hi) {
        const int mid = lo + (hi - lo) / 2;
        if (keys[mid] < k) lo = mid + 1; else hi = mid;
    }
    return lo;
}
// The same by a warp, which probes 32 places at a time: four rounds for a million keys instead of twenty.
__device__ __forceinline__ int lower_place_warp(const uint32_t* keys, int lo, int hi, uint32_t k) {
    const int lane = threadIdx.x & 31;
    while (hi - lo > 32) {
        const long long span = hi - lo;
        const int at = lo + (int)(span * (lane + 1) / 33);
        const int less = __popc(__ballot_sync(0xFFFFFFFFu, keys[at] < k));     // the first `less` probes are
        const int from = lo;
        if (less > 0) lo = from + (int)(span * less / 33) + 1;
        if (less < 32) hi = from + (int)(span * (less + 1) / 33);
    }
    const int at = lo + lane;
    return lo + __popc(__ballot_sync(0xFFFFFFFFu, at < hi && keys[at] < k));
}

// Zeros in the table rows that no id names: 256 rows per CTA, looked up in the part of the sorted ids that theirs lie in.
// Clearing the whole table first would write the rows with ids twice.
__device__ __forceinline__ void zero_rows(const uint32_t* keys, int n, int rows, int nvec, uint32_t block, void* out, int type) {
    __shared__ int ends[2];
    __shared__ bool named[kLookupThreads];
    const uint32_t r0 = block * kLookupThreads;
    const int here = (int)min((uint32_t)kLookupThreads, (uint32_t)rows - r0), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    named[threadIdx.x] = false;
    if (warp < 2) {
        const int at = lower_place_warp(keys, 0, n, warp ? r0 + here : r0);
        if (lane == 0) ends[warp] = at;
    }
    __syncthreads();
    const int lo = ends[0], hi = ends[1];
    if (hi - lo <= 16 * kLookupThreads) {
        for (int i = lo + threadIdx.x; i < hi; i += kLookupThreads) named[keys[i] - r0] = true;
    } else {                                                              // long runs of few ids
        const int at = lower_place(keys, lo, hi, r0 + threadIdx.x);
        named[threadIdx.x] = at < hi && keys[at] == r0 + threadIdx.x;
    }
    __syncthreads();
    for (int k = warp; k < here; k += kLookupThreads / 32)
        if (!named[k])
            for (int v = lane; v < nvec; v += 32) store_row4(out, (size_t)(r0 + k) * nvec + v, make_float4(0.f, 0.f, 0.f, 0.f), type);
}

struct SumArgs {
    const uint32_t* keys;
    const uint32_t* vals;
    const void* dout;
    void* dtable;
    float scale;
    int n, rows, nvec, log, type, items;
    int parts;                  // CTAs that sum; those behind them clear the rows without ids beside them
    RunEnds* ends;              // [parts]
    float4* partial;            // [CTAs][2][nvec]: sums of head and tail
};

// A group of lanes adds up `items` places of the sorted list; the CTA then joins its groups in order.  The rows of
// several places are requested before the first is added.  Bound by the latency of rows in any order at the warps that the
// requested rows leave room for: 1.2 million rows of 80 fp32 channels into 600,000, 145 us, 4.0 TB/s; 960,000 rows of 64 bf16
// channels into 16, 44 us, 2.8 TB/s.
template <int K, bool kHalf>
__global__ void __launch_bounds__(kLookupThreads, K == 1 ? 4 : K <= 3 ? 3 : 2) lookup_sum_kernel(SumArgs a) {
    await_predecessor();
    using Raw = std::conditional_t<kHalf, uint2, float4>;

    if ((int)blockIdx.x >= a.parts) {
        zero_rows(a.keys, a.n, a.rows, a.nvec, blockIdx.x - a.parts, a.dtable, a.type);
        return;
    }
    extern __shared__ float4 part[];            // [groups][2][nvec], behind it the CTA's keys (one more at each end) and places
    __shared__ RunEnds ends[kLookupThreads];
    const int lanes = 1 << a.log, lane = threadIdx.x & (lanes - 1), group = threadIdx.x >> a.log, groups = kLookupThreads >> a.log;
    const uint32_t none = (uint32_t)a.rows;
    uint32_t* keys = reinterpret_cast<uint32_t*>(part + groups * 2 * a.nvec) + 1;
    uint32_t* vals = keys + groups * kRunItems + 1;
    RunEnds mine = {-1, 0, -1, 0};
    constexpr int U = (kHalf ? 2 : 1) * (K <= 2 ? 4 : K == 3 ? 2 : 1);
    float4 acc[K];
#pragma unroll
    for (int i = 0; i < K; ++i) acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](const Raw (&x)[K]) {
#pragma unroll
        for (int i = 0; i < K; ++i) {
            float4 f;
            if constexpr (kHalf) f = as_floats(x[i], a.type); else f = x[i];
            acc[i].x += f.x; acc[i].y += f.y; acc[i].z += f.z; acc[i].w += f.w;
        }
    };
    bool begun = false;                                               // the open run begins in this group's places
    // Pieces of kRunItems places per group; only very long lists have more than one.
    const long long cta0 = (long long)blockIdx.x * groups * a.items;
    for (int piece = 0; piece < a.items; piece += kRunItems) {
        __syncthreads();
        for (int i = (int)threadIdx.x - 1; i <= groups * kRunItems; i += kLookupThreads) {
            // Place i of the staged ones belongs to group i / kRunItems; -1 and the one behind the last are neighbours.
            const int g = i < 0 ? 0 : min(i / kRunItems, groups - 1), k = i - g * kRunItems;
            const long long p = cta0 + (long long)g * a.items + piece + k;
            keys[i] = p >= 0 && p < a.n ? a.keys[p] : p < 0 ? 0xFFFFFFFFu : none;
            if (i >= 0 && i < groups * kRunItems) vals[i] = p < a.n ? a.vals[p] : 0u;
        }
        __syncthreads();
        const long long p0 = cta0 + (long long)group * a.items + piece;
        const int here = (int)max(0LL, min((long long)min(kRunItems, a.items - piece), (long long)a.n - p0)), at = group * kRunItems;
        if (here > 0) {
            // With several pieces a group's neighbours are not its neighbours in the staged list.
            const uint32_t before = a.items == kRunItems ? keys[at - 1] : p0 > 0 ? a.keys[p0 - 1] : 0xFFFFFFFFu;
            const uint32_t behind = a.items == kRunItems ? keys[at + here] : p0 + here < a.n ? a.keys[p0 + here] : none;
            if (before != keys[at]) begun = true;
            else if (piece == 0) begun = false;
            for (int k = 0; k < here; k += U) {
                if (keys[at + k] == none) break;
                Raw x[U][K];
                int rows = 1;
#pragma unroll
                for (int q = 0; q < U; ++q) {
                    const bool in = k + q < here && keys[at + k + q] != none;
                    rows = in ? q + 1 : rows;
                    const Raw* from = static_cast<const Raw*>(a.dout) + (size_t)(in ? vals[at + k + q] : 0u) * a.nvec;
#pragma unroll
                    for (int i = 0; i < K; ++i) {
                        const int v = lane + (i << a.log);
                        x[q][i] = in && v < a.nvec ? __ldg(from + v) : Raw{};
                    }
                }
#pragma unroll
                for (int q = 0; q < U; ++q) {
                    if (q >= rows) break;
                    const uint32_t key = keys[at + k + q], next = k + q + 1 < here ? keys[at + k + q + 1] : behind;
                    add(x[q]);
                    const bool over = next != key, last = piece + k + q + 1 >= a.items || p0 + k + q + 1 >= a.n;
                    if (!over && !last) continue;
#pragma unroll
                    for (int i = 0; i < K; ++i) {
                        const int v = lane + (i << a.log);
                        if (v < a.nvec) {
                            if (begun && over) store_row4(a.dtable, (size_t)key * a.nvec + v, scaled(acc[i], a.scale), a.type);
                            else part[(group * 2 + (begun ? 1 : 0)) * a.nvec + v] = acc[i];
                        }
                        acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                    }
                    if (!begun) { mine.head = (int)key; mine.through = !over; }
                    else if (!over) mine.tail = (int)key;
                    begun = true;
                }
            }
        }
    }
    if (lane == 0) ends[group] = mine;
    __syncthreads();
    for (int v = threadIdx.x; v < a.nvec; v += kLookupThreads) {
        float4 run = make_float4(0.f, 0.f, 0.f, 0.f);
        bool in_cta = false;                                          // the open run begins in this CTA
        RunEnds all = {-1, 0, -1, 0};
        float4* partial = a.partial + (size_t)blockIdx.x * 2 * a.nvec + v;
        for (int g = 0; g < groups; ++g) {
            const RunEnds r = ends[g];
            if (r.head >= 0) {
                const float4 x = part[g * 2 * a.nvec + v];
                run.x += x.x; run.y += x.y; run.z += x.z; run.w += x.w;
                if (!in_cta) { all.head = r.head; all.through = r.through; }
                if (!r.through) {
                    if (in_cta) store_row4(a.dtable, (size_t)r.head * a.nvec + v, scaled(run, a.scale), a.type);
                    else partial[0] = run;
                    run = make_float4(0.f, 0.f, 0.f, 0.f);
                    in_cta = false;
                    all.tail = -1;
                }
            }
            if (r.tail >= 0) {
                run = part[(g * 2 + 1) * a.nvec + v];
                in_cta = true;
                all.tail = r.tail;
            }
        }
        if (all.tail >= 0) partial[a.nvec] = run;
        else if (all.through) partial[0] = run;
        if (v == 0) a.ends[blockIdx.x] = all;
    }
    release_successor();
}

// The runs that the CTAs' parts divide: CTA i joins the one that begins in part i, its warps every eighth part of it.  All
// latency, 4 to 8 us.
__global__ void __launch_bounds__(kLookupThreads) lookup_join_kernel(SumArgs a, int parts) {
    await_predecessor();
    constexpr int kWarps = kLookupThreads / 32;
    extern __shared__ float4 part[];            // [warps][nvec]
    const int i = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int id = a.ends[i].tail;
    if (id < 0) return;
    // Parts i + 1 .. last hold the rest of the run: it ends in the first whose head does not go through.
    int last = parts - 1;
    for (int j0 = i + 1; j0 < parts; j0 += 32) {
        const int j = j0 + lane;
        const unsigned stop = __ballot_sync(0xFFFFFFFFu, j < parts && !a.ends[j].through);
        if (stop) { last = j0 + __ffs(stop) - 1; break; }
    }
    for (int v0 = 0; v0 < a.nvec; v0 += 32) {
        const int v = v0 + lane;
        if (v >= a.nvec) continue;
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        if (warp == 0) s = a.partial[((size_t)i * 2 + 1) * a.nvec + v];
        for (int j = i + 1 + warp; j <= last; j += kWarps) {
            if (a.ends[j].head != id) continue;
            const float4 x = a.partial[(size_t)j * 2 * a.nvec + v];
            s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
        }
        part[warp * a.nvec + v] = s;
    }
    __syncthreads();
    for (int v = threadIdx.x; v < a.nvec; v += kLookupThreads) {
        float4 s = part[v];
        for (int w = 1; w < kWarps; ++w) {
            const float4 x = part[w * a.nvec + v];
            s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
        }
        store_row4(a.dtable, (size_t)id * a.nvec + v, scaled(s, a.scale), a.type);
    }
    release_successor();
}

template <int K, bool kHalf>
cudaError_t launch_sum_of(const SumArgs& a, int ctas, size_t shared, cudaStream_t st) {
    // Sums of a CTA's groups, two of up to K vectors per thread, and the keys and places of up to a group per thread.
    constexpr size_t most = (size_t)kLookupThreads * (2 * K * sizeof(float4) + kRunItems * 2 * sizeof(uint32_t)) + 4 * sizeof(uint32_t);
    if (shared > 40 * 1024) {
        const cudaError_t e = allow_shared(lookup_sum_kernel<K, kHalf>, most);
        if (e != cudaSuccess) return e;
    }
    launch_chained(lookup_sum_kernel<K, kHalf>, dim3(ctas), kLookupThreads, shared, st, a);
    return cudaSuccess;
}
template <int K>
cudaError_t launch_sum(const SumArgs& a, int ctas, size_t shared, cudaStream_t st) {
    return a.type == EMC2_F32 ? launch_sum_of<K, false>(a, ctas, shared, st) : launch_sum_of<K, true>(a, ctas, shared, st);
}

int check_lookup(const emc2_bridge* h, int n, int rows, int channels, int type, const void* ids) {
    if (!h || n < 0 || rows < 0 || (int64_t)n > (int64_t)h->cfg.max_batch * h->cfg.max_points) return EMC2_ERR_INVALID_ARG;
    if (channels < 4 || channels > kMaxRowChannels || (channels & 3) || !is_type(type)) return EMC2_ERR_INVALID_ARG;
    // Vectors of the rows are counted in 32 bits.
    if ((uint64_t)std::max(n, rows) * (uint64_t)(channels / 4) > 0xFFFF0000ull) return EMC2_ERR_INVALID_ARG;
    if (n > 0 && !ids) return EMC2_ERR_INVALID_ARG;
    if (!on_4_bytes(ids)) return EMC2_ERR_INVALID_ARG;
    return EMC2_OK;
}

}  // namespace

size_t lookup_scratch_bytes(const emc2_bridge* h, int max_channels) {
    return lookup_scratch_most(h->num_sms, (long long)h->cfg.max_batch * h->cfg.max_points, max_channels);
}

}  // namespace emc2

using namespace emc2;

extern "C" int emc2_row_lookup(emc2_bridge_t* h, int32_t n, int32_t rows, int32_t channels, int32_t type, const int32_t* d_ids,
                               const void* d_table, float scale, void* d_out, void* cuda_stream) {
    const int rc = check_lookup(h, n, rows, channels, type, d_ids);
    if (rc != EMC2_OK) return rc;
    if (!on_16_bytes(d_table) || !on_16_bytes(d_out)) return EMC2_ERR_INVALID_ARG;
    if (n == 0) return EMC2_OK;
    if (!d_out || (rows > 0 && !d_table) || d_out == d_table) return EMC2_ERR_INVALID_ARG;
    RowsDevice device(h->cfg.device);
    if (!device.ok) return EMC2_ERR_CUDA;
    const int row_bytes = channels * type_bytes(type), unit = row_bytes % 16 == 0 ? 16 : 8;
    LookupArgs a;
    a.ids = d_ids; a.table = d_table; a.out = d_out; a.scale = scale; a.rows = rows; a.type = type;
    a.row = make_fast_div((uint32_t)(row_bytes / unit));
    a.units = (uint32_t)n * (uint32_t)(row_bytes / unit);
    a.status = h->d_status;
    const uint32_t per_cta = kLookupThreads * kLookupUnroll, ctas = (a.units + per_cta - 1) / per_cta;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    LaunchScope ls(h, K_ROW_LOOKUP, st);
    if (unit == 16) lookup_kernel<uint4><<<ctas, kLookupThreads, 0, st>>>(a);
    else lookup_kernel<uint2><<<ctas, kLookupThreads, 0, st>>>(a);
    return check_cuda(h, cudaGetLastError());
}

extern "C" int emc2_row_lookup_grad(emc2_bridge_t* h, int32_t n, int32_t rows, int32_t channels, int32_t type, const int32_t* d_ids,
                                    const void* d_grad_out, float scale, void* d_grad_table, void* cuda_stream) {
    const int rc = check_lookup(h, n, rows, channels, type, d_ids);
    if (rc != EMC2_OK) return rc;
    if (!on_16_bytes(d_grad_out) || !on_16_bytes(d_grad_table)) return EMC2_ERR_INVALID_ARG;
    if (rows > 0 && !d_grad_table) return EMC2_ERR_INVALID_ARG;
    if (n > 0 && (!d_grad_out || d_grad_out == d_grad_table)) return EMC2_ERR_INVALID_ARG;
    if (!h->rows_scratch.slab || channels > h->rows_scratch.max_channels) return EMC2_ERR_TOO_LARGE;
    RowsDevice device(h->cfg.device);
    if (!device.ok) return EMC2_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (n == 0) {
        if (rows == 0) return EMC2_OK;
        return check_cuda(h, cudaMemsetAsync(d_grad_table, 0, (size_t)rows * channels * type_bytes(type), st));
    }
    SumArgs a;
    a.nvec = channels / 4;
    const RowSplit split = row_split(a.nvec, 3);
    const LookupParts parts = lookup_parts(h->num_sms, n, a.nvec);
    const int groups = parts.groups, ctas = parts.ctas;
    a.items = parts.items;
    const LookupScratch s = lookup_scratch(n, ctas, a.nvec);
    if (s.bytes > h->rows_scratch.bytes) return EMC2_ERR_TOO_LARGE;
    char* base = static_cast<char*>(h->rows_scratch.slab);
    uint32_t* keys[2] = {reinterpret_cast<uint32_t*>(base + s.keys[0]), reinterpret_cast<uint32_t*>(base + s.keys[1])};
    uint32_t* vals[2] = {reinterpret_cast<uint32_t*>(base + s.vals[0]), reinterpret_cast<uint32_t*>(base + s.vals[1])};
    int bits = 1;
    while (bits < 32 && ((uint64_t)1 << bits) < (uint64_t)rows + 1) ++bits;         // the keys are 0 .. rows
    const int passes = (bits + 9) / 10, digit = (bits + passes - 1) / passes;
    int at = 1;
    for (int p = 0; p < passes; ++p, at ^= 1) {
        SortArgs o;
        o.ids = p == 0 ? d_ids : nullptr;
        o.keys_in = keys[at]; o.vals_in = vals[at]; o.keys_out = keys[at ^ 1]; o.vals_out = vals[at ^ 1];
        o.counts = reinterpret_cast<int*>(base + s.counts); o.totals = reinterpret_cast<int*>(base + s.row_tot); o.status = h->d_status;
        o.n = n; o.rows = rows; o.tiles = (n + kSortItems - 1) / kSortItems; o.stride = (o.tiles + 3) / 4 * 4; o.shift = p * digit; o.digits = 1 << digit;
        LaunchScope ls(h, K_LOOKUP_SORT, st);
        launch_kernel(p > 0, sort_count_kernel, dim3(o.tiles), kSortThreads, 0, st, o);
        launch_chained(sort_scan_kernel, dim3((o.digits + kSortWarps - 1) / kSortWarps), kSortThreads, 0, st, o);
        launch_chained(sort_move_kernel, dim3(o.tiles), kSortThreads, 0, st, o);
    }
    a.keys = keys[at]; a.vals = vals[at]; a.dout = d_grad_out; a.dtable = d_grad_table; a.scale = scale; a.n = n; a.rows = rows;
    a.log = split.log; a.type = type;
    a.ends = reinterpret_cast<RunEnds*>(base + s.ends);
    a.partial = reinterpret_cast<float4*>(base + s.partial);
    a.parts = ctas;
    const int grid = ctas + (int)(((long long)rows + kLookupThreads - 1) / kLookupThreads);
    {
        const size_t shared = (size_t)groups * 2 * a.nvec * sizeof(float4) + ((size_t)groups * kRunItems * 2 + 4) * sizeof(uint32_t);
        LaunchScope ls(h, K_LOOKUP_SUM, st);
        cudaError_t e;
        switch (split.per) {
            case 1: e = launch_sum<1>(a, grid, shared, st); break;
            case 2: e = launch_sum<2>(a, grid, shared, st); break;
            case 3: e = launch_sum<3>(a, grid, shared, st); break;
            case 4: e = launch_sum<4>(a, grid, shared, st); break;
            case 5: e = launch_sum<5>(a, grid, shared, st); break;
            case 6: e = launch_sum<6>(a, grid, shared, st); break;
            case 7: e = launch_sum<7>(a, grid, shared, st); break;
            default: e = launch_sum<8>(a, grid, shared, st); break;
        }
        if (e != cudaSuccess) return check_cuda(h, e);
    }
    {
        LaunchScope ls(h, K_LOOKUP_JOIN, st);
        launch_chained(lookup_join_kernel, dim3(ctas), kLookupThreads, (size_t)(kLookupThreads / 32) * a.nvec * sizeof(float4), st, a, ctas);
    }
    return check_cuda(h, cudaGetLastError());
}
