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

#include "rows.cuh"

namespace emc2 {
namespace {

constexpr int kLookupThreads = 256;
constexpr int kLookupUnroll = 4;
constexpr int kRunItems = 16;                 // sorted places per group of lanes, at least
constexpr int kMaxSumCtas = 16384;

__device__ __forceinline__ float4 scaled(float4 f, float s) {
    return make_float4(f.x * s, f.y * s, f.z * s, f.w * s);
}

struct LookupArgs {
    const int32_t* ids;
    const void* table;
    void* out;
    float scale;
    int n, rows, nvec, type;
    FastDiv row;                // division by nvec
    uint32_t vectors;           // n * nvec
    int* status;
};

// A vector of four elements per thread and step, kLookupUnroll of them requested before the first is stored.
__global__ void __launch_bounds__(kLookupThreads) lookup_kernel(LookupArgs a) {
    const uint32_t t0 = blockIdx.x * (kLookupThreads * kLookupUnroll) + threadIdx.x;
    float4 f[kLookupUnroll];
    bool bad = false;
#pragma unroll
    for (int u = 0; u < kLookupUnroll; ++u) {
        const uint32_t t = t0 + u * kLookupThreads;
        f[u] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (t >= a.vectors) continue;
        uint32_t i, v;
        a.row.divmod(t, i, v);
        const int id = __ldg(a.ids + i);
        bad |= id >= a.rows;
        if (id >= 0 && id < a.rows) f[u] = load_row4(a.table, (size_t)id * a.nvec + v, a.type);
    }
#pragma unroll
    for (int u = 0; u < kLookupUnroll; ++u) {
        const uint32_t t = t0 + u * kLookupThreads;
        if (t < a.vectors) store_row4(a.out, t, scaled(f[u], a.scale), a.type);
    }
    if (bad) atomicOr(a.status, kStatusBadRows);
}

// Keys of the sort: the id, or `rows` (sorted behind all of them) where there is none.
__global__ void __launch_bounds__(kLookupThreads)
lookup_keys_kernel(const int32_t* ids, int n, int rows, uint32_t* keys, uint32_t* vals, int* status) {
    const int i = blockIdx.x * kLookupThreads + threadIdx.x;
    if (i >= n) return;
    const int id = ids[i];
    if (id >= rows) atomicOr(status, kStatusBadRows);
    keys[i] = id >= 0 && id < rows ? (uint32_t)id : (uint32_t)rows;
    vals[i] = (uint32_t)i;
}

// First place in [lo, hi) of the ascending keys whose key is at least k; hi if there is none.
__device__ __forceinline__ int lower_place(const uint32_t* keys, int lo, int hi, uint32_t k) {
    while (lo < hi) {
        const int mid = lo + (hi - lo) / 2;
        if (keys[mid] < k) lo = mid + 1; else hi = mid;
    }
    return lo;
}

// Zeros in the table rows that no id names: 256 rows per CTA, looked up in the part of the sorted ids that theirs lie in.
// Clearing the whole table first would write the rows with ids twice.
__global__ void __launch_bounds__(kLookupThreads) lookup_zero_kernel(const uint32_t* keys, int n, int rows, int nvec, FastDiv row, void* out, int type) {
    __shared__ int ends[2];
    __shared__ bool named[kLookupThreads];
    const uint32_t r0 = blockIdx.x * kLookupThreads;
    const int here = (int)min((uint32_t)kLookupThreads, (uint32_t)rows - r0);
    if ((threadIdx.x & 31) == 0 && threadIdx.x < 64) ends[threadIdx.x >> 5] = lower_place(keys, 0, n, threadIdx.x ? r0 + here : r0);
    __syncthreads();
    const uint32_t r = r0 + threadIdx.x;
    const int at = lower_place(keys, ends[0], ends[1], r);
    named[threadIdx.x] = at < ends[1] && keys[at] == r;
    __syncthreads();
    for (int t = threadIdx.x; t < here * nvec; t += kLookupThreads) {
        uint32_t k, v;
        row.divmod((uint32_t)t, k, v);
        if (!named[k]) store_row4(out, (size_t)r0 * nvec + t, make_float4(0.f, 0.f, 0.f, 0.f), type);
    }
}

// What a part of the sorted list leaves of the runs that its ends divide.
struct RunEnds {
    int head;                   // id of a run that begins before the part, or -1
    int through;                // that run also goes on behind the part
    int tail;                   // id of a run that begins in the part and goes on behind it, or -1
    int pad;
};

struct SumArgs {
    const uint32_t* keys;
    const uint32_t* vals;
    const void* dout;
    void* dtable;
    float scale;
    int n, rows, nvec, log, type, items;
    RunEnds* ends;              // [CTAs]
    float4* partial;            // [CTAs][2][nvec]: sums of head and tail
};

// A group of lanes adds up `items` places of the sorted list; the CTA then joins its groups in order.
template <int K>
__global__ void __launch_bounds__(kLookupThreads) lookup_sum_kernel(SumArgs a) {
    extern __shared__ float4 part[];            // [groups][2][nvec]
    __shared__ RunEnds ends[kLookupThreads];
    const int lanes = 1 << a.log, lane = threadIdx.x & (lanes - 1), group = threadIdx.x >> a.log, groups = kLookupThreads >> a.log;
    const uint32_t none = (uint32_t)a.rows;
    const long long p0 = ((long long)blockIdx.x * groups + group) * a.items;
    const int from = (int)min(p0, (long long)a.n), to = (int)min(p0 + a.items, (long long)a.n);
    RunEnds mine = {-1, 0, -1, 0};
    float4 acc[K];
#pragma unroll
    for (int i = 0; i < K; ++i) acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (from < to) {
        uint32_t key = a.keys[from];
        bool begun = from == 0 || a.keys[from - 1] != key;            // the run begins here
        for (int p = from; p < to && key != none; ++p) {
            const uint32_t next = p + 1 < a.n ? a.keys[p + 1] : none;
            const size_t row = a.vals[p];
            float4 x[K];
            load_row<K>(x, a.dout, row * a.nvec, lane, a.log, a.nvec, a.type);
#pragma unroll
            for (int i = 0; i < K; ++i) { acc[i].x += x[i].x; acc[i].y += x[i].y; acc[i].z += x[i].z; acc[i].w += x[i].w; }
            const bool over = next != key;
            if (!over && p + 1 < to) continue;
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
            key = next;
            begun = true;
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
}

// The runs that the CTAs' parts divide: CTA i joins the one that begins in part i, its warps every eighth part of it.
__global__ void __launch_bounds__(kLookupThreads) lookup_join_kernel(SumArgs a, int parts) {
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
}

template <int K>
void launch_sum(const SumArgs& a, int ctas, size_t shared, cudaStream_t st) {
    if (shared > 40 * 1024) cudaFuncSetAttribute(lookup_sum_kernel<K>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)shared);
    lookup_sum_kernel<K><<<ctas, kLookupThreads, shared, st>>>(a);
}

int check_lookup(const emc2_bridge* h, int n, int rows, int channels, int type, const void* ids) {
    if (!h || n < 0 || rows < 0 || (int64_t)n > (int64_t)h->cfg.max_batch * h->cfg.max_points) return EMC2_ERR_INVALID_ARG;
    if (channels < 4 || channels > kMaxRowChannels || (channels & 3) || !is_type(type)) return EMC2_ERR_INVALID_ARG;
    // Vectors of the rows are counted in 32 bits.
    if ((uint64_t)std::max(n, rows) * (uint64_t)(channels / 4) > 0xFFFF0000ull) return EMC2_ERR_INVALID_ARG;
    if (n > 0 && !ids) return EMC2_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(ids) & 3) return EMC2_ERR_INVALID_ARG;
    return EMC2_OK;
}

// Places per group and CTAs of lookup_sum_kernel.
int sum_items(long long n, int groups, int* ctas) {
    long long items = kRunItems;
    const long long most = (long long)groups * kMaxSumCtas;
    if (n > items * most) items = (n + most - 1) / most;
    *ctas = (int)((n + items * groups - 1) / (items * groups));
    return (int)items;
}

struct LookupScratch {
    size_t keys[2], vals[2], counts, row_tot, ends, partial, bytes;
};

// Scratch of the gradient for n ids and rows of nvec vectors, as offsets.
LookupScratch lookup_scratch(long long n, int ctas, int nvec) {
    LookupScratch s;
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t o = off; off += (bytes + 255) & ~(size_t)255; return o; };
    for (int k = 0; k < 2; ++k) { s.keys[k] = take((size_t)n * 4); s.vals[k] = take((size_t)n * 4); }
    s.counts = take((size_t)256 * sort_tiles((size_t)n) * 4);
    s.row_tot = take(256 * 4);
    s.ends = take((size_t)ctas * sizeof(RunEnds));
    s.partial = take((size_t)ctas * 2 * nvec * sizeof(float4));
    s.bytes = off;
    return s;
}

}  // namespace

size_t lookup_scratch_bytes(const emc2_bridge* h, int max_channels) {
    const long long n = (long long)h->cfg.max_batch * h->cfg.max_points;
    size_t most = 0;
    // Narrower rows have more groups per CTA, so fewer CTAs: which width needs most depends on n.
    for (int c = 4; c <= max_channels; c += 4) {
        int ctas;
        sum_items(n, kLookupThreads >> row_split(c / 4).log, &ctas);
        most = std::max(most, lookup_scratch(n, ctas, c / 4).bytes);
    }
    return most;
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
    LookupArgs a;
    a.ids = d_ids; a.table = d_table; a.out = d_out; a.scale = scale; a.n = n; a.rows = rows; a.nvec = channels / 4; a.type = type;
    a.row = make_fast_div((uint32_t)a.nvec);
    a.vectors = (uint32_t)n * (uint32_t)a.nvec;
    a.status = h->d_status;
    const uint32_t per_cta = kLookupThreads * kLookupUnroll;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    LaunchScope ls(h, K_ROW_LOOKUP, st);
    lookup_kernel<<<(a.vectors + per_cta - 1) / per_cta, kLookupThreads, 0, st>>>(a);
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
    const RowSplit split = row_split(a.nvec);
    const int groups = kLookupThreads >> split.log;
    int ctas;
    a.items = sum_items(n, groups, &ctas);
    const LookupScratch s = lookup_scratch(n, ctas, a.nvec);
    char* base = static_cast<char*>(h->rows_scratch.slab);
    uint32_t* keys[2] = {reinterpret_cast<uint32_t*>(base + s.keys[0]), reinterpret_cast<uint32_t*>(base + s.keys[1])};
    uint32_t* vals[2] = {reinterpret_cast<uint32_t*>(base + s.vals[0]), reinterpret_cast<uint32_t*>(base + s.vals[1])};
    {
        LaunchScope ls(h, K_LOOKUP_SORT, st);
        lookup_keys_kernel<<<(n + kLookupThreads - 1) / kLookupThreads, kLookupThreads, 0, st>>>(d_ids, n, rows, keys[0], vals[0], h->d_status);
    }
    int bits = 0;
    while (bits < 32 && ((uint64_t)1 << bits) < (uint64_t)rows + 1) ++bits;         // the keys are 0 .. rows
    const int at = radix_sort(h, K_LOOKUP_SORT, n, bits, keys, vals, true, reinterpret_cast<int*>(base + s.counts),
                              reinterpret_cast<int*>(base + s.row_tot), st);
    a.keys = keys[at]; a.vals = vals[at]; a.dout = d_grad_out; a.dtable = d_grad_table; a.scale = scale; a.n = n; a.rows = rows;
    a.log = split.log; a.type = type;
    a.ends = reinterpret_cast<RunEnds*>(base + s.ends);
    a.partial = reinterpret_cast<float4*>(base + s.partial);
    if (rows > 0) {
        LaunchScope ls(h, K_LOOKUP_SUM, st);
        lookup_zero_kernel<<<(rows + kLookupThreads - 1) / kLookupThreads, kLookupThreads, 0, st>>>(
            a.keys, n, rows, a.nvec, make_fast_div((uint32_t)a.nvec), d_grad_table, type);
    }
    {
        const size_t shared = (size_t)groups * 2 * a.nvec * sizeof(float4);
        LaunchScope ls(h, K_LOOKUP_SUM, st);
        switch (split.per) {
            case 1: launch_sum<1>(a, ctas, shared, st); break;
            case 2: launch_sum<2>(a, ctas, shared, st); break;
            case 3: launch_sum<3>(a, ctas, shared, st); break;
            case 4: launch_sum<4>(a, ctas, shared, st); break;
            case 5: launch_sum<5>(a, ctas, shared, st); break;
            case 6: launch_sum<6>(a, ctas, shared, st); break;
            case 7: launch_sum<7>(a, ctas, shared, st); break;
            default: launch_sum<8>(a, ctas, shared, st); break;
        }
    }
    {
        LaunchScope ls(h, K_LOOKUP_JOIN, st);
        lookup_join_kernel<<<ctas, kLookupThreads, (size_t)(kLookupThreads / 32) * a.nvec * sizeof(float4), st>>>(a, ctas);
    }
    return check_cuda(h, cudaGetLastError());
}
