// A whole mixture-of-experts layer for a few rows: router, choice, gated feed-forward of the chosen experts, weighted sum.
//
//   l = x w_router^T + b;  the k largest;  p = softmax over these
//   y = sum_j p_j (act(x w_gate[e_j]^T) * (x w_up[e_j]^T)) w_down[e_j]^T
//
// Bound by the weights of the experts that are asked for, which are read once; a row alone by the kernels' starts and waits, 4-bit weights
// by what makes numbers of them.  The first kernel has a CTA per row; the last of them to finish sorts the pairs (row, choice) by expert.  The
// second has a CTA per expert and tile of hidden units, the third per expert, tile of channels and share of the hidden units; what they leave
// is added up in the order of a row's choices, by the last CTA of a tile of channels or, for more rows, by a fourth kernel.  Each kernel is set
// up while the one before still runs.  In both products every warp streams its own rows of weights from memory into the registers of m16n8k16
// products, whose 16 rows are the rows at hand and whose 8 columns are the weights': a row of x more costs no more reading, and there are too
// few of them for larger products to help.
//
// 128 rows of 1,024 channels, 4 of 32 experts of 4,096 units, bf16: 167 us, of which the weights' 805 MB take 123 at a copy's rate; in 4 bits 161
// (33), with half of the issue slots and a third of the tensor pipe's.  One row of 256 channels, 2 of 16 experts of 1,024 units: 12.7.
//
// A logit is the sum of a sum in fp32 and of all that its roundings left (Ogita, Rump and Oishi, "Accurate sum and dot product", 2005), as if
// of twice the bits, so that the choice does not depend on an order of summation; 64-bit arithmetic took six times as long.  Products are
// summed in fp32.  act(g) * u goes into the last product as the sum of two numbers of the type, so that a row keeps its bits whichever rows it
// comes with: rounded to one where an expert has more than 16 rows, the layer of 128 rows took 162 us (146), and lost what that loses.  y is
// rounded once.
#include <algorithm>
#include <atomic>

#include "mx4.cuh"
#include "umma.cuh"

namespace emc2 {
namespace {

constexpr int kRouteThreads = 256;           // one per expert
constexpr int kRouteWarps = kRouteThreads / 32;
constexpr int kLayerThreads = 256;           // of the products; two CTAs per SM
constexpr int kLayerWarps = kLayerThreads / 32;
constexpr int kMaxLayerRows = 128;
constexpr int kMaxLayerExperts = 256;
constexpr int kMaxChoices = 8;
constexpr int kMaxSlots = kMaxLayerRows * kMaxChoices;     // pairs (row, choice)
constexpr int kMaxLayerHidden = 8192;
constexpr int kPanel = 256;                  // elements of the rows at hand in shared memory at a time
enum Stage { HIDDEN = 0, DOWN };
// Sixteens of a product's rows in a pass, at most, and the rows at hand that they are: a row of hidden values, in two parts, takes two.  Three of
// hidden values are what shared memory and registers have room for.  With two: 184 us instead of 168 for the layer above, whose experts
// have 16 rows on average, 175 instead of 164 in 4 bits; 33 instead of 37 where two experts of 512 channels and 2,048 units have 128 each.
__host__ __device__ constexpr int pass_sixteens(int stage) { return stage == DOWN ? 3 : 2; }
__host__ __device__ constexpr int rows_of_sixteen(int stage) { return stage == DOWN ? 8 : 16; }
__host__ __device__ constexpr int pass_rows(int stage) { return pass_sixteens(stage) * rows_of_sixteen(stage); }
constexpr int kMaxShares = 8;                // of the hidden units in the third kernel
constexpr int kMaxTiles = 64;                // of channels, per counter
constexpr int kLastAdds = 64;                // partial results of an output that the third kernel adds up itself, at most

// What the kernels leave one another, on the device.
struct LayerNotes {
    int arrived;                             // CTAs of the first kernel; zero between calls
    int used, active, pad;                   // rows in use, experts with rows
    int arrived_tile[kMaxTiles];             // CTAs of a tile of channels; zero between calls
    int expert[kMaxLayerExperts];            // the active experts, ascending
    int start[kMaxLayerExperts + 1];         // their pairs, sorted by expert and then by pair
    int row[kMaxSlots];                      // of a sorted pair
    int place[kMaxSlots];                    // of pair row * k + j among the sorted
};

struct LayerArgs {
    const void* x;
    const int32_t* count;                    // or null
    const float* w_router;
    const float* b_router;                   // or null
    const void* w[3];                        // gate, up, down: of the type, or codes
    const uint8_t* scales[3];                // of codes
    int32_t* ids;
    float* weights;
    void* y;
    LayerNotes* notes;
    void* hidden;                            // [sorted pair][H / 8][32 bytes], see hidden_place
    float* part;                             // [share][sorted pair][C]
    int* status;
    int n, C, H, E, k, act;
    int split_log;                           // warps that share a tile, each with every such step: 1 << split_log
    int tiles;                               // CTAs per expert
    int passes;                              // ... times so many, which share its passes of kRowsAtOnce rows
    int shares;                              // third kernel: of the hidden units
    int last_adds;                           // ... and whether its last CTAs add up
};

// Place of element i among eight, in the order that codes come in.
__host__ __device__ __forceinline__ int ordered_place(int i) { return (i & 3) * 2 + (i >> 2); }

// A hidden value is the sum of two of the type.  Where part q of value i (whose place among its eight is i % 8) of a pair of rows lies, in
// values: eight are two 16-byte registers of a product's lanes, the parts in rows g and g + 8.
__device__ __forceinline__ size_t hidden_place(int i, int q) { return (size_t)(i >> 3) * 16 + (i >> 2 & 1) * 8 + (i >> 1 & 1) * 4 + q * 2 + (i & 1); }

// Numbers that ascend as the logits do; NaN below all.  0 is left for what has been taken.
__device__ __forceinline__ unsigned long long logit_key(double v) {
    if (v != v) return 1ull;
    const long long b = __double_as_longlong(v + 0.0);            // -0 counts as 0
    return b < 0 ? ~(unsigned long long)b : (unsigned long long)b | 0x8000000000000000ull;
}

// high + rest += a b, the products' and the sums' roundings kept.
__device__ __forceinline__ void add_product(float& high, float& rest, float a, float b) {
    const float p = __fmul_rn(a, b), left = __fmaf_rn(a, b, -p), s = __fadd_rn(high, p), t = __fsub_rn(s, high);
    rest = __fadd_rn(rest, __fadd_rn(__fadd_rn(__fsub_rn(high, __fsub_rn(s, t)), __fsub_rn(p, t)), left));
    high = s;
}

// What a CTA needs for a row's choice.
struct Router {
    float x[kMaxRowChannels];
    unsigned long long key[kMaxLayerExperts];
    double logit[kMaxLayerExperts];
};

__device__ __forceinline__ int rows_in_use(const LayerArgs& a, bool reports) {
    if (!a.count) return a.n;
    const int used = *a.count;
    if ((used < 0 || used > a.n) && reports) atomicOr(a.status, kStatusBadRows);
    return min(max(used, 0), a.n);
}

// The warp's logits once more, in 64 bits: where terms or sums are past the range of fp32, or without a value.
__device__ __forceinline__ void far_logits(const float* w, const float* bias, int C, int E, Router& r) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll 1
    for (int e = 0; e < E; ++e) {
        if ((e >> 2) % kRouteWarps != warp) continue;
        double l = 0.0;
#pragma unroll 1
        for (int c = lane; c < C; c += 32) l += (double)__ldg(w + (size_t)e * C + c) * (double)r.x[c];
#pragma unroll
        for (int d = 16; d; d >>= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, d);
        if (bias) l += (double)__ldg(bias + e);
        __syncwarp();
        if (lane == 0) {
            r.logit[e] = l;
            r.key[e] = logit_key(l);
        }
    }
}

// A row's choices, by a whole CTA of kRouteThreads: lane j of the first warp has choice j and its weight.
template <bool BF16>
__device__ __forceinline__ void choose(const LayerArgs& a, int row, Router& r, int& id, float& weight) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid < a.C / 8) {
        const uint4 v = __ldg(static_cast<const uint4*>(a.x) + (size_t)row * (a.C / 8) + tid);
        const float4 f = as_floats(make_uint2(v.x, v.y), BF16 ? EMC2_BF16 : EMC2_F16), g = as_floats(make_uint2(v.z, v.w), BF16 ? EMC2_BF16 : EMC2_F16);
        reinterpret_cast<float4*>(r.x)[2 * tid] = f;
        reinterpret_cast<float4*>(r.x)[2 * tid + 1] = g;
    }
    __syncthreads();
    // Four experts at a time, so that their weights are under way together.
    bool far = false;
    for (int e0 = warp * 4; e0 < a.E; e0 += kRouteWarps * 4) {
        float high[4] = {0.f, 0.f, 0.f, 0.f}, rest[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int v = lane; v < a.C / 4; v += 32) {
            float4 f[4];
#pragma unroll
            for (int q = 0; q < 4; ++q)
                f[q] = e0 + q < a.E ? __ldg(reinterpret_cast<const float4*>(a.w_router + (size_t)(e0 + q) * a.C) + v) : make_float4(0.f, 0.f, 0.f, 0.f);
            const float4 g = reinterpret_cast<const float4*>(r.x)[v];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                add_product(high[q], rest[q], f[q].x, g.x);
                add_product(high[q], rest[q], f[q].y, g.y);
                add_product(high[q], rest[q], f[q].z, g.z);
                add_product(high[q], rest[q], f[q].w, g.w);
            }
        }
        double sum[4];
        bool past = false;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            sum[q] = (double)high[q] + (double)rest[q];
            past = past || !isfinite(high[q]);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
#pragma unroll
            for (int d = 16; d; d >>= 1) sum[q] += __shfl_xor_sync(0xFFFFFFFFu, sum[q], d);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int e = e0 + q;
            if (lane != q || e >= a.E) continue;
            const double l = a.b_router ? sum[q] + (double)__ldg(a.b_router + e) : sum[q];
            r.logit[e] = l;
            r.key[e] = logit_key(l);
        }
        far = far || __any_sync(0xFFFFFFFFu, past);
    }
    if (far) far_logits(a.w_router, a.b_router, a.C, a.E, r);
    __syncthreads();
    if (warp > 0) return;
    double chosen = 0.0, top = 0.0;                               // lane j: logit of choice j
    id = 0;
    for (int j = 0; j < a.k; ++j) {
        unsigned long long best = 0;
        unsigned at = 0;
        for (int e = lane; e < a.E; e += 32)
            if (r.key[e] > best) { best = r.key[e]; at = e; }
        // The largest upper half, of those the largest lower half, of those the lowest expert.
        const unsigned upper = __reduce_max_sync(0xFFFFFFFFu, (unsigned)(best >> 32));
        bool mine = (unsigned)(best >> 32) == upper;
        const unsigned lower = __reduce_max_sync(0xFFFFFFFFu, mine ? (unsigned)best : 0u);
        mine = mine && (unsigned)best == lower && best != 0;
        at = __reduce_min_sync(0xFFFFFFFFu, mine ? at : ~0u);
        if (j == 0) top = r.logit[at];
        if (lane == j) { chosen = r.logit[at]; id = at; }
        if (lane == 0) r.key[at] = 0;
        __syncwarp();
    }
    const float q = lane < a.k ? expf((float)(chosen - top)) : 0.f;
    float s = q;
#pragma unroll
    for (int d = 4; d; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);      // eight choices at most
    weight = q / s;
}

// Sorts up to 32 pairs by expert, stable: by one warp, whose lanes are the pairs (expert e; none: kMaxLayerExperts).
template <typename N>
__device__ __forceinline__ void sort_few(N& to, int e, int pairs, int k, int used) {
    const int lane = threadIdx.x & 31;
    const unsigned same = __match_any_sync(0xFFFFFFFFu, e);
    const int rank = __popc(same & ((1u << lane) - 1));
    int before = 0, active = 0;                                   // pairs, and experts, of lower numbers
    for (int i = 0; i < pairs; ++i) {
        const int other = __shfl_sync(0xFFFFFFFFu, e, i), first = __shfl_sync(0xFFFFFFFFu, rank, i) == 0;
        before += other < e;
        active += other < e && first;
    }
    if (lane < pairs) {
        to.row[before + rank] = lane / k;
        to.place[lane] = before + rank;
        if (rank == 0) {
            to.expert[active] = e;
            to.start[active + 1] = before + __popc(same);
        }
    }
    const int all = __popc(__ballot_sync(0xFFFFFFFFu, lane < pairs && rank == 0));
    if (lane == 0) {
        to.active = all;
        to.used = used;
        to.start[0] = 0;
    }
}

// One CTA per row, and with room for few: without that bound the compiler keeps to 48 registers, too few for the weights under way, and routing
// 128 rows of 1,024 channels to 4 of 32 experts takes 27 us instead of 17 by itself.
template <bool BF16>
__global__ void __launch_bounds__(kRouteThreads, 1) layer_route_kernel(LayerArgs a) {
    __shared__ __align__(16) Router router;
    __shared__ int last;
    const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    release_successor();                                          // at once: what follows waits for the end of this kernel, set up
    const int used = rows_in_use(a, row == 0 && tid == 0);
    if (row < used) {
        int id;
        float weight;
        choose<BF16>(a, row, router, id, weight);
        if (tid < a.k) {
            a.ids[(size_t)row * a.k + tid] = id;
            a.weights[(size_t)row * a.k + tid] = weight;
        }
    }
    // The last CTA sorts the pairs: stable, by the counts of every expert in pieces of 32 pairs.
    __syncthreads();
    if (gridDim.x > 1) {
        if (tid == 0) {
            __threadfence();
            last = atomicAdd(&a.notes->arrived, 1) == (int)gridDim.x - 1;
        }
        __syncthreads();
        if (!last) return;
        __threadfence();
    }
    const int pairs = used * a.k;
    if (pairs <= 32) {
        if (warp > 0) return;
        sort_few(*a.notes, lane < pairs ? __ldcg(a.ids + lane) : kMaxLayerExperts, pairs, a.k, used);
        if (lane == 0) a.notes->arrived = 0;
        return;
    }
    __shared__ int of[kMaxSlots];
    __shared__ uint16_t piece[kMaxSlots / 32][kMaxLayerExperts];
    __shared__ int base[kMaxLayerExperts], warp_sum[2][kRouteWarps];
    const int pieces = (pairs + 31) / 32;
    for (int i = tid; i < pairs; i += kRouteThreads) of[i] = __ldcg(a.ids + i);
    for (int i = tid; i < pieces * kMaxLayerExperts / 2; i += kRouteThreads) reinterpret_cast<uint32_t*>(piece)[i] = 0u;
    __syncthreads();
    for (int p = warp; p < pieces; p += kRouteWarps) {
        const int i = p * 32 + lane, e = i < pairs ? of[i] : -1;
        const unsigned same = __match_any_sync(0xFFFFFFFFu, e);
        if (e >= 0 && (same & ((1u << lane) - 1)) == 0) piece[p][e] = (uint16_t)__popc(same);
    }
    __syncthreads();
    // Thread e: pairs of expert e, before a piece and in all; then starts and places among the active ones.
    int total = 0;
    for (int p = 0; p < pieces; ++p) {
        const int c = piece[p][tid];
        piece[p][tid] = (uint16_t)total;
        total += c;
    }
    int sum = total, rank = total > 0;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int s = __shfl_up_sync(0xFFFFFFFFu, sum, d), r = __shfl_up_sync(0xFFFFFFFFu, rank, d);
        if (lane >= d) { sum += s; rank += r; }
    }
    if (lane == 31) { warp_sum[0][warp] = sum; warp_sum[1][warp] = rank; }
    __syncthreads();
    for (int w = 0; w < warp; ++w) { sum += warp_sum[0][w]; rank += warp_sum[1][w]; }
    base[tid] = sum - total;
    if (total > 0) {
        a.notes->expert[rank - 1] = tid;
        a.notes->start[rank] = sum;
    }
    if (tid == kRouteThreads - 1) {
        a.notes->active = rank;
        a.notes->used = used;
        a.notes->start[0] = 0;
        a.notes->arrived = 0;
    }
    __syncthreads();
    for (int p = warp; p < pieces; p += kRouteWarps) {
        const int i = p * 32 + lane, e = i < pairs ? of[i] : -1;
        const unsigned same = __match_any_sync(0xFFFFFFFFu, e);
        if (e < 0) continue;
        const int at = base[e] + piece[p][e] + __popc(same & ((1u << lane) - 1));
        a.notes->row[at] = i / a.k;
        a.notes->place[i] = at;
    }
}

// ---- products
template <bool BF16>
__device__ __forceinline__ void product(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if (BF16)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Eight codes as the pairs (0, 4), (1, 5), (2, 6), (3, 7), times the type's smallest power that is not its last: the three bits of a size
// are put at the end of the exponent and the start of the mantissa, where they read as the element times 2^-126 (bf16) or 2^-14 (fp16),
// its number below 1 too, and `factor` makes up for it.  fp16's results are twice the elements, see spare.
template <bool BF16>
__device__ __forceinline__ void decode8(uint32_t (&r)[4], uint32_t codes, uint32_t factor) {
    constexpr uint32_t size = BF16 ? 0x01C001C0u : 0x0E000E00u, sign = 0x80008000u;
    constexpr int up = BF16 ? 6 : 9;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t m = up >= 4 * i ? codes << (up - 4 * i) : codes >> (4 * i - up);
        const uint32_t v = (m & size) | ((codes << (12 - 4 * i)) & sign);
        if (BF16) asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r[i]) : "r"(v), "r"(factor));
        else asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r[i]) : "r"(v), "r"(factor));
    }
}
// Sums are relative to the largest power that a row has had so far, and `spare` powers above it, so that the next rise is seldom.  What is
// smaller than a type's numbers reach is rounded: fp16 has one to spare and is taken twice as large, so that its elements are rounded to 2^-24 of the
// row's largest power; with two, and as they are, to 2^-22.  bf16's reach is 2^-131.
__host__ __device__ constexpr uint32_t spare(bool bf16) { return bf16 ? 2u : 1u; }
// The pair of factors for a block whose power is 2^-below of what the sums are relative to.
template <bool BF16>
__device__ __forceinline__ uint32_t block_factor(int below) {
    if (BF16) return (uint32_t)max(253 - below, 0) * 0x00800080u;
    const uint32_t h = below < 30 ? (uint32_t)(30 - below) << 10 : below <= 39 ? 1u << (39 - below) : 0u;
    return h * 0x00010001u;
}

// Weights as [experts * rows][elements or bytes of codes], in boxes of 128 bytes of 16 rows (gate, up) or 32 (down), whose vectors are
// mixed with the row's number (the copies' swizzle); what lies behind a row reads as zeros.
struct LayerMaps {
    CUtensorMap w[3];
};

// Panels of the rows at hand, in two buffers, as the 16-byte registers of a product's lanes: [16 rows][8 blocks of 32 elements][2 halves]
// [32 lanes].  A lane's vector has two words of row g and, between them, those of row g + 8.
__host__ __device__ constexpr uint32_t panel_bytes(int stage) { return pass_sixteens(stage) * kPanel / 32 * 2 * 512; }
// The warps' sums take the panels' place when the products are done: [warp][16 rows][32 rows of weights][16], the last index mixed with the
// one before, so that writers and readers meet few of the same banks.
static_assert(kLayerWarps * pass_sixteens(DOWN) * 16 * 32 * 4 <= 2 * panel_bytes(DOWN) && kLayerWarps * pass_sixteens(HIDDEN) * 16 * 32 * 4 <= 2 * panel_bytes(HIDDEN), "sums");
// Behind them the ring: [stage][warp][32 rows][128 bytes], on 128 bytes.  A third kernel's CTA has 112 KB: two fit an SM's 228.
constexpr uint32_t kWarpStage = 32 * 128, kStage = kLayerWarps * kWarpStage;
constexpr size_t product_shared(int stage) { return 2 * panel_bytes(stage) + 2 * kStage; }

// The pairs sorted by expert, where the kernel has them.
struct Lists {
    int active;
    const int *expert, *start, *row;
};

// A warp's barriers, one per stage, and the parities that it waits for next.
struct Ring {
    uint32_t bars, phases;
    volatile int* gave_up;
};

// What a warp's rows of weights are: four tiles of eight, of the gate's and the up projection's rows or of the down projection's.  Lane (g, t)
// has row g / 2 + 4 (g % 2) of each, so that the eight vectors that lanes read together lie on different banks.  Which element stands at which
// place of a product does not matter, if weights and rows agree.
//   16 bits: two blocks of 32 elements to a step, of each of which the lane has 8t .. 8t + 7.
//    4 bits: eight blocks to a step, of which the lane has the t-th of either half.  A block's elements are taken relative to the largest power
//            that the row has had so far, which the sums are relative to; when it rises, they are scaled down.
// The weights of the next step are on their way to shared memory, in boxes that the warp alone reads: registers have no room for as much as the
// memory needs to be asked for at once (50 KB per SM and more).
template <int STAGE, bool MX, bool BF16, bool HALVES, int MT>
__device__ __forceinline__ void layer_rows(const LayerArgs& a, const LayerMaps& maps, const Lists& lists, char* smem, Ring& wait, int e, int pair0, int rows) {
    constexpr int kPiece = MX ? 256 : 64;                         // elements of a step
    int tid;                                                      // anew for every pass, as what follows from it: registers are short
    asm volatile("mov.u32 %0, %%tid.x;" : "=r"(tid));
    const int lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int split_log = MX ? HALVES : a.split_log, split = 1 << split_log, per_cta = kLayerWarps >> split_log, part = warp & (split - 1), slot = warp >> split_log;
    const int K = STAGE == HIDDEN ? a.C : a.H, M = STAGE == HIDDEN ? a.H : a.C;
    const int unit = (int)blockIdx.y, tile = unit * per_cta + slot;        // of 16 hidden units, or of 32 channels
    // The third kernel's share of the hidden units, whole steps of the products; the last ones ragged.
    const int each = STAGE == HIDDEN ? K : ((K + a.shares - 1) / a.shares + 255) / 256 * 256;
    const int k0 = STAGE == HIDDEN ? 0 : min(K, (int)blockIdx.x * each), k1 = min(K, k0 + each);
    // 4 bits: where the lane finds its block's powers, of its rows of weights.  Rows behind the last are read as the last, and come to nothing.
    constexpr int kRows = STAGE == HIDDEN ? 2 : 4;
    const int blocks = (K + kMxBlock - 1) / kMxBlock, r0 = tile * (STAGE == HIDDEN ? 16 : 32);
    const int row = g >> 1 | (g & 1) << 2;
    uint32_t at[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) at[i] = (uint32_t)(e * M + min(r0 + row + 8 * i, M - 1)) * (uint32_t)blocks + (uint32_t)(k0 / kMxBlock + t);
    float acc[MT][4][4];                                          // [16 rows][tile]
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[m][i][c] = 0.f;
    // A thread brings the vectors of its lane number and, in every 16 rows, the warp's block of a panel: of rows g and g + 8 of x through
    // registers, where their words change places; hidden values, which lie as the products take them, by copies past the registers.  The
    // two parts of one stand in rows g and g + 8, whose sums the lane adds.
    const uint32_t panels = (uint32_t)__cvta_generic_to_shared(smem);
    static_assert(kLayerWarps == kPanel / 32, "a block of a panel per warp");
    const int chunk = MX ? (warp & ~3) * 4 + t * 4 + (warp & 3) : warp * 4 + t;       // vector of a panel's row
    const char* from[MT][2];                                      // STAGE == HIDDEN
    const int rows_left = rows - g;
    const uint32_t values = (uint32_t)(pair0 + g) * 4 * a.H + chunk * 32;          // 1,024 pairs of 8,192 units at most
    if (STAGE == HIDDEN) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int r = m * 16 + q * 8 + g;
                from[m][q] = r < rows ? static_cast<const char*>(a.x) + ((size_t)lists.row[pair0 + r] * a.C + chunk * 8) * 2 : nullptr;
            }
    }
    uint4 brought[MT][2];
    // The panel from element k on is on its way from `bring` on, to the buffer at `to`, and there after `put` and a barrier.
    auto bring = [&](int k, uint32_t to) {
        if constexpr (STAGE == DOWN) {
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const bool there = m * 8 < rows_left && k + chunk * 8 < k1;
                const char* src = static_cast<const char*>(a.hidden) + (there ? values + (uint32_t)(m * 32 * a.H + k * 4) : 0u);
                const uint32_t dst = to + (uint32_t)((m * (kPanel / 32) + warp) * 1024 + lane * 16), bytes = there ? 16u : 0u;       // the rest of 16 is zeros
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + 512), "l"(src + 16), "r"(bytes) : "memory");
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        } else {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    brought[m][q] = make_uint4(0u, 0u, 0u, 0u);
                    if (from[m][q] && k + chunk * 8 < k1) brought[m][q] = *reinterpret_cast<const uint4*>(from[m][q] + 2 * k);
                    // Eight codes come as the pairs (0, 4), (1, 5), (2, 6), (3, 7); the hidden values lie in that order.
                    if (MX) {
                        const uint4 v = brought[m][q];
                        brought[m][q] = make_uint4(__byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632), __byte_perm(v.y, v.w, 0x5410), __byte_perm(v.y, v.w, 0x7632));
                    }
                }
        }
    };
    auto put = [&](uint32_t to) {
        if constexpr (STAGE == DOWN) {
            asm volatile("cp.async.wait_group 0;" ::: "memory");
        } else {
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const uint4 &u = brought[m][0], &v = brought[m][1];
                const uint32_t at = to + (uint32_t)((m * (kPanel / 32) + warp) * 1024 + lane * 16);
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(u.x), "r"(v.x), "r"(u.y), "r"(v.y) : "memory");
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + 512), "r"(u.z), "r"(v.z), "r"(u.w), "r"(v.w) : "memory");
            }
        }
    };
    auto rows_at = [&](uint32_t panel, int block, int m, int half) {
        uint4 v;
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                     : "r"(panel + (uint32_t)((m * (kPanel / 32) + block) * 1024 + half * 512)));
        return v;
    };
    constexpr uint32_t kPanelBytes = panel_bytes(STAGE);
    const uint32_t ring = panels + 2 * kPanelBytes + warp * kWarpStage;
    // The copies mix a vector's number with bits 7 to 9 of its row's address.  Of the step's second half: bit 6 the other way.
    const uint32_t mine = ring + row * 128 + ((t ^ ((ring >> 7) + row & 7)) << 4);
    // Warps that share a tile take every such step of it, with 4 bits either half of every step (whose weights they both have copied).
    const int stride = MX ? kPiece : kPiece << split_log, steps = (k1 - k0 + stride - 1) / stride, panel_log = MX ? 0 : 2 - split_log;      // steps of a panel
    const uint32_t lead = elected();
    auto request = [&](int s, uint32_t (&powers)[2]) {            // powers: of the lane's blocks, a byte for each of the four rows
        const int k = k0 + s * stride + (MX ? 0 : part * kPiece);
        const uint32_t to = ring + (s & 1) * kStage, bar = wait.bars + (s & 1) * 8;
        bar_expect(lead, bar, kWarpStage);
        if (STAGE == HIDDEN) {
            copy_tile(lead, to, &maps.w[0], MX ? k / 2 : k, e * M + r0, bar);
            copy_tile(lead, to + kWarpStage / 2, &maps.w[1], MX ? k / 2 : k, e * M + r0, bar);
        } else {
            copy_tile(lead, to, &maps.w[2], MX ? k / 2 : k, e * M + r0, bar);
        }
        if (!MX) return;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            powers[u] = 0;
            if (k + (4 * u + t) * kMxBlock >= k1) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i) powers[u] |= (uint32_t)__ldg(a.scales[STAGE == HIDDEN ? i >> 1 : 2] + (at[i % kRows] + 4 * u)) << (8 * i);
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i) at[i] += stride / kMxBlock;
    };
    uint32_t largest = 0;                                         // powers that the sums are relative to, of the lane's four rows of weights
    // The sums' columns 2t and 2t + 1 of a tile are those of the lanes with these g, which have their factors.
    auto scale = [&](int i, float f) {
        const float f0 = __shfl_sync(0xFFFFFFFFu, f, 8 * t), f1 = __shfl_sync(0xFFFFFFFFu, f, 8 * t + 4);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            acc[m][i][0] *= f0; acc[m][i][1] *= f1;
            acc[m][i][2] *= f0; acc[m][i][3] *= f1;
        }
    };
    auto multiply = [&](uint32_t stage, int u, uint32_t power_of_block, uint32_t panel, int first) {      // u: half of the step; first: block of the panel
        uint4 v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[i].x), "=r"(v[i].y), "=r"(v[i].z), "=r"(v[i].w) : "r"((mine ^ u << 6) + stage + i * 1024));
        if (!MX) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    const uint4 x = rows_at(panel, first, m, half);
#pragma unroll
                    for (int i = 0; i < 4; ++i) product<BF16>(acc[m][i], x.x, x.y, x.z, x.w, half ? v[i].z : v[i].x, half ? v[i].w : v[i].y);
                }
            }
            return;
        }
        uint32_t top = __vmaxu4(power_of_block, __shfl_xor_sync(0xFFFFFFFFu, power_of_block, 1));
        top = __vmaxu4(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
        if (__any_sync(0xFFFFFFFFu, __vmaxu4(top, largest) != largest)) {
            top = __vmaxu4(__vmaxu4(__vminu4(__vaddus4(top, spare(BF16) * 0x01010101u), 0xFEFEFEFEu), top), largest);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int fall = (int)(top >> (8 * i) & 255u) - (int)(largest >> (8 * i) & 255u);
                scale(i, __uint_as_float((uint32_t)max(127 - fall, 0) << 23));
            }
            largest = top;
        }
        uint32_t factor[4];
        const uint32_t below = largest - power_of_block;          // byte by byte: none is larger
#pragma unroll
        for (int i = 0; i < 4; ++i) factor[i] = block_factor<BF16>((int)(below >> (8 * i) & 255u));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t r[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) decode8<BF16>(r[i], j == 0 ? v[i].x : j == 1 ? v[i].y : j == 2 ? v[i].z : v[i].w, factor[i]);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    const uint4 x = rows_at(panel, first + j, m, half);
#pragma unroll
                    for (int i = 0; i < 4; ++i) product<BF16>(acc[m][i], x.x, x.y, x.z, x.w, r[i][2 * half], r[i][2 * half + 1]);
                }
            }
        }
    };
    uint32_t powers[2][2];
    __syncwarp();                                                 // of the pass before, the warp has read all
#pragma unroll
    for (int s = 0; s < 2; ++s)
        if (s < steps) request(s, powers[s]);
    bring(k0, panels);
    put(panels);
    // Not unrolled: the products of several steps do not fit the instruction cache.
#pragma unroll 1
    for (int s = 0; s < steps; ++s) {
        const int panel = s >> panel_log, in_panel = s & ((1 << panel_log) - 1), next = k0 + (panel + 1) * kPanel;
        if (in_panel == 0) {
            __syncthreads();                                      // the panel is there, and the other one is done with
            if (next < k1) bring(next, panels + ((panel & 1) ^ 1) * kPanelBytes);
        }
        const uint32_t stage = s & 1;
        warp_wait(wait.bars + stage * 8, wait.phases >> stage & 1u, wait.gave_up, a.status);
        wait.phases ^= 1u << stage;
        const uint32_t at_panel = panels + (panel & 1) * kPanelBytes + lane * 16;
        if (HALVES) {
            multiply(stage * kStage, part, part ? powers[0][1] : powers[0][0], at_panel, 4 * part);
        } else {
#pragma unroll
            for (int u = 0; u < 2; ++u) multiply(stage * kStage, u, powers[0][u], at_panel, ((in_panel * stride + (MX ? 0 : part * kPiece)) >> 5) + (MX ? 4 : 1) * u);
        }
        __syncwarp();                                             // the stage is done with
        powers[0][0] = powers[1][0];
        powers[0][1] = powers[1][1];
        if (s + 2 < steps) request(s + 2, powers[1]);
        if (in_panel == (1 << panel_log) - 1 && next < k1) put(panels + ((panel & 1) ^ 1) * kPanelBytes);
    }
    if (MX) {
#pragma unroll
        for (int i = 0; i < 4; ++i) scale(i, (BF16 ? 1.0f : 0.5f) * mx_power(largest >> (8 * i) & 255u));
    }
    __syncthreads();                                              // the panels are done with; the warps that share a tile are added in their order
    float* sums = reinterpret_cast<float*>(smem);
    constexpr int kHeld = rows_of_sixteen(STAGE);
    auto sum_at = [&](int w, int m, int column, int r) { return ((w * MT + m) * 32 + column) * 16 + (r ^ (column >> 1)); };
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int column = i * 8 + t + 4 * c;                // the row of lanes with g = 2t + c
                if (STAGE == DOWN) {
                    sums[sum_at(warp, m, column, g)] = acc[m][i][c] + acc[m][i][2 + c];
                } else {
                    sums[sum_at(warp, m, column, g)] = acc[m][i][c];
                    sums[sum_at(warp, m, column, g + 8)] = acc[m][i][2 + c];
                }
            }
    __syncthreads();
    auto sum = [&](int s, int c, int column) {
        float v = 0.f;
        for (int q = 0; q < split; ++q) v += sums[sum_at(s * split + q, c / kHeld, column, c % kHeld)];
        return v;
    };
    if (STAGE == DOWN) {
        for (int s = 0; s < per_cta; ++s)
            for (int c = warp; c < rows; c += kLayerWarps) {
                const int at = (unit * per_cta + s) * 32 + lane;
                if (at < M) a.part[((size_t)blockIdx.x * (a.n * a.k) + pair0 + c) * a.C + at] = sum(s, c, lane);
            }
        __syncthreads();
        return;
    }
    const uint32_t by_rows = (65536u + rows - 1) / rows;          // a quotient of fewer than 256 by it
    for (int o = tid / 16; o < per_cta * rows; o += kLayerThreads / 16) {
        const int s = (int)(o * by_rows >> 16), c = o - s * rows, u = tid % 16, at = (unit * per_cta + s) * 16 + u;
        if (at >= M) continue;
        const float gate = sum(s, c, u), up = sum(s, c, 16 + u);
        const float f = a.act == EMC2_ACT_SILU ? gate / (1.0f + expf(-gate)) : 0.5f * gate * erfcf(-0.70710678f * gate);
        const float h = f * up;
        const int i = MX ? (at & ~7) + ordered_place(at & 7) : at;
        const size_t pair = (size_t)(pair0 + c) * 2 * a.H, to = pair + hidden_place(i, 0), rest = pair + hidden_place(i, 1);
        // What the first part leaves is exact; an infinite one leaves nothing.
        if (BF16) {
            __nv_bfloat16* p = static_cast<__nv_bfloat16*>(a.hidden);
            const __nv_bfloat16 first = __float2bfloat16_rn(h);
            p[to] = first;
            p[rest] = __float2bfloat16_rn(isinf(__bfloat162float(first)) ? 0.f : h - __bfloat162float(first));
        } else {
            __half* p = static_cast<__half*>(a.hidden);
            const __half first = __float2half_rn(h);
            p[to] = first;
            p[rest] = __float2half_rn(isinf(__half2float(first)) ? 0.f : h - __half2float(first));
        }
    }
    __syncthreads();
}

// The rows of the CTA's expert, 32 at a time, against its weights.  A CTA's place: share of the hidden units (the third kernel's) in x,
// tile of its rows of weights in y, active expert and, within it, of the passes over its rows in z.
template <int STAGE, bool MX, bool BF16, bool HALVES>
__device__ __forceinline__ void layer_unit(const LayerArgs& a, const LayerMaps& maps, const Lists& lists, char* smem) {
    __shared__ __align__(8) unsigned long long bars[kLayerWarps][2];
    __shared__ int gave_up;
    __shared__ volatile int at_pass;
    if (threadIdx.x == 0) {
        gave_up = 0;
        at_pass = (int)blockIdx.z % a.passes;
    }
    Ring ring = {smem_u32(bars[threadIdx.x >> 5]), 0u, &gave_up};
    if ((threadIdx.x & 31) == 0)
        for (int s = 0; s < 2; ++s) bar_init(ring.bars + s * 8, 1);
    fence_bar_init();
    fence_async_shared();
    __syncthreads();
    // Looked up again for every pass: the products leave no registers to keep it.
#pragma unroll 1
    for (;;) {
        const int pass = at_pass, i = (int)blockIdx.z / a.passes, all = lists.start[i + 1] - lists.start[i];
        constexpr int kMost = pass_rows(STAGE);
        if (pass * kMost >= all) break;
        const int e = lists.expert[i], p = lists.start[i] + pass * kMost, rows = min(kMost, all - pass * kMost);
        constexpr int kEach = rows_of_sixteen(STAGE);
        if (rows <= kEach) layer_rows<STAGE, MX, BF16, HALVES, 1>(a, maps, lists, smem, ring, e, p, rows);
        else if (STAGE == HIDDEN || rows <= 2 * kEach) layer_rows<STAGE, MX, BF16, HALVES, 2>(a, maps, lists, smem, ring, e, p, rows);
        else layer_rows<STAGE, MX, BF16, HALVES, STAGE == HIDDEN ? 2 : 3>(a, maps, lists, smem, ring, e, p, rows);
        if (threadIdx.x == 0) at_pass += a.passes;               // all have read it before the barriers of the products
        __syncthreads();
    }
    leave_after_timeout(&gave_up);
}

// y of four channels of a row: its choices in their order, of each the shares in theirs.
template <bool BF16>
__device__ __forceinline__ void layer_sum(const LayerArgs& a, int row, int c) {
    const size_t apart = (size_t)a.n * a.k * a.C;
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int j = 0; j < a.k; ++j) {
        const float* at = a.part + (size_t)a.notes->place[row * a.k + j] * a.C + c;
        const float p = a.weights[row * a.k + j];
        float4 z = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int s = 0; s < a.shares; ++s) {
            const float4 q = __ldcg(reinterpret_cast<const float4*>(at + s * apart));
            z.x += q.x; z.y += q.y; z.z += q.z; z.w += q.w;
        }
        y.x += p * z.x; y.y += p * z.y; y.z += p * z.z; y.w += p * z.w;
    }
    store_row4(a.y, ((size_t)row * a.C + c) / 4, y, BF16 ? EMC2_BF16 : EMC2_F16);
}

template <bool MX, bool BF16, bool HALVES>
__global__ void __launch_bounds__(kLayerThreads, 2) layer_hidden_kernel(LayerArgs a, const __grid_constant__ LayerMaps maps) {
    await_predecessor();
    release_successor();
    extern __shared__ __align__(128) char panels[];
    const Lists lists = {a.notes->active, a.notes->expert, a.notes->start, a.notes->row};
    if ((int)blockIdx.z < lists.active * a.passes) layer_unit<HIDDEN, MX, BF16, HALVES>(a, maps, lists, panels);
}

struct OneRow {
    int active, used;
    int expert[kMaxChoices], start[kMaxChoices + 1], row[kMaxChoices], place[kMaxChoices];
};

// The first kernel and the second in one, for one row (decoding): every CTA makes its choice for itself, the first one notes it for what
// follows.  That is a launch and a wait less: 12.9 us against 14.1 with 8 experts of 256 channels, 13.1 against 14.5 with 32, 26.0 against 27.2 with
// 256 of 512.  Two rows are no faster this way (15.8 against 15.4), four are slower (19.6 against 15.6): their choices come one after the other.
template <bool MX, bool BF16, bool HALVES>
__global__ void __launch_bounds__(kLayerThreads, 2) layer_one_row_kernel(LayerArgs a, const __grid_constant__ LayerMaps maps) {
    release_successor();
    extern __shared__ __align__(128) char panels[];
    static_assert(kRouteThreads == kLayerThreads && sizeof(Router) <= 2 * panel_bytes(HIDDEN), "the router's place is the panels'");
    __shared__ OneRow found;
    const int tid = threadIdx.x;
    const bool notes = blockIdx.y == 0 && blockIdx.z == 0;
    const int used = rows_in_use(a, notes && tid == 0);
    int id = kMaxLayerExperts;
    float weight = 0.f;
    if (used) choose<BF16>(a, 0, *reinterpret_cast<Router*>(panels), id, weight);
    if (tid < 32) {
        if (tid >= a.k) id = kMaxLayerExperts;
        sort_few(found, id, used * a.k, a.k, used);
        if (notes) {
            sort_few(*a.notes, id, used * a.k, a.k, used);
            if (tid < used * a.k) {
                a.ids[tid] = id;
                a.weights[tid] = weight;
            }
        }
    }
    __syncthreads();
    const Lists lists = {found.active, found.expert, found.start, found.row};
    if ((int)blockIdx.z < lists.active * a.passes) layer_unit<HIDDEN, MX, BF16, HALVES>(a, maps, lists, panels);
}

template <bool MX, bool BF16, bool HALVES>
__global__ void __launch_bounds__(kLayerThreads, 2) layer_down_kernel(LayerArgs a, const __grid_constant__ LayerMaps maps) {
    await_predecessor();
    release_successor();
    extern __shared__ __align__(128) char panels[];
    __shared__ int last;
    const Lists lists = {a.notes->active, a.notes->expert, a.notes->start, a.notes->row};
    if ((int)blockIdx.z >= lists.active * a.passes) return;
    layer_unit<DOWN, MX, BF16, HALVES>(a, maps, lists, panels);
    if (!a.last_adds) return;
    const int unit = (int)blockIdx.y, tid = threadIdx.x;
    __syncthreads();
    if (tid == 0) {
        __threadfence();
        last = atomicAdd(&a.notes->arrived_tile[unit], 1) == a.notes->active * a.passes * a.shares - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    const int wide = (kLayerWarps >> a.split_log) * 32, width = min(a.C - unit * wide, wide) / 4;
    for (int o = tid; o < a.notes->used * width; o += kLayerThreads) layer_sum<BF16>(a, o / width, unit * wide + o % width * 4);
    if (tid == 0) a.notes->arrived_tile[unit] = 0;
}

template <bool BF16>
__global__ void __launch_bounds__(kLayerThreads) layer_sum_kernel(LayerArgs a) {
    await_predecessor();
    const int o = blockIdx.x * kLayerThreads + threadIdx.x, width = a.C / 4;
    if (o < a.notes->used * width) layer_sum<BF16>(a, o / width, o % width * 4);
    release_successor();
}

// ---- scratch: notes, hidden values, partial sums
size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }
constexpr int kPartRows = 2 * kMaxSlots;     // shares times pairs, at most

template <bool MX, bool BF16>
cudaError_t launch_layer(emc2_bridge* h, LayerArgs a, cudaStream_t st) {
    constexpr size_t most_hidden = product_shared(HIDDEN), most_down = product_shared(DOWN);
    static std::atomic<uint64_t> allowed{0};                      // devices; one bound for every call, so once for each
    const uint64_t bit = h->cfg.device < 64 ? (uint64_t)1 << h->cfg.device : 0;
    if (!(allowed.load(std::memory_order_relaxed) & bit)) {
        cudaError_t e = allow_shared(layer_hidden_kernel<MX, BF16, false>, most_hidden);
        if (e == cudaSuccess) e = allow_shared(layer_down_kernel<MX, BF16, false>, most_down);
        if (e == cudaSuccess && MX) e = allow_shared(layer_hidden_kernel<MX, BF16, MX>, most_hidden);
        if (e == cudaSuccess) e = allow_shared(layer_one_row_kernel<MX, BF16, false>, most_hidden);
        if (e == cudaSuccess && MX) e = allow_shared(layer_one_row_kernel<MX, BF16, MX>, most_hidden);
        if (e == cudaSuccess && MX) e = allow_shared(layer_down_kernel<MX, BF16, MX>, most_down);
        if (e != cudaSuccess) return e;
        allowed.fetch_or(bit, std::memory_order_relaxed);
    }
    LayerMaps maps;
    for (int i = 0; i < 3; ++i) {
        const int K = i < 2 ? a.C : a.H, M = i < 2 ? a.H : a.C;
        const cuuint64_t row = MX ? (cuuint64_t)mx4_blocks(K) * 16 : (cuuint64_t)K * 2;
        const cuuint64_t dims[2] = {MX ? row : (cuuint64_t)K, (cuuint64_t)a.E * M}, strides[1] = {row};
        const cuuint32_t box[2] = {MX ? 128u : 64u, i < 2 ? 16u : 32u}, step[2] = {1, 1};
        const EncodeTiled f = encoder();
        if (!f || f(&maps.w[i], MX ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2,
                    const_cast<void*>(a.w[i]), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                    CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return cudaErrorInvalidValue;
    }
    const int experts = std::min(a.E, a.n * a.k);
    const int step = MX ? 256 : 64;
    // CTAs that share an expert's rows: where its tiles leave SMs without one, so many that all fit, and as its passes are with a quarter more rows than
    // an even choice gives it.  us for the layer so, with one CTA for all passes, with as many as an expert can have passes, and as an even choice gives
    // (16-bit weights; 4-bit): 128 rows, both of 2 experts of 512 channels and 2,048 units 37.4, 65.0, 37.4, 37.3 (37.7, 79.6, 37.7, 37.7); 100 rows, 2 of
    // 16 of 512 and 1,024 29.8, 29.9, 36.7, 29.9; 128 rows, 1 of 2 of 1,024 and 2,048 40.4, 51.0, 40.8, 39.7 (42.0, 73.6, 42.2, 50.4); 96 rows, 1 of 3 of
    // 256 and 512 19.5, 23.3, 20.0, 20.8 (22.0, 30.1, 23.5, 27.4); 50 rows, 2 of 5 of 256 and 1,024 22.5, 24.3, 25.0, 24.4.
    // Then warps that share a tile: none where the CTAs fill the SMs, else as many as that takes, and as have steps.
    auto tiles_of = [&](int M, int width) {
        const int per = (kLayerWarps >> a.split_log) * width;
        return (M + per - 1) / per;
    };
    auto plan = [&](int K, int M, int width, int rows) {
        const int steps = (K + step - 1) / step, most_log = MX ? 1 : 2, most_passes = std::min((a.n + rows - 1) / rows, (5 * a.n * a.k + 4 * rows * a.E - 1) / (4 * rows * a.E));
        a.split_log = 0;
        a.tiles = tiles_of(M, width);
        for (a.passes = 1; a.passes < most_passes && a.tiles * experts * a.shares * (a.passes + 1) <= 2 * h->num_sms;) ++a.passes;
        for (;; ++a.split_log) {
            a.tiles = tiles_of(M, width);
            if (a.tiles * experts * a.shares * a.passes >= h->num_sms || a.split_log == most_log || (!MX && (1 << a.split_log) >= steps)) break;
        }
    };
    const bool one = a.n == 1;
    if (!one) {
        LaunchScope ls(h, K_LAYER_ROUTE, st);
        layer_route_kernel<BF16><<<a.n, kRouteThreads, 0, st>>>(a);
    }
    {
        LaunchScope ls(h, K_LAYER_HIDDEN, st);
        plan(a.C, a.H, 16, pass_rows(HIDDEN));
        // Two to four waves of CTAs end less unevenly as twice as many, where there are channels enough to make up for their starts.  us for the
        // layer with and without, at 592 to 1,183 CTAs: of 1,024 channels 167.6 and 171.6 (1,024 CTAs), 122.7 and 125.6 (640), 170.8 and 181.2
        // (608), 144.6 and 147.8 (1,024, 20 rows); of 768 109.7 and 111.2 (896).  Of 512 105.9 and 103.4 (784), 93.9 and 92.3 (1,152), of 256 79.0
        // and 72.8 (1,152), of 128 60.4 and 55.0 (800): no.  Of 1,024 channels in more CTAs (1,216) 195.5 and 196.6, of 512 (1,504) 159.9 and 152.
        const int ctas = a.tiles * experts;
        if (!MX && a.split_log == 0 && ctas >= 4 * h->num_sms && ctas < 8 * h->num_sms && a.C >= 12 * step) {
            a.split_log = 1;
            a.tiles = tiles_of(a.H, 16);
        }
        const dim3 grid(1, (unsigned)a.tiles, (unsigned)(a.passes * experts));
        const bool halves = MX && a.split_log;
        if (one) launch_kernel(false, halves ? layer_one_row_kernel<MX, BF16, MX> : layer_one_row_kernel<MX, BF16, false>, grid, kLayerThreads, most_hidden, st, a, maps);
        else launch_chained(halves ? layer_hidden_kernel<MX, BF16, MX> : layer_hidden_kernel<MX, BF16, false>, grid, kLayerThreads, most_hidden, st, a, maps);
    }
    {
        LaunchScope ls(h, K_LAYER_DOWN, st);
        // Shares of the hidden units, of 256 at least: so many that there is a CTA per SM, which then has one or two, all at once.  With twice as many
        // there are two waves, and more to add up: 32 experts of 1,024 channels and 4,096 units 173.9 us instead of 167.5, of 2,560 units 128.6 instead of 121.5,
        // of 512 and 2,048 75.1 and 75.1; in 4 bits 159.5 instead of 167.5, 118.3 instead of 115.2 and 69.3 instead of 69.7.
        const int tiles = (a.C + kLayerWarps * 32 - 1) / (kLayerWarps * 32);
        while (a.shares < kMaxShares && tiles * experts * a.shares < h->num_sms && a.H >= 2 * a.shares * 256 && 2 * a.shares * a.n * a.k <= kPartRows)
            a.shares *= 2;
        plan(a.H / a.shares, a.C, 32, pass_rows(DOWN));
        // Where the CTAs fill the SMs, the few experts with more rows than a pass get CTAs for a second one, which the others' leave at once: one CTA
        // with both would be the last by far.  us for the layer so and without, means of eight choices of experts: 32 of 1,024 channels and 4,096 units 167.2 and
        // 173.5 (188 where an expert has 25 rows), in 4 bits 160.9 and 173.5; 28 experts of 512 channels and 3,584 units 95.2 and 102.3; 16 of 1,024
        // and 4,864, of 32 rows on average, 164.0 and 171.8.  With rarer ones, up to 8 rows on average, or SMs to spare it gains nothing: 8 experts of 1,024
        // channels and units, 64 rows, 31.6 and 30.8.
        if (a.passes == 1 && a.split_log == 0 && a.n > pass_rows(DOWN) && 3 * a.n * a.k > pass_rows(DOWN) * a.E) a.passes = 2;
        a.last_adds = a.n * a.k * a.shares <= kLastAdds;
        launch_chained(MX && a.split_log ? layer_down_kernel<MX, BF16, MX> : layer_down_kernel<MX, BF16, false>, dim3((unsigned)a.shares, (unsigned)a.tiles, (unsigned)(a.passes * experts)), kLayerThreads, most_down, st, a, maps);
    }
    if (!a.last_adds) {
        LaunchScope ls(h, K_LAYER_SUM, st);
        launch_chained(layer_sum_kernel<BF16>, dim3((unsigned)(a.n * a.C / 4 + kLayerThreads - 1) / kLayerThreads), kLayerThreads, 0, st, a);
    }
    return cudaGetLastError();
}

int run_layer(emc2_bridge* h, LayerArgs a, int type, bool mx, cudaStream_t st) {
    if (!h || a.n < 0 || a.n > kMaxLayerRows || a.C < 8 || a.C > kMaxRowChannels || (a.C & 7) || a.H < 8 || a.H > kMaxLayerHidden || (a.H & 7))
        return EMC2_ERR_INVALID_ARG;
    if (a.E < 1 || a.E > kMaxLayerExperts || a.k < 1 || a.k > kMaxChoices || a.k > a.E) return EMC2_ERR_INVALID_ARG;
    if ((type != EMC2_BF16 && type != EMC2_F16) || (a.act != EMC2_ACT_SILU && a.act != EMC2_ACT_GELU)) return EMC2_ERR_INVALID_ARG;
    if (!on_16_bytes(a.x) || !on_16_bytes(a.y) || !on_4_bytes(a.count) || !a.w_router || !on_16_bytes(a.w_router) || !on_4_bytes(a.b_router) ||
        !on_4_bytes(a.ids) || !on_4_bytes(a.weights))
        return EMC2_ERR_INVALID_ARG;
    for (int i = 0; i < 3; ++i)
        if (!a.w[i] || !on_16_bytes(a.w[i]) || (mx && !a.scales[i])) return EMC2_ERR_INVALID_ARG;
    if (a.n == 0) return EMC2_OK;
    if (!a.x || !a.y || !a.ids || !a.weights || a.x == a.y) return EMC2_ERR_INVALID_ARG;
    const RowsScratch& r = h->rows_scratch;
    if (!r.slab || a.C > r.max_channels || a.H > r.max_hidden) return EMC2_ERR_TOO_LARGE;
    RowsDevice device(h->cfg.device);
    if (!device.ok) return EMC2_ERR_CUDA;
    a.status = h->d_status;
    a.notes = static_cast<LayerNotes*>(r.notes);
    char* at = static_cast<char*>(r.slab);
    a.hidden = at;
    at += up256((size_t)kMaxSlots * 2 * a.H * 2);
    a.part = reinterpret_cast<float*>(at);
    a.tiles = a.shares = a.passes = 1;
    const cudaError_t e = type == EMC2_BF16 ? (mx ? launch_layer<true, true>(h, a, st) : launch_layer<false, true>(h, a, st))
                                            : (mx ? launch_layer<true, false>(h, a, st) : launch_layer<false, false>(h, a, st));
    return check_cuda(h, e);
}

}  // namespace

size_t layer_notes_bytes() { return up256(sizeof(LayerNotes)); }
size_t layer_scratch_bytes(int max_channels, int max_hidden) {
    if (max_hidden <= 0) return 0;
    return up256((size_t)kMaxSlots * 2 * max_hidden * 2) + (size_t)kPartRows * max_channels * sizeof(float);
}

}  // namespace emc2

using namespace emc2;

extern "C" int emc2_expert_layer(emc2_bridge_t* h, int32_t n, int32_t channels, int32_t hidden, int32_t experts, int32_t choices, int32_t type,
                                 int32_t act, const void* d_x, const int32_t* d_count, const float* d_w_router, const float* d_b_router,
                                 const void* d_w_gate, const void* d_w_up, const void* d_w_down, void* d_y, int32_t* d_ids, float* d_weights,
                                 void* cuda_stream) {
    LayerArgs a = {};
    a.x = d_x; a.count = d_count; a.w_router = d_w_router; a.b_router = d_b_router; a.y = d_y; a.ids = d_ids; a.weights = d_weights;
    a.w[0] = d_w_gate; a.w[1] = d_w_up; a.w[2] = d_w_down;
    a.n = n; a.C = channels; a.H = hidden; a.E = experts; a.k = choices; a.act = act;
    return run_layer(h, a, type, false, static_cast<cudaStream_t>(cuda_stream));
}

extern "C" int emc2_expert_layer_mx4(emc2_bridge_t* h, int32_t n, int32_t channels, int32_t hidden, int32_t experts, int32_t choices, int32_t type,
                                     int32_t act, const void* d_x, const int32_t* d_count, const float* d_w_router, const float* d_b_router,
                                     const uint8_t* d_gate_codes, const uint8_t* d_gate_scales, const uint8_t* d_up_codes,
                                     const uint8_t* d_up_scales, const uint8_t* d_down_codes, const uint8_t* d_down_scales, void* d_y,
                                     int32_t* d_ids, float* d_weights, void* cuda_stream) {
    LayerArgs a = {};
    a.x = d_x; a.count = d_count; a.w_router = d_w_router; a.b_router = d_b_router; a.y = d_y; a.ids = d_ids; a.weights = d_weights;
    a.w[0] = d_gate_codes; a.w[1] = d_up_codes; a.w[2] = d_down_codes;
    a.scales[0] = d_gate_scales; a.scales[1] = d_up_scales; a.scales[2] = d_down_scales;
    a.n = n; a.C = channels; a.H = hidden; a.E = experts; a.k = choices; a.act = act;
    return run_layer(h, a, type, true, static_cast<cudaStream_t>(cuda_stream));
}
