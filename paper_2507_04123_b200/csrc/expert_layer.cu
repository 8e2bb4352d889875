// A whole mixture-of-experts layer for a few rows: router, choice, gated feed-forward of the chosen experts, weighted sum.
//
//   l = x w_router^T + b;  the k largest;  p = softmax over these
//   y = sum_j p_j (act(x w_gate[e_j]^T) * (x w_up[e_j]^T)) w_down[e_j]^T
//
// Bound by the weights of the experts that are asked for, which are read once: three kernels, each set up while the one before still
// runs.  The first has a CTA per row; the last of them to finish sorts the pairs (row, choice) by expert.  The second has a CTA per expert
// and tile of hidden units, the third per expert, tile of channels and share of the hidden units; the last CTA of a tile of channels adds up
// what all left for it, in the order of a row's choices.  In both, every warp streams its own rows of weights from memory into the registers
// of m16n8k16 products, whose 16 rows are the weights' and whose 8 columns are the rows at hand: a row of x more costs no
// more reading, and there are too few of them for larger products to help.
//
// The logits are summed in 64 bits, so that the choice does not depend on an order of summation; products in fp32; act(g) * u is rounded to
// the type, y once.
#include <algorithm>

#include "mx4.cuh"

namespace emc2 {
namespace {

constexpr int kLayerThreads = 256;
constexpr int kLayerWarps = kLayerThreads / 32;
constexpr int kMaxLayerRows = 128;
constexpr int kMaxLayerExperts = 256;
constexpr int kMaxChoices = 8;
constexpr int kMaxSlots = kMaxLayerRows * kMaxChoices;     // pairs (row, choice)
constexpr int kMaxLayerHidden = 8192;
constexpr int kPanel = 512;                  // elements of the rows at hand in shared memory at a time
constexpr int kRowsAtOnce = 32;
constexpr int kMaxShares = 8;                // of the hidden units in the third kernel
constexpr int kMaxTiles = 64;                // of channels, per counter

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
    void* hidden;                            // [sorted pair][H]
    float* part;                             // [share][sorted pair][C]
    int* status;
    int n, C, H, E, k, act;
    int split;                               // warps that share a tile, each with every split-th block
    int tiles;                               // CTAs per expert
    int shares;                              // third kernel: of the hidden units
};

__device__ __forceinline__ float type_float(const void* p, size_t i, bool bf16) {
    return bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]) : __half2float(static_cast<const __half*>(p)[i]);
}

// Numbers that ascend as the logits do; NaN below all.  0 is left for what has been taken.
__device__ __forceinline__ unsigned long long logit_key(double v) {
    if (v != v) return 1ull;
    const long long b = __double_as_longlong(v + 0.0);            // -0 counts as 0
    return b < 0 ? ~(unsigned long long)b : (unsigned long long)b | 0x8000000000000000ull;
}

// One CTA per row.
template <bool BF16>
__global__ void __launch_bounds__(kLayerThreads) layer_route_kernel(LayerArgs a) {
    __shared__ __align__(16) float x[kMaxRowChannels];
    __shared__ unsigned long long key[kMaxLayerExperts];
    __shared__ double logit[kMaxLayerExperts];
    __shared__ int last;
    const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int used = a.n;
    if (a.count) {
        used = *a.count;
        if (used < 0 || used > a.n) {
            if (row == 0 && tid == 0) atomicOr(a.status, kStatusBadRows);
            used = min(max(used, 0), a.n);
        }
    }
    if (row < used) {
        for (int i = tid; i < a.C; i += kLayerThreads) x[i] = type_float(a.x, (size_t)row * a.C + i, BF16);
        __syncthreads();
        for (int e = warp; e < a.E; e += kLayerWarps) {
            const float4* w = reinterpret_cast<const float4*>(a.w_router + (size_t)e * a.C);
            double s = 0.0, t = 0.0;
#pragma unroll 4
            for (int v = lane; v < a.C / 4; v += 32) {
                const float4 f = __ldg(w + v), g = *reinterpret_cast<const float4*>(x + 4 * v);
                s += (double)f.x * (double)g.x;
                t += (double)f.y * (double)g.y;
                s += (double)f.z * (double)g.z;
                t += (double)f.w * (double)g.w;
            }
            s += t;
#pragma unroll
            for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
            if (lane == 0) {
                if (a.b_router) s += (double)__ldg(a.b_router + e);
                logit[e] = s;
                key[e] = logit_key(s);
            }
        }
        __syncthreads();
        if (warp == 0) {
            double chosen = 0.0, top = 0.0;                       // lane j: logit of choice j
            int id = 0;
            for (int j = 0; j < a.k; ++j) {
                unsigned long long best = 0;
                int at = 0;
                for (int e = lane; e < a.E; e += 32)
                    if (key[e] > best) { best = key[e]; at = e; }
#pragma unroll
                for (int d = 16; d; d >>= 1) {
                    const unsigned long long other = __shfl_xor_sync(0xFFFFFFFFu, best, d);
                    const int o = __shfl_xor_sync(0xFFFFFFFFu, at, d);
                    if (other > best || (other == best && o < at)) { best = other; at = o; }
                }
                if (j == 0) top = logit[at];
                if (lane == j) { chosen = logit[at]; id = at; }
                if (lane == 0) key[at] = 0;
                __syncwarp();
            }
            const float q = lane < a.k ? expf((float)(chosen - top)) : 0.f;
            float s = q;
#pragma unroll
            for (int d = 4; d; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);      // eight choices at most
            if (lane < a.k) {
                a.ids[(size_t)row * a.k + lane] = id;
                a.weights[(size_t)row * a.k + lane] = q / s;
            }
        }
    }
    // The last CTA sorts the pairs: stable, by the counts of every expert in pieces of 32 pairs.
    __syncthreads();
    if (tid == 0) {
        __threadfence();
        last = atomicAdd(&a.notes->arrived, 1) == (int)gridDim.x - 1;
    }
    __syncthreads();
    release_successor();
    if (!last) return;
    __threadfence();
    __shared__ int of[kMaxSlots];
    __shared__ uint16_t piece[kMaxSlots / 32][kMaxLayerExperts];
    __shared__ int base[kMaxLayerExperts], warp_sum[2][kLayerWarps];
    const int pairs = used * a.k, pieces = (pairs + 31) / 32;
    for (int i = tid; i < pairs; i += kLayerThreads) of[i] = __ldcg(a.ids + i);
    for (int i = tid; i < pieces * kMaxLayerExperts / 2; i += kLayerThreads) reinterpret_cast<uint32_t*>(piece)[i] = 0u;
    __syncthreads();
    for (int p = warp; p < pieces; p += kLayerWarps) {
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
    if (tid == kLayerThreads - 1) {
        a.notes->active = rank;
        a.notes->used = used;
        a.notes->start[0] = 0;
        a.notes->arrived = 0;
    }
    __syncthreads();
    for (int p = warp; p < pieces; p += kLayerWarps) {
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
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Eight codes as four pairs of the type, by the bytes of the eight magnitudes.
template <bool BF16>
__device__ __forceinline__ void decode8(uint32_t (&r)[4], uint32_t codes) {
    constexpr uint32_t top_low = BF16 ? 0x3F3F3F00u : 0x3E3C3800u, top_high = BF16 ? 0x40404040u : 0x46444240u;
    constexpr uint32_t end_low = 0xC0800000u, end_high = 0xC0804000u;
    const uint32_t m = codes & 0x77777777u;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t at = m >> (16 * i), s = codes >> (16 * i);
        const uint32_t top = __byte_perm(top_low, top_high, at);
        const uint32_t end = BF16 ? __byte_perm(end_low, end_high, at) : 0u;
        r[2 * i] = __byte_perm(end, top, 0x5140) | (s << 12 & 0x00008000u) | (s << 24 & 0x80000000u);
        r[2 * i + 1] = __byte_perm(end, top, 0x7362) | (s << 4 & 0x00008000u) | (s << 16 & 0x80000000u);
    }
}

// A block of 32 elements of a product: lane (g, t) has elements 8t .. 8t + 7 of rows g and g + 8 of the weights and of row g of the rows at
// hand; which element stands at which place of an instruction does not matter, if both sides agree.
__device__ __forceinline__ uint4 load_weights(const void* p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

enum Stage { HIDDEN = 0, DOWN };

// Panels of the rows at hand, in two buffers: [row][kPanel] and 64 bytes more, so that the eight rows that lanes read together lie on
// different banks.
constexpr int kPanelStride = kPanel * 2 + 64;
constexpr int kPanelBytes = kRowsAtOnce * kPanelStride;

// What a warp's rows of weights are: two tiles of 16, of the gate's and the up projection's rows or of the down projection's.
template <int STAGE, bool MX, bool BF16, int NT>
__device__ __forceinline__ void layer_rows(const LayerArgs& a, char* smem, int e, int pair0, int rows) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int per_cta = kLayerWarps / a.split, part = warp % a.split, slot = warp / a.split;
    const int K = STAGE == HIDDEN ? a.C : a.H, M = STAGE == HIDDEN ? a.H : a.C;
    const int unit = blockIdx.x % a.tiles, tile = unit * per_cta + slot;        // of 16 hidden units, or of 32 channels
    // The third kernel's share of the hidden units, whole steps of the products; the last ones ragged.
    const int each = STAGE == HIDDEN ? K : ((K + a.shares - 1) / a.shares + 127) / 128 * 128;
    const int k0 = STAGE == HIDDEN ? 0 : min(K, (int)blockIdx.y * each), k1 = min(K, k0 + each);
    // The rows of weights that this lane reads: the first, in units of 16 bytes (all of a call's have fewer than 2^29), and how many of
    // those after every eighth there are.
    const int blocks = (K + kMxBlock - 1) / kMxBlock, units = MX ? blocks : K / 8, r0 = tile * (STAGE == HIDDEN ? 16 : 32) + g;
    const uint32_t w0 = (uint32_t)(e * M + r0) * (uint32_t)units;
    const int there = max(0, (M - r0 + 7) / 8);
    auto has = [&](int i) { return (STAGE == HIDDEN ? i & 1 : i) < there; };
    auto row_of = [&](int i) { return w0 + (uint32_t)((STAGE == HIDDEN ? i & 1 : i) * 8 * units); };
    auto weights_of = [&](int i) { return static_cast<const uint4*>(a.w[STAGE == HIDDEN ? i >> 1 : 2]); };
    auto scales_of = [&](int i) { return a.scales[STAGE == HIDDEN ? i >> 1 : 2]; };
    float acc[2][NT][4];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[m][n][c] = 0.f;
    // Copies a panel; what lies behind the rows or behind K is zero.
    const uint32_t panels = (uint32_t)__cvta_generic_to_shared(smem), mine_at = g * kPanelStride + t * 16;
    auto copy_panel = [&](int at, uint32_t to) {
        constexpr int chunks = kPanel / 8;
        for (int i = tid; i < 8 * NT * chunks; i += kLayerThreads) {
            const int r = i / chunks, c = i % chunks, k = at + c * 8;
            const bool in = r < rows && k < k1;
            const void* from = a.x;
            if (in) {
                if (STAGE == HIDDEN) from = static_cast<const char*>(a.x) + ((size_t)a.notes->row[pair0 + r] * a.C + k) * 2;
                else from = static_cast<const char*>(a.hidden) + ((size_t)(pair0 + r) * a.H + k) * 2;
            }
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + (uint32_t)(r * kPanelStride + c * 16)),
                         "l"(from), "r"(in ? 16 : 0) : "memory");
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto rows_at = [&](uint32_t panel, int block, int n) {
        uint4 v;
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                     : "r"(panel + (uint32_t)(n * 8 * kPanelStride + block * 64)));
        return v;
    };
    copy_panel(k0, panels);
    int buffer = 0;
    for (int p = k0; p < k1; p += kPanel, buffer ^= 1) {
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();                                          // the panel is there, and the other one is done with
        if (p + kPanel < k1) copy_panel(p + kPanel, panels + (buffer ^ 1) * kPanelBytes);
        const uint32_t panel = panels + buffer * kPanelBytes + mine_at;
        const int end = min(kPanel, k1 - p);
        if (!MX) {
            // Blocks of weights under way at once, as the registers have room.
            constexpr int kAtOnce = NT == 4 ? 3 : 4;
            for (int b = part * 32; b < end; b += a.split * 32 * kAtOnce) {
                uint4 v[kAtOnce][4];
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) {
                    const int k = b + u * a.split * 32 + t * 8;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        v[u][i] = make_uint4(0u, 0u, 0u, 0u);
                        if (has(i) && k < end) v[u][i] = load_weights(weights_of(i) + (row_of(i) + (uint32_t)(p + k) / 8));
                    }
                }
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) {
                    const int k = b + u * a.split * 32;
                    if (k >= end) break;
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const uint4 x = rows_at(panel, k >> 5, n);
#pragma unroll
                        for (int m = 0; m < 2; ++m) {
                            const uint4 &lo = v[u][2 * m], &hi = v[u][2 * m + 1];
                            product<BF16>(acc[m][n], lo.x, hi.x, lo.y, hi.y, x.x, x.y);
                            product<BF16>(acc[m][n], lo.z, hi.z, lo.w, hi.w, x.z, x.w);
                        }
                    }
                }
            }
        } else {
            // Four blocks to a step: lane t reads the codes of block t and passes them round the four lanes, so that each has its eight
            // elements of every block.
            for (int b = part * 128; b < end; b += a.split * 128) {
                const int block = (p + b) / kMxBlock;
                uint4 v[4];
                uint32_t powers = 0;                              // of block t, a byte for each of the four rows
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[i] = make_uint4(0u, 0u, 0u, 0u);
                    if (has(i) && block + t < blocks) v[i] = load_weights(weights_of(i) + (row_of(i) + (uint32_t)(block + t)));
                    if (has(i) && block + t < blocks) powers |= (uint32_t)__ldg(scales_of(i) + (row_of(i) + (uint32_t)(block + t))) << (8 * i);
                }
                uint32_t mine[4][4];                              // [row][block]
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t c[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
                    uint32_t got[4];                              // by the distance of the lane that it came from
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                        const int to = t ^ d;
                        const uint32_t out = to == 0 ? c[0] : to == 1 ? c[1] : to == 2 ? c[2] : c[3];
                        got[d] = d ? __shfl_xor_sync(0xFFFFFFFFu, out, d) : out;
                    }
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int d = q ^ t;
                        mine[i][q] = d == 0 ? got[0] : d == 1 ? got[1] : d == 2 ? got[2] : got[3];
                    }
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if (b + q * 32 >= end) break;
                    uint32_t r[4][4];
                    float s[4];
                    const uint32_t power = __shfl_sync(0xFFFFFFFFu, powers, (lane & 28) | q);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        decode8<BF16>(r[i], mine[i][q]);
                        s[i] = mx_power(power >> (8 * i) & 255u);
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const uint4 x = rows_at(panel, (b >> 5) + q, n);
#pragma unroll
                        for (int m = 0; m < 2; ++m) {
                            float c[4] = {0.f, 0.f, 0.f, 0.f};
                            product<BF16>(c, r[2 * m][0], r[2 * m + 1][0], r[2 * m][1], r[2 * m + 1][1], x.x, x.y);
                            product<BF16>(c, r[2 * m][2], r[2 * m + 1][2], r[2 * m][3], r[2 * m + 1][3], x.z, x.w);
                            acc[m][n][0] += s[2 * m] * c[0];
                            acc[m][n][1] += s[2 * m] * c[1];
                            acc[m][n][2] += s[2 * m + 1] * c[2];
                            acc[m][n][3] += s[2 * m + 1] * c[3];
                        }
                    }
                }
            }
        }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");         // an empty share has its panel of zeros under way
    // The warps' sums in shared memory, [warp][2][column][16]; those that share a tile are added in their order.
    __syncthreads();
    float* sums = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                sums[((warp * 2 + m) * (8 * NT) + n * 8 + 2 * t + (c & 1)) * 17 + g + (c >> 1) * 8] = acc[m][n][c];
    __syncthreads();
    const int width = STAGE == HIDDEN ? 16 : 32;
    for (int i = tid; i < per_cta * 8 * NT * width; i += kLayerThreads) {
        const int u = i % width, c = i / width % (8 * NT), s = i / (width * 8 * NT), at = (unit * per_cta + s) * width + u;
        if (c >= rows || at >= M) continue;
        auto sum = [&](int m, int r) {
            float v = 0.f;
            for (int q = 0; q < a.split; ++q) v += sums[(((s * a.split + q) * 2 + m) * (8 * NT) + c) * 17 + r];
            return v;
        };
        if (STAGE == HIDDEN) {
            const float gate = sum(0, u), up = sum(1, u);
            const float f = a.act == EMC2_ACT_SILU ? gate / (1.0f + expf(-gate)) : 0.5f * gate * erfcf(-0.70710678f * gate);
            const float h = f * up;
            const size_t to = (size_t)(pair0 + c) * a.H + at;
            if (BF16) static_cast<__nv_bfloat16*>(a.hidden)[to] = __float2bfloat16_rn(h);
            else static_cast<__half*>(a.hidden)[to] = __float2half_rn(h);
        } else {
            a.part[((size_t)blockIdx.y * (a.n * a.k) + pair0 + c) * a.C + at] = sum(u >> 4, u & 15);
        }
    }
    __syncthreads();
}

// The rows of the CTA's expert, 32 at a time, against its weights.
template <int STAGE, bool MX, bool BF16>
__device__ __forceinline__ void layer_unit(const LayerArgs& a, char* smem) {
    const int i = blockIdx.x / a.tiles;
    for (int p = a.notes->start[i]; p < a.notes->start[i + 1]; p += kRowsAtOnce) {
        const int e = a.notes->expert[i], rows = min(kRowsAtOnce, a.notes->start[i + 1] - p);
        if (rows <= 8) layer_rows<STAGE, MX, BF16, 1>(a, smem, e, p, rows);
        else if (rows <= 16) layer_rows<STAGE, MX, BF16, 2>(a, smem, e, p, rows);
        else layer_rows<STAGE, MX, BF16, 4>(a, smem, e, p, rows);
    }
}

template <bool MX, bool BF16>
__global__ void __launch_bounds__(kLayerThreads, 2) layer_hidden_kernel(LayerArgs a) {
    await_predecessor();
    extern __shared__ __align__(16) char panels[];
    if ((int)blockIdx.x < a.notes->active * a.tiles) layer_unit<HIDDEN, MX, BF16>(a, panels);
    release_successor();
}

template <bool MX, bool BF16>
__global__ void __launch_bounds__(kLayerThreads, 2) layer_down_kernel(LayerArgs a) {
    await_predecessor();
    extern __shared__ __align__(16) char panels[];
    __shared__ int last;
    if ((int)blockIdx.x >= a.notes->active * a.tiles) return;
    layer_unit<DOWN, MX, BF16>(a, panels);
    const int unit = blockIdx.x % a.tiles, tid = threadIdx.x;
    __syncthreads();
    if (tid == 0) {
        __threadfence();
        last = atomicAdd(&a.notes->arrived_tile[unit], 1) == a.notes->active * a.shares - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    const int width = min(a.C - unit * (kLayerWarps / a.split) * 32, (kLayerWarps / a.split) * 32), used = a.notes->used, pairs = a.n * a.k;
    for (int o = tid; o < used * width; o += kLayerThreads) {
        const int row = o / width, c = unit * (kLayerWarps / a.split) * 32 + o % width;
        float y = 0.f;
        for (int j = 0; j < a.k; ++j) {
            const int at = a.notes->place[row * a.k + j];
            float z = 0.f;
            for (int s = 0; s < a.shares; ++s) z += __ldcg(a.part + ((size_t)s * pairs + at) * a.C + c);
            y += a.weights[row * a.k + j] * z;
        }
        if (BF16) static_cast<__nv_bfloat16*>(a.y)[(size_t)row * a.C + c] = __float2bfloat16_rn(y);
        else static_cast<__half*>(a.y)[(size_t)row * a.C + c] = __float2half_rn(y);
    }
    if (tid == 0) a.notes->arrived_tile[unit] = 0;
}

// ---- scratch: notes, hidden values, partial sums
size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }
constexpr int kPartRows = 2 * kMaxSlots;     // shares times pairs, at most

template <bool MX, bool BF16>
cudaError_t launch_layer(emc2_bridge* h, LayerArgs a, cudaStream_t st) {
    constexpr size_t most = 2 * kPanelBytes;
    cudaError_t e = allow_shared(layer_hidden_kernel<MX, BF16>, most);
    if (e == cudaSuccess) e = allow_shared(layer_down_kernel<MX, BF16>, most);
    if (e != cudaSuccess) return e;
    const int experts = std::min(a.E, a.n * a.k);
    const int step = MX ? 128 : 32;
    // Warps that share a tile: as many as fill the SMs, and as have blocks.
    auto plan = [&](int K, int M, int width) {
        const int blocks = (K + step - 1) / step, most_split = std::min(kPanel / step, kLayerWarps);
        a.split = 1;
        for (;; a.split *= 2) {
            const int per = kLayerWarps / a.split * width;
            a.tiles = (M + per - 1) / per;
            if (a.tiles * experts >= 2 * h->num_sms || 2 * a.split > most_split || a.split >= blocks) break;
        }
    };
    {
        LaunchScope ls(h, K_LAYER_ROUTE, st);
        layer_route_kernel<BF16><<<a.n, kLayerThreads, 0, st>>>(a);
    }
    {
        LaunchScope ls(h, K_LAYER_HIDDEN, st);
        plan(a.C, a.H, 16);
        launch_chained(layer_hidden_kernel<MX, BF16>, dim3((unsigned)(a.tiles * experts)), kLayerThreads, most, st, a);
    }
    {
        LaunchScope ls(h, K_LAYER_DOWN, st);
        plan(a.H, a.C, 32);
        a.shares = 1;
        while (a.shares < kMaxShares && a.tiles * experts * a.shares < 4 * h->num_sms && a.H >= 2 * a.shares * 256 &&
               2 * a.shares * a.n * a.k <= kPartRows)
            a.shares *= 2;
        launch_chained(layer_down_kernel<MX, BF16>, dim3((unsigned)(a.tiles * experts), (unsigned)a.shares), kLayerThreads, most, st, a);
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
    a.hidden = r.slab;
    a.part = reinterpret_cast<float*>(static_cast<char*>(r.slab) + up256((size_t)kMaxSlots * a.H * 2));
    a.split = a.tiles = a.shares = 1;
    const cudaError_t e = type == EMC2_BF16 ? (mx ? launch_layer<true, true>(h, a, st) : launch_layer<false, true>(h, a, st))
                                            : (mx ? launch_layer<true, false>(h, a, st) : launch_layer<false, false>(h, a, st));
    return check_cuda(h, e);
}

}  // namespace

size_t layer_notes_bytes() { return up256(sizeof(LayerNotes)); }
size_t layer_scratch_bytes(int max_channels, int max_hidden) {
    if (max_hidden <= 0) return 0;
    return up256((size_t)kMaxSlots * max_hidden * 2) + (size_t)kPartRows * max_channels * sizeof(float);
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
