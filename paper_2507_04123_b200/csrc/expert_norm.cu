// Layer norm of dispatched rows with a weight and a bias per expert, and its gradients.
//
//   m = mean(x), r = 1 / sqrt(mean((x - m)^2) + eps), h = (x - m) r, y = h w_e + b_e
//   g = dy w_e:  dx = r (g - mean(g) - h mean(g h)),  dw_e = sum dy h,  db_e = sum dy   over the expert's rows
//
// Bound by memory: a row is read once, held in the registers of a group of lanes (see row_split), and written once.  The
// weights are read from shared memory, so that registers are left for enough warps to keep the loads in flight.
// Sums, means and gradients of the parameters are held in fp32; y and dx are rounded once.
#include <algorithm>

#include "rows.cuh"

namespace emc2 {
namespace {

constexpr int kNormThreads = 256;
constexpr int kNormShared = 24 * 1024;       // of weights; more are read through the L1 cache

struct NormArgs {
    RowSegments seg;
    FastDiv frame;               // division by N
    const void* x;
    const float* weight;
    const float* bias;           // or null
    void* y;
    float* mean;                 // or null
    float* rstd;                 // or null
    float eps, inv_c;
    int nvec, log, type_x, type_y, shared;
};

// Weights (and biases) of all experts in shared memory, or where they are.  The caller synchronises the CTA.
__device__ __forceinline__ void stage_weights(const float* w, const float* bias, int vectors, bool shared, float4* at, const float4*& ws, const float4*& bs) {
    ws = reinterpret_cast<const float4*>(w);
    bs = reinterpret_cast<const float4*>(bias);
    if (!shared) return;
    for (int i = threadIdx.x; i < vectors; i += blockDim.x) {
        at[i] = ws[i];
        if (bias) at[vectors + i] = bs[i];
    }
    ws = at;
    if (bias) bs = at + vectors;
}

// Rows in the caller's order, one per group of lanes and step.  1.2 million rows of 80 channels, fp32 to bf16: 105 us, 5.6 TB/s
// of the rows read and written (133 us with the weights in registers).
template <int K>
__global__ void __launch_bounds__(kNormThreads, K <= 2 ? 6 : K <= 4 ? 4 : K <= 6 ? 3 : 2) norm_kernel(NormArgs a) {
    __shared__ int bounds[kMaxBounds];
    extern __shared__ float4 weights[];
    const float4 *ws, *bs;
    stage_weights(a.weight, a.bias, a.seg.E * a.nvec, a.shared, weights, ws, bs);
    load_bounds(a.seg, bounds);
    const int lane = threadIdx.x & ((1 << a.log) - 1);
    const uint32_t rows = (uint32_t)a.seg.B * a.seg.N, groups = (gridDim.x * kNormThreads) >> a.log;
    const uint32_t sub = (threadIdx.x & 31) >> a.log, first = (blockIdx.x * kNormThreads + threadIdx.x) >> a.log;
    const int E = a.seg.E;
    // All groups of a warp make the same number of steps: the sums are taken by the whole warp.
    for (uint32_t r0 = first - sub; r0 < rows; r0 += groups) {
        const uint32_t row = r0 + sub;
        int e = E;
        if (row < rows) {
            uint32_t b, j;
            a.frame.divmod(row, b, j);
            const int* of = bounds + b * (E + 1);
            if ((int)j >= of[0]) {
                e = 0;
                while (e < E && (int)j >= of[e + 1]) ++e;
            }
        }
        const bool in = e < E;
        float4 x[K];
        load_row<K>(x, a.x, (size_t)row * a.nvec, lane, a.log, in ? a.nvec : 0, a.type_x);
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < K; ++i) s += (x[i].x + x[i].y) + (x[i].z + x[i].w);
        const float m = group_sum(s, a.log) * a.inv_c;
        // The variance from the differences: the squares of values far from zero would lose it.
        float q = 0.f;
#pragma unroll
        for (int i = 0; i < K; ++i) {
            if (lane + (i << a.log) >= a.nvec) continue;
            x[i].x -= m; x[i].y -= m; x[i].z -= m; x[i].w -= m;
            q += (x[i].x * x[i].x + x[i].y * x[i].y) + (x[i].z * x[i].z + x[i].w * x[i].w);
        }
        const float r = rsqrtf(group_sum(q, a.log) * a.inv_c + a.eps);
        if (!in) continue;
#pragma unroll
        for (int i = 0; i < K; ++i) {
            const int v = lane + (i << a.log);
            if (v >= a.nvec) continue;
            const float4 w = ws[e * a.nvec + v];
            float4 o = make_float4(x[i].x * r * w.x, x[i].y * r * w.y, x[i].z * r * w.z, x[i].w * r * w.w);
            if (a.bias) {
                const float4 c = bs[e * a.nvec + v];
                o.x += c.x; o.y += c.y; o.z += c.z; o.w += c.w;
            }
            store_row4(a.y, (size_t)row * a.nvec + v, o, a.type_y);
        }
        if (lane == 0) {
            if (a.mean) a.mean[row] = m;
            if (a.rstd) a.rstd[row] = r;
        }
    }
}

struct NormGradArgs {
    RowSegments seg;
    const void* x;
    const void* dy;
    const float* weight;
    const float* mean;
    const float* rstd;
    void* dx;
    float* part;                 // [gridDim.x + E][2][C]: sums of dw and db of a CTA's rows of an expert
    int* share;                  // [E][2]: first CTA with rows of the expert and the one behind the last
    float inv_c;
    int nvec, log, type_x, type_y;
};

// The rows are taken expert by expert, an equal run of them per CTA: a CTA meets few experts, and sums the parameters'
// gradients of each in registers.  Entry i + e of `part` holds those of CTA i and expert e: along the run of all rows
// either i or e goes up, so no two share an entry.  Rows and sums fill the registers, so
// that few warps have loads in flight, which is what it waits for: 960,000 rows of 64 fp32 channels 117 us, 5.3 TB/s of the rows.
template <int K>
__global__ void __launch_bounds__(kNormThreads, K <= 2 ? 3 : K <= 4 ? 2 : 1) norm_grad_kernel(NormGradArgs a) {
    __shared__ int bounds[kMaxBounds];
    __shared__ int start[kMaxSegments + 1];
    extern __shared__ float4 sums[];             // [warps][2][nvec]
    __shared__ float4 ws[kMaxRowChannels / 4];
    // A warp's next rows are requested before it works on these, where the registers of two CTAs per SM, or else of one, allow it
    // (us for 100,000 rows of 256 fp32 channels 57.8, without 68.4; of 1,024 225 and 253; of 512, where it would cost the
    // second CTA, 142 and 114).
    constexpr bool kAhead = K != 4;
    load_bounds(a.seg, bounds);
    segment_starts(a.seg, bounds, 1, start);
    // CTA i has rows total * i / ctas .. total * (i + 1) / ctas - 1 of the run of all rows, one at least.
    const int B = a.seg.B, E = a.seg.E, total = start[B * E], ctas = min((int)gridDim.x, total);
    if (blockIdx.x == 0 && threadIdx.x < E) {
        const long long from = start[threadIdx.x * B], to = start[(threadIdx.x + 1) * B];
        a.share[2 * threadIdx.x] = from < to ? (int)(((from + 1) * ctas - 1) / total) : 0;
        a.share[2 * threadIdx.x + 1] = from < to ? (int)((to * ctas - 1) / total) + 1 : 0;
    }
    if ((int)blockIdx.x >= ctas) return;
    // Ends of the CTA's run, in shared memory for want of registers.
    __shared__ int run[2];
    if (threadIdx.x < 2) run[threadIdx.x] = (int)((long long)total * (blockIdx.x + threadIdx.x) / ctas);
    __syncthreads();
    const int lanes = 1 << a.log, lane = threadIdx.x & (lanes - 1), warp = threadIdx.x >> 5;
    const int per_warp = 32 >> a.log, sub = (threadIdx.x & 31) >> a.log, step = kNormThreads >> a.log;
    for (int e = segment_of(start, B * E, run[0]) / B; e < E && start[e * B] < run[1]; ++e) {
        const int from = max(run[0], start[e * B]), to = min(run[1], start[(e + 1) * B]);
        if (from >= to) continue;
        float4 dw[K], db[K];
        __syncthreads();                                          // the weights of the expert before are done with
        for (int v = threadIdx.x; v < a.nvec; v += kNormThreads) ws[v] = __ldg(reinterpret_cast<const float4*>(a.weight) + e * a.nvec + v);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < K; ++i) {
            dw[i] = db[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
        int q = e * B;
        uint4 next_x[K], next_g[K];
        float next_m = 0.f, next_r = 0.f;
        uint32_t next_row = 0;                                    // 2^24 rows at most
        auto request = [&](int p) {
            int n = 0;                                            // vectors of the row, none behind the last
            if (p < to) {
                n = a.nvec;
                while (p >= start[q + 1]) ++q;                    // p < start[(e + 1) * B]
                const int b = q - e * B;
                next_row = (uint32_t)(b * a.seg.N + bounds[b * (E + 1) + e] + (p - start[q]));
                next_m = __ldg(a.mean + next_row);
                next_r = __ldg(a.rstd + next_row);
            }
            request_row<K>(next_x, a.x, (size_t)next_row * a.nvec, lane, a.log, n, a.type_x);
            request_row<K>(next_g, a.dy, (size_t)next_row * a.nvec, lane, a.log, n, a.type_y);
        };
        int p = from + warp * per_warp + sub;                     // the group's; a warp goes on while any of its groups has one
        if (kAhead) request(p);
        while (p - sub < to) {
            if (!kAhead) request(p);
            const bool in = p < to;
            const uint32_t row = next_row;
            const float m = next_m, r = next_r;
            uint4 raw_x[K], raw_g[K];
#pragma unroll
            for (int i = 0; i < K; ++i) { raw_x[i] = next_x[i]; raw_g[i] = next_g[i]; }
            p += step;
            if (kAhead) request(p);
            float4 x[K], g[K];
#pragma unroll
            for (int i = 0; i < K; ++i) { x[i] = row_floats(raw_x[i], a.type_x); g[i] = row_floats(raw_g[i], a.type_y); }
            float s = 0.f, t = 0.f;
#pragma unroll
            for (int i = 0; i < K; ++i) {
                if (!in || lane + (i << a.log) >= a.nvec) continue;
                x[i].x = (x[i].x - m) * r; x[i].y = (x[i].y - m) * r; x[i].z = (x[i].z - m) * r; x[i].w = (x[i].w - m) * r;
                dw[i].x += g[i].x * x[i].x; dw[i].y += g[i].y * x[i].y; dw[i].z += g[i].z * x[i].z; dw[i].w += g[i].w * x[i].w;
                db[i].x += g[i].x; db[i].y += g[i].y; db[i].z += g[i].z; db[i].w += g[i].w;
                const float4 w = ws[lane + (i << a.log)];
                g[i].x *= w.x; g[i].y *= w.y; g[i].z *= w.z; g[i].w *= w.w;
                s += (g[i].x + g[i].y) + (g[i].z + g[i].w);
                t += (g[i].x * x[i].x + g[i].y * x[i].y) + (g[i].z * x[i].z + g[i].w * x[i].w);
            }
            s = group_sum(s, a.log) * a.inv_c;
            t = group_sum(t, a.log) * a.inv_c;
            if (!in) continue;
#pragma unroll
            for (int i = 0; i < K; ++i) {
                const int v = lane + (i << a.log);
                if (v >= a.nvec) continue;
                const float4 o = make_float4(r * (g[i].x - s - x[i].x * t), r * (g[i].y - s - x[i].y * t),
                                             r * (g[i].z - s - x[i].z * t), r * (g[i].w - s - x[i].w * t));
                store_row4(a.dx, (size_t)row * a.nvec + v, o, a.type_x);
            }
        }
        // The groups of a warp hold the same columns in the same lanes, then the warps' sums in their order.
#pragma unroll
        for (int i = 0; i < K; ++i) {
            float* f = &dw[i].x;
            float* h = &db[i].x;
#pragma unroll
            for (int c = 0; c < 4; ++c)
                for (int d = lanes; d < 32; d <<= 1) {
                    f[c] += __shfl_xor_sync(0xFFFFFFFFu, f[c], d);
                    h[c] += __shfl_xor_sync(0xFFFFFFFFu, h[c], d);
                }
            const int v = lane + (i << a.log);
            if (sub == 0 && v < a.nvec) {
                sums[(warp * 2 + 0) * a.nvec + v] = dw[i];
                sums[(warp * 2 + 1) * a.nvec + v] = db[i];
            }
        }
        __syncthreads();
        float4* part = reinterpret_cast<float4*>(a.part) + (size_t)(blockIdx.x + e) * 2 * a.nvec;
        for (int v = threadIdx.x; v < 2 * a.nvec; v += kNormThreads) {
            float4 o = sums[v];
            for (int k = 1; k < kNormThreads / 32; ++k) {
                const float4 y = sums[k * 2 * a.nvec + v];
                o.x += y.x; o.y += y.y; o.z += y.z; o.w += y.w;
            }
            part[v] = o;
        }
        __syncthreads();
    }
}

struct NormSumArgs {
    const float* part;
    const int* share;
    float* dweight;
    float* dbias;                // or null
    int C;
};

// dw_e and db_e: the entries of the CTAs that had rows of expert e, every 32nd by one warp, then the warps' sums in their
// order; 32 columns per CTA.
constexpr int kNormSumThreads = 1024;
__global__ void __launch_bounds__(kNormSumThreads) norm_sum_kernel(NormSumArgs a) {
    await_predecessor();
    constexpr int kWarps = kNormSumThreads / 32;
    __shared__ float sum[kWarps][33];
    const int e = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;     // column of [dw | db]
    const int i0 = a.share[2 * e], i1 = a.share[2 * e + 1];
    float s = 0.f;
    if (c < 2 * a.C) {
#pragma unroll 4
        for (int i = i0 + warp; i < i1; i += kWarps) s += a.part[(size_t)(i + e) * 2 * a.C + c];
    }
    sum[warp][lane] = s;
    __syncthreads();
    // Warp w adds up column w: its lanes hold the warps' sums.
    float v = sum[lane][warp];
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    const int mine = blockIdx.x * 32 + warp;
    if (lane == 0 && mine < 2 * a.C) {
        if (mine < a.C) a.dweight[e * a.C + mine] = v;
        else if (a.dbias) a.dbias[e * a.C + mine - a.C] = v;
    }
    release_successor();
}

template <template <int> class F, typename... A>
cudaError_t by_vectors(int per, const A&... args) {
    switch (per) {
        case 1: return F<1>::go(args...);
        case 2: return F<2>::go(args...);
        case 3: return F<3>::go(args...);
        case 4: return F<4>::go(args...);
        case 5: return F<5>::go(args...);
        case 6: return F<6>::go(args...);
        case 7: return F<7>::go(args...);
        default: return F<8>::go(args...);
    }
}

template <int K>
struct Norm {
    static cudaError_t go(const NormArgs& a, int ctas, size_t shared, cudaStream_t st) {
        norm_kernel<K><<<ctas, kNormThreads, shared, st>>>(a);
        return cudaSuccess;
    }
};
template <int K>
struct NormGrad {
    static cudaError_t go(const NormGradArgs& a, int ctas, size_t shared, cudaStream_t st) {
        if (shared > 24 * 1024) {                // the sums of eight warps, two of up to 32 * K vectors each
            const cudaError_t e = allow_shared(norm_grad_kernel<K>, (size_t)(kNormThreads / 32) * 2 * 32 * K * sizeof(float4));
            if (e != cudaSuccess) return e;
        }
        norm_grad_kernel<K><<<ctas, kNormThreads, shared, st>>>(a);
        return cudaSuccess;
    }
};

// As many as are resident, see the kernel's launch bounds.
int norm_grad_ctas(const emc2_bridge* h, int per) { return (per <= 2 ? 3 : per <= 4 ? 2 : 1) * h->num_sms; }
constexpr int kShareInts = 64;               // 2 * EMC2_MAX_EXPERTS and up to a multiple of 256 bytes

int check_norm(const emc2_bridge* h, int B, int N, int channels, int type_x, int type_y, const void* x, const int32_t* offsets,
               const float* weight) {
    if (!h || B < 0 || N < 0 || B > h->cfg.max_batch || N > h->cfg.max_points) return EMC2_ERR_INVALID_ARG;
    if (channels < 4 || channels > kMaxRowChannels || (channels & 3) || !is_type(type_x) || !is_type(type_y)) return EMC2_ERR_INVALID_ARG;
    if (!weight || !on_16_bytes(weight) || !on_16_bytes(x)) return EMC2_ERR_INVALID_ARG;
    if (B > 0 && N > 0 && !x) return EMC2_ERR_INVALID_ARG;
    if (!on_4_bytes(offsets)) return EMC2_ERR_INVALID_ARG;
    return EMC2_OK;
}

}  // namespace

size_t norm_scratch_bytes(const emc2_bridge* h, int max_channels) {
    return kShareInts * sizeof(int) + (size_t)(norm_grad_ctas(h, 1) + EMC2_MAX_EXPERTS) * 2 * max_channels * sizeof(float);
}

}  // namespace emc2

using namespace emc2;

extern "C" int emc2_expert_norm(emc2_bridge_t* h, int32_t B, int32_t N, int32_t channels, int32_t type_x, int32_t type_y,
                                const void* d_x, const int32_t* d_offsets, const float* d_weight, const float* d_bias, float eps,
                                void* d_y, float* d_mean, float* d_rstd, void* cuda_stream) {
    const int rc = check_norm(h, B, N, channels, type_x, type_y, d_x, d_offsets, d_weight);
    if (rc != EMC2_OK) return rc;
    if (!on_16_bytes(d_bias) || !on_16_bytes(d_y) || !on_4_bytes(d_mean) || !on_4_bytes(d_rstd) || !(eps >= 0.0f)) return EMC2_ERR_INVALID_ARG;
    if (B == 0 || N == 0) return EMC2_OK;
    if (!d_y || d_y == d_x) return EMC2_ERR_INVALID_ARG;
    RowsDevice device(h->cfg.device);
    if (!device.ok) return EMC2_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    NormArgs a;
    a.seg = row_segments(h, B, N, d_offsets);
    a.frame = make_fast_div((uint32_t)N);
    a.x = d_x; a.weight = d_weight; a.bias = d_bias; a.y = d_y; a.mean = d_mean; a.rstd = d_rstd;
    a.eps = eps; a.inv_c = 1.0f / (float)channels; a.nvec = channels / 4; a.type_x = type_x; a.type_y = type_y;
    const RowSplit split = row_split(a.nvec, 8);
    a.log = split.log;
    const size_t weights = (size_t)(d_bias ? 2 : 1) * a.seg.E * channels * sizeof(float);
    a.shared = weights <= kNormShared;
    const long long rows = (long long)B * N, per_cta = kNormThreads >> split.log;
    const int ctas = (int)std::min<long long>((rows + per_cta - 1) / per_cta, 8LL * h->num_sms);
    LaunchScope ls(h, K_NORM, st);
    const cudaError_t e = by_vectors<Norm>(split.per, a, ctas, a.shared ? weights : 0, st);
    return check_cuda(h, e != cudaSuccess ? e : cudaGetLastError());
}

extern "C" int emc2_expert_norm_grad(emc2_bridge_t* h, int32_t B, int32_t N, int32_t channels, int32_t type_x, int32_t type_y,
                                     const void* d_x, const int32_t* d_offsets, const float* d_weight, const float* d_mean,
                                     const float* d_rstd, const void* d_grad_y, void* d_grad_x, float* d_grad_weight,
                                     float* d_grad_bias, void* cuda_stream) {
    const int rc = check_norm(h, B, N, channels, type_x, type_y, d_x, d_offsets, d_weight);
    if (rc != EMC2_OK) return rc;
    if (!d_grad_weight || !on_16_bytes(d_grad_y) || !on_16_bytes(d_grad_x) || !on_4_bytes(d_mean) || !on_4_bytes(d_rstd) ||
        !on_4_bytes(d_grad_weight) || !on_4_bytes(d_grad_bias))
        return EMC2_ERR_INVALID_ARG;
    const bool empty = B == 0 || N == 0;
    if (!empty && (!d_mean || !d_rstd || !d_grad_y || !d_grad_x || d_grad_x == d_x || d_grad_x == d_grad_y)) return EMC2_ERR_INVALID_ARG;
    if (!h->rows_scratch.slab || channels > h->rows_scratch.max_channels) return EMC2_ERR_TOO_LARGE;
    RowsDevice device(h->cfg.device);
    if (!device.ok) return EMC2_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const RowSegments seg = row_segments(h, B, N, d_offsets);
    if (empty) {
        const size_t bytes = (size_t)seg.E * channels * sizeof(float);
        cudaError_t e = cudaMemsetAsync(d_grad_weight, 0, bytes, st);
        if (e == cudaSuccess && d_grad_bias) e = cudaMemsetAsync(d_grad_bias, 0, bytes, st);
        return check_cuda(h, e);
    }
    NormGradArgs a;
    a.seg = seg;
    a.x = d_x; a.dy = d_grad_y; a.weight = d_weight; a.mean = d_mean; a.rstd = d_rstd; a.dx = d_grad_x;
    a.share = static_cast<int*>(h->rows_scratch.slab);
    a.part = reinterpret_cast<float*>(a.share + kShareInts);
    a.inv_c = 1.0f / (float)channels; a.nvec = channels / 4; a.type_x = type_x; a.type_y = type_y;
    const RowSplit split = row_split(a.nvec, 3);
    a.log = split.log;
    const long long rows = (long long)B * N, per_cta = kNormThreads >> split.log;
    const int ctas = (int)std::min<long long>((rows + per_cta - 1) / per_cta, norm_grad_ctas(h, split.per));
    NormSumArgs t;
    t.part = a.part; t.share = a.share; t.dweight = d_grad_weight; t.dbias = d_grad_bias; t.C = channels;
    {
        LaunchScope ls(h, K_NORM_GRAD, st);
        const cudaError_t e = by_vectors<NormGrad>(split.per, a, ctas, (size_t)(kNormThreads / 32) * 2 * a.nvec * sizeof(float4), st);
        if (e != cudaSuccess) return check_cuda(h, e);
    }
    {
        LaunchScope ls(h, K_NORM_SUM, st);
        launch_chained(norm_sum_kernel, dim3((2 * channels + 31) / 32, seg.E), kNormSumThreads, 0, st, t);
    }
    return check_cuda(h, cudaGetLastError());
}
