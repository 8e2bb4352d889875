// What follows an expert's block: its result normed, dropped out, gated, scaled and added to the rows, and the norm before the
// next block; and the gradients of all that.
//
//   h = (f - m) r, m = mean(f), r = 1 / sqrt(mean((f - m)^2) + eps)     (h = f without the norm behind the block)
//   o = x + s_e gate k (h w_e + b_e),     k = 1 / (1 - p) or 0 per element, see dropout.cuh
//   y = (o - m') r' w'_e + b'_e
//
//   do = d out + r' (g - mean(g) - h' mean(g h')), g = dy w', h' = (o - m') r'          dx = do
//   q = gate k do:  d gate = sum_c s k do (h w + b);  df = r (g - mean(g) - h mean(g h)), g = q s w
//   with S1 = sum q and S2 = sum q h over an expert's rows:  dw = s S2,  db = s S1,  ds = w S2 + b S1
//   dw' = sum dy h',  db' = sum dy
//
// Bound by memory: every row is read and written once, in the registers of a group of lanes.  The five parameter gradients need four
// sums.  Sums, means and statistics are held in fp32; y is normed from the unrounded o; out, y, dx and df are rounded once.
#include <algorithm>

#include "dropout.cuh"

namespace emc2 {
namespace {

constexpr int kResThreads = 256;
constexpr int kResShared = 40 * 1024;        // of parameters; more are read through the L1 cache
constexpr int kParams = 5;
enum Param { POST_W = 0, POST_B, SCALE, PRE_W, PRE_B };

struct ResParams {
    const float* p[kParams];                 // [E][C]; null: ones for weights and the scale, zeros for biases
};

// Eight entries of a parameter at vector v of an expert's; `hi`: the second four are there.
__device__ __forceinline__ void param8(float (&f)[8], const float4* p, int v, bool hi, float missing) {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = missing;
    if (!p) return;
    const float4 a = p[v];
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
    if (hi) {
        const float4 b = p[v + 1];
        f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
}

struct ResArgs {
    RowSegments seg;
    FastDiv frame;                           // division by N
    const void* x;
    const void* f;
    const float* gate;                       // or null
    ResParams par;
    void* out;
    void* y;                                 // null without PRE_W
    float4* stats;                           // or null
    Dropout drop;
    float eps, inv_c;
    int nvec, log, type_x, type_f, type_y, shared;
};

template <int K, bool WIDE>
__global__ void __launch_bounds__(kResThreads, K <= 1 ? 4 : K <= 2 ? 3 : 2) residual_kernel(ResArgs a) {
    __shared__ int bounds[kMaxBounds];
    extern __shared__ float4 staged[];
    const float4* par[kParams];
    {
        float4* at = staged;
        const int vectors = a.seg.E * a.nvec;
#pragma unroll
        for (int i = 0; i < kParams; ++i) {
            par[i] = reinterpret_cast<const float4*>(a.par.p[i]);
            if (!a.shared || !par[i]) continue;
            for (int v = threadIdx.x; v < vectors; v += kResThreads) at[v] = __ldg(par[i] + v);
            par[i] = at;
            at += vectors;
        }
    }
    load_bounds(a.seg, bounds);
    const int lane = threadIdx.x & ((1 << a.log) - 1), E = a.seg.E;
    const uint32_t rows = (uint32_t)a.seg.B * a.seg.N, groups = (gridDim.x * kResThreads) >> a.log;
    const uint32_t sub = (threadIdx.x & 31) >> a.log, first = (blockIdx.x * kResThreads + threadIdx.x) >> a.log;
    DropoutSeed seed = {};
    if (a.drop.threshold) seed = dropout_seed(a.drop);
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
        Raw8 rx[K], rf[K];
#pragma unroll
        for (int i = 0; i < K; ++i) {
            const int v = 2 * (lane + (i << a.log));
            const size_t at = (size_t)row * a.nvec + v;
            rf[i] = request8<WIDE>(a.f, at, in && v < a.nvec, in && v + 1 < a.nvec, a.type_f);
            rx[i] = request8<WIDE>(a.x, at, in && v < a.nvec, in && v + 1 < a.nvec, a.type_x);
        }
        const float gate = in && a.gate ? __ldg(a.gate + row) : 1.0f;
        float o[K][8];
#pragma unroll
        for (int i = 0; i < K; ++i) floats8(o[i], rf[i], a.type_f);
        float m = 0.f, r = 1.f;
        if (a.par.p[POST_W]) {
            float s = 0.f, q = 0.f;
#pragma unroll
            for (int i = 0; i < K; ++i)
                s += ((o[i][0] + o[i][1]) + (o[i][2] + o[i][3])) + ((o[i][4] + o[i][5]) + (o[i][6] + o[i][7]));
            m = group_sum(s, a.log) * a.inv_c;
            // The variance from the differences: the squares of values far from zero would lose it.
#pragma unroll
            for (int i = 0; i < K; ++i) {
                const int v = 2 * (lane + (i << a.log));
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (v + j / 4 >= a.nvec) continue;
                    o[i][j] -= m;
                    q += o[i][j] * o[i][j];
                }
            }
            r = rsqrtf(group_sum(q, a.log) * a.inv_c + a.eps);
        }
        float s2 = 0.f;
#pragma unroll
        for (int i = 0; i < K; ++i) {
            const int v = 2 * (lane + (i << a.log));
            if (!in || v >= a.nvec) continue;
            const bool hi = WIDE || v + 1 < a.nvec;
            float w[8], c[8], x[8];
            param8(w, par[POST_W], e * a.nvec + v, hi, 1.f);
            param8(c, par[POST_B], e * a.nvec + v, hi, 0.f);
#pragma unroll
            for (int j = 0; j < 8; ++j) o[i][j] = o[i][j] * r * w[j] + c[j];
            if (a.drop.threshold) {
                const uint4 bits = dropout_bits(seed, row, (uint32_t)(v >> 1));
#pragma unroll
                for (int j = 0; j < 8; ++j) o[i][j] = dropout_keeps(bits, j, a.drop.threshold) ? o[i][j] * a.drop.factor : 0.f;
            }
            param8(w, par[SCALE], e * a.nvec + v, hi, 1.f);
            floats8(x, rx[i], a.type_x);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                o[i][j] = x[j] + w[j] * gate * o[i][j];
                if (WIDE || j < 4 || hi) s2 += o[i][j];
            }
            store8<WIDE>(a.out, (size_t)row * a.nvec + v, hi, o[i], a.type_x);
        }
        float m2 = 0.f, r2 = 1.f;
        if (a.par.p[PRE_W]) {
            m2 = group_sum(s2, a.log) * a.inv_c;
            float q = 0.f;
#pragma unroll
            for (int i = 0; i < K; ++i) {
                const int v = 2 * (lane + (i << a.log));
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (v + j / 4 >= a.nvec) continue;
                    o[i][j] -= m2;
                    q += o[i][j] * o[i][j];
                }
            }
            r2 = rsqrtf(group_sum(q, a.log) * a.inv_c + a.eps);
#pragma unroll
            for (int i = 0; i < K; ++i) {
                const int v = 2 * (lane + (i << a.log));
                if (!in || v >= a.nvec) continue;
                const bool hi = WIDE || v + 1 < a.nvec;
                float w[8], c[8];
                param8(w, par[PRE_W], e * a.nvec + v, hi, 1.f);
                param8(c, par[PRE_B], e * a.nvec + v, hi, 0.f);
#pragma unroll
                for (int j = 0; j < 8; ++j) o[i][j] = o[i][j] * r2 * w[j] + c[j];
                store8<WIDE>(a.y, (size_t)row * a.nvec + v, hi, o[i], a.type_y);
            }
        }
        if (lane == 0 && in && a.stats) a.stats[row] = make_float4(m, r, m2, r2);
    }
}

struct ResGradArgs {
    RowSegments seg;
    const void* o;                           // the new rows; null without PRE_W
    const void* f;
    const void* dout;                        // or null
    const void* dy;                          // null without PRE_W
    const float* gate;                       // or null
    ResParams par;
    const float4* stats;                     // null without both norms
    void* dx;
    void* df;
    float* dgate;                            // or null
    Dropout drop;
    float* part;                             // [gridDim.x + E][4][C]: S2, S1, dw', db' of a CTA's rows of an expert
    int* share;                              // [E][2]: first CTA with rows of the expert and the one behind the last
    float inv_c;
    int nvec, log, type_x, type_f, type_y;
};

// The rows are taken expert by expert, an equal run of them per CTA, which sums its rows of an expert before it goes to the next;
// entry i + e of `part` holds those of CTA i and expert e (along the run of all rows either i or e goes up, so no two share one).
// The sums stay in registers for rows of up to 256 channels (K = 1); wider rows, whose values alone fill the registers, have them
// in shared memory, an entry per warp and column that one lane adds to.
template <int K, bool WIDE>
__global__ void __launch_bounds__(kResThreads, K == 1 ? 2 : 1) residual_grad_kernel(ResGradArgs a) {
    constexpr bool kInShared = K > 1;
    constexpr int kWarps = kResThreads / 32;
    __shared__ int bounds[kMaxBounds];
    __shared__ int start[kMaxSegments + 1];
    __shared__ int run[2];
    extern __shared__ float4 sums[];         // [warps][4][nvec]
    load_bounds(a.seg, bounds);
    segment_starts(a.seg, bounds, 1, start);
    const int B = a.seg.B, E = a.seg.E, total = start[B * E], ctas = min((int)gridDim.x, total);
    if (blockIdx.x == 0 && threadIdx.x < E) {
        const long long from = start[threadIdx.x * B], to = start[(threadIdx.x + 1) * B];
        a.share[2 * threadIdx.x] = from < to ? (int)(((from + 1) * ctas - 1) / total) : 0;
        a.share[2 * threadIdx.x + 1] = from < to ? (int)((to * ctas - 1) / total) + 1 : 0;
    }
    if ((int)blockIdx.x >= ctas) return;
    if (threadIdx.x < 2) run[threadIdx.x] = (int)((long long)total * (blockIdx.x + threadIdx.x) / ctas);
    __syncthreads();
    const int lanes = 1 << a.log, lane = threadIdx.x & (lanes - 1), warp = threadIdx.x >> 5;
    const int per_warp = 32 >> a.log, sub = (threadIdx.x & 31) >> a.log, step = kResThreads >> a.log;
    const bool pre = a.par.p[PRE_W] != nullptr, post = a.par.p[POST_W] != nullptr;
    DropoutSeed seed = {};
    if (a.drop.threshold) seed = dropout_seed(a.drop);
    float4* mine = sums + warp * 4 * a.nvec;
    for (int e = segment_of(start, B * E, run[0]) / B; e < E && start[e * B] < run[1]; ++e) {
        const int from = max(run[0], start[e * B]), to = min(run[1], start[(e + 1) * B]);
        if (from >= to) continue;
        const float4* par[kParams];
#pragma unroll
        for (int i = 0; i < kParams; ++i) par[i] = a.par.p[i] ? reinterpret_cast<const float4*>(a.par.p[i]) + e * a.nvec : nullptr;
        float acc[kInShared ? 1 : 4][8];
        if (kInShared) {
            for (int v = threadIdx.x; v < kWarps * 4 * a.nvec; v += kResThreads) sums[v] = make_float4(0.f, 0.f, 0.f, 0.f);
            __syncthreads();
        } else {
#pragma unroll
            for (int i = 0; i < (kInShared ? 1 : 4); ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[i][j] = 0.f;
        }
        auto add = [&](int plane, int i, int v, bool hi, const float (&t)[8]) {
            if (!kInShared) {
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[kInShared ? 0 : plane][j] += t[j];
                return;
            }
            float4* at = mine + plane * a.nvec + v;
            float4 s = at[0];
            at[0] = make_float4(s.x + t[0], s.y + t[1], s.z + t[2], s.w + t[3]);
            if (!hi) return;
            s = at[1];
            at[1] = make_float4(s.x + t[4], s.y + t[5], s.z + t[6], s.w + t[7]);
        };
        int q = e * B;
        // A warp goes on while any of its groups has a row.
        for (int p = from + warp * per_warp + sub; p - sub < to; p += step) {
            const bool in = p < to;
            uint32_t row = 0;
            if (in) {
                while (p >= start[q + 1]) ++q;                    // p < start[(e + 1) * B]
                const int b = q - e * B;
                row = (uint32_t)(b * a.seg.N + bounds[b * (E + 1) + e] + (p - start[q]));
            }
            Raw8 ro[K], rf[K], rd[K], ry[K];
#pragma unroll
            for (int i = 0; i < K; ++i) {
                const int v = 2 * (lane + (i << a.log));
                const bool lo = in && v < a.nvec, hi = in && v + 1 < a.nvec;
                const size_t at = (size_t)row * a.nvec + v;
                if (pre) {
                    ro[i] = request8<WIDE>(a.o, at, lo, hi, a.type_x);
                    ry[i] = request8<WIDE>(a.dy, at, lo, hi, a.type_y);
                }
                rd[i] = request8<WIDE>(a.dout, at, lo && a.dout, hi && a.dout, a.type_x);
                rf[i] = request8<WIDE>(a.f, at, lo, hi, a.type_f);
            }
            float4 st = make_float4(0.f, 1.f, 0.f, 1.f);
            if (in && a.stats) st = __ldg(a.stats + row);
            const float gate = in && a.gate ? __ldg(a.gate + row) : 1.0f;
            float d[K][8];
#pragma unroll
            for (int i = 0; i < K; ++i) floats8(d[i], rd[i], a.type_x);
            if (pre) {
                float o[K][8], g[K][8], s = 0.f, t = 0.f;
#pragma unroll
                for (int i = 0; i < K; ++i) {
                    const int v = 2 * (lane + (i << a.log));
                    floats8(o[i], ro[i], a.type_x);
                    floats8(g[i], ry[i], a.type_y);
                    if (!in || v >= a.nvec) continue;
                    const bool hi = WIDE || v + 1 < a.nvec;
                    float w[8];
                    add(3, i, v, hi, g[i]);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        o[i][j] = (o[i][j] - st.z) * st.w;
                        if (!WIDE && j >= 4 && !hi) o[i][j] = 0.f;
                        w[j] = g[i][j] * o[i][j];
                    }
                    add(2, i, v, hi, w);
                    param8(w, par[PRE_W], v, hi, 0.f);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        g[i][j] *= w[j];
                        s += g[i][j];
                        t += g[i][j] * o[i][j];
                    }
                }
                s = group_sum(s, a.log) * a.inv_c;
                t = group_sum(t, a.log) * a.inv_c;
#pragma unroll
                for (int i = 0; i < K; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) d[i][j] += st.w * (g[i][j] - s - o[i][j] * t);
            }
            float h[K][8], s = 0.f, t = 0.f, u = 0.f;
#pragma unroll
            for (int i = 0; i < K; ++i) {
                const int v = 2 * (lane + (i << a.log));
                floats8(h[i], rf[i], a.type_f);
                if (!in || v >= a.nvec) continue;
                const bool hi = WIDE || v + 1 < a.nvec;
                store8<WIDE>(a.dx, (size_t)row * a.nvec + v, hi, d[i], a.type_x);
                uint4 bits = make_uint4(0u, 0u, 0u, 0u);
                if (a.drop.threshold) bits = dropout_bits(seed, row, (uint32_t)(v >> 1));
                float w[8], c[8];
                param8(w, par[POST_W], v, hi, 1.f);
                param8(c, par[POST_B], v, hi, 0.f);
                float sc[8], k[8];
                param8(sc, par[SCALE], v, hi, 1.f);
                // What is dropped passes nothing on, whatever it holds.
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const bool kept = (!a.drop.threshold || dropout_keeps(bits, j, a.drop.threshold)) && (WIDE || j < 4 || hi);
                    h[i][j] = (h[i][j] - st.x) * st.y;
                    const float through = kept ? (a.drop.threshold ? d[i][j] * a.drop.factor : d[i][j]) : 0.f;
                    u += kept ? sc[j] * through * (h[i][j] * w[j] + c[j]) : 0.f;
                    d[i][j] = through * gate;
                    k[j] = kept ? d[i][j] * h[i][j] : 0.f;
                }
                add(1, i, v, hi, d[i]);
                add(0, i, v, hi, k);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    d[i][j] *= sc[j] * w[j];
                    if (!WIDE && j >= 4 && !hi) h[i][j] = 0.f;
                    s += d[i][j];
                    t += d[i][j] * h[i][j];
                }
            }
            if (post) {
                s = group_sum(s, a.log) * a.inv_c;
                t = group_sum(t, a.log) * a.inv_c;
            }
            if (a.dgate) {
                u = group_sum(u, a.log);
                if (in && lane == 0) a.dgate[row] = u;
            }
#pragma unroll
            for (int i = 0; i < K; ++i) {
                const int v = 2 * (lane + (i << a.log));
                if (!in || v >= a.nvec) continue;
                if (post) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) d[i][j] = st.y * (d[i][j] - s - h[i][j] * t);
                }
                store8<WIDE>(a.df, (size_t)row * a.nvec + v, WIDE || v + 1 < a.nvec, d[i], a.type_f);
            }
        }
        // The groups of a warp hold the same columns in the same lanes, then the warps' sums in their order.
        if (!kInShared) {
            const int v = 2 * lane;
#pragma unroll
            for (int i = 0; i < (kInShared ? 1 : 4); ++i) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    for (int w = lanes; w < 32; w <<= 1) acc[i][j] += __shfl_xor_sync(0xFFFFFFFFu, acc[i][j], w);
                if (sub == 0 && v < a.nvec) {
                    mine[i * a.nvec + v] = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
                    if (v + 1 < a.nvec) mine[i * a.nvec + v + 1] = make_float4(acc[i][4], acc[i][5], acc[i][6], acc[i][7]);
                }
            }
        }
        __syncthreads();
        float4* part = reinterpret_cast<float4*>(a.part) + (size_t)(blockIdx.x + e) * 4 * a.nvec;
        for (int v = threadIdx.x; v < 4 * a.nvec; v += kResThreads) {
            float4 o = sums[v];
            for (int w = 1; w < kWarps; ++w) {
                const float4 y = sums[w * 4 * a.nvec + v];
                o.x += y.x; o.y += y.y; o.z += y.z; o.w += y.w;
            }
            part[v] = o;
        }
        __syncthreads();
    }
}

struct ResSumArgs {
    const float* part;
    const int* share;
    ResParams par;
    float* grad[kParams];                    // each may be null
    int C;
};

// The entries of the CTAs that had rows of expert e, every eighth by one warp, then the warps' sums in their order; 32 columns per
// CTA, four sums each.
constexpr int kResSumThreads = 1024;
__global__ void __launch_bounds__(kResSumThreads) residual_sum_kernel(const __grid_constant__ ResSumArgs a) {
    await_predecessor();
    __shared__ float sum[32][32];
    const int e = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, plane = warp & 3, c = blockIdx.x * 32 + lane;
    const int i0 = a.share[2 * e], i1 = a.share[2 * e + 1];
    float s = 0.f;
    if (c < a.C) {
#pragma unroll 4
        for (int i = i0 + (warp >> 2); i < i1; i += 8) s += a.part[((size_t)(i + e) * 4 + plane) * a.C + c];
    }
    sum[warp][lane] = s;
    __syncthreads();
    if (warp < kParams && c < a.C && a.grad[warp]) {
        float t[4];
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            t[p] = sum[p][lane];
            for (int k = 1; k < 8; ++k) t[p] += sum[4 * k + p][lane];
        }
        const size_t at = (size_t)e * a.C + c;
        auto value = [&](int p, float missing) { return a.par.p[p] ? a.par.p[p][at] : missing; };
        float g = t[3];
        if (warp == POST_W) g = value(SCALE, 1.f) * t[0];
        if (warp == POST_B) g = value(SCALE, 1.f) * t[1];
        // Without the weights h is the block's result itself.
        if (warp == SCALE) g = value(POST_W, 1.f) * t[0] + value(POST_B, 0.f) * t[1];
        if (warp == PRE_W) g = t[2];
        a.grad[warp][at] = g;
    }
    release_successor();
}

template <int K>
struct Residual {
    static cudaError_t go(const ResArgs& a, bool wide, int ctas, size_t shared, cudaStream_t st) {
        if (wide) residual_kernel<K, true><<<ctas, kResThreads, shared, st>>>(a);
        else residual_kernel<K, false><<<ctas, kResThreads, shared, st>>>(a);
        return cudaSuccess;
    }
};
template <int K>
struct ResidualGrad {
    static cudaError_t go(const ResGradArgs& a, bool wide, int ctas, size_t shared, cudaStream_t st) {
        auto kernel = wide ? residual_grad_kernel<K, true> : residual_grad_kernel<K, false>;
        if (shared > 24 * 1024) {            // the sums of eight warps, four of up to 64 * K vectors each
            const cudaError_t e = allow_shared(kernel, (size_t)(kResThreads / 32) * 4 * 64 * K * sizeof(float4));
            if (e != cudaSuccess) return e;
        }
        kernel<<<ctas, kResThreads, shared, st>>>(a);
        return cudaSuccess;
    }
};

// Lanes of a row: groups of eight channels, one per lane up to 32 lanes, and vectors of them per lane.
RowSplit residual_split(int channels) { return row_split((channels + 7) / 8, 1); }

int residual_grad_ctas(const emc2_bridge* h, int per) { return (per == 1 ? 2 : 1) * h->num_sms; }
constexpr int kShareInts = 64;               // 2 * EMC2_MAX_EXPERTS and up to a multiple of 256 bytes

int check_residual(const emc2_bridge* h, int B, int N, int channels, int type_x, int type_f, int type_y, const void* f, const int32_t* offsets,
                   const float* gate, const ResParams& par, float p, const int64_t* seed) {
    if (!h || B < 0 || N < 0 || B > h->cfg.max_batch || N > h->cfg.max_points) return EMC2_ERR_INVALID_ARG;
    if (channels < 4 || channels > kMaxRowChannels || (channels & 3) || !is_type(type_x) || !is_type(type_f) || !is_type(type_y)) return EMC2_ERR_INVALID_ARG;
    for (int i = 0; i < kParams; ++i)
        if (!on_16_bytes(par.p[i])) return EMC2_ERR_INVALID_ARG;
    if ((par.p[POST_B] && !par.p[POST_W]) || (par.p[PRE_B] && !par.p[PRE_W])) return EMC2_ERR_INVALID_ARG;
    if (!is_share(p) || !on_8_bytes(seed) || (p > 0.0f && !seed)) return EMC2_ERR_INVALID_ARG;
    if (!on_16_bytes(f) || !on_4_bytes(offsets) || !on_4_bytes(gate)) return EMC2_ERR_INVALID_ARG;
    if (B > 0 && N > 0 && !f) return EMC2_ERR_INVALID_ARG;
    return EMC2_OK;
}

}  // namespace

size_t residual_scratch_bytes(const emc2_bridge* h, int max_channels) {
    return kShareInts * sizeof(int) + (size_t)(residual_grad_ctas(h, 1) + EMC2_MAX_EXPERTS) * 4 * max_channels * sizeof(float);
}

}  // namespace emc2

using namespace emc2;

extern "C" int emc2_expert_residual(emc2_bridge_t* h, int32_t B, int32_t N, int32_t channels, int32_t type_x, int32_t type_f, int32_t type_y,
                                    const void* d_x, const void* d_f, const int32_t* d_offsets, const float* d_gate,
                                    const float* d_post_weight, const float* d_post_bias, const float* d_scale, const float* d_pre_weight,
                                    const float* d_pre_bias, float eps, float p, const int64_t* d_seed, void* d_out, void* d_y,
                                    float* d_stats, void* cuda_stream) {
    const ResParams par = {{d_post_weight, d_post_bias, d_scale, d_pre_weight, d_pre_bias}};
    const int rc = check_residual(h, B, N, channels, type_x, type_f, type_y, d_f, d_offsets, d_gate, par, p, d_seed);
    if (rc != EMC2_OK) return rc;
    if (!on_16_bytes(d_x) || !on_16_bytes(d_out) || !on_16_bytes(d_y) || !on_16_bytes(d_stats) || !(eps >= 0.0f)) return EMC2_ERR_INVALID_ARG;
    if (B == 0 || N == 0) return EMC2_OK;
    if (!d_x || !d_out || (d_pre_weight != nullptr) != (d_y != nullptr)) return EMC2_ERR_INVALID_ARG;
    if (d_out == d_x || d_out == d_f || (d_y && (d_y == d_x || d_y == d_f || d_y == d_out))) return EMC2_ERR_INVALID_ARG;
    RowsDevice device(h->cfg.device);
    if (!device.ok) return EMC2_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    ResArgs a;
    a.seg = row_segments(h, B, N, d_offsets);
    a.frame = make_fast_div((uint32_t)N);
    a.x = d_x; a.f = d_f; a.gate = d_gate; a.par = par; a.out = d_out; a.y = d_y; a.stats = reinterpret_cast<float4*>(d_stats);
    a.drop = make_dropout(p, d_seed);
    a.eps = eps; a.inv_c = 1.0f / (float)channels; a.nvec = channels / 4; a.type_x = type_x; a.type_f = type_f; a.type_y = type_y;
    const RowSplit split = residual_split(channels);
    a.log = split.log;
    int given = 0;
    for (const float* q : par.p) given += q != nullptr;
    const size_t staged = (size_t)given * a.seg.E * channels * sizeof(float);
    a.shared = staged <= kResShared;
    const bool wide = is_wide(channels, type_x, d_x) && is_wide(channels, type_x, d_out) && is_wide(channels, type_f, d_f) &&
                      (!d_y || is_wide(channels, type_y, d_y));
    const long long rows = (long long)B * N, per_cta = kResThreads >> split.log;
    const int ctas = (int)std::min<long long>((rows + per_cta - 1) / per_cta, 8LL * h->num_sms);
    LaunchScope ls(h, K_RESIDUAL, st);
    const size_t shared = a.shared ? staged : 0;
    cudaError_t e;
    switch (split.per) {
        case 1: e = Residual<1>::go(a, wide, ctas, shared, st); break;
        case 2: e = Residual<2>::go(a, wide, ctas, shared, st); break;
        case 3: e = Residual<3>::go(a, wide, ctas, shared, st); break;
        default: e = Residual<4>::go(a, wide, ctas, shared, st);
    }
    return check_cuda(h, e != cudaSuccess ? e : cudaGetLastError());
}

extern "C" int emc2_expert_residual_grad(emc2_bridge_t* h, int32_t B, int32_t N, int32_t channels, int32_t type_x, int32_t type_f, int32_t type_y,
                                         const void* d_out, const void* d_f, const int32_t* d_offsets, const float* d_stats,
                                         const void* d_grad_out, const void* d_grad_y, const float* d_gate, const float* d_post_weight,
                                         const float* d_post_bias, const float* d_scale, const float* d_pre_weight, float p,
                                         const int64_t* d_seed, void* d_grad_x, void* d_grad_f, float* d_grad_gate,
                                         float* d_grad_post_weight, float* d_grad_post_bias, float* d_grad_scale,
                                         float* d_grad_pre_weight, float* d_grad_pre_bias, void* cuda_stream) {
    const ResParams par = {{d_post_weight, d_post_bias, d_scale, d_pre_weight, nullptr}};
    const int rc = check_residual(h, B, N, channels, type_x, type_f, type_y, d_f, d_offsets, d_gate, par, p, d_seed);
    if (rc != EMC2_OK) return rc;
    ResSumArgs t;
    t.par = par; t.C = channels;
    float* const grads[kParams] = {d_grad_post_weight, d_grad_post_bias, d_grad_scale, d_grad_pre_weight, d_grad_pre_bias};
    for (int i = 0; i < kParams; ++i) {
        t.grad[i] = grads[i];
        if (!on_4_bytes(grads[i])) return EMC2_ERR_INVALID_ARG;
    }
    if (!on_16_bytes(d_out) || !on_16_bytes(d_stats) || !on_16_bytes(d_grad_out) || !on_16_bytes(d_grad_y) || !on_16_bytes(d_grad_x) ||
        !on_16_bytes(d_grad_f) || !on_4_bytes(d_grad_gate))
        return EMC2_ERR_INVALID_ARG;
    // No gradients of what there is not.
    if ((!d_post_weight && (d_grad_post_weight || d_grad_post_bias)) || (!d_pre_weight && (d_grad_pre_weight || d_grad_pre_bias)) ||
        (!d_gate && d_grad_gate))
        return EMC2_ERR_INVALID_ARG;
    const bool empty = B == 0 || N == 0;
    if (!empty) {
        if (!d_grad_x || !d_grad_f || (d_pre_weight ? !d_out || !d_grad_y : !d_grad_out) || ((d_pre_weight || d_post_weight) && !d_stats)) return EMC2_ERR_INVALID_ARG;
        for (const void* q : {d_out, d_f, d_grad_out, d_grad_y})
            if (q && (q == d_grad_x || q == d_grad_f)) return EMC2_ERR_INVALID_ARG;
        if (d_grad_x == d_grad_f) return EMC2_ERR_INVALID_ARG;
    }
    if (!h->rows_scratch.slab || channels > h->rows_scratch.max_channels) return EMC2_ERR_TOO_LARGE;
    RowsDevice device(h->cfg.device);
    if (!device.ok) return EMC2_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const RowSegments seg = row_segments(h, B, N, d_offsets);
    if (empty) {
        for (float* g : grads)
            if (g) {
                const cudaError_t e = cudaMemsetAsync(g, 0, (size_t)seg.E * channels * sizeof(float), st);
                if (e != cudaSuccess) return check_cuda(h, e);
            }
        return EMC2_OK;
    }
    ResGradArgs a;
    a.seg = seg;
    a.o = d_out; a.f = d_f; a.dout = d_grad_out; a.dy = d_grad_y; a.gate = d_gate; a.par = par;
    a.stats = d_pre_weight || d_post_weight ? reinterpret_cast<const float4*>(d_stats) : nullptr;
    a.dx = d_grad_x; a.df = d_grad_f; a.dgate = d_grad_gate; a.drop = make_dropout(p, d_seed);
    a.share = static_cast<int*>(h->rows_scratch.slab);
    a.part = reinterpret_cast<float*>(a.share + kShareInts);
    a.inv_c = 1.0f / (float)channels; a.nvec = channels / 4; a.type_x = type_x; a.type_f = type_f; a.type_y = type_y;
    t.part = a.part; t.share = a.share;
    const RowSplit split = residual_split(channels);
    a.log = split.log;
    const bool wide = is_wide(channels, type_x, d_grad_x) && is_wide(channels, type_f, d_f) && is_wide(channels, type_f, d_grad_f) &&
                      (!d_grad_out || is_wide(channels, type_x, d_grad_out)) &&
                      (!d_pre_weight || (is_wide(channels, type_x, d_out) && is_wide(channels, type_y, d_grad_y)));
    const long long rows = (long long)B * N, per_cta = kResThreads >> split.log;
    const int ctas = (int)std::min<long long>((rows + per_cta - 1) / per_cta, residual_grad_ctas(h, split.per));
    const size_t shared = (size_t)(kResThreads / 32) * 4 * a.nvec * sizeof(float4);
    {
        LaunchScope ls(h, K_RESIDUAL_GRAD, st);
        cudaError_t e;
        switch (split.per) {
            case 1: e = ResidualGrad<1>::go(a, wide, ctas, shared, st); break;
            case 2: e = ResidualGrad<2>::go(a, wide, ctas, shared, st); break;
            case 3: e = ResidualGrad<3>::go(a, wide, ctas, shared, st); break;
            default: e = ResidualGrad<4>::go(a, wide, ctas, shared, st);
        }
        if (e != cudaSuccess) return check_cuda(h, e);
    }
    {
        LaunchScope ls(h, K_RESIDUAL_SUM, st);
        launch_chained(residual_sum_kernel, dim3((channels + 31) / 32, seg.E), kResSumThreads, 0, st, t);
    }
    return check_cuda(h, cudaGetLastError());
}
