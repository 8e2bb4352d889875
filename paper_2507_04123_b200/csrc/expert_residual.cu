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
// Bound by memory: every row is read and written once, in the registers of a group of lanes, where the same steps one by one read or write
// it a dozen times.  The five parameter gradients need four
// sums.  Sums, means and statistics are held in fp32; y is normed from the unrounded o; out, y, dx and df are rounded once.
#include <algorithm>

#include "dropout.cuh"
#include "umma.cuh"

namespace emc2 {
namespace {

constexpr int kResThreads = 256;
constexpr int kResShared = 64 * 1024;        // of parameters; more are read through the L1 cache
// CTAs per SM.  Each stages the parameters and works out where its rows are, but few of them end unevenly.  us with 2, 4 and 8: 1.2 million rows
// of 80 channels, fp32 209, 192 and 193; 60,000 of 1,024, bf16 117, 127 and 144; 240,000 of 36, fp32 37, 40 and 46.
constexpr int kResGrid = 4;
constexpr int kParams = 5;
enum Param { POST_W = 0, POST_B, SCALE, PRE_W, PRE_B };

struct ResParams {
    const float* p[kParams];                 // [E][C]; null: ones for weights and the scale, zeros for biases
};

// What the kernels take of them: s w and s b of the block's side, and w' and b'; one vector, at v of all experts' rows.
enum Folded { SIDE_W = 0, SIDE_B, NEXT_W, NEXT_B, kFolded };
__device__ __forceinline__ float4 folded_param(const ResParams& par, int i, int v) {
    auto of = [&](const float* p, float missing) {
        return p ? __ldg(reinterpret_cast<const float4*>(p) + v) : make_float4(missing, missing, missing, missing);
    };
    if (i >= NEXT_W) return of(i == NEXT_W ? par.p[PRE_W] : par.p[PRE_B], 0.f);
    const float4 s = of(par.p[SCALE], 1.f), w = i == SIDE_W ? of(par.p[POST_W], 1.f) : of(par.p[POST_B], 0.f);
    return make_float4(s.x * w.x, s.y * w.y, s.z * w.z, s.w * w.w);
}

// The usual calls have kernels of their own, without the branches on what a call can lack, which were half of the instructions: both norms, a
// gradient from behind, rows of a multiple of eight channels, all bf16 or fp16, or fp32 with bf16 blocks.
enum Usual { ANY = 0, F32_ROWS, BF16_ROWS, F16_ROWS };
inline int usual_of(int type_x, int type_f, int type_y) {
    if (type_f != type_y) return ANY;
    if (type_f == EMC2_F16) return type_x == EMC2_F16 ? F16_ROWS : ANY;
    if (type_f != EMC2_BF16) return ANY;
    return type_x == EMC2_F32 ? F32_ROWS : type_x == EMC2_BF16 ? BF16_ROWS : ANY;
}
template <int U>
__device__ __forceinline__ int rows_type(int type) { return U == F32_ROWS ? EMC2_F32 : U == BF16_ROWS ? EMC2_BF16 : U == F16_ROWS ? EMC2_F16 : type; }
template <int U>
__device__ __forceinline__ int block_type(int type) { return U == ANY ? type : U == F16_ROWS ? EMC2_F16 : EMC2_BF16; }

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
    uint32_t params_bytes;                   // of the parameters in shared memory
};

// ---- A thread's next rows on their way to shared memory, in places that it alone reads.
template <int BYTES>
__device__ __forceinline__ void copy_ahead(uint32_t dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
}
// Eight elements take a slot of 16 bytes a thread, in fp32 two.
constexpr uint32_t kSlotBytes = kResThreads * 16;
template <bool WIDE, uint32_t SLOT = kSlotBytes>
__device__ __forceinline__ void ahead8(uint32_t dst, const void* p, uint32_t vec, bool hi, int type) {
    if (type == EMC2_F32) {
        copy_ahead<16>(dst, static_cast<const float4*>(p) + vec);
        if (WIDE || hi) copy_ahead<16>(dst + SLOT, static_cast<const float4*>(p) + vec + 1);
    } else if (WIDE) {
        copy_ahead<16>(dst, static_cast<const uint2*>(p) + vec);
    } else {
        copy_ahead<8>(dst, static_cast<const uint2*>(p) + vec);
        if (hi) copy_ahead<8>(dst + 8, static_cast<const uint2*>(p) + vec + 1);
    }
}
__device__ __forceinline__ Raw8 slot8(const char* at, int type) {
    Raw8 r;
    r.a = *reinterpret_cast<const uint4*>(at);
    r.b = type == EMC2_F32 ? *reinterpret_cast<const uint4*>(at + kSlotBytes) : make_uint4(0u, 0u, 0u, 0u);
    return r;
}
__device__ __forceinline__ void clear_second(Raw8& r, int type) {
    if (type == EMC2_F32) r.b = make_uint4(0u, 0u, 0u, 0u);
    else r.a.z = r.a.w = 0u;
}

// Rows in the caller's order, one per group of lanes and step, with few lanes and up to five groups of eight channels per lane: the
// more a lane requests at once, the more is in flight, and the fewer steps its four sums over the lanes take.  A row's copies are on their
// way while the one before is worked on and the generator runs.  1.2 million rows of 80 fp32 channels, a tenth dropped: 192 us, 6.1 TB/s, 93 % of a
// copy's rate.  60,000 of 1,024 bf16 channels: 127 us.
template <int K, bool WIDE, int U, bool DROP>
__global__ void __launch_bounds__(kResThreads, K <= 1 ? 4 : K <= 2 ? 3 : 2) residual_kernel(ResArgs a) {
    __shared__ int bounds[kMaxBounds];
    extern __shared__ float4 staged[];       // [kFolded][E][nvec] if they fit, then slots of the rows on their way
    const int E = a.seg.E, plane = E * a.nvec;
    const bool post = U || a.par.p[POST_W] != nullptr, pre = U || a.par.p[PRE_W] != nullptr, drop = U ? DROP : a.drop.any != 0;
    const bool shared = U || a.shared;
    const int type_x = rows_type<U>(a.type_x), type_f = block_type<U>(a.type_f), type_y = block_type<U>(a.type_y);
    if (shared)
        for (int i = 0; i < kFolded; ++i)
            for (int v = threadIdx.x; v < plane; v += kResThreads) staged[i * plane + v] = folded_param(a.par, i, v);
    load_bounds(a.seg, bounds);
    auto param8 = [&](float (&f)[8], int i, int v, bool hi) {
        const float4 p = shared ? staged[i * plane + v] : folded_param(a.par, i, v);
        float4 q = make_float4(0.f, 0.f, 0.f, 0.f);
        if (hi) q = shared ? staged[i * plane + v + 1] : folded_param(a.par, i, v + 1);
        f[0] = p.x; f[1] = p.y; f[2] = p.z; f[3] = p.w;
        f[4] = q.x; f[5] = q.y; f[6] = q.z; f[7] = q.w;
    };
    const int lane = threadIdx.x & ((1 << a.log) - 1);
    const uint32_t rows = (uint32_t)a.seg.B * a.seg.N, groups = (gridDim.x * kResThreads) >> a.log;
    const uint32_t sub = (threadIdx.x & 31) >> a.log, first = (blockIdx.x * kResThreads + threadIdx.x) >> a.log;
    DropoutSeed seed = {};
    if (drop) seed = dropout_seed(a.drop);
    const uint32_t f_slots = type_f == EMC2_F32 ? 2u : 1u, x_slots = type_x == EMC2_F32 ? 2u : 1u;
    char* const slots_f = reinterpret_cast<char*>(staged) + a.params_bytes + threadIdx.x * 16;
    char* const slots_x = slots_f + K * f_slots * kSlotBytes;
    auto expert_of = [&](uint32_t row) {                          // E: none
        if (row >= rows) return E;
        uint32_t b, j;
        a.frame.divmod(row, b, j);
        const int* of = bounds + b * (E + 1);
        if ((int)j < of[0]) return E;
        int e = 0;
        while (e < E && (int)j >= of[e + 1]) ++e;
        return e;
    };
    auto request = [&](char* slots, uint32_t per, const void* p, uint32_t row, int type, bool in) {
#pragma unroll
        for (int i = 0; i < K; ++i) {
            const int v = 2 * (lane + (i << a.log));
            if (in && (U || v < a.nvec)) ahead8<WIDE>((uint32_t)__cvta_generic_to_shared(slots + i * per * kSlotBytes), p, row * (uint32_t)a.nvec + v, v + 1 < a.nvec, type);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto taken = [&](float (&f)[8], const char* slots, uint32_t per, int i, int type, bool hi) {
        Raw8 raw = slot8(slots + i * per * kSlotBytes, type);
        if (!WIDE && !hi) clear_second(raw, type);
        floats8(f, raw, type);
    };
    int e_next = expert_of(first);
    request(slots_f, f_slots, a.f, first, type_f, e_next < E);
    request(slots_x, x_slots, a.x, first, type_x, e_next < E);
    // All groups of a warp make the same number of steps: the sums are taken by the whole warp.
    for (uint32_t r0 = first - sub; r0 < rows; r0 += groups) {
        const uint32_t row = r0 + sub, after = row + groups;
        const int e = e_next;
        const bool in = e < E;
        float gate = in && a.gate ? __ldg(a.gate + row) : 1.0f;
        e_next = expert_of(after);
        uint4 bits[K];                       // worked out while the rows are on their way
        if (drop) {
            uint32_t of[K], group[K];
#pragma unroll
            for (int i = 0; i < K; ++i) { of[i] = row; group[i] = (uint32_t)(lane + (i << a.log)); }
            dropout_bits(bits, seed, of, group);
            gate *= a.drop.factor;
        }
        asm volatile("cp.async.wait_group 1;" ::: "memory");
        float o[K][8];
#pragma unroll
        for (int i = 0; i < K; ++i) {
            const int v = 2 * (lane + (i << a.log));
#pragma unroll
            for (int j = 0; j < 8; ++j) o[i][j] = 0.f;
            if (in && (U || v < a.nvec)) taken(o[i], slots_f, f_slots, i, type_f, v + 1 < a.nvec);
        }
        request(slots_f, f_slots, a.f, after, type_f, e_next < E);
        float m = 0.f, r = 1.f;
        if (post) {
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
                    if (!U && v + (WIDE ? 0 : j / 4) >= a.nvec) continue;
                    o[i][j] -= m;
                    q += o[i][j] * o[i][j];
                }
            }
            r = rsqrtf(group_sum(q, a.log) * a.inv_c + a.eps);
        }
        float s2 = 0.f;
        asm volatile("cp.async.wait_group 1;" ::: "memory");
#pragma unroll
        for (int i = 0; i < K; ++i) {
            const int v = 2 * (lane + (i << a.log));
            if (!in || (!U && v >= a.nvec)) continue;
            const bool hi = WIDE || v + 1 < a.nvec;
            float w[8], c[8], x[8];
            param8(w, SIDE_W, e * a.nvec + v, hi);
            param8(c, SIDE_B, e * a.nvec + v, hi);
            taken(x, slots_x, x_slots, i, type_x, hi);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float t = x[j] + gate * (o[i][j] * r * w[j] + c[j]);
                o[i][j] = !drop || dropout_keeps(bits[i], j, a.drop.above) ? t : x[j];
                if (WIDE || j < 4 || hi) s2 += o[i][j];
            }
            store8<WIDE>(a.out, (size_t)row * a.nvec + v, hi, o[i], type_x);
        }
        request(slots_x, x_slots, a.x, after, type_x, e_next < E);
        float m2 = 0.f, r2 = 1.f;
        if (pre) {
            m2 = group_sum(s2, a.log) * a.inv_c;
            float q = 0.f;
#pragma unroll
            for (int i = 0; i < K; ++i) {
                const int v = 2 * (lane + (i << a.log));
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (!U && v + (WIDE ? 0 : j / 4) >= a.nvec) continue;
                    o[i][j] -= m2;
                    q += o[i][j] * o[i][j];
                }
            }
            r2 = rsqrtf(group_sum(q, a.log) * a.inv_c + a.eps);
#pragma unroll
            for (int i = 0; i < K; ++i) {
                const int v = 2 * (lane + (i << a.log));
                if (!in || (!U && v >= a.nvec)) continue;
                const bool hi = WIDE || v + 1 < a.nvec;
                float w[8], c[8];
                param8(w, NEXT_W, e * a.nvec + v, hi);
                param8(c, NEXT_B, e * a.nvec + v, hi);
#pragma unroll
                for (int j = 0; j < 8; ++j) o[i][j] = o[i][j] * r2 * w[j] + c[j];
                store8<WIDE>(a.y, (size_t)row * a.nvec + v, hi, o[i], type_y);
            }
        }
        if (lane == 0 && in && a.stats) a.stats[row] = make_float4(m, r, m2, r2);
    }
}

__device__ __forceinline__ uint4 lds128(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
    return v;
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
    int nvec, lanes, type_x, type_f, type_y; // lanes of a row, any number; more than 32 across a CTA
};

// Sums of N values over the lanes of a row's group, `l` a lane's place in it and `base` the warp's lane of its first; every
// lane gets them.  Any number of lanes: rows of 80 channels take ten, three of them a warp.
template <int N>
__device__ __forceinline__ void group_sums(float (&v)[N], int lanes, int l, int base) {
    if ((lanes & (lanes - 1)) == 0) {
        for (int d = 1; d < lanes; d <<= 1) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xFFFFFFFFu, v[i], d);
        }
        return;
    }
    for (int n = lanes; n > 1;) {
        const int half = (n + 1) >> 1;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float x = __shfl_down_sync(0xFFFFFFFFu, v[i], half);
            if (l + half < n) v[i] += x;
        }
        n = half;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = __shfl_sync(0xFFFFFFFFu, v[i], base);
}

// The same over a CTA, by way of `meet` [warps][N], which nobody reads behind the next barrier.
template <int N>
__device__ __forceinline__ void cta_sums(float (&v)[N], float (*meet)[6]) {
#pragma unroll
    for (int d = 16; d; d >>= 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xFFFFFFFFu, v[i], d);
    }
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) meet[threadIdx.x >> 5][i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = meet[0][i];
    for (int w = 1; w < (int)blockDim.x / 32; ++w) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += meet[w][i];
    }
}

// The run of rows that a CTA has, as a part of all rows expert by expert.  The first CTA notes which CTAs have rows of an expert.
// Called by a whole CTA; false: it has none.
__device__ __forceinline__ bool take_run(const ResGradArgs& a, int* bounds, int* start, int* run) {
    load_bounds(a.seg, bounds);
    segment_starts(a.seg, bounds, 1, start);
    const int B = a.seg.B, E = a.seg.E, total = start[B * E], ctas = min((int)gridDim.x, total);
    if (blockIdx.x == 0 && threadIdx.x < E) {
        const long long from = start[threadIdx.x * B], to = start[(threadIdx.x + 1) * B];
        a.share[2 * threadIdx.x] = from < to ? (int)(((from + 1) * ctas - 1) / total) : 0;
        a.share[2 * threadIdx.x + 1] = from < to ? (int)((to * ctas - 1) / total) + 1 : 0;
    }
    if ((int)blockIdx.x >= ctas) return false;
    if (threadIdx.x < 2) run[threadIdx.x] = (int)((long long)total * (blockIdx.x + threadIdx.x) / ctas);
    __syncthreads();
    return true;
}
// Rows at places of the run of an expert's rows, for ascending places.
struct RowAt {
    const int *bounds, *start;
    int N, E, e, b, until, shift;
    __device__ __forceinline__ RowAt(const ResGradArgs& a, const int* bounds_, const int* start_, int e_)
        : bounds(bounds_), start(start_ + e_ * a.seg.B), N(a.seg.N), E(a.seg.E), e(e_), b(-1), until(start[0]), shift(0) {}
    __device__ __forceinline__ uint32_t operator()(int p) {
        while (p >= until) {                                      // p is before the end of the expert's rows
            ++b;
            shift = b * N + bounds[b * (E + 1) + e] - start[b];
            until = start[b + 1];
        }
        return (uint32_t)(p + shift);
    }
};
// Sums of the warps, [warps][4][nvec], in their order to the entry of the CTA and expert.
template <int THREADS>
__device__ __forceinline__ void give_sums(const ResGradArgs& a, const float4* sums, int e) {
    __syncthreads();
    float4* part = reinterpret_cast<float4*>(a.part) + (size_t)(blockIdx.x + e) * 4 * a.nvec;
    for (int v = threadIdx.x; v < 4 * a.nvec; v += THREADS) {
        float4 o = sums[v];
        for (int w = 1; w < THREADS / 32; ++w) {
            const float4 y = sums[w * 4 * a.nvec + v];
            o.x += y.x; o.y += y.y; o.z += y.z; o.w += y.w;
        }
        part[v] = o;
    }
    __syncthreads();
}

// Contiguous bytes to shared memory; both on 16 bytes.
__device__ __forceinline__ void copy_bytes(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

// Rows with eight channels per lane: several in a warp, or (ACROSS, more than 256 channels) one across two to four warps, a CTA, whose sums
// meet in shared memory.  The rows are taken expert by expert, an equal run of them per CTA, which sums its rows of an
// expert before it goes to the next; entry i + e of `part` holds those of CTA i and expert e (along the run of all rows either i or e
// goes up, so no two share one).  The sums stay in registers; a group of lanes has two rows in work, whose waits for one another's lanes
// and for shared memory fill each other.  The next rows, which lie side by side within a frame, are on their way to shared memory, for
// which no registers are left, as one piece of every buffer (lane by lane, the copies' own way through the SM's memory pipe was what the kernel
// waited for: 147 us instead of 109).  Rows of four channels more than a multiple of eight need not begin on 16 bytes: their lanes copy their
// own.  480,000 rows of 64 fp32 channels, a tenth dropped: 109 us, 5.2 TB/s, with half of the issue slots of few warps, which the registers of sums and
// rows allow; 90,000 of 256 bf16 channels: 65 us; 28,000 of 1,024 fp32 channels 93 us, 5.6 TB/s (with a warp per row and its sums in shared memory
// 153), 60,000 of 512 bf16 channels 87 us (164).
constexpr int kGradThreads = 128;
// Ragged rows, and unusual calls across a CTA, have one row in work, and the registers for four CTAs: 120,000 rows of 132 bf16 channels 169 us, with
// two rows and two CTAs 222; 28,000 of 772, fp32, 138 and 177.  Others have two: 120,000 of 72, fp16 without kernels of its own, 64, with one 71.
__host__ __device__ constexpr int rows_at_once(bool wide, int usual, bool across) { return usual || (wide && !across) ? 2 : 1; }
constexpr int grad_ctas(bool wide, int usual, bool across) { return rows_at_once(wide, usual, across) == 1 ? 4 : 3; }      // per SM, as the registers have room
constexpr uint32_t kGradSlot = kGradThreads * 16;
template <bool WIDE, int U, bool DROP, bool ACROSS>
__global__ void __launch_bounds__(kGradThreads, grad_ctas(WIDE, U, ACROSS)) residual_grad_kernel(ResGradArgs a) {
    constexpr int R = rows_at_once(WIDE, U, ACROSS);
    constexpr int kTeams = ACROSS ? 1 : kGradThreads / 32;      // that have rows of their own: warps, or the CTA
    __shared__ int bounds[kMaxBounds];
    __shared__ int start[kMaxSegments + 1];
    __shared__ int run[2];
    __shared__ float4 folded[kFolded - 1][ACROSS ? 256 : 64];                    // the expert's s w, s b and w'
    __shared__ __align__(8) unsigned long long bars[kTeams][2];
    __shared__ float meet[ACROSS ? 2 : 1][kGradThreads / 32][6];
    __shared__ int gave_up;
    extern __shared__ float4 sums[];         // [teams][4][nvec], then two stages of the rows in work per group; across a CTA the latter only
    if (!take_run(a, bounds, start, run)) return;
    const int B = a.seg.B, E = a.seg.E;
    const int type_x = rows_type<U>(a.type_x), type_f = block_type<U>(a.type_f), type_y = block_type<U>(a.type_y);
    const int lanes = a.lanes, team = ACROSS ? 0 : threadIdx.x >> 5, per_warp = ACROSS ? 1 : 32 / lanes, chunk = R * per_warp;
    auto in_team = [] { return (int)(ACROSS ? threadIdx.x : threadIdx.x & 31); };
    // Threads behind the last lane of a row that takes warps read what that one reads, and count as zeros.
    const int sub = ACROSS ? 0 : in_team() / lanes, base = sub * lanes, l = ACROSS ? min(in_team(), lanes - 1) : in_team() - base;
    const bool lane_in = !ACROSS || in_team() < lanes;
    auto team_sync = [] {
        if (ACROSS) __syncthreads();
        else __syncwarp();
    };
    const bool pre = U || a.par.p[PRE_W] != nullptr, post = U || a.par.p[POST_W] != nullptr, behind = U || a.dout, noted = U || a.stats;
    const bool drop = U ? DROP : a.drop.any != 0, active = ACROSS ? lane_in : sub < per_warp, hi = WIDE || 2 * l + 1 < a.nvec;
    DropoutSeed seed = {};
    if (drop) seed = dropout_seed(a.drop);
    // Bytes of a row in each buffer, and where a stage of the warp has the buffer's rows; with copies by lanes, where it has a lane's
    // vectors, which are 16 bytes at the thread's number.
    auto slots = [](int type) { return type == EMC2_F32 ? 2u : 1u; };
    const uint32_t row_x = slots(type_x) * a.nvec * 8, row_y = slots(type_y) * a.nvec * 8, row_f = slots(type_f) * a.nvec * 8;
    const uint32_t at_y = pre ? (WIDE ? chunk * row_x : slots(type_x) * kGradSlot) : 0u;
    const uint32_t at_d = at_y + (pre ? (WIDE ? chunk * row_y : slots(type_y) * kGradSlot) : 0u);
    const uint32_t at_f = at_d + (behind ? (WIDE ? chunk * row_x : slots(type_x) * kGradSlot) : 0u);
    const uint32_t at_s = at_f + (WIDE ? chunk * row_f : slots(type_f) * kGradSlot);
    const uint32_t row_bytes = at_s + (noted ? (WIDE ? chunk * 16 : kGradSlot) : 0u);      // of a stage of the warp; by lanes, of a row
    const uint32_t ring_at = smem_u32(sums + (ACROSS ? 0 : kTeams * 4 * a.nvec)) + (WIDE ? team * 2 * row_bytes : threadIdx.x * 16), bar = smem_u32(bars[team]);
    if (WIDE) {
        if (threadIdx.x == 0) gave_up = 0;
        if (in_team() == 0) { bar_init(bar, 1); bar_init(bar + 8, 1); }
        fence_bar_init();
        fence_async_shared();
        __syncthreads();
    }
    const bool leads = in_team() == 0;
    const int place = min(sub, per_warp - 1);                     // lanes behind the last group read its row, for nothing
    uint32_t phases = 0;
    for (int e = segment_of(start, B * E, run[0]) / B; e < E && start[e * B] < run[1]; ++e) {
        const int from = max(run[0], start[e * B]), to = min(run[1], start[(e + 1) * B]);
        if (from >= to) continue;
        for (int v = threadIdx.x; v < a.nvec; v += blockDim.x)
            for (int i = SIDE_W; i <= NEXT_W; ++i) folded[i][v] = folded_param(a.par, i, e * a.nvec + v);
        __syncthreads();
        auto param8 = [&](float (&f)[8], int i) {
            const float4 x = folded[i][2 * l];
            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
            if (hi) y = folded[i][2 * l + 1];
            f[0] = x.x; f[1] = x.y; f[2] = x.z; f[3] = x.w;
            f[4] = y.x; f[5] = y.y; f[6] = y.z; f[7] = y.w;
        };
        float acc[4][8];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[i][j] = 0.f;
        RowAt row_at(a, bounds, start, e), ahead_at(a, bounds, start, e);
        uint32_t next[R] = {};                              // rows under way; with copies by lanes
        // The warp's rows from place p on; a lane's are p + sub and p + per_warp + sub.
        auto request = [&](int p, uint32_t stage) {
            uint32_t dst = ring_at + stage * (WIDE ? row_bytes : R * row_bytes);
            if (WIDE) {
                uint32_t dst_y = dst + at_y, dst_d = dst + at_d, dst_f = dst + at_f, dst_s = dst + at_s;
                if (p >= to) return;
                const int end = min(p + chunk, to);
                if (end - p < chunk) {                            // places without a row are zeros, which add nothing
                    auto clear = [&](uint32_t buffer, uint32_t bytes) {
                        for (uint32_t o = (uint32_t)(end - p) * bytes + in_team() * 16; o < chunk * bytes; o += (ACROSS ? blockDim.x : 32) * 16)
                            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(buffer + o), "r"(0u) : "memory");
                    };
                    if (pre) {
                        clear(dst, row_x);
                        clear(dst_y, row_y);
                    }
                    if (behind) clear(dst_d, row_x);
                    clear(dst_f, row_f);
                    if (noted) clear(dst_s, 16);
                    fence_async_shared();                         // before the next expert's copies
                    team_sync();
                }
                if (!leads) return;
                const uint32_t full = bar + stage * 8;
                bar_expect(1, full, (uint32_t)(end - p) * ((pre ? row_x + row_y : 0u) + (behind ? row_x : 0u) + row_f + (noted ? 16u : 0u)));
                do {                                              // one piece of every frame
                    const uint32_t row = ahead_at(p);
                    const uint32_t len = (uint32_t)(min(end, ahead_at.until) - p);
                    auto copy = [&](uint32_t to_bytes, const void* rows, uint32_t bytes) {
                        copy_bytes(to_bytes, static_cast<const char*>(rows) + (unsigned long long)row * bytes, len * bytes, full);
                    };
                    if (pre) {
                        copy(dst, a.o, row_x);
                        copy(dst_y, a.dy, row_y);
                    }
                    if (behind) copy(dst_d, a.dout, row_x);
                    copy(dst_f, a.f, row_f);
                    if (noted) copy(dst_s, a.stats, 16);
                    p += (int)len;
                    dst += len * row_x; dst_y += len * row_y; dst_d += len * row_x; dst_f += len * row_f; dst_s += len * 16;
                } while (p < end);
                return;
            }
#pragma unroll
            for (int k = 0; k < R; ++k, dst += row_bytes) {
                const int q = p + k * per_warp + sub;
                if (q >= to || !active) continue;
                const uint32_t row = next[k] = ahead_at(q);
                const uint32_t at = row * (uint32_t)a.nvec + 2 * l;             // 2^24 rows of 64 vectors at most
                if (pre) {
                    ahead8<WIDE, kGradSlot>(dst, a.o, at, hi, type_x);
                    ahead8<WIDE, kGradSlot>(dst + at_y, a.dy, at, hi, type_y);
                }
                if (behind) ahead8<WIDE, kGradSlot>(dst + at_d, a.dout, at, hi, type_x);
                ahead8<WIDE, kGradSlot>(dst + at_f, a.f, at, hi, type_f);
                if (noted) copy_ahead<16>(dst + at_s, a.stats + row);
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        uint32_t stage = 0;
        team_sync();
        request(from + team * chunk, 0);
        for (int p = from + team * chunk; p < to; p += kTeams * chunk) {
            bool in[R];
            uint32_t row[R];
            float gate[R];
#pragma unroll
            for (int k = 0; k < R; ++k) {
                in[k] = active && p + k * per_warp + sub < to;
                row[k] = !WIDE ? next[k] : in[k] ? row_at(p + k * per_warp + sub) : 0u;
                gate[k] = in[k] && a.gate ? __ldg(a.gate + row[k]) : 1.0f;
            }
            const uint32_t now = stage;
            const uint32_t at = ring_at + stage * (WIDE ? row_bytes : R * row_bytes);
            stage ^= 1;
            request(p + kTeams * chunk, stage);
            uint4 bits[R];
            if (drop) {                                           // while the rows are on their way
                uint32_t group[R];
#pragma unroll
                for (int k = 0; k < R; ++k) group[k] = (uint32_t)l;
                dropout_bits(bits, seed, row, group);
            }
            if (WIDE) {
                warp_wait(bar + now * 8, phases >> now & 1u, &gave_up, a.seg.status);
                phases ^= 1u << now;
            } else {
                asm volatile("cp.async.wait_group 1;" ::: "memory");
            }
            float d[R][8], h[R][8];
            float4 st[R];
            auto taken = [&](float (&f)[8], int k, uint32_t buffer, uint32_t bytes, int type) {
                Raw8 raw;
                if (WIDE) {
                    const uint32_t mine = at + buffer + (uint32_t)(k * per_warp + place) * bytes + (type == EMC2_F32 ? 32u : 16u) * l;
                    raw.a = lds128(mine);
                    if (type == EMC2_F32) raw.b = lds128(mine + 16);
                } else {
                    raw.a = raw.b = make_uint4(0u, 0u, 0u, 0u);
                    if (in[k]) {
                        raw.a = lds128(at + k * row_bytes + buffer);
                        if (type == EMC2_F32) raw.b = lds128(at + k * row_bytes + buffer + kGradSlot);
                    }
                    if (!hi) clear_second(raw, type);
                }
                floats8(f, raw, type);
            };
#pragma unroll
            for (int k = 0; k < R; ++k) {
                st[k] = make_float4(0.f, 1.f, 0.f, 1.f);
                if (noted && (WIDE || in[k])) {
                    const uint4 v = lds128(WIDE ? at + at_s + (uint32_t)(k * per_warp + place) * 16 : at + k * row_bytes + at_s);
                    st[k] = make_float4(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w));
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) d[k][j] = 0.f;
                if (behind) taken(d[k], k, at_d, row_x, type_x);
                taken(h[k], k, at_f, row_f, type_f);
            }
            if (pre) {
                float o[R][8], g[R][8], w[8], means[2 * R] = {};
                param8(w, NEXT_W);
#pragma unroll
                for (int k = 0; k < R; ++k) {
                    taken(o[k], k, 0, row_x, type_x);
                    taken(g[k], k, at_y, row_y, type_y);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        o[k][j] = (o[k][j] - st[k].z) * st[k].w;
                        if (!WIDE && j >= 4 && !hi) o[k][j] = 0.f;
                        if (ACROSS && !lane_in) o[k][j] = g[k][j] = 0.f;
                        acc[2][j] += g[k][j] * o[k][j];
                        acc[3][j] += g[k][j];
                        g[k][j] *= w[j];
                        means[k] += g[k][j];
                        means[R + k] += g[k][j] * o[k][j];
                    }
                }
                if (ACROSS) cta_sums(means, meet[0]);
                else group_sums(means, lanes, l, base);
#pragma unroll
                for (int k = 0; k < R; ++k) {
                    const float m = means[k] * a.inv_c, t = means[R + k] * a.inv_c;
#pragma unroll
                    for (int j = 0; j < 8; ++j) d[k][j] += st[k].w * ((g[k][j] - m) - o[k][j] * t);
                }
            }
            float w[8], means[3 * R] = {};
            param8(w, SIDE_W);
#pragma unroll
            for (int k = 0; k < R; ++k) {
                if (in[k]) store8<WIDE>(a.dx, (size_t)row[k] * a.nvec + 2 * l, hi, d[k], type_x);
                // What is dropped passes nothing on, whatever it holds; behind a norm no element of a row with NaN or infinities has a
                // value.
                if (drop) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        d[k][j] = dropout_keeps(bits[k], j, a.drop.above) ? d[k][j] : 0.f;
                        if (!post) h[k][j] = dropout_keeps(bits[k], j, a.drop.above) ? h[k][j] : 0.f;
                    }
                }
                if (post) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) h[k][j] = (h[k][j] - st[k].x) * st[k].y;
                }
                if (!WIDE && !hi) {
#pragma unroll
                    for (int j = 4; j < 8; ++j) d[k][j] = h[k][j] = 0.f;
                }
                if (ACROSS && !lane_in) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) d[k][j] = h[k][j] = 0.f;
                }
            }
            if (a.dgate) {
                float c[8];
                param8(c, SIDE_B);
#pragma unroll
                for (int k = 0; k < R; ++k)
#pragma unroll
                    for (int j = 0; j < 8; ++j) means[2 * R + k] += d[k][j] * (h[k][j] * w[j] + c[j]);
            }
#pragma unroll
            for (int k = 0; k < R; ++k) {
                const float through = drop ? a.drop.factor * gate[k] : gate[k];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    d[k][j] *= through;
                    acc[1][j] += d[k][j];
                    acc[0][j] += d[k][j] * h[k][j];
                    d[k][j] *= w[j];
                    means[k] += d[k][j];
                    means[R + k] += d[k][j] * h[k][j];
                }
            }
            if (post || a.dgate) {
                if (ACROSS) cta_sums(means, meet[ACROSS]);
                else group_sums(means, lanes, l, base);
            }
#pragma unroll
            for (int k = 0; k < R; ++k) {
                if (!in[k]) continue;
                if (a.dgate && l == 0) a.dgate[row[k]] = drop ? means[2 * R + k] * a.drop.factor : means[2 * R + k];
                if (post) {
                    const float m = means[k] * a.inv_c, t = means[R + k] * a.inv_c;
#pragma unroll
                    for (int j = 0; j < 8; ++j) d[k][j] = st[k].y * ((d[k][j] - m) - h[k][j] * t);
                }
                store8<WIDE>(a.df, (size_t)row[k] * a.nvec + 2 * l, hi, d[k], type_f);
            }
            team_sync();                                          // the stage has been read by all
        }
        if (ACROSS) {
            float4* part = reinterpret_cast<float4*>(a.part) + (size_t)(blockIdx.x + e) * 4 * a.nvec + 2 * l;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (!lane_in) break;
                part[i * a.nvec] = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
                if (hi) part[i * a.nvec + 1] = make_float4(acc[i][4], acc[i][5], acc[i][6], acc[i][7]);
            }
            continue;                                             // the rows of this expert are done with by all
        }
        // The groups of a warp hold the same columns at the same places.
        float4* mine = sums + team * 4 * a.nvec + 2 * l;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float total = acc[i][j];
                for (int w = 1; w < per_warp; ++w) total += __shfl_sync(0xFFFFFFFFu, acc[i][j], (l + w * lanes) & 31);
                acc[i][j] = total;
            }
            if (sub == 0) {
                mine[i * a.nvec] = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
                if (hi) mine[i * a.nvec + 1] = make_float4(acc[i][4], acc[i][5], acc[i][6], acc[i][7]);
            }
        }
        give_sums<kGradThreads>(a, sums, e);
    }
    if (WIDE) leave_after_timeout(&gave_up);
    else asm volatile("cp.async.wait_group 0;" ::: "memory");
}

struct ResSumArgs {
    const float* part;
    const int* share;
    ResParams par;
    float* grad[kParams];                    // each may be null
    int C;
};

// The entries of the CTAs that had rows of expert e, every eighth by one warp, then the warps' sums in their order; 32 columns per
// CTA, four sums each.  Bound by the wait for the entries, which the L2 holds: 2 us behind the gradients' kernel.
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
    template <typename F>
    static cudaError_t go(F kernel, const ResArgs& a, int ctas, size_t shared, cudaStream_t st) {
        if (shared > 24 * 1024) {
            const cudaError_t e = allow_shared(kernel, kResShared + K * 4 * kSlotBytes);
            if (e != cudaSuccess) return e;
        }
        kernel<<<ctas, kResThreads, shared, st>>>(a);
        return cudaSuccess;
    }
    static cudaError_t go(const ResArgs& a, bool wide, int usual, int ctas, cudaStream_t st) {
        auto slots = [](int type) { return type == EMC2_F32 ? 2 : 1; };
        const size_t shared = a.params_bytes + (size_t)K * (slots(a.type_x) + slots(a.type_f)) * kSlotBytes;
        if (usual == F32_ROWS)
            return a.drop.any ? go(residual_kernel<K, true, F32_ROWS, true>, a, ctas, shared, st) : go(residual_kernel<K, true, F32_ROWS, false>, a, ctas, shared, st);
        if (usual == BF16_ROWS)
            return a.drop.any ? go(residual_kernel<K, true, BF16_ROWS, true>, a, ctas, shared, st) : go(residual_kernel<K, true, BF16_ROWS, false>, a, ctas, shared, st);
        if (usual == F16_ROWS)
            return a.drop.any ? go(residual_kernel<K, true, F16_ROWS, true>, a, ctas, shared, st) : go(residual_kernel<K, true, F16_ROWS, false>, a, ctas, shared, st);
        return wide ? go(residual_kernel<K, true, ANY, true>, a, ctas, shared, st) : go(residual_kernel<K, false, ANY, true>, a, ctas, shared, st);
    }
};
// Warps of a row of more than 256 channels, which a CTA then has one at a time; 1: a warp has one or more.
int row_warps(int channels) { return (channels + 255) / 256; }
template <bool ACROSS>
cudaError_t launch_grad(const ResGradArgs& a, bool wide, int usual, int ctas, int threads, cudaStream_t st) {
    auto slots = [](int type) { return type == EMC2_F32 ? 2 : 1; };
    constexpr int teams = ACROSS ? 1 : kGradThreads / 32;
    const bool pre = a.par.p[PRE_W] != nullptr;
    const int n = (pre ? slots(a.type_x) + slots(a.type_y) : 0) + (a.dout ? slots(a.type_x) : 0) + slots(a.type_f);
    const size_t own = ACROSS ? 0 : (size_t)teams * 4 * a.nvec * sizeof(float4);
    // Two stages of the rows in work: per team of `chunk` rows, or per thread of its vectors and a row's statistics.
    const size_t at_once = rows_at_once(wide, usual, ACROSS), chunk = ACROSS ? at_once : at_once * (32 / a.lanes);
    const size_t stages = wide ? (size_t)teams * 2 * chunk * ((size_t)n * a.nvec * 8 + (a.stats ? 16 : 0)) : (size_t)2 * at_once * (n + (a.stats ? 1 : 0)) * kGradSlot;
    const size_t shared = own + stages;
    // 16 KB of sums and the two stages of four fp32 buffers and the statistics: of rows of eight channels, two in work, 64 of 144 bytes per warp.  Others
    // need less: lanes' vectors 9 slots of one row, rows across a CTA 16 KB and 16 bytes each, two at once, and no sums.
    constexpr size_t most = 16 * 1024 + 8 * 64 * 144;
    static_assert(2 * 9 * kGradSlot <= 8 * 64 * 144 && 2 * 2 * (16 * 1024 + 16) <= 8 * 64 * 144, "stages");
    static_assert(rows_at_once(false, ANY, false) == 1 && rows_at_once(false, ANY, true) == 1, "lanes' vectors of one row");
    auto kernel = wide ? residual_grad_kernel<true, ANY, true, ACROSS> : residual_grad_kernel<false, ANY, true, ACROSS>;
    if (usual == F32_ROWS) kernel = a.drop.any ? residual_grad_kernel<true, F32_ROWS, true, ACROSS> : residual_grad_kernel<true, F32_ROWS, false, ACROSS>;
    if (usual == BF16_ROWS) kernel = a.drop.any ? residual_grad_kernel<true, BF16_ROWS, true, ACROSS> : residual_grad_kernel<true, BF16_ROWS, false, ACROSS>;
    if (usual == F16_ROWS) kernel = a.drop.any ? residual_grad_kernel<true, F16_ROWS, true, ACROSS> : residual_grad_kernel<true, F16_ROWS, false, ACROSS>;
    if (shared > 24 * 1024) {
        const cudaError_t e = allow_shared(kernel, most);
        if (e != cudaSuccess) return e;
    }
    kernel<<<ctas, threads, shared, st>>>(a);
    return cudaSuccess;
}

// As many as the registers have room for.
int residual_grad_ctas(const emc2_bridge* h, int warps, bool wide, int usual) {
    const int full = grad_ctas(wide, usual, warps > 1);         // of kGradThreads
    return (warps == 1 ? full : full * (kGradThreads / 32) / warps) * h->num_sms;
}
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
    return kShareInts * sizeof(int) + (size_t)(residual_grad_ctas(h, 2, true, ANY) + EMC2_MAX_EXPERTS) * 4 * max_channels * sizeof(float);
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
    // Rows whose last group is half empty are accessed by 8 and 16 bytes, which few lanes that are far apart do worse: 240,000 rows of 36 fp32
    // channels by one lane each 49 us, by two 46.
    const RowSplit split = row_split((channels + 7) / 8, channels % 8 ? 3 : 5);
    a.log = split.log;
    const size_t staged = (size_t)kFolded * a.seg.E * channels * sizeof(float);
    a.shared = staged <= kResShared;
    const bool wide = is_wide(channels, type_x, d_x) && is_wide(channels, type_x, d_out) && is_wide(channels, type_f, d_f) &&
                      (!d_y || is_wide(channels, type_y, d_y));
    const long long rows = (long long)B * N, per_cta = kResThreads >> split.log;
    const int ctas = (int)std::min<long long>((rows + per_cta - 1) / per_cta, (long long)kResGrid * h->num_sms);
    LaunchScope ls(h, K_RESIDUAL, st);
    a.params_bytes = a.shared ? (uint32_t)staged : 0u;
    // Every lane of a row full, and the parameters in shared memory.
    const bool full = wide && a.shared && d_post_weight && d_pre_weight && (channels / 8) == split.per << split.log;
    const int usual = full ? usual_of(type_x, type_f, type_y) : ANY;
    cudaError_t e;
    switch (split.per) {
        case 1: e = Residual<1>::go(a, wide, usual, ctas, st); break;
        case 2: e = Residual<2>::go(a, wide, usual, ctas, st); break;
        case 3: e = Residual<3>::go(a, wide, usual, ctas, st); break;
        case 4: e = Residual<4>::go(a, wide, usual, ctas, st); break;
        default: e = Residual<5>::go(a, wide, usual, ctas, st);
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
    const int warps = row_warps(channels);
    a.lanes = (channels + 7) / 8;
    const bool wide = is_wide(channels, type_x, d_grad_x) && is_wide(channels, type_f, d_f) && is_wide(channels, type_f, d_grad_f) &&
                      (!d_grad_out || is_wide(channels, type_x, d_grad_out)) &&
                      (!d_pre_weight || (is_wide(channels, type_x, d_out) && is_wide(channels, type_y, d_grad_y)));
    const long long rows = (long long)B * N, per_cta = warps == 1 ? 2 * (kGradThreads / 32) * (32 / a.lanes) : 4;
    const int usual = wide && d_post_weight && d_pre_weight && d_grad_out ? usual_of(type_x, type_f, type_y) : ANY;
    const int ctas = (int)std::min<long long>((rows + per_cta - 1) / per_cta, residual_grad_ctas(h, warps, wide, usual));
    {
        LaunchScope ls(h, K_RESIDUAL_GRAD, st);
        const cudaError_t e = warps == 1 ? launch_grad<false>(a, wide, usual, ctas, kGradThreads, st) : launch_grad<true>(a, wide, usual, ctas, warps * 32, st);
        if (e != cudaSuccess) return check_cuda(h, e);
    }
    {
        LaunchScope ls(h, K_RESIDUAL_SUM, st);
        launch_chained(residual_sum_kernel, dim3((channels + 31) / 32, seg.E), kResSumThreads, 0, st, t);
    }
    return check_cuda(h, cudaGetLastError());
}
