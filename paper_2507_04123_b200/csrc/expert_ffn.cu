// Gated feed-forward block on dispatched rows, with weights per expert, and its gradients.
//
//   g = x Wg^T, u = x Wu^T, h = act(g) u, y = h Wd^T                       rows [., C], hidden width H
//   dh = dy Wd, dg = dh u act'(g), du = dh act(g), dx = dg Wg + du Wu
//   dWg = dg^T x, dWu = du^T x, dWd = dy^T h                               sums over the expert's rows
//
// All products run on the tensor cores (tcgen05, fp32 accumulators in TMEM).  Nothing of width H reaches device memory:
// tiles of 128 rows stay in shared memory while the hidden units pass by in chunks, whose weights are copied in beside the
// products.  What bounds the kernels are the products' own times at these widths and the activation beside them.  A product of
// 128 x N x 16 takes N / 2 clocks by its arithmetic; issued back to back it was measured at 45 clocks for N = 32, 49 for 64, 65
// for 128, 129 for 256, and at no less than 63 with A in TMEM.  So chunks are as wide as TMEM allows.  The hidden values go
// back to TMEM for the second product of y and dx, as its A, which leaves the shared memory to the copies; where TMEM is
// needed for wider chunks they go to shared memory.  What lies between the two products of a chunk (h, or dg and du) is
// rounded to the rows' type, as the tensor cores take it; all sums are held in fp32, results are rounded once.
//
// Warps of several kinds pass tiles along with mbarriers: one copies (tiled bulk copies), two issue the products before the
// activation and one those behind it (one for all was what all waited for), sixteen apply the activation from TMEM to TMEM or
// shared memory, eight per accumulator so that one is filled while the other is read.
#include <algorithm>

#include "rows.cuh"
#include "umma.cuh"

namespace emc2 {
namespace {

constexpr int kTileRows = 128;
constexpr int kBlockBytes = kTileRows * 128;     // a tile's 64 columns
constexpr int kEpilogueWarps = 16, kCopyWarp = 16, kFirstWarp = 17, kSecondWarp = 18, kOtherFirstWarp = 19, kFixWarp = 19;
constexpr int kFfnThreads = 640;
constexpr int kTmemColumns = 512;
constexpr int kMaxFfnChannels = 256, kMaxFfnHidden = 8192;
constexpr int kMaxStages = 4;
constexpr size_t kMaxShared = 232448 - 1024;     // what a CTA can have, less the kernels' static part
constexpr size_t kMaxWeightShared = kMaxShared - 4096;                     // ffn_weights_kernel's tables of the segments are static

enum { FORWARD = 0, GRAD_X = 1 };
// Where the hidden values go: to TMEM, to shared memory, or there with h beside dg and du.
enum { TO_TMEM = 0, TO_SHARED = 1, TO_SHARED_WITH_H = 2 };

// ---------------------------------------------------------------- a walk over the tiles, expert by expert
// Tiles hold up to 128 * NT rows of one (expert, frame) segment.
struct TileWalk {
    int q;              // segment e * B + b
    int row;            // first row of the tile in [B * N]
    int left;           // rows of the segment from there on
};

__device__ __forceinline__ void segment_rows(const RowSegments& s, int q, int& lo, int& hi) {
    const int e = q / s.B, b = q - e * s.B;
    if (!s.offsets) { lo = 0; hi = s.N; return; }
    const int32_t* of = s.offsets + b * (s.E + 1);
    int at = 0;
    for (int k = 0; k <= e; ++k) at = max(at, min(__ldg(of + k), s.N));
    lo = at;
    hi = max(at, min(__ldg(of + e + 1), s.N));
}

// From the tables of load_bounds and segment_starts.
__device__ __forceinline__ TileWalk tile_at(const RowSegments& s, const int* bounds, const int* start, int tile, int tile_rows) {
    TileWalk w;
    w.q = segment_of(start, s.B * s.E, tile);
    const int e = w.q / s.B, b = w.q - e * s.B, skip = (tile - start[w.q]) * tile_rows;
    const int* of = bounds + b * (s.E + 1) + e;
    w.row = b * s.N + of[0] + skip;
    w.left = of[1] - of[0] - skip;
    return w;
}

__device__ __forceinline__ void next_tile(const RowSegments& s, TileWalk& w, int tile_rows) {
    w.row += tile_rows;
    w.left -= tile_rows;
    while (w.left <= 0 && ++w.q < s.B * s.E) {
        int lo, hi;
        segment_rows(s, w.q, lo, hi);
        w.row = (w.q % s.B) * s.N + lo;
        w.left = hi - lo;
    }
}

// An item is a tile, or one of `splits` shares of its hidden units.
struct ItemWalk {
    TileWalk tile;
    int split;
};
__device__ __forceinline__ void next_item(const RowSegments& s, ItemWalk& w, int tile_rows, int splits) {
    if (++w.split < splits) return;
    w.split = 0;
    next_tile(s, w.tile, tile_rows);
}

// ---------------------------------------------------------------- activations, two values at a time
// The special-function unit is what the activation waits for (16 results a clock and SM), so exponentials and reciprocals are
// what is saved.

// g / (1 + exp(-g)) and the sigmoid 1 / (1 + exp(-g)), by exponentials and one reciprocal for two (a reciprocal each: 260 us
// instead of 220 for 1.2 million rows of 80 channels, 320 units).  Both are right to a few units of fp32 relative to themselves,
// which the roundings behind them need: for negative g they are small, and a form that is right to 2^-12 of 1, like
// (1 + tanh.approx(g / 2)) / 2 (183 us), has none of their bits left at g = -9.  The exponentials of one pair in four, or of every
// other, by a polynomial on the fp32 units: 233 and 236 us.  Gates below -41.5 are taken as -41.5, where the result
// is above -2^-54: the denominators' product then stays below 2^120.  A NaN stays one.
__device__ __forceinline__ uint64_t silu2(uint64_t g, uint64_t& sigmoid) {
    const float2 x = unpair(g);
    const uint64_t c = pair(max_nan(x.x, -41.5f), max_nan(x.y, -41.5f));
    const float2 e = unpair(mul2(c, pair(-1.44269504f, -1.44269504f)));
    const float2 d = unpair(add2(pair(fast_exp2(e.x), fast_exp2(e.y)), pair(1.0f, 1.0f)));
    sigmoid = reciprocals(d.x, d.y);
    return mul2(c, sigmoid);
}

// The normal distribution at g and its density times sqrt(2 pi): Abramowitz and Stegun 7.1.26 for the error function at
// g / sqrt(2), off by 0.75e-7 at most.  Its exponential is the density's, so that both take one exponential and half a
// reciprocal; the constants are the published ones, halved.
__device__ __forceinline__ uint64_t normal2(uint64_t g, uint64_t& density) {
    const float2 x = unpair(g), e = unpair(mul2(mul2(g, g), pair(-0.72134752f, -0.72134752f)));
    density = pair(fast_exp2(e.x), fast_exp2(e.y));
    constexpr float p = 0.3275911f * 0.70710678f;
    const uint64_t t = reciprocals(fmaf(p, fminf(fabsf(x.x), 1e6f), 1.0f), fmaf(p, fminf(fabsf(x.y), 1e6f), 1.0f));
    auto all = [](float v) { return pair(v, v); };
    uint64_t q = fma2(t, all(0.5307027145f), all(-0.7265760135f));
    q = fma2(t, q, all(0.7107068705f));
    q = fma2(t, q, all(-0.142248368f));
    q = fma2(t, q, all(0.127414796f));
    const float2 tail = unpair(mul2(mul2(t, q), density));
    return pair(x.x < 0.0f ? tail.x : 1.0f - tail.x, x.y < 0.0f ? tail.y : 1.0f - tail.y);
}

template <int ACT>
__device__ __forceinline__ uint64_t activation2(uint64_t g) {
    uint64_t beside;
    return ACT == EMC2_ACT_SILU ? silu2(g, beside) : mul2(g, normal2(g, beside));
}
template <int ACT>
__device__ __forceinline__ void activation_grad2(uint64_t g, uint64_t& a, uint64_t& da) {
    if (ACT == EMC2_ACT_SILU) {
        uint64_t s;
        a = silu2(g, s);
        da = fma2(a, fma2(s, pair(-1.0f, -1.0f), pair(1.0f, 1.0f)), s);        // s + a (1 - s)
    } else {
        uint64_t density;
        const uint64_t phi = normal2(g, density);
        a = mul2(g, phi);
        da = fma2(mul2(g, pair(0.39894228f, 0.39894228f)), density, phi);
    }
}

template <bool BF16>
__device__ __forceinline__ uint32_t pack(float a, float b) { return as_halves(a, b, BF16 ? EMC2_BF16 : EMC2_F16); }
template <bool BF16>
__device__ __forceinline__ uint32_t pack(uint64_t p) {
    const float2 f = unpair(p);
    return pack<BF16>(f.x, f.y);
}

__device__ __forceinline__ void store_shared(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// 16-byte piece `piece` of row r in a block of rows of HC 16-bit values, with the swizzle that its width has.
template <int HC>
__device__ __forceinline__ uint32_t swizzled(int r, int piece) {
    return HC == 64 ? r * 128 + ((piece ^ (r & 7)) << 4) : r * 64 + ((piece ^ ((r >> 1) & 3)) << 4);
}

// The same for a block of `width` columns: 64, 32 or 16.
__device__ __forceinline__ uint32_t swizzled(int width, int r, int piece) {
    return width == 64 ? swizzled<64>(r, piece) : width == 32 ? swizzled<32>(r, piece) : r * 32 + ((piece ^ ((r >> 2) & 1)) << 4);
}

// Columns c .. c + 7 of a chunk, at j of the arrays: the values that go on to the second product, a 16-byte piece of row r.
template <int MODE, int HC, int ACT, bool BF16, int TO, int W>
__device__ __forceinline__ void hidden8(const uint32_t (&g)[W], const uint32_t (&u)[W], const uint32_t (&dh)[W], int j0, uint32_t to, int r, int c) {
    constexpr uint32_t kBlock = kTileRows * HC * 2;
    uint32_t p[4], q[4], t[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int j = j0 + 2 * i;
        uint32_t first = g[j];
        if (TO != TO_TMEM) asm volatile("" : "+r"(first));           // and pair by pair here, see hidden_half
        const uint64_t gg = pair(first, g[j + 1]), uu = pair(u[j], u[j + 1]);
        if (MODE == FORWARD) {
            p[i] = pack<BF16>(mul2(activation2<ACT>(gg), uu));
        } else {
            const uint64_t dd = pair(dh[j], dh[j + 1]);
            uint64_t a, da;
            activation_grad2<ACT>(gg, a, da);
            p[i] = pack<BF16>(mul2(mul2(dd, uu), da));
            q[i] = pack<BF16>(mul2(dd, a));
            if (TO == TO_SHARED_WITH_H) t[i] = pack<BF16>(mul2(a, uu));
        }
    }
    if (TO == TO_TMEM) {
        tmem_store(to + c / 2, p[0], p[1], p[2], p[3]);
        if (MODE == GRAD_X) tmem_store(to + (HC + c) / 2, q[0], q[1], q[2], q[3]);
    } else {
        const uint32_t at = to + swizzled<HC>(r, c / 8);
        store_shared(at, p[0], p[1], p[2], p[3]);
        if (MODE == GRAD_X) store_shared(at + kBlock, q[0], q[1], q[2], q[3]);
        if (TO == TO_SHARED_WITH_H) store_shared(at + 2 * kBlock, t[0], t[1], t[2], t[3]);
    }
}

// One arrival per warp, for what all its threads have done.
__device__ __forceinline__ void warp_arrive(uint32_t bar) {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) bar_arrive(bar);
}

// The activation of half of the columns of one chunk of one tile: accumulators of g and u, HC columns each, and of dh, of the
// warp's 32 rows into the blocks at `to`.  The accumulators are given back as soon as they are in registers (which hold 32
// columns of two or 8 to 16 of three), before the arithmetic, so that the next products run beside it.
template <int MODE, int HC, int ACT, bool BF16, int TO>
__device__ __forceinline__ void hidden_half(uint32_t acc, uint32_t acc_dh, int half, uint32_t to, int r, uint32_t acc_empty, uint32_t hid_empty,
                                            uint32_t parity, volatile int* gave_up, int* status) {
    constexpr int W = MODE == FORWARD ? HC / 2 : HC == 64 || (ACT == EMC2_ACT_GELU && TO != TO_TMEM) ? 8 : 16;
#pragma unroll
    for (int c = 0; c < HC / 2; c += W) {
        uint32_t g[W], u[W], dh[W];
        const int at = half * (HC / 2) + c;
        tmem_load(g, acc + at);
        tmem_load(u, acc + HC + at);
        if (MODE == GRAD_X) tmem_load(dh, acc_dh + at);
        tmem_wait(g);
        tmem_wait(u);
        if (MODE == GRAD_X) tmem_wait(dh);
        if (c + W == HC / 2) {
            tmem_fence_before();
            warp_arrive(acc_empty);
        }
        if (c == 0) {
            bar_wait_inline(hid_empty, parity, gave_up, status);           // a call would save the values around it
            __syncwarp();                                                  // stores to TMEM, and its loads, are for whole warps
        }
#pragma unroll
        for (int j = 0; j < W; j += 8) {
            // One piece after the other: the arithmetic of two would not fit in the registers.
#pragma unroll
            for (int i = j; i < j + 8; ++i) asm volatile("" : "+r"(g[i]));
            hidden8<MODE, HC, ACT, BF16, TO>(g, u, dh, j, to, r, at + j);
        }
    }
    if (TO != TO_TMEM) {
        fence_async_shared();
    } else {
        tmem_wait_stores();
        tmem_fence_before();
    }
}

// ---------------------------------------------------------------- rows: y, or dx
struct RowArgs {
    RowSegments seg;
    void* out;
    int C, H, c16, chunks;                  // c16: C rounded up to 16; chunks of HC hidden units
    int full, tail;                         // blocks of 64 columns, and the columns of a narrower one behind them: 0, 16 or 32
    int xn, gn, dn;                         // stages of the rows' tiles, of Wg and Wu, of Wd
    int splits;                             // shares of the hidden units, each an item of its own; 1 unless NT is
    float* part;                            // [items][128][C]: what the shares leave, or null
    int2* tiles;                            // then [max_tiles] for ffn_join_kernel: a tile's first row and how many it has
    int max_tiles;
    uint32_t off_g, off_d, off_h;           // in the dynamic shared memory, behind the rows' tiles
    uint32_t x_bytes, g_bytes, d_bytes, h_bytes;   // of a stage; h: of a unit's hidden values, two of them, if they go there
    uint32_t tile_bytes;                    // of one tensor's tile
};
struct Maps {
    CUtensorMap x, dy, gate, up, down, out;
    CUtensorMap x_tail, dy_tail, gate_tail, up_tail, out_tail;              // of the last block of columns, where it is narrower
};

// 1.2 million rows of 80 bf16 channels, 320 units, SiLU: 220 us, 0.84 PFLOP/s in products of N = 128 and 80 (fp16 223; GELU
// 293).  What it waits for is the activation: three results of the special-function unit for two values, 59 % of that unit's rate beside
// 52 % of the issue slots; a fourth result costs 40 us.  dx of 480,000 fp16 rows of 64 channels, 256 units, GELU: 162 us; of 95,000 bf16 rows
// of 256, 1,024 units, SiLU: 346 us, 0.72 PFLOP/s, where products of N = 64 and 32 take as long as twice as wide ones would.
template <int MODE, int HC, int NT, int TO, int ACT, bool BF16, bool SHARES>
__global__ void __launch_bounds__(kFfnThreads, 1) ffn_rows_kernel(const RowArgs a, const __grid_constant__ Maps maps) {
    // TMEM: the output of NT tiles, two accumulators of g and u, for dx two of dh, and the hidden values of two units unless
    // those go to shared memory.
    constexpr int kHidColumns = MODE == FORWARD ? HC / 2 : HC, kHidBlock = kTileRows * HC * 2;
    extern __shared__ uint8_t dynamic[];
    __shared__ __align__(8) uint64_t bars[4 * kMaxStages * 2 + 16];
    __shared__ uint32_t tmem_at;
    __shared__ int gave_up;
    const uint32_t base = uniform((smem_u32(dynamic) + 1023u) & ~1023u);
    const int warp = uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31;
    const uint32_t bar0 = smem_u32(bars);
    auto x_full = [&](int s) { return bar0 + 8 * s; };
    auto x_empty = [&](int s) { return bar0 + 8 * (4 + s); };
    auto g_full = [&](int s) { return bar0 + 8 * (8 + s); };
    auto g_empty = [&](int s) { return bar0 + 8 * (12 + s); };
    auto d_full = [&](int s) { return bar0 + 8 * (16 + s); };
    auto d_empty = [&](int s) { return bar0 + 8 * (20 + s); };
    auto acc_full = [&](int s) { return bar0 + 8 * (24 + s); };
    auto acc_empty = [&](int s) { return bar0 + 8 * (26 + s); };
    auto hid_full = [&](int s) { return bar0 + 8 * (28 + s); };
    auto hid_empty = [&](int s) { return bar0 + 8 * (30 + s); };
    auto out_full = [&](int t) { return bar0 + 8 * (32 + t); };
    auto out_empty = [&](int t) { return bar0 + 8 * (34 + t); };
    auto staged = [&](int s) { return bar0 + 8 * (36 + s); };

    // The tables lie where the tiles come later.
    int* bounds = reinterpret_cast<int*>(dynamic + (base - smem_u32(dynamic)));
    int* start = bounds + kMaxBounds;
    load_bounds(a.seg, bounds);
    segment_starts(a.seg, bounds, kTileRows * NT, start);
    const int splits = SHARES ? a.splits : 1, total = start[a.seg.B * a.seg.E] * splits;
    const int lo = uniform((int)((long long)total * blockIdx.x / gridDim.x)), hi = (int)((long long)total * (blockIdx.x + 1) / gridDim.x);
    if (SHARES && blockIdx.x == 0)
        for (int t = threadIdx.x; t < a.max_tiles; t += kFfnThreads) {
            int2 rows = make_int2(0, 0);
            if (t * splits < total) {
                const TileWalk w = tile_at(a.seg, bounds, start, t, kTileRows);
                rows = make_int2(w.row, min(w.left, kTileRows));
            }
            a.tiles[t] = rows;
        }
    if (lo >= hi) return;
    ItemWalk walk = {tile_at(a.seg, bounds, start, lo / splits, kTileRows * NT), lo % splits};
    auto advance = [&](ItemWalk& w) { next_item(a.seg, w, kTileRows * NT, splits); };
    auto first_chunk = [&](int split) { return SHARES ? split * a.chunks / splits : split > 0 ? a.chunks : 0; };
    if (threadIdx.x == 0) {
        gave_up = 0;
        for (int s = 0; s < kMaxStages; ++s) {
            bar_init(x_full(s), 1); bar_init(x_empty(s), 1);
            bar_init(g_full(s), 1); bar_init(g_empty(s), MODE == FORWARD ? NT : 1);
            bar_init(d_full(s), 1); bar_init(d_empty(s), 1);
            bar_init(staged(s), NT == 2 ? 8 : 16);
        }
        for (int s = 0; s < 2; ++s) {
            bar_init(acc_full(s), 1); bar_init(acc_empty(s), 8);
            bar_init(hid_full(s), 8); bar_init(hid_empty(s), 1);
            bar_init(out_full(s), 1); bar_init(out_empty(s), NT == 2 ? 8 : 16);
        }
        fence_bar_init();
    }
    if (warp == 0) tmem_alloc(smem_u32(&tmem_at), kTmemColumns);
    fence_async_shared();
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tmem = uniform(tmem_at);
    const uint32_t acc0 = tmem + NT * a.c16, dh0 = acc0 + 4 * HC, hid0 = dh0 + (MODE == GRAD_X ? 2 * HC : 0);
    const int items = uniform(hi - lo);
#define WAIT(bar, parity) bar_wait(bar, parity, &gave_up, a.seg.status)

    if (warp == kCopyWarp) {
        // One warp copies rows and weights, each as soon as a stage of theirs is free, and stores finished tiles from where
        // their rows were: the wait for one must not hold up the others.
        const uint32_t lead = elected();
        Ring x(a.xn), g(a.gn), d(a.dn), done(a.xn);
        ItemWalk rows = walk, stored = walk;
        int t = 0, left = items * NT, st = 0, pending = items * NT;        // tiles to copy, tiles to store
        auto copy_rows = [&] {
            const uint32_t to = base + x.at * a.x_bytes, bar = x_full(x.at);
            const int row = uniform(rows.tile.row) + t * kTileRows;
            bar_expect(lead, bar, a.x_bytes);
            for (int b = 0; b < a.full; ++b) {
                copy_tile(lead, to + b * kBlockBytes, &maps.x, 64 * b, row, bar);
                if (MODE == GRAD_X) copy_tile(lead, to + a.tile_bytes + b * kBlockBytes, &maps.dy, 64 * b, row, bar);
            }
            if (a.tail) {
                copy_tile(lead, to + a.full * kBlockBytes, &maps.x_tail, 64 * a.full, row, bar);
                if (MODE == GRAD_X) copy_tile(lead, to + a.tile_bytes + a.full * kBlockBytes, &maps.dy_tail, 64 * a.full, row, bar);
            }
            x.next();
            --left;
            if (++t == NT) { t = 0; advance(rows); }
        };
        auto store_rows = [&] {
            const int row = uniform(stored.tile.row) + st * kTileRows;
            if (!SHARES && uniform(stored.tile.left) - st * kTileRows >= kTileRows) {      // others have left directly
                const uint32_t from = base + done.at * a.x_bytes;
                for (int b = 0; b < a.full; ++b) store_tile(lead, &maps.out, 64 * b, row, from + b * kBlockBytes);
                if (a.tail) store_tile(lead, &maps.out_tail, 64 * a.full, row, from + a.full * kBlockBytes);
                stores_read();
                __syncwarp();
            }
            if (lead) bar_arrive(x_empty(done.at));
            done.next();
            --pending;
            if (++st == NT) { st = 0; advance(stored); }
        };
        auto over = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xFFFFFFFFu, bar_test(bar, parity)) != 0; };
        auto given_up = [&] { return __any_sync(0xFFFFFFFFu, *(volatile int*)&gave_up) != 0; };
        auto poll = [&] {
            if (pending > 0 && over(staged(done.at), done.parity)) store_rows();
            if (left > 0 && over(x_empty(x.at), x.parity ^ 1)) copy_rows();
        };
        auto wait = [&](uint32_t bar, uint32_t parity) {
            for (int i = 0; !__all_sync(0xFFFFFFFFu, bar_try(bar, parity)); ++i) {
                poll();
                if (i > kWaitTries) { gave_up = 1; atomicOr(a.seg.status, kStatusTimeout); }
                if (given_up()) break;
            }
        };
        copy_rows();
        for (int it = 0; it < items && !given_up(); ++it, advance(walk)) {
            const int e = uniform(walk.tile.q / a.seg.B), split = uniform(walk.split), end = first_chunk(split + 1);
            for (int j = first_chunk(split); j < end; ++j, g.next(), d.next()) {
                wait(g_empty(g.at), g.parity ^ 1);
                const uint32_t to = base + a.off_g + g.at * a.g_bytes, bar = g_full(g.at);
                bar_expect(lead, bar, a.g_bytes);
                // The gradients take Wg and Wu both ways: their last block is a whole one.
                const int whole = MODE == GRAD_X && a.tail ? a.full + 1 : a.full;
                for (int b = 0; b < whole; ++b) {
                    copy_tile(lead, to + b * (2 * HC * 128), &maps.gate, 64 * b, j * HC, e, bar);
                    copy_tile(lead, to + b * (2 * HC * 128) + HC * 128, &maps.up, 64 * b, j * HC, e, bar);
                }
                if (MODE == FORWARD && a.tail) {
                    copy_tile(lead, to + a.full * (2 * HC * 128), &maps.gate_tail, 64 * a.full, j * HC, e, bar);
                    copy_tile(lead, to + a.full * (2 * HC * 128) + HC * a.tail * 2, &maps.up_tail, 64 * a.full, j * HC, e, bar);
                }
                wait(d_empty(d.at), d.parity ^ 1);
                bar_expect(lead, d_full(d.at), a.d_bytes);
                copy_tile(lead, base + a.off_d + d.at * a.d_bytes, &maps.down, j * HC, 0, e, d_full(d.at));
                poll();
            }
        }
        // What is left: the last tiles' results, and rows whose stage one of them held.
        while (pending > 0 && !given_up()) {
            WAIT(staged(done.at), done.parity);
            __syncwarp();
            poll();
        }
        stores_written();
    } else if (warp == kFirstWarp || warp == kOtherFirstWarp) {
        // Unit n is chunk j of tile t of an item; two warps take them in turn.  Issuing returns little before the last product
        // begins, and every wait takes 100 clocks even if it is over: one waits while the other's products run.
        // A barrier's parity says no more than whether its last use is over.  So a warp waits for every use of a stage in
        // turn, and no stage comes round before both are done with it: each tile of an item, or each second chunk where an
        // item is one tile, has stages of its own (their numbers are even), and an item is not over before both have issued a
        // chunk of it; if it has a single one, the first warp takes all.
        const int mine = warp == kFirstWarp ? 0 : 1;
        const uint32_t lead = elected(), kind_gu = product_kind(2 * HC, BF16, false, false), kind_dh = product_kind(HC, BF16, false, true);
        // Wd's stage ends with the channels, where the other tiles' last block is a whole one (see `tail`).
        const int steps = 4 * a.full, tail_steps = a.tail / 16, dh_steps = a.c16 / 16 - tail_steps;
        const uint64_t tail_x0 = operand(base + a.full * kBlockBytes, a.tail * 2, 0);
        const uint64_t tail_w0 = operand(base + a.off_g + a.full * (2 * HC * 128), MODE == FORWARD ? a.tail * 2 : 128, 0);
        const uint64_t x0 = operand(base, 128, 0), w0 = operand(base + a.off_g, 128, 0), wd0 = operand(base + a.off_d, HC * 2, 0);
        Ring x(a.xn), g(a.gn), d(a.dn);
        if (NT == 2 && mine == 1) x.next();
        const bool alone = NT == 1 && a.chunks == 1;
        const int mine_items = alone && mine == 1 ? 0 : items;
        for (int it = 0, n = 0, split = lo % splits; it < mine_items; ++it, split = split + 1 < splits ? split + 1 : 0) {
            WAIT(x_full(x.at), x.parity);
            const uint64_t xa = operand_at(x0, x.at * a.x_bytes), xt = operand_at(tail_x0, x.at * a.x_bytes);
            for (int j = first_chunk(split); j < first_chunk(split + 1); ++j, ++n, g.next(), d.next()) {
                if (NT == 1 && (n & 1) != mine && !alone) continue;
                const int slot = NT == 2 ? mine : n & 1;               // of the accumulators
                const uint32_t acc = acc0 + slot * 2 * HC, dh = dh0 + slot * HC;
                WAIT(g_full(g.at), g.parity);
                if (MODE == GRAD_X) WAIT(d_full(d.at), d.parity);
                WAIT(acc_empty(slot), ((NT == 2 ? n : n >> 1) & 1) ^ 1);
                tmem_fence_after();
                product_blocks(lead, acc, xa, kBlockBytes, operand_at(w0, g.at * a.g_bytes), 2 * HC * 128, steps, kind_gu);
                product_blocks(lead, acc, xt, 0, operand_at(tail_w0, g.at * a.g_bytes), 0, tail_steps, kind_gu, steps > 0);
                if (MODE == GRAD_X) {
                    const uint64_t wd = operand_at(wd0, d.at * a.d_bytes);
                    product_blocks_mn(lead, dh, operand_at(xa, a.tile_bytes), kBlockBytes, wd, 32 * HC, dh_steps, kind_dh);
                    product_blocks_mn(lead, dh, operand_at(xt, a.tile_bytes), 0, operand_at(wd, dh_steps * 32 * HC), 32 * HC, tail_steps, kind_dh, dh_steps > 0);
                }
                products_done(lead, acc_full(slot));
                // The gradients' second products take Wg and Wu again: their warp gives them back.
                products_done(lead, MODE == FORWARD ? g_empty(g.at) : d_empty(d.at));
            }
            for (int k = 0; k < NT; ++k) x.next();
        }
    } else if (warp == kSecondWarp) {
        const uint32_t lead = elected(), kind_out = product_kind(a.c16, BF16, false, MODE == GRAD_X);
        const uint64_t w0 = MODE == FORWARD ? operand(base + a.off_d, HC * 2, 0) : operand(base + a.off_g, 128, 2 * HC * 128);
        const uint64_t hs0 = operand(base + a.off_h, HC * 2, 0);
        Ring w(MODE == FORWARD ? a.dn : a.gn);
        for (int it = 0, n = 0, split = lo % splits; it < items; ++it, split = split + 1 < splits ? split + 1 : 0) {
            const int from = first_chunk(split), end = first_chunk(split + 1);
            for (int j = from; j < end; ++j, w.next())
                for (int t = 0; t < NT; ++t, ++n) {
                    // The first products of this unit have waited for the gradients' Wg and Wu, but not this warp.
                    if (t == 0) WAIT(MODE == FORWARD ? d_full(w.at) : g_full(w.at), w.parity);
                    if (j == from) WAIT(out_empty(t), (it & 1) ^ 1);
                    WAIT(hid_full(n & 1), n >> 1 & 1);
                    tmem_fence_after();
                    const uint32_t out = tmem + t * a.c16;
                    const uint64_t ww = operand_at(w0, w.at * (MODE == FORWARD ? a.d_bytes : a.g_bytes));
#pragma unroll
                    for (int k = 0; k < kHidColumns / 8; ++k) {
                        const uint64_t b = operand_at(ww, MODE == FORWARD ? 32 * k : k * 16 * 128);
                        if (TO == TO_TMEM) product_tmem(lead, out, hid0 + (n & 1) * kHidColumns + 8 * k, b, kind_out, j > from || k > 0);
                        else product(lead, out, operand_at(hs0, (n & 1) * a.h_bytes + k / (HC / 16) * kHidBlock + k % (HC / 16) * 32), b, kind_out, j > from || k > 0);
                    }
                    products_done(lead, hid_empty(n & 1));
                    if (t == NT - 1) products_done(lead, MODE == FORWARD ? d_empty(w.at) : g_empty(w.at));
                    if (j == end - 1) products_done(lead, out_full(t));
                }
        }
    } else if (warp < kEpilogueWarps) {
        const int group = warp >> 3, half = warp >> 2 & 1, quarter = warp & 3, r = quarter * 32 + lane;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        Ring x(a.xn);
        int n = 0;
        for (int it = 0; it < items; ++it, advance(walk)) {
            for (int k = (first_chunk(walk.split + 1) - first_chunk(walk.split)) * NT; k > 0; --k, ++n) {
                if ((n & 1) != group) continue;
                warp_wait(acc_full(group), n >> 1 & 1, &gave_up, a.seg.status);
                tmem_fence_after();
                hidden_half<MODE, HC, ACT, BF16, TO>(acc0 + group * 2 * HC + lanes, dh0 + group * HC + lanes, half,
                                                     TO == TO_TMEM ? hid0 + group * kHidColumns + lanes : base + a.off_h + group * a.h_bytes, r, acc_empty(group), hid_empty(group),
                                                     (n >> 1 & 1) ^ 1, &gave_up, a.seg.status);
                warp_arrive(hid_full(group));
            }
            // The result takes the place of the tile's rows, which no product reads any more, and leaves from there as
            // whole lines (a thread's own row would be 16 bytes of each: 1,300 clocks a tile); rows of a ragged tile leave directly.
            const int t = NT == 2 ? group : 0, xs = x.at + t < a.xn ? x.at + t : x.at + t - a.xn, left = walk.tile.left - t * kTileRows;
            warp_wait(out_full(t), it & 1, &gave_up, a.seg.status);
            tmem_fence_after();
            const uint32_t stage = base + xs * a.x_bytes;
            uint16_t* to = static_cast<uint16_t*>(a.out) + (size_t)(walk.tile.row + t * kTileRows + r) * a.C;
            for (int c = 16 * (NT == 2 ? half : 2 * group + half); c < a.c16; c += NT == 2 ? 32 : 64) {
                uint32_t v[16];
                __syncwarp();                                          // behind stores by some lanes
                tmem_load(v, tmem + t * a.c16 + c + lanes);
                tmem_wait(v);
                if constexpr (SHARES) {                                // part of the sum: ffn_join_kernel adds them up and rounds
                    float4* part = reinterpret_cast<float4*>(a.part + ((size_t)(lo + it) * kTileRows + r) * a.C + c);
#pragma unroll
                    for (int k = 0; k < 16; k += 4)
                        if (c + k < a.C)
                            part[k / 4] = make_float4(__uint_as_float(v[k]), __uint_as_float(v[k + 1]), __uint_as_float(v[k + 2]), __uint_as_float(v[k + 3]));
                } else {
#pragma unroll
                    for (int k = 0; k < 16; k += 8) {
                        const uint32_t p0 = pack<BF16>(pair(v[k], v[k + 1])), p1 = pack<BF16>(pair(v[k + 2], v[k + 3]));
                        const uint32_t p2 = pack<BF16>(pair(v[k + 4], v[k + 5])), p3 = pack<BF16>(pair(v[k + 6], v[k + 7]));
                        if (left >= kTileRows) store_shared(stage + (c >> 6) * kBlockBytes + swizzled(c >> 6 < a.full ? 64 : a.tail, r, (c & 63) / 8 + k / 8), p0, p1, p2, p3);
                        else if (r < left && c + k < a.C) *reinterpret_cast<uint4*>(to + c + k) = make_uint4(p0, p1, p2, p3);
                    }
                }
            }
            tmem_fence_before();
            warp_arrive(out_empty(t));
            fence_async_shared();
            warp_arrive(staged(xs));                                       // of the stage: it has no next use before this one is stored
            for (int k = 0; k < NT; ++k) x.next();
        }
    }
    __syncwarp();
    leave_after_timeout(&gave_up);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    if (warp == 0) tmem_free(tmem, kTmemColumns);
}

struct JoinArgs {
    const float* part;
    const int2* tiles;
    void* out;
    int C, splits, type;
};

// Rows of one tile, a vector of four channels per thread: the shares in their order, rounded once.
__global__ void __launch_bounds__(256) ffn_join_kernel(JoinArgs a) {
    await_predecessor();
    const int2 rows = a.tiles[blockIdx.x];
    const int v = blockIdx.y * 256 + threadIdx.x;
    const size_t step = (size_t)kTileRows * (a.C / 4);
    if (v < rows.y * (a.C / 4)) {
        const float4* part = reinterpret_cast<const float4*>(a.part) + (size_t)blockIdx.x * a.splits * step + v;
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
        for (int k = 0; k < a.splits; ++k) {
            const float4 x = part[k * step];
            s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
        }
        store_row4(a.out, (size_t)rows.x * (a.C / 4) + v, s, a.type);
    }
    release_successor();
}

// ---------------------------------------------------------------- weights: dWg, dWu, dWd
constexpr int kShareInts = 64;              // 2 * EMC2_MAX_EXPERTS and up to a multiple of 256 bytes
struct WeightArgs {
    RowSegments seg;
    float* part;                            // [ranges + E][slices][3 * HC][C]
    int* share;                             // see WeightSumArgs
    int C, H, c16, blocks, slices, ranges;
    int xn, hn;
    uint32_t off_w, off_h;
    uint32_t x_bytes, w_bytes, h_bytes;
};

// Zeros in rows `rows` .. 127 of the blocks of a tile (one warp): they belong to other experts, and whatever they hold,
// infinities and NaN too, must not reach the sums.
__device__ __forceinline__ void clear_rows(uint32_t tile, int blocks, int rows, int lane) {
    const int pieces = (kTileRows - rows) * 8;
    for (int b = 0; b < blocks; ++b)
        for (int i = lane; i < pieces; i += 32) store_shared(tile + b * kBlockBytes + rows * 128 + i * 16, 0u, 0u, 0u, 0u);
}

// A unit of work is a slice of hidden units and a range of the tiles, with accumulators for the three gradients of the
// slice, [C, HC] each (the channels in the lanes).  All slices of a range are taken at about the same time, so that its
// tiles are read from device memory once.  A range that meets several experts has a part of the result for each: entry
// r + e of `part`, which along the run of all tiles no other pair of range and expert has.
// 480,000 fp16 rows of 64 channels, 256 units, GELU: 200 us; 95,000 bf16 rows of 256, 1,024 units, SiLU: 545 us, 0.55 PFLOP/s:
// of a tile's products those of the transposed rows have N = 64 and 32 columns at C > 128, which take 49 and 45 clocks for 32 and 16.
template <int HC, int ACT, bool BF16>
__global__ void __launch_bounds__(kFfnThreads, 1) ffn_weights_kernel(const WeightArgs a, const __grid_constant__ Maps maps) {
    constexpr int kOut = 3 * HC, kTwoDh = HC == 32 ? 1 : 0, kHidBlock = kTileRows * HC * 2;
    extern __shared__ uint8_t dynamic[];
    __shared__ __align__(8) uint64_t bars[36];
    __shared__ int bounds[kMaxBounds];
    __shared__ int start[kMaxSegments + 1];
    __shared__ uint32_t tmem_at;
    __shared__ int gave_up;
    const uint32_t base = uniform((smem_u32(dynamic) + 1023u) & ~1023u);
    const int warp = uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31;
    const uint32_t bar0 = smem_u32(bars);
    // A tile's stage comes and goes in parts: its rows' channels by 128, then those of dy.
    auto x_land = [&](int p) { return bar0 + 8 * p; };
    auto x_full = [&](int p) { return bar0 + 8 * (8 + p); };
    auto x_empty = [&](int p) { return bar0 + 8 * (16 + p); };
    auto acc_full = [&](int s) { return bar0 + 8 * (24 + s); };
    auto acc_empty = [&](int s) { return bar0 + 8 * (26 + s); };
    auto hid_full = [&](int s) { return bar0 + 8 * (28 + s); };
    auto hid_empty = [&](int s) { return bar0 + 8 * (30 + s); };
    const uint32_t w_full = bar0 + 8 * 32, w_empty = bar0 + 8 * 33, out_full = bar0 + 8 * 34, out_empty = bar0 + 8 * 35;

    load_bounds(a.seg, bounds);
    segment_starts(a.seg, bounds, kTileRows, start);
    const int total = uniform(start[a.seg.B * a.seg.E]), ranges = min(a.ranges, total), work = ranges * a.slices;
    // Range r has tiles total * r / ranges .. total * (r + 1) / ranges - 1, one at least.
    if (blockIdx.x == 0 && threadIdx.x < a.seg.E) {
        const long long from = start[threadIdx.x * a.seg.B], to = start[(threadIdx.x + 1) * a.seg.B];
        a.share[2 * threadIdx.x] = from < to ? (int)(((from + 1) * ranges - 1) / total) : 0;
        a.share[2 * threadIdx.x + 1] = from < to ? (int)((to * ranges - 1) / total) + 1 : 0;
    }
    if (total == 0) return;
    if (threadIdx.x == 0) {
        gave_up = 0;
        for (int p = 0; p < 8; ++p) { bar_init(x_land(p), 1); bar_init(x_full(p), 1); bar_init(x_empty(p), 1); }
        for (int s = 0; s < 2; ++s) {
            bar_init(acc_full(s), 1); bar_init(acc_empty(s), 8);
            bar_init(hid_full(s), 8); bar_init(hid_empty(s), 1);
        }
        bar_init(w_full, 1); bar_init(w_empty, 1); bar_init(out_full, 1); bar_init(out_empty, 16);
        fence_bar_init();
    }
    if (warp == 0) tmem_alloc(smem_u32(&tmem_at), kTmemColumns);
    fence_async_shared();
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tmem = uniform(tmem_at);
    const int halves = (a.c16 + 127) / 128, parts = 2 * halves;        // of the channels, 128 lanes each
    auto blocks_of = [&](int m) { return a.blocks - 2 * m < 2 ? a.blocks - 2 * m : 2; };
    const uint32_t acc0 = tmem + halves * kOut, dh0 = acc0 + 4 * HC;
    // Every role makes the same walk: for each unit of work its tiles, a piece for each expert.
    auto expert_of = [&](int tile) { return tile < total ? segment_of(start, a.seg.B * a.seg.E, tile) / a.seg.B : a.seg.E; };
    auto first_tile = [&](int r) { return (int)((long long)total * r / ranges); };

    if (warp == kCopyWarp) {
        const uint32_t lead = elected();
        Ring x(a.xn);
        int piece = 0;
        for (int k = blockIdx.x; k < work && !__any_sync(0xFFFFFFFFu, *(volatile int*)&gave_up); k += gridDim.x) {
            const int r = k / a.slices, c = k - r * a.slices, lo = first_tile(r), hi = first_tile(r + 1);
            TileWalk walk = tile_at(a.seg, bounds, start, lo, kTileRows);
            int e = -1;
            for (int i = lo; i < hi; ++i, x.next(), next_tile(a.seg, walk, kTileRows)) {
                const int now = uniform(walk.q / a.seg.B), row = uniform(walk.row);
                if (now != e) {
                    e = now;
                    WAIT(w_empty, (piece & 1) ^ 1);
                    bar_expect(lead, w_full, a.w_bytes);
                    for (int b = 0; b < a.blocks; ++b) {
                        const uint32_t to = base + a.off_w + b * (2 * HC * 128);
                        copy_tile(lead, to, &maps.gate, 64 * b, c * HC, e, w_full);
                        copy_tile(lead, to + HC * 128, &maps.up, 64 * b, c * HC, e, w_full);
                    }
                    copy_tile(lead, base + a.off_w + a.blocks * (2 * HC * 128), &maps.down, c * HC, 0, e, w_full);
                    ++piece;
                }
                const uint32_t to = base + x.at * a.x_bytes;
                for (int p = 0; p < parts; ++p) {
                    const int m = p < halves ? p : p - halves, index = x.at * parts + p;
                    WAIT(x_empty(index), x.parity ^ 1);
                    bar_expect(lead, x_land(index), blocks_of(m) * kBlockBytes);
                    for (int b = 2 * m; b < 2 * m + blocks_of(m); ++b) {
                        if (p < halves) copy_tile(lead, to + b * kBlockBytes, &maps.x, 64 * b, row, x_land(index));
                        else copy_tile(lead, to + (a.blocks + b) * kBlockBytes, &maps.dy, 64 * b, row, x_land(index));
                    }
                }
            }
        }
    } else if (warp == kFixWarp) {
        Ring x(a.xn);
        for (int k = blockIdx.x; k < work; k += gridDim.x) {
            const int r = k / a.slices, lo = first_tile(r), hi = first_tile(r + 1);
            TileWalk walk = tile_at(a.seg, bounds, start, lo, kTileRows);
            for (int i = lo; i < hi; ++i, x.next(), next_tile(a.seg, walk, kTileRows)) {
                for (int p = 0; p < parts; ++p) {
                    const int m = p < halves ? p : p - halves, index = x.at * parts + p;
                    WAIT(x_land(index), x.parity);
                    if (walk.left < kTileRows) {
                        __syncwarp();
                        clear_rows(base + x.at * a.x_bytes + ((p < halves ? 0 : a.blocks) + 2 * m) * kBlockBytes, blocks_of(m), walk.left, lane);
                        fence_async_shared();
                    }
                    __syncwarp();
                    if (lane == 0) bar_arrive(x_full(index));
                }
            }
        }
    } else if (warp == kFirstWarp || warp == kSecondWarp) {
        // Both warps make the walk; each has its own waits.
        const uint32_t lead = elected(), kind_gu = product_kind(2 * HC, BF16, false, false), kind_dh = product_kind(HC, BF16, false, true);
        const uint32_t kind_w2 = product_kind(2 * HC, BF16, true, true), kind_w1 = product_kind(HC, BF16, true, true);
        const bool second = warp == kSecondWarp;
        const uint64_t x0 = operand(base, 128, second ? kBlockBytes : 0), w0 = operand(base + a.off_w, 128, 0);
        const uint64_t wd0 = operand(base + a.off_w + a.blocks * (2 * HC * 128), HC * 2, 0), hid0 = operand(base + a.off_h, HC * 2, kHidBlock);
        Ring x(a.xn), hid(a.hn);
        int n = 0, piece = 0;
        for (int k = blockIdx.x; k < work; k += gridDim.x) {
            const int r = k / a.slices, lo = first_tile(r), hi = first_tile(r + 1);
            int end = lo;                                                  // of the piece
            for (int i = lo; i < hi; ++i, ++n, x.next()) {
                const bool first = i == end;
                if (first) end = uniform(min(hi, start[(expert_of(i) + 1) * a.seg.B]));
                const bool last = i + 1 == end;
                const uint64_t xa = operand_at(x0, x.at * a.x_bytes);
                if (!second) {
                    if (first) WAIT(w_full, piece & 1);
                    WAIT(acc_empty(n & 1), (n >> 1 & 1) ^ 1);
                    for (int m = 0; m < halves; ++m) {
                        WAIT(x_full(x.at * parts + m), x.parity);
                        tmem_fence_after();
                        product_blocks(lead, acc0 + (n & 1) * 2 * HC, operand_at(xa, 2 * m * kBlockBytes), kBlockBytes, operand_at(w0, 2 * m * (2 * HC * 128)),
                                       2 * HC * 128, min(8, a.c16 / 16 - 8 * m), kind_gu, m > 0);
                    }
                    if (!kTwoDh && n > 0) WAIT(acc_empty((n - 1) & 1), (n - 1) >> 1 & 1);
                    for (int m = 0; m < halves; ++m) {
                        WAIT(x_full(x.at * parts + halves + m), x.parity);
                        tmem_fence_after();
                        product_blocks_mn(lead, dh0 + kTwoDh * (n & 1) * HC, operand_at(xa, (a.blocks + 2 * m) * kBlockBytes), kBlockBytes,
                                          operand_at(wd0, 8 * m * 32 * HC), 32 * HC, min(8, a.c16 / 16 - 8 * m), kind_dh, m > 0);
                    }
                    products_done(lead, acc_full(n & 1));
                    if (last) products_done(lead, w_empty);
                } else {
                    if (first) WAIT(out_empty, (piece & 1) ^ 1);
                    WAIT(hid_full(n & 1), n >> 1 & 1);                     // so the tile is there, and the first products are through with it
                    tmem_fence_after();
                    const uint64_t h = operand_at(hid0, hid.at * a.h_bytes);
                    for (int p = 0; p < parts; ++p) {
                        const int m = p < halves ? p : p - halves;
                        if (p < halves) {
                            const uint64_t xm = operand_at(xa, 2 * m * kBlockBytes);
#pragma unroll
                            for (int q = 0; q < kTileRows / 16; ++q)
                                product(lead, tmem + m * kOut, operand_at(xm, q * 16 * 128), operand_at(h, q * 32 * HC), kind_w2, !first || q > 0);
                        } else {
                            const uint64_t ym = operand_at(xa, (a.blocks + 2 * m) * kBlockBytes);
#pragma unroll
                            for (int q = 0; q < kTileRows / 16; ++q)
                                product(lead, tmem + m * kOut + 2 * HC, operand_at(ym, q * 16 * 128), operand_at(h, 2 * kHidBlock + q * 32 * HC), kind_w1, !first || q > 0);
                        }
                        products_done(lead, x_empty(x.at * parts + p));
                    }
                    products_done(lead, hid_empty(n & 1));
                    if (last) products_done(lead, out_full);
                    hid.next();
                }
                if (last) ++piece;
            }
        }
    } else if (warp < kEpilogueWarps) {
        const int group = warp >> 3, half = warp >> 2 & 1, quarter = warp & 3, row = quarter * 32 + lane;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16, hid = base + a.off_h;
        int n = 0, piece = 0;
        for (int k = blockIdx.x; k < work; k += gridDim.x) {
            const int r = k / a.slices, c = k - r * a.slices, lo = first_tile(r), hi = first_tile(r + 1);
            for (int i = lo, e = expert_of(lo); i < hi; e = expert_of(i)) {
                for (const int end = min(hi, start[(e + 1) * a.seg.B]); i < end; ++i, ++n) {
                    if ((n & 1) != group) continue;
                    warp_wait(acc_full(group), n >> 1 & 1, &gave_up, a.seg.status);
                    tmem_fence_after();
                    const int before = n - a.hn, slot = before & 1;        // a group waits for every use of a barrier in turn
                    hidden_half<GRAD_X, HC, ACT, BF16, TO_SHARED_WITH_H>(acc0 + group * 2 * HC + lanes, dh0 + kTwoDh * group * HC + lanes, half,
                                                             hid + (a.hn == 2 ? group * a.h_bytes : 0), row, acc_empty(group), hid_empty(slot), before >> 1 & 1,
                                                             &gave_up, a.seg.status);
                    warp_arrive(hid_full(group));
                }
                warp_wait(out_full, piece & 1, &gave_up, a.seg.status);
                ++piece;
                tmem_fence_after();
                float* part = a.part + ((size_t)(r + e) * a.slices + c) * kOut * a.C;
                for (int m = 0; m < halves; ++m) {
                    const int ch = m * 128 + row;
                    for (int j = 16 * (warp >> 2); j < kOut; j += 64) {
                        uint32_t v[16];
                        __syncwarp();
                        tmem_load(v, tmem + m * kOut + j + lanes);
                        tmem_wait(v);
#pragma unroll
                        for (int q = 0; q < 16; ++q)
                            if (ch < a.C) part[(size_t)(j + q) * a.C + ch] = __uint_as_float(v[q]);
                    }
                }
                tmem_fence_before();
                warp_arrive(out_empty);
            }
        }
    }
#undef WAIT
    __syncwarp();
    leave_after_timeout(&gave_up);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    if (warp == 0) tmem_free(tmem, kTmemColumns);
}

struct WeightSumArgs {
    const float* part;
    const int* share;               // [E][2]: first range with tiles of the expert and the one behind the last; as ffn_weights_kernel left it
    void* gate;
    void* up;
    void* down;
    int C, H, slice, slices, type;
};

// dW of 32 / RS hidden units and 32 channels: the parts of the ranges that met the expert.  Four units per warp; every RS-th
// part by one warp where there are many, then the warps' sums in their order.
template <int RS>
__global__ void __launch_bounds__(256) ffn_sum_kernel(WeightSumArgs a) {
    await_predecessor();
    constexpr int kUnits = 32 / RS;
    __shared__ float sums[RS][kUnits][33];
    const int columns = (a.C + 31) / 32, kind = blockIdx.y, e = blockIdx.z, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c0 = blockIdx.x % columns * 32, h0 = blockIdx.x / columns * kUnits, mine = warp % RS, u0 = warp / RS * 4;
    const int r0 = a.share[2 * e], r1 = a.share[2 * e + 1];
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    if (c0 + lane < a.C) {
        const size_t step = (size_t)a.slices * 3 * a.slice * a.C;             // from a range to the next
        const float* p = a.part + ((size_t)e * a.slices + h0 / a.slice) * 3 * a.slice * a.C + ((size_t)kind * a.slice + h0 % a.slice + u0) * a.C + c0 + lane;
#pragma unroll 4
        for (int r = r0 + mine; r < r1; r += RS)
#pragma unroll
            for (int k = 0; k < 4; ++k) s[k] += p[r * step + (size_t)k * a.C];
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) sums[mine][u0 + k][lane] = s[k];
    __syncthreads();
    uint16_t* out = static_cast<uint16_t*>(kind == 0 ? a.gate : kind == 1 ? a.up : a.down);
    for (int i = threadIdx.x; i < kUnits * 32; i += 256) {
        // Consecutive threads write consecutive addresses: channels of [E, H, C], hidden units of [E, C, H].
        const int h = kind < 2 ? i >> 5 : i % kUnits, c = kind < 2 ? i & 31 : i / kUnits;
        float v = sums[0][h][c];
#pragma unroll
        for (int w = 1; w < RS; ++w) v += sums[w][h][c];
        if (h0 + h < a.H && c0 + c < a.C)
            out[kind < 2 ? ((size_t)e * a.H + h0 + h) * a.C + c0 + c : ((size_t)e * a.C + c0 + c) * a.H + h0 + h] = (uint16_t)as_halves(v, 0.f, a.type);
    }
    release_successor();
}

// ---------------------------------------------------------------- host
// [z, y, x] of 16-bit values, copied as boxes of x_box columns (64, 32 or 16, with the swizzle of that width) and y_box rows;
// what lies outside reads as zeros.
bool encode(CUtensorMap* map, const void* p, int type, uint64_t x, uint64_t y, uint64_t z, int x_box, int y_box) {
    const cuuint64_t dims[3] = {x, y, z}, strides[2] = {x * 2, x * y * 2};
    const cuuint32_t box[3] = {(cuuint32_t)x_box, (cuuint32_t)y_box, 1}, step[3] = {1, 1, 1};
    const EncodeTiled f = encoder();
    return f && f(map, type == EMC2_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, z ? 3 : 2, const_cast<void*>(p), dims,
                  strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, x_box == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : x_box == 32 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_32B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct FfnCall {
    RowSegments seg;
    int C, H, type, act;
    const void* x;
    const void* dy;
    const void* gate;
    const void* up;
    const void* down;
    void* out;
};

bool make_maps(const FfnCall& f, int hc, int tail, Maps* m) {
    const int c16 = (f.C + 15) / 16 * 16;
    const uint64_t rows = (uint64_t)f.seg.B * f.seg.N, E = (uint64_t)f.seg.E;
    if (tail && !(encode(&m->x_tail, f.x, f.type, f.C, rows, 0, tail, kTileRows) && encode(&m->dy_tail, f.dy ? f.dy : f.x, f.type, f.C, rows, 0, tail, kTileRows) &&
                  encode(&m->out_tail, f.out, f.type, f.C, rows, 0, tail, kTileRows) && encode(&m->gate_tail, f.gate, f.type, f.C, f.H, E, tail, hc) &&
                  encode(&m->up_tail, f.up, f.type, f.C, f.H, E, tail, hc)))
        return false;
    return encode(&m->x, f.x, f.type, f.C, rows, 0, 64, kTileRows) && encode(&m->dy, f.dy ? f.dy : f.x, f.type, f.C, rows, 0, 64, kTileRows) &&
           encode(&m->out, f.out, f.type, f.C, rows, 0, 64, kTileRows) &&
           encode(&m->gate, f.gate, f.type, f.C, f.H, E, 64, hc) && encode(&m->up, f.up, f.type, f.C, f.H, E, 64, hc) &&
           encode(&m->down, f.down, f.type, f.H, f.C, E, hc, c16);
}

template <typename F, typename A>
int launch_ffn(emc2_bridge* h, int kind, F kernel, const A& a, const Maps& m, int ctas, int threads, size_t shared, size_t most, cudaStream_t st) {
    const cudaError_t e = allow_shared(kernel, most);
    if (e != cudaSuccess) return check_cuda(h, e);
    LaunchScope ls(h, kind, st);
    kernel<<<ctas, threads, shared, st>>>(a, m);
    return check_cuda(h, cudaGetLastError());
}

// Tiles of 128 * NT rows there can be.
long long row_tiles(const RowSegments& s, int NT) {
    return ((long long)s.B * s.N + kTileRows * NT - 1) / (kTileRows * NT) + (long long)s.B * s.E;
}

template <int MODE, int HC, int NT, int TO, bool SHARES>
int launch_rows_kernel(emc2_bridge* h, const FfnCall& f, const RowArgs& a, const Maps& m, int ctas, size_t shared, cudaStream_t st) {
    const int kind = MODE == FORWARD ? K_FFN : K_FFN_GRAD_X;
    const bool bf16 = f.type == EMC2_BF16;
    if (f.act == EMC2_ACT_SILU)
        return bf16 ? launch_ffn(h, kind, ffn_rows_kernel<MODE, HC, NT, TO, EMC2_ACT_SILU, true, SHARES>, a, m, ctas, kFfnThreads, shared, kMaxShared, st)
                    : launch_ffn(h, kind, ffn_rows_kernel<MODE, HC, NT, TO, EMC2_ACT_SILU, false, SHARES>, a, m, ctas, kFfnThreads, shared, kMaxShared, st);
    if constexpr (TO == TO_TMEM)
        return bf16 ? launch_ffn(h, kind, ffn_rows_kernel<MODE, HC, NT, TO, EMC2_ACT_GELU, true, SHARES>, a, m, ctas, kFfnThreads, shared, kMaxShared, st)
                    : launch_ffn(h, kind, ffn_rows_kernel<MODE, HC, NT, TO, EMC2_ACT_GELU, false, SHARES>, a, m, ctas, kFfnThreads, shared, kMaxShared, st);
    return EMC2_ERR_INTERNAL;
}

template <int MODE, int HC, int NT, int TO>
int launch_rows(emc2_bridge* h, const FfnCall& f, cudaStream_t st) {
    RowArgs a;
    a.seg = f.seg; a.out = f.out; a.C = f.C; a.H = f.H;
    a.c16 = (f.C + 15) / 16 * 16;
    a.chunks = (f.H + HC - 1) / HC;
    a.full = a.c16 / 64;
    a.tail = a.c16 % 64;
    if (a.tail == 48) { a.tail = 0; ++a.full; }                              // no swizzle of that width
    a.tile_bytes = a.full * kBlockBytes + kTileRows * a.tail * 2;            // these are all multiples of 1 KB
    a.x_bytes = (MODE == FORWARD ? 1 : 2) * a.tile_bytes;
    a.g_bytes = 2 * HC * (MODE == FORWARD ? a.full * 128 + a.tail * 2 : (a.full + (a.tail > 0)) * 128);
    a.d_bytes = a.c16 * HC * 2;
    a.h_bytes = TO == TO_TMEM ? 0 : (MODE == FORWARD ? 1 : 2) * kTileRows * HC * 2;
    // As many stages as there is room for: first two of each, then more of the rows.
    a.xn = NT; a.gn = 2; a.dn = 2;
    auto room = [&] { return (size_t)a.xn * a.x_bytes + (size_t)a.gn * a.g_bytes + (size_t)a.dn * a.d_bytes + 2 * a.h_bytes + 1024; };
    // What is left goes to the next item's rows and to twice the stages of the weights (see the first products' warps for the
    // even numbers).
    auto more_rows = [&](int n) { while (a.xn < n && room() + NT * a.x_bytes <= kMaxShared) a.xn += NT; };
    if (NT == 2) more_rows(4);
    if (room() + 2 * (a.g_bytes + a.d_bytes) <= kMaxShared) { a.gn += 2; a.dn += 2; }
    if (NT == 1) more_rows(2);
    a.off_g = a.xn * a.x_bytes;
    a.off_d = a.off_g + a.gn * a.g_bytes;
    a.off_h = a.off_d + a.dn * a.d_bytes;
    Maps m;
    if (!make_maps(f, HC, a.tail, &m)) return check_cuda(h, cudaErrorInvalidValue);
    const size_t shared = std::max(room(), (size_t)(kMaxBounds + kMaxSegments + 1) * 4 + 1024);
    // Few rows: shares of their hidden units, of four chunks at least, keep the other SMs busy, if there is scratch for what
    // they leave and more than 16 chunks.  us in one piece, and in shares with their join: 64 rows of 64 channels, 4,096 units
    // 47.2 and 21.5; 1,280 units 26.6 and 21.2; 512 units 20.5 and 21.4.
    const long long tiles = row_tiles(f.seg, NT);
    const RowsScratch& r = h->rows_scratch;
    a.splits = 1;
    if (NT == 1 && 2 * tiles <= h->num_sms && r.slab && f.C <= r.max_channels && r.max_hidden > 0 && a.chunks > 16)
        a.splits = (int)std::min<long long>(a.chunks / 4, h->num_sms / tiles);
    a.part = a.splits > 1 ? static_cast<float*>(r.slab) : nullptr;
    a.max_tiles = (int)std::min<long long>(tiles, h->num_sms);
    a.tiles = a.part ? reinterpret_cast<int2*>(a.part + (size_t)h->num_sms * kTileRows * f.C) : nullptr;
    const int ctas = (int)std::min<long long>(tiles * a.splits, h->num_sms);
    if (a.splits == 1) return launch_rows_kernel<MODE, HC, NT, TO, false>(h, f, a, m, ctas, shared, st);
    const int rc = launch_rows_kernel<MODE, HC, 1, TO, true>(h, f, a, m, ctas, shared, st);
    if (rc != EMC2_OK) return rc;
    const JoinArgs join = {a.part, a.tiles, f.out, f.C, a.splits, f.type};
    LaunchScope ls(h, K_FFN_JOIN, st);
    launch_chained(ffn_join_kernel, dim3((unsigned)tiles, (kTileRows * f.C / 4 + 255) / 256), 256, 0, st, join);
    return check_cuda(h, cudaGetLastError());
}

// Ranges of the tiles: four units of work per SM, but eight tiles in each while that leaves one unit per SM.
int weight_ranges(const emc2_bridge* h, int slices, long long tiles) {
    const long long most = std::max(1, 4 * h->num_sms / slices), few = std::max<long long>(tiles / 8, (h->num_sms + slices - 1) / slices);
    return (int)std::max<long long>(1, std::min({most, few, tiles}));
}

// Stages that fit: of the hidden values two, of the tiles up to three.  The product of the transposed rows takes 128
// channels at a time: with fewer than that it reads up to one block behind a tile's last (the results go to lanes that
// nobody reads), which the weights' room has to cover.
template <int HC>
size_t plan_weights(WeightArgs& a, const FfnCall& f) {
    a.seg = f.seg; a.C = f.C; a.H = f.H;
    a.c16 = (f.C + 15) / 16 * 16;
    a.blocks = (f.C + 63) / 64;
    a.slices = (f.H + HC - 1) / HC;
    a.x_bytes = 2 * a.blocks * kBlockBytes;
    a.w_bytes = a.blocks * 2 * HC * 128 + a.c16 * HC * 2;
    a.h_bytes = 3 * kTileRows * HC * 2;
    a.xn = 1; a.hn = 1;
    constexpr size_t most = kMaxWeightShared;
    auto room = [&] { return (size_t)a.xn * a.x_bytes + std::max<size_t>(a.w_bytes + (size_t)a.hn * a.h_bytes, kBlockBytes) + 1024; };
    if (room() + a.x_bytes <= most) ++a.xn;
    if (room() + a.h_bytes <= most) ++a.hn;
    if (a.xn == 2 && room() + a.x_bytes <= most) ++a.xn;
    a.off_w = a.xn * a.x_bytes;
    a.off_h = a.off_w + a.w_bytes;
    return room();
}

template <int HC>
int launch_slices(emc2_bridge* h, const FfnCall& f, WeightArgs& a, cudaStream_t st) {
    const size_t shared = plan_weights<HC>(a, f);
    a.share = static_cast<int*>(h->rows_scratch.slab);
    a.part = reinterpret_cast<float*>(a.share + kShareInts);
    a.ranges = weight_ranges(h, a.slices, row_tiles(f.seg, 1));
    Maps m;
    if (!make_maps(f, HC, 0, &m)) return check_cuda(h, cudaErrorInvalidValue);
    const int ctas = std::min(a.ranges * a.slices, h->num_sms);
    const bool bf16 = f.type == EMC2_BF16;
    if (f.act == EMC2_ACT_SILU)
        return bf16 ? launch_ffn(h, K_FFN_GRAD_W, ffn_weights_kernel<HC, EMC2_ACT_SILU, true>, a, m, ctas, kFfnThreads, shared, kMaxWeightShared, st)
                    : launch_ffn(h, K_FFN_GRAD_W, ffn_weights_kernel<HC, EMC2_ACT_SILU, false>, a, m, ctas, kFfnThreads, shared, kMaxWeightShared, st);
    return bf16 ? launch_ffn(h, K_FFN_GRAD_W, ffn_weights_kernel<HC, EMC2_ACT_GELU, true>, a, m, ctas, kFfnThreads, shared, kMaxWeightShared, st)
                : launch_ffn(h, K_FFN_GRAD_W, ffn_weights_kernel<HC, EMC2_ACT_GELU, false>, a, m, ctas, kFfnThreads, shared, kMaxWeightShared, st);
}

// Slices of 64 hidden units where two stages of tiles fit beside them (up to 96 channels): half the products, which below
// N = 128 take little less for half the columns.  us with 64 and with 32, 60,000 rows: 64 channels, 1,024 units 96.8 and
// 125.4; 96 channels, 512 units 80.3 and 87.6.
bool wide_slices(const FfnCall& f) {
    WeightArgs a;
    plan_weights<64>(a, f);
    return a.c16 <= 128 && a.xn >= 2;
}

int launch_weights(emc2_bridge* h, const FfnCall& f, void* gate, void* up, void* down, cudaStream_t st) {
    WeightArgs a;
    const bool wide = wide_slices(f);
    const int rc = wide ? launch_slices<64>(h, f, a, st) : launch_slices<32>(h, f, a, st);
    if (rc != EMC2_OK) return rc;
    WeightSumArgs s;
    s.part = a.part; s.share = a.share; s.gate = gate; s.up = up; s.down = down; s.C = f.C; s.H = f.H;
    s.slice = wide ? 64 : 32; s.slices = a.slices; s.type = f.type;
    LaunchScope ls(h, K_FFN_SUM, st);
    // Where the CTAs with 32 units each would be two per SM or fewer, eight times as many share out the parts.  us with 32 units
    // and with 4: 60,000 rows of 64 channels and 256 units, four experts (192 CTAs) 14.5 and 9.2; of 128 and 512 (768 CTAs)
    // 13.7 and 17.8.
    const int columns = (f.C + 31) / 32;
    if ((f.H + 31) / 32 * columns * 3 * f.seg.E <= 2 * h->num_sms) launch_chained(ffn_sum_kernel<8>, dim3((f.H + 3) / 4 * columns, 3, f.seg.E), 256, 0, st, s);
    else launch_chained(ffn_sum_kernel<1>, dim3((f.H + 31) / 32 * columns, 3, f.seg.E), 256, 0, st, s);
    return check_cuda(h, cudaGetLastError());
}

int check_ffn(const emc2_bridge* h, int B, int N, int C, int H, int type, int act, const void* x, const int32_t* offsets, const void* gate,
              const void* up, const void* down) {
    if (!h || B < 0 || N < 0 || B > h->cfg.max_batch || N > h->cfg.max_points) return EMC2_ERR_INVALID_ARG;
    if (C < 8 || C > kMaxFfnChannels || (C & 7) || H < 8 || H > kMaxFfnHidden || (H & 7)) return EMC2_ERR_INVALID_ARG;
    if ((type != EMC2_BF16 && type != EMC2_F16) || (act != EMC2_ACT_SILU && act != EMC2_ACT_GELU)) return EMC2_ERR_INVALID_ARG;
    if (!gate || !up || !down || !on_16_bytes(gate) || !on_16_bytes(up) || !on_16_bytes(down) || !on_16_bytes(x)) return EMC2_ERR_INVALID_ARG;
    if (B > 0 && N > 0 && !x) return EMC2_ERR_INVALID_ARG;
    if (!on_4_bytes(offsets)) return EMC2_ERR_INVALID_ARG;
    return EMC2_OK;
}

}  // namespace

size_t ffn_scratch_bytes(const emc2_bridge* h, int max_channels, int max_hidden) {
    if (max_hidden <= 0) return 0;
    const int C = std::min(max_channels, kMaxFfnChannels);
    size_t most = 0;
    for (int slice : {32, 64})
        for (int slices = 1; slices <= (max_hidden + slice - 1) / slice; ++slices)
            most = std::max(most, (size_t)(weight_ranges(h, slices, 1LL << 40) + EMC2_MAX_EXPERTS) * slices * 3 * slice * C * sizeof(float));
    most += kShareInts * sizeof(int);
    return std::max(most, (size_t)h->num_sms * (kTileRows * C * sizeof(float) + sizeof(int2)));      // the shares of few rows
}

}  // namespace emc2

using namespace emc2;

extern "C" int emc2_expert_ffn(emc2_bridge_t* h, int32_t B, int32_t N, int32_t channels, int32_t hidden, int32_t type, int32_t act,
                               const void* d_x, const int32_t* d_offsets, const void* d_w_gate, const void* d_w_up, const void* d_w_down,
                               void* d_y, void* cuda_stream) {
    const int rc = check_ffn(h, B, N, channels, hidden, type, act, d_x, d_offsets, d_w_gate, d_w_up, d_w_down);
    if (rc != EMC2_OK) return rc;
    if (!on_16_bytes(d_y)) return EMC2_ERR_INVALID_ARG;
    if (B == 0 || N == 0) return EMC2_OK;
    if (!d_y || d_y == d_x) return EMC2_ERR_INVALID_ARG;
    RowsDevice device(h->cfg.device);
    if (!device.ok) return EMC2_ERR_CUDA;
    const FfnCall f = {row_segments(h, B, N, d_offsets), channels, hidden, type, act, d_x, nullptr, d_w_gate, d_w_up, d_w_down, d_y};
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    // Chunks of hidden units, and tiles that share their weights, as TMEM has room for (see ffn_rows_kernel).  Two tiles share
    // a chunk's weights where there can be more than one per SM, counted by the rows and one more per segment: where the segments
    // end is known on the device only.  Calls of many short segments therefore run tiles that are mostly empty.  us
    // of one and of two: 15,000 rows of 64 channels, 1,024 units 23.3 and 31.5; 20,000 30.7 and 30.7; 60,000 52.0 and 51.2 (but
    // 40,000, whose pairs are just more than the SMs, 41.7 and 50.0); 60,000 of 80 channels, 320 units 31.5 and 29.4; of 128 channels,
    // 512 units 47.1 and 41.0.
    const bool pairs = row_tiles(f.seg, 1) > h->num_sms;
    if (channels <= 96) return pairs ? launch_rows<FORWARD, 64, 2, TO_TMEM>(h, f, st) : launch_rows<FORWARD, 64, 1, TO_TMEM>(h, f, st);
    return channels <= 128 && pairs ? launch_rows<FORWARD, 32, 2, TO_TMEM>(h, f, st) : launch_rows<FORWARD, 32, 1, TO_TMEM>(h, f, st);
}

extern "C" int emc2_expert_ffn_grad(emc2_bridge_t* h, int32_t B, int32_t N, int32_t channels, int32_t hidden, int32_t type, int32_t act,
                                    const void* d_x, const int32_t* d_offsets, const void* d_w_gate, const void* d_w_up,
                                    const void* d_w_down, const void* d_grad_y, void* d_grad_x, void* d_grad_gate, void* d_grad_up,
                                    void* d_grad_down, void* cuda_stream) {
    int rc = check_ffn(h, B, N, channels, hidden, type, act, d_x, d_offsets, d_w_gate, d_w_up, d_w_down);
    if (rc != EMC2_OK) return rc;
    if (!d_grad_gate || !d_grad_up || !d_grad_down || !on_16_bytes(d_grad_y) || !on_16_bytes(d_grad_x) || !on_16_bytes(d_grad_gate) ||
        !on_16_bytes(d_grad_up) || !on_16_bytes(d_grad_down))
        return EMC2_ERR_INVALID_ARG;
    const bool empty = B == 0 || N == 0;
    if (!empty && (!d_grad_y || !d_grad_x || d_grad_x == d_x || d_grad_x == d_grad_y)) return EMC2_ERR_INVALID_ARG;
    if (!h->rows_scratch.slab || channels > h->rows_scratch.max_channels || hidden > h->rows_scratch.max_hidden) return EMC2_ERR_TOO_LARGE;
    RowsDevice device(h->cfg.device);
    if (!device.ok) return EMC2_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const FfnCall f = {row_segments(h, B, N, d_offsets), channels, hidden, type, act, d_x, d_grad_y, d_w_gate, d_w_up, d_w_down, d_grad_x};
    if (empty) {
        const size_t bytes = (size_t)f.seg.E * hidden * channels * 2;
        cudaError_t e = cudaMemsetAsync(d_grad_gate, 0, bytes, st);
        if (e == cudaSuccess) e = cudaMemsetAsync(d_grad_up, 0, bytes, st);
        if (e == cudaSuccess) e = cudaMemsetAsync(d_grad_down, 0, bytes, st);
        return check_cuda(h, e);
    }
    // The weights' gradients need nothing of dx: they run on a stream of the handle, whose CTAs take the SMs over as those of
    // dx end, instead of waiting for the last.  Not where dx is in shares, which lie in the same scratch, nor for few channels,
    // where it was measured to be slower.  us on one stream and on two: 15,000 rows of 128
    // channels, 512 units 70.7 and 63.5; 60,000 of 256, 1,024 units 607 and 582; of 64, 1,024 units 179 and 182; 120,000 of 64, 1,024
    // units, GELU 345 and 363.
    const bool aside = h->overlap && 2 * row_tiles(f.seg, 1) > h->num_sms && channels > 96;
    const cudaStream_t weights_st = aside ? h->side : st;
    if (aside) {
        cudaError_t e = cudaEventRecord(h->ev_fork, st);
        if (e == cudaSuccess) e = cudaStreamWaitEvent(h->side, h->ev_fork, 0);
        if (e != cudaSuccess) return check_cuda(h, e);
    }
    // Hidden values in shared memory leave TMEM to chunks of 64 units; GELU's arithmetic has no registers for those.  us of dx
    // with them and with chunks of 32: 60,000 rows of 64 channels, 1,024 units, SiLU 75.8 and 81.9; 256 units 34.9 and 35.7.
    rc = channels <= 64 && act == EMC2_ACT_SILU ? launch_rows<GRAD_X, 64, 1, TO_SHARED>(h, f, st) : launch_rows<GRAD_X, 32, 1, TO_TMEM>(h, f, st);
    if (rc == EMC2_OK) rc = launch_weights(h, f, d_grad_gate, d_grad_up, d_grad_down, weights_st);
    if (aside) {                                                           // also after an error: `st` never runs ahead
        cudaError_t e = cudaEventRecord(h->ev_join, h->side);
        if (e == cudaSuccess) e = cudaStreamWaitEvent(st, h->ev_join, 0);
        if (rc == EMC2_OK) rc = check_cuda(h, e);
    }
    return rc;
}
