// Thin wrappers over the sm_100a instructions that the matrix kernels use: mbarriers with bounded waits, tiled bulk
// copies, and tcgen05 with its accumulators in tensor memory (TMEM).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace emc2 {

// The driver's encoder of tensor maps, or null.
using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                 const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiled encoder() {
    static const EncodeTiled f = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return f;
}

#ifdef __CUDACC__

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ uint32_t elected() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p;
}
// The value of lane 0, which the compiler then knows to be the same in all lanes.
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __shfl_sync(0xFFFFFFFFu, v, 0); }
__device__ __forceinline__ int uniform(int v) { return __shfl_sync(0xFFFFFFFFu, v, 0); }
// ---- mbarriers, by shared-memory address
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t arrivals) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(arrivals) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t lead, uint32_t bar, uint32_t bytes) {
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t"
                 "@q mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}" ::"r"(bar), "r"(bytes), "r"(lead) : "memory");
}
// Whether the phase of that parity is over; try_wait suspends the thread for a while first, test_wait does not.
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}
__device__ __forceinline__ bool bar_test(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}

// A wait that ends: after kWaitTries tries it sets *gave_up, and from then on every wait of the CTA that is not over at once
// is given up.  The CTA then runs through the rest of its steps without waiting (what it computes is void, as the status
// says) and winds up, see leave_after_timeout.  A hint for a long suspension made everything 10 % slower, polling without any
// 3 % (forward, 1.2 M rows of 80 channels, at 183 us).  Only the first try is in line: the warps that copy and issue products run
// through little else, and what they fetch counts.
constexpr int kWaitTries = 1 << 22;
constexpr int kStatusTimeout = 2;            // device status: EMC2_ERR_TIMEOUT
__device__ __forceinline__ void bar_wait_inline(uint32_t bar, uint32_t parity, volatile int* gave_up, int* status) {
    for (int i = 0; i < kWaitTries; ++i) {
        if (bar_try(bar, parity)) return;
        if ((i & 255) == 1 && *gave_up) return;
    }
    *gave_up = 1;
    atomicOr(status, kStatusTimeout);
}
__device__ __noinline__ static void bar_wait_on(uint32_t bar, uint32_t parity, volatile int* gave_up, int* status) {
    bar_wait_inline(bar, parity, gave_up, status);
}
__device__ __forceinline__ void bar_wait(uint32_t bar, uint32_t parity, volatile int* gave_up, int* status) {
    if (!bar_try(bar, parity)) bar_wait_on(bar, parity, gave_up, status);
}
// The same by whole warps before instructions that a warp has to reach together (all loads and stores of TMEM): lanes can
// leave the loop of a wait in different turns.
__device__ __forceinline__ void warp_wait(uint32_t bar, uint32_t parity, volatile int* gave_up, int* status) {
    bar_wait(bar, parity, gave_up, status);
    __syncwarp();
}
// Copies and products still in flight get this long to land before the CTA gives its memory back.
__device__ __forceinline__ void leave_after_timeout(volatile int* gave_up) {
    if (*gave_up)
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);
}

__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void fence_bar_init() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }

// ---- tiled bulk copies; x counts elements of the innermost dimension (a multiple of 16 bytes)
// As with the products below, a whole warp comes here with the same arguments and one lane (`lead`) issues.
__device__ __forceinline__ void copy_tile(uint32_t lead, uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %5, 0;\n\t"
                 "@q cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n\t}"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar), "r"(lead) : "memory");
}
__device__ __forceinline__ void copy_tile(uint32_t lead, uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %6, 0;\n\t"
                 "@q cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n\t}"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar), "r"(lead) : "memory");
}
// And back: the tile at src, whose reads the lane that issued waits for with stores_read.
__device__ __forceinline__ void store_tile(uint32_t lead, const CUtensorMap* map, int x, int y, uint32_t src) {
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %4, 0;\n\t"
                 "@q cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];\n\t}"
                 ::"l"(map), "r"(x), "r"(y), "r"(src), "r"(lead) : "memory");
}
__device__ __forceinline__ void stores_read() {
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
}
__device__ __forceinline__ void stores_written() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

// ---- TMEM
__device__ __forceinline__ void tmem_alloc(uint32_t dst, uint32_t columns) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t columns) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(columns) : "memory");
}
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 8, 16 or 32 columns of the warp's 32 lanes: lane l of the warp gets row 32 * (warp % 4) + l.  Valid after tmem_wait, through
// which the registers pass, so that nothing that reads them moves ahead of it.
__device__ __forceinline__ void tmem_load(uint32_t (&r)[8], uint32_t addr) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x8.b32 {"
        "%0, %1, %2, %3, %4, %5, %6, %7"
        "}, [%8];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_load(uint32_t (&r)[16], uint32_t addr) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {"
        "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15"
        "}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_load(uint32_t (&r)[32], uint32_t addr) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
        "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, "
        "%23, %24, %25, %26, %27, %28, %29, %30, %31"
        "}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_wait(uint32_t (&a)[8]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(a[0]), "+r"(a[1]), "+r"(a[2]), "+r"(a[3]), "+r"(a[4]), "+r"(a[5]), "+r"(a[6]), "+r"(a[7])::"memory");
}
__device__ __forceinline__ void tmem_wait(uint32_t (&a)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(a[0]), "+r"(a[1]), "+r"(a[2]), "+r"(a[3]), "+r"(a[4]), "+r"(a[5]), "+r"(a[6]), "+r"(a[7]), "+r"(a[8]), "+r"(a[9]),
                   "+r"(a[10]), "+r"(a[11]), "+r"(a[12]), "+r"(a[13]), "+r"(a[14]), "+r"(a[15])::"memory");
}
__device__ __forceinline__ void tmem_wait(uint32_t (&a)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(a[0]), "+r"(a[1]), "+r"(a[2]), "+r"(a[3]), "+r"(a[4]), "+r"(a[5]), "+r"(a[6]), "+r"(a[7]), "+r"(a[8]), "+r"(a[9]),
                   "+r"(a[10]), "+r"(a[11]), "+r"(a[12]), "+r"(a[13]), "+r"(a[14]), "+r"(a[15]), "+r"(a[16]), "+r"(a[17]), "+r"(a[18]),
                   "+r"(a[19]), "+r"(a[20]), "+r"(a[21]), "+r"(a[22]), "+r"(a[23]), "+r"(a[24]), "+r"(a[25]), "+r"(a[26]), "+r"(a[27]),
                   "+r"(a[28]), "+r"(a[29]), "+r"(a[30]), "+r"(a[31])::"memory");
}

// Four columns of the warp's 32 lanes; complete after tmem_wait_stores.
__device__ __forceinline__ void tmem_store(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void tmem_wait_stores() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// ---- pairs of floats in one instruction
__device__ __forceinline__ uint64_t pair(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ uint64_t pair(uint32_t a, uint32_t b) { return pair(__uint_as_float(a), __uint_as_float(b)); }
__device__ __forceinline__ float2 unpair(uint64_t p) {
    float2 f;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(p));
    return f;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ float fast_exp2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// The larger of both; NaN if one is.
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// Both reciprocals from one: a and b from 1 to 2^60.
__device__ __forceinline__ uint64_t reciprocals(float a, float b) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(a * b));
    return mul2(pair(r, r), pair(b, a));
}

// ---- products: D[128, N] (+)= A[128, 16] B[16, N], fp32 accumulators
// A whole warp comes here, with the same arguments in every lane, and its elected lane issues: the descriptors then stay in
// uniform registers.  Issued by a thread on a branch of its own each product took 71 clocks or more; so it takes what the
// tensor core does: 45 up to N = 32, 49 at 64, 65 at 128, 97 at 192, 129 at 256, and with A in TMEM 63 up to N = 128 (B200).
// Shared-memory operands are tiles of rows of `row_bytes` (128, 64 or 32, with the swizzle of that width): groups of eight
// rows follow one another every 8 * row_bytes.
//   K-major  (a row holds consecutive k of one m or n): a step of 16 k is 32 bytes further in the row
//   MN-major (a row holds consecutive m or n of one k): a step of 16 k is 16 rows further; blocks of row_bytes / 2
//            columns are `block` bytes apart
__device__ __forceinline__ uint64_t operand(uint32_t addr, int row_bytes, uint32_t block) {
    const uint64_t swizzle = row_bytes == 128 ? 2 : row_bytes == 64 ? 4 : 6;
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)((block & 0x3FFFFu) >> 4) << 16 | (uint64_t)((8 * row_bytes) >> 4) << 32 |
           1ull << 46 | swizzle << 61;
}
// Instruction descriptor: fp32 accumulators, both operands bf16 or both fp16.
__device__ __forceinline__ uint32_t product_kind(int n, bool bf16, bool a_mn, bool b_mn) {
    return 1u << 4 | (bf16 ? 1u : 0u) << 7 | (bf16 ? 1u : 0u) << 10 | (a_mn ? 1u : 0u) << 15 | (b_mn ? 1u : 0u) << 16 |
           (uint32_t)(n >> 3) << 17 | (uint32_t)(128 >> 4) << 24;
}
__device__ __forceinline__ void product(uint32_t lead, uint32_t d, uint64_t a, uint64_t b, uint32_t kind, bool add) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(kind), "r"((uint32_t)add), "r"(lead) : "memory");
}
// The same with A in TMEM: row m in lane m, two values of k per column, a step of 16 k in eight columns.
__device__ __forceinline__ void product_tmem(uint32_t lead, uint32_t d, uint32_t a, uint64_t b, uint32_t kind, bool add) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d), "r"(a), "l"(b), "r"(kind), "r"((uint32_t)add), "r"(lead) : "memory");
}
// Further on by a multiple of 16 bytes.
__device__ __forceinline__ uint64_t operand_at(uint64_t op, uint32_t bytes) { return op + (bytes >> 4); }
// `steps` steps of 16 k with both operands K-major in blocks of 64 columns.  What is computed
// between two products counts: four steps are written out.
__device__ __forceinline__ void product_blocks(uint32_t lead, uint32_t d, uint64_t a, uint32_t a_block, uint64_t b, uint32_t b_block, int steps, uint32_t kind,
                                               bool add = false) {
    for (; steps >= 4; steps -= 4) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            product(lead, d, operand_at(a, 32 * k), operand_at(b, 32 * k), kind, add);
            add = true;
        }
        a = operand_at(a, a_block);
        b = operand_at(b, b_block);
    }
    for (int k = 0; k < steps; ++k) {
        product(lead, d, operand_at(a, 32 * k), operand_at(b, 32 * k), kind, add);
        add = true;
    }
}
// The same with B MN-major in one block, a step of it `b_step` bytes further.
__device__ __forceinline__ void product_blocks_mn(uint32_t lead, uint32_t d, uint64_t a, uint32_t a_block, uint64_t b, uint32_t b_step, int steps, uint32_t kind,
                                                  bool add = false) {
    for (; steps >= 4; steps -= 4) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            product(lead, d, operand_at(a, 32 * k), operand_at(b, b_step * k), kind, add);
            add = true;
        }
        a = operand_at(a, a_block);
        b = operand_at(b, 4 * b_step);
    }
    for (int k = 0; k < steps; ++k) {
        product(lead, d, operand_at(a, 32 * k), operand_at(b, b_step * k), kind, add);
        add = true;
    }
}

// The stages of a ring in turn: the stage, and the parity of its use.
struct Ring {
    int n, at = 0;
    uint32_t parity = 0;
    __device__ __forceinline__ explicit Ring(int n_) : n(n_) {}
    __device__ __forceinline__ void next() {
        if (++at == n) { at = 0; parity ^= 1; }
    }
};

// Arrives at `bar` when all products issued so far by the elected lane are done.
__device__ __forceinline__ void products_done(uint32_t lead, uint32_t bar) {
    asm volatile(
        "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar), "r"(lead) : "memory");
}

#endif  // __CUDACC__

}  // namespace emc2
