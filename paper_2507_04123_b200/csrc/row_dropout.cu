// Dropout of rows: y = x / (1 - p) where the generator keeps the element, else 0.  The gradient is the same call on dy.
//
// Bound by memory, next by the generator: eight elements share one of its numbers, see dropout.cuh, and a thread requests its elements
// before it computes theirs.  1.2 million rows of 80 bf16 channels: 66 us, 5.8 TB/s read and written, with 62 % of the issue slots; a thread
// per eight elements, the type looked up at run time, took 92.
#include <algorithm>

#include "dropout.cuh"

namespace emc2 {
namespace {

constexpr int kDropThreads = 256;
constexpr int kDropGroups = 4;               // of eight elements per thread

struct DropArgs {
    const void* x;
    void* y;
    FastDiv width;                           // division by the groups of a row
    Dropout drop;
    uint32_t groups;                         // of all rows
    int nvec;
};

// The type is a constant: a branch on it per pair of elements was a quarter of the instructions.
template <bool WIDE, int TYPE>
__global__ void __launch_bounds__(kDropThreads) dropout_kernel(DropArgs a) {
    const uint32_t first = blockIdx.x * (kDropThreads * kDropGroups) + threadIdx.x;
    Raw8 raw[kDropGroups];
    uint32_t row[kDropGroups], at[kDropGroups];
#pragma unroll
    for (int i = 0; i < kDropGroups; ++i) {
        const uint32_t g = first + i * kDropThreads;
        const bool in = g < a.groups;
        a.width.divmod(g, row[i], at[i]);
        raw[i] = request8<WIDE>(a.x, (size_t)row[i] * a.nvec + 2 * at[i], in, in && 2 * at[i] + 1 < (uint32_t)a.nvec, TYPE);
    }
    uint4 bits[kDropGroups];
    dropout_bits(bits, dropout_seed(a.drop), row, at);
    if (!a.drop.any) {
#pragma unroll
        for (int i = 0; i < kDropGroups; ++i) bits[i] = make_uint4(~0u, ~0u, ~0u, ~0u);
    }
    const uint32_t above = a.drop.any ? a.drop.above : 0u;
#pragma unroll
    for (int i = 0; i < kDropGroups; ++i) {
        float f[8];
        floats8(f, raw[i], TYPE);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = dropout_keeps(bits[i], j, above) ? f[j] * a.drop.factor : 0.0f;
        if (first + i * kDropThreads < a.groups) store8<WIDE>(a.y, (size_t)row[i] * a.nvec + 2 * at[i], 2 * at[i] + 1 < (uint32_t)a.nvec, f, TYPE);
    }
}

template <int TYPE>
void launch_dropout(const DropArgs& a, bool wide, unsigned ctas, cudaStream_t st) {
    if (wide) dropout_kernel<true, TYPE><<<ctas, kDropThreads, 0, st>>>(a);
    else dropout_kernel<false, TYPE><<<ctas, kDropThreads, 0, st>>>(a);
}

}  // namespace
}  // namespace emc2

using namespace emc2;

extern "C" int emc2_row_dropout(emc2_bridge_t* h, int32_t n, int32_t channels, int32_t type, const void* d_x, float p,
                                const int64_t* d_seed, void* d_y, void* cuda_stream) {
    if (!h || n < 0 || (int64_t)n > (int64_t)h->cfg.max_batch * h->cfg.max_points) return EMC2_ERR_INVALID_ARG;
    if (channels < 4 || channels > kMaxRowChannels || (channels & 3) || !is_type(type) || !is_share(p)) return EMC2_ERR_INVALID_ARG;
    if (!d_seed || !on_8_bytes(d_seed) || !on_16_bytes(d_x) || !on_16_bytes(d_y)) return EMC2_ERR_INVALID_ARG;
    if (n == 0) return EMC2_OK;
    if (!d_x || !d_y || d_x == d_y) return EMC2_ERR_INVALID_ARG;
    RowsDevice device(h->cfg.device);
    if (!device.ok) return EMC2_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    DropArgs a;
    a.x = d_x; a.y = d_y; a.drop = make_dropout(p, d_seed); a.nvec = channels / 4;
    const uint32_t width = (uint32_t)(channels + 7) / 8;
    a.width = make_fast_div(width);
    a.groups = (uint32_t)n * width;                              // 2^24 rows of 128 at most
    const unsigned ctas = (a.groups + kDropThreads * kDropGroups - 1) / (kDropThreads * kDropGroups);
    LaunchScope ls(h, K_ROW_DROPOUT, st);
    const bool wide = is_wide(channels, type, d_x) && is_wide(channels, type, d_y);
    if (type == EMC2_F32) launch_dropout<EMC2_F32>(a, wide, ctas, st);
    else if (type == EMC2_BF16) launch_dropout<EMC2_BF16>(a, wide, ctas, st);
    else launch_dropout<EMC2_F16>(a, wide, ctas, st);
    return check_cuda(h, cudaGetLastError());
}
