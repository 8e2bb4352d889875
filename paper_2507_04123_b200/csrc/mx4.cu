// Rows to microscaled 4-bit floating point (see mx4.cuh).  Per block of 32 elements
//
//   power = 2^(floor(log2 max|x|) - 2), at least 2^-127;  code = x / power rounded to the nearest element, halves to even, 6 at most
//
// so that the largest element lies in [4, 8) before it is rounded.  A block with an infinity or NaN gets the power NaN.
// Bound by memory, with 73 % of the issue slots: four lanes share a block, eight elements each, and a thread requests several before it works
// on the first.  131,072 rows of 1,024 bf16 channels, their values written as bf16: 102 us, 6.0 TB/s read and written.
#include "dropout.cuh"
#include "mx4.cuh"

namespace emc2 {
namespace {

constexpr int kMxThreads = 256;
constexpr int kMxGroups = 4;                 // of eight elements per thread

struct MxArgs {
    const void* x;
    uint32_t* codes;                         // of eight elements each; or null
    uint8_t* scales;                         // or null
    void* values;                            // or null
    FastDiv width;                           // division by the groups of eight of a row, blocks whole
    uint32_t groups;                         // of all rows
    int nvec;
};

// Eight codes, the first in the lowest bits.
__device__ __forceinline__ uint32_t e2m1_codes(const float (&f)[8]) {
    uint32_t c;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(c) : "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7]));
    return c;
}

template <bool WIDE, int TYPE>
__global__ void __launch_bounds__(kMxThreads) mx4_kernel(MxArgs a) {
    const uint32_t first = blockIdx.x * (kMxThreads * kMxGroups) + threadIdx.x;
    Raw8 raw[kMxGroups];
#pragma unroll
    for (int i = 0; i < kMxGroups; ++i) {
        const uint32_t g = first + i * kMxThreads;
        uint32_t row, at;
        a.width.divmod(g, row, at);
        const bool in = g < a.groups && (int)(2 * at) < a.nvec;
        raw[i] = request8<WIDE>(a.x, (size_t)row * a.nvec + 2 * at, in, in && (int)(2 * at + 1) < a.nvec, TYPE);
    }
#pragma unroll
    for (int i = 0; i < kMxGroups; ++i) {
        const uint32_t g = first + i * kMxThreads;
        float f[8];
        floats8(f, raw[i], TYPE);
        // As numbers without sign, so that NaN is the largest.
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(f[j]) & 0x7FFFFFFFu);
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
        const uint32_t e = top >> 23;
        const uint32_t power = e == 255u ? 255u : e > 2u ? e - 2u : 0u;
        const float inverse = __uint_as_float(power == 255u ? 0u : (254u - power) << 23);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = power == 255u ? 0.f : f[j] * inverse;
        const uint32_t codes = e2m1_codes(f);
        if (g >= a.groups) continue;
        if (a.codes) a.codes[g] = codes;
        if (a.scales && (g & 3) == 0) a.scales[g >> 2] = (uint8_t)power;
        if (!a.values) continue;
        uint32_t row, at;
        a.width.divmod(g, row, at);
        if ((int)(2 * at) >= a.nvec) continue;
        const float scale = mx_power(power);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t c = codes >> (4 * j);
            // The code's bits as those of a fp32 number: the element times 2^-126.
            f[j] = __uint_as_float((c & 8u) << 28 | (c & 7u) << 22) * 0x1p126f * scale;
        }
        store8<WIDE>(a.values, (size_t)row * a.nvec + 2 * at, (int)(2 * at + 1) < a.nvec, f, TYPE);
    }
}

template <int TYPE>
void launch_mx4(const MxArgs& a, bool wide, unsigned ctas, cudaStream_t st) {
    if (wide) mx4_kernel<true, TYPE><<<ctas, kMxThreads, 0, st>>>(a);
    else mx4_kernel<false, TYPE><<<ctas, kMxThreads, 0, st>>>(a);
}

}  // namespace
}  // namespace emc2

using namespace emc2;

extern "C" int emc2_mx4_quantise(emc2_bridge_t* h, int32_t rows, int32_t channels, int32_t type, const void* d_x, uint8_t* d_codes,
                                 uint8_t* d_scales, void* d_values, void* cuda_stream) {
    if (!h || rows < 0 || channels < 4 || channels > kMaxMxChannels || (channels & 3) || !is_type(type)) return EMC2_ERR_INVALID_ARG;
    const int64_t blocks = (int64_t)rows * mx4_blocks(channels);
    if (blocks > (int64_t)1 << 29) return EMC2_ERR_INVALID_ARG;
    if (!on_16_bytes(d_x) || !on_16_bytes(d_codes) || !on_16_bytes(d_values)) return EMC2_ERR_INVALID_ARG;
    if (rows == 0) return EMC2_OK;
    if (!d_x || d_x == d_values || (d_codes != nullptr) != (d_scales != nullptr) || (!d_codes && !d_values)) return EMC2_ERR_INVALID_ARG;
    RowsDevice device(h->cfg.device);
    if (!device.ok) return EMC2_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    MxArgs a;
    a.x = d_x; a.codes = reinterpret_cast<uint32_t*>(d_codes); a.scales = d_scales; a.values = d_values; a.nvec = channels / 4;
    a.width = make_fast_div((uint32_t)mx4_blocks(channels) * 4);
    a.groups = (uint32_t)blocks * 4;
    const unsigned ctas = (a.groups + kMxThreads * kMxGroups - 1) / (kMxThreads * kMxGroups);
    const bool wide = is_wide(channels, type, d_x) && (!d_values || is_wide(channels, type, d_values));
    LaunchScope ls(h, K_MX4, st);
    if (type == EMC2_F32) launch_mx4<EMC2_F32>(a, wide, ctas, st);
    else if (type == EMC2_BF16) launch_mx4<EMC2_BF16>(a, wide, ctas, st);
    else launch_mx4<EMC2_F16>(a, wide, ctas, st);
    return check_cuda(h, cudaGetLastError());
}
