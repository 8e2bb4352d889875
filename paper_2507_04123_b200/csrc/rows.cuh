// What the operators on dispatched rows share: element types, the experts' segments, the split of a row over lanes.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "bridge_internal.cuh"
#include "row_sizes.cuh"

namespace emc2 {

constexpr int kStatusBadRows = 4;            // device status: EMC2_ERR_INVALID_ARG
constexpr int kMaxRowChannels = 1024;        // row_lookup, expert_norm
constexpr int kMaxSegments = EMC2_MAX_BATCH * EMC2_MAX_EXPERTS;
constexpr int kMaxBounds = EMC2_MAX_BATCH * (EMC2_MAX_EXPERTS + 1);

inline int type_bytes(int type) { return type == EMC2_F32 ? 4 : 2; }
inline bool is_type(int type) { return type >= EMC2_F32 && type <= EMC2_F16; }
inline bool on_16_bytes(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
inline bool on_4_bytes(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }

// Makes the handle's device current for a call.  It is set where it is current already too: a host thread that has made no CUDA
// call yet has the device's number but not its context, which the encoding of a tensor map needs.
struct RowsDevice {
    int prev = -1;
    bool ok = true;
    explicit RowsDevice(int dev) {
        ok = cudaGetDevice(&prev) == cudaSuccess && cudaSetDevice(dev) == cudaSuccess;
        if (prev == dev) prev = -1;
    }
    ~RowsDevice() {
        if (prev >= 0) cudaSetDevice(prev);
    }
};

// Lets a kernel be launched with up to `most` bytes of dynamic shared memory, the largest that any call of it has.  The setting is
// the process's: a call's own size could be lowered by another handle's call on another thread before the launch, which
// would then be refused.
template <typename F>
cudaError_t allow_shared(F kernel, size_t most) {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most);
}

// The experts' segments of a call.  offsets null: one expert owns all rows.
struct RowSegments {
    const int32_t* offsets;
    int B, N, E;
    int* status;
};

inline RowSegments row_segments(const emc2_bridge* h, int B, int N, const int32_t* offsets) {
    return {offsets, B, N, offsets ? h->cfg.num_experts : 1, h->d_status};
}

#ifdef __CUDACC__

__device__ __forceinline__ float4 as_floats(uint2 v, int type) {
    float4 f;
    if (type == EMC2_BF16) {
        f.x = __uint_as_float(v.x << 16);
        f.y = __uint_as_float(v.x & 0xFFFF0000u);
        f.z = __uint_as_float(v.y << 16);
        f.w = __uint_as_float(v.y & 0xFFFF0000u);
    } else {
        const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&v.x)), b = __half22float2(*reinterpret_cast<const __half2*>(&v.y));
        f = make_float4(a.x, a.y, b.x, b.y);
    }
    return f;
}

// Two floats rounded to a 16-bit type, to nearest even; the first in the low half.
__device__ __forceinline__ uint32_t as_halves(float a, float b, int type) {
    if (type == EMC2_BF16) {
        const __nv_bfloat162 r = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&r);
    }
    const __half2 r = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&r);
}

// Vector v (four elements) of a buffer of `type`.
__device__ __forceinline__ void store_row4(void* p, size_t v, const float4& f, int type) {
    if (type == EMC2_F32) static_cast<float4*>(p)[v] = f;
    else static_cast<uint2*>(p)[v] = make_uint2(as_halves(f.x, f.y, type), as_halves(f.z, f.w, type));
}

// The vectors lane + i * lanes of a row as they lie in memory (a 16-bit type's in the first half), zeros past nvec, and the
// values of one.  Apart, so that a thread can request several rows before it converts the first: behind a conversion, which
// branches on the type, the compiler puts no earlier load.
template <int K>
__device__ __forceinline__ void request_row(uint4 (&r)[K], const void* p, size_t v0, int lane, int log, int nvec, int type) {
#pragma unroll
    for (int i = 0; i < K; ++i) r[i] = make_uint4(0u, 0u, 0u, 0u);
    if (type == EMC2_F32) {
#pragma unroll
        for (int i = 0; i < K; ++i) {
            const int v = lane + (i << log);
            if (v < nvec) r[i] = __ldg(static_cast<const uint4*>(p) + v0 + v);
        }
    } else {
#pragma unroll
        for (int i = 0; i < K; ++i) {
            const int v = lane + (i << log);
            if (v >= nvec) continue;
            const uint2 h = __ldg(static_cast<const uint2*>(p) + v0 + v);
            r[i].x = h.x;
            r[i].y = h.y;
        }
    }
}
__device__ __forceinline__ float4 row_floats(const uint4& r, int type) {
    if (type == EMC2_F32) return make_float4(__uint_as_float(r.x), __uint_as_float(r.y), __uint_as_float(r.z), __uint_as_float(r.w));
    return as_floats(make_uint2(r.x, r.y), type);
}

// The row's values at once, for a kernel that has one row to wait for.
template <int K>
__device__ __forceinline__ void load_row(float4 (&f)[K], const void* p, size_t v0, int lane, int log, int nvec, int type) {
    if (type == EMC2_F32) {
#pragma unroll
        for (int i = 0; i < K; ++i) {
            const int v = lane + (i << log);
            f[i] = v < nvec ? __ldg(static_cast<const float4*>(p) + v0 + v) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
    } else {
        uint2 h[K];
#pragma unroll
        for (int i = 0; i < K; ++i) {
            const int v = lane + (i << log);
            h[i] = v < nvec ? __ldg(static_cast<const uint2*>(p) + v0 + v) : make_uint2(0u, 0u);
        }
#pragma unroll
        for (int i = 0; i < K; ++i) f[i] = as_floats(h[i], type);
    }
}

// Sum over the 1 << log lanes of a row's group; every lane gets it.
__device__ __forceinline__ float group_sum(float v, int log) {
    for (int d = 1; d < 1 << log; d <<= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    return v;
}

// bounds[b * (E + 1) + e]: first row of expert e in frame b, [.. + E]: the end.  Offsets that do not ascend within
// 0 .. N are pulled to the nearest that do, so that whatever they hold every row belongs to one expert at most and
// lies inside the frame; the first CTA then reports them.  Called by a whole CTA; ready on return.
__device__ __forceinline__ void load_bounds(const RowSegments& s, int* bounds) {
    const int n = s.B * (s.E + 1);
    for (int i = threadIdx.x; i < n; i += blockDim.x)
        bounds[i] = s.offsets ? __ldg(s.offsets + i) : (i & 1) * s.N;
    __syncthreads();
    for (int b = threadIdx.x; b < s.B; b += blockDim.x) {
        int at = 0;
        bool bad = false;
        for (int e = 0; e <= s.E; ++e) {
            const int raw = bounds[b * (s.E + 1) + e];
            bad |= raw < at || raw > s.N;
            at = max(at, min(raw, s.N));
            bounds[b * (s.E + 1) + e] = at;
        }
        if (bad && blockIdx.x == 0 && blockIdx.y == 0) atomicOr(s.status, kStatusBadRows);
    }
    __syncthreads();
}

// start[q], q = e * B + b: rows of the segments before (expert e, frame b) when the segments are put one behind another,
// expert by expert; start[E * B]: all of them.  `unit` > 1 counts units of that many rows, the last of a segment ragged.
// Called by a whole CTA behind load_bounds; ready on return.
__device__ __forceinline__ void segment_starts(const RowSegments& s, const int* bounds, int unit, int* start) {
    const int n = s.B * s.E;
    if (threadIdx.x < 32) {
        int run = 0;
        for (int q0 = 0; q0 < n; q0 += 32) {
            const int q = q0 + (int)threadIdx.x, e = q / s.B, b = q - e * s.B;
            int len = 0;
            if (q < n) len = bounds[b * (s.E + 1) + e + 1] - bounds[b * (s.E + 1) + e];
            len = (len + unit - 1) / unit;
            int inc = len;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int y = __shfl_up_sync(0xFFFFFFFFu, inc, d);
                if ((int)threadIdx.x >= d) inc += y;
            }
            if (q < n) start[q] = run + inc - len;
            run += __shfl_sync(0xFFFFFFFFu, inc, 31);
        }
        if (threadIdx.x == 0) start[n] = run;
    }
    __syncthreads();
}

// Last q with start[q] <= p, for 0 <= p < start[n]: the segment that p lies in (empty ones are passed over).
__device__ __forceinline__ int segment_of(const int* start, int n, int p) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= p) lo = mid; else hi = mid;
    }
    return lo;
}

#endif  // __CUDACC__

}  // namespace emc2
