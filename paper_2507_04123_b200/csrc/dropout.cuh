// Dropout without a stored mask: eight elements of a row share one number of the counter-based generator Philox4x32 with
// 10 rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011).
//
//   counter = (row, channel / 8, call, call >> 32), key = (seed, seed >> 32); element j of the eight takes 16 bits: the low
//   half of word j / 2 for even j, the high half for odd j; it is kept where these are >= round(65536 p)
//
// 16 bits, not 32, because the generator is what a pass over 16-bit rows would wait for: it takes 20 wide products per number.
// The kept share is therefore a multiple of 2^-16, and the factor is exact for that share.
#pragma once

#include <cmath>

#include "rows.cuh"

namespace emc2 {

struct Dropout {
    const unsigned long long* seed;      // {seed, number of the call} on the device
    uint32_t any;                        // 0: nothing is dropped
    uint32_t above;                      // else 16 bits are compared as the upper half of a word that has to be above this
    float factor;
};

inline bool is_share(float p) { return p >= 0.0f && p <= 1.0f; }
inline Dropout make_dropout(float p, const int64_t* d_seed) {
    Dropout d;
    d.seed = reinterpret_cast<const unsigned long long*>(d_seed);
    const int threshold = (int)std::floor((double)p * 65536.0 + 0.5);
    d.any = threshold > 0;
    d.above = (uint32_t)threshold * 65536u - 1u;         // of 65536: no word is above it
    d.factor = threshold < 65536 ? (float)(65536.0 / (65536 - threshold)) : 0.0f;
    return d;
}

#ifdef __CUDACC__

struct DropoutSeed {
    uint32_t key0, key1, call0, call1;
};
__device__ __forceinline__ DropoutSeed dropout_seed(const Dropout& d) {
    const unsigned long long key = __ldg(d.seed), call = __ldg(d.seed + 1);
    return {(uint32_t)key, (uint32_t)(key >> 32), (uint32_t)call, (uint32_t)(call >> 32)};
}

// Bits of K groups at once, round by round: the rounds' keys are worked out once for all, and the products of one group fill the
// waits of another's.
template <int K>
__device__ __forceinline__ void dropout_bits(uint4 (&bits)[K], const DropoutSeed& s, const uint32_t (&row)[K], const uint32_t (&group)[K]) {
    uint32_t k0 = s.key0, k1 = s.key1;
#pragma unroll
    for (int i = 0; i < K; ++i) bits[i] = make_uint4(row[i], group[i], s.call0, s.call1);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
#pragma unroll
        for (int i = 0; i < K; ++i) {
            uint4& c = bits[i];
            const unsigned long long a = (unsigned long long)c.x * 0xD2511F53u, b = (unsigned long long)c.z * 0xCD9E8D57u;
            c = make_uint4((uint32_t)(b >> 32) ^ c.y ^ k0, (uint32_t)b, (uint32_t)(a >> 32) ^ c.w ^ k1, (uint32_t)a);
        }
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
}

// Whether element j (known at compile time) of the eight is kept.
__device__ __forceinline__ bool dropout_keeps(const uint4& bits, int j, uint32_t above) {
    const uint32_t w = j < 2 ? bits.x : j < 4 ? bits.y : j < 6 ? bits.z : bits.w;
    return ((j & 1) ? w : w << 16) > above;              // the lower half of an odd element's word decides nothing: above ends in 0xFFFF
}

// ---- Eight elements of a row, at a multiple of eight channels.  `hi`: the row has the second four.  WIDE: rows of a multiple of eight
// channels, fp32 ones in buffers on 32 bytes, so that they are one access (a lane that stores 16 bytes of every 32 leaves half sectors).
struct Raw8 {
    uint4 a, b;                          // 16-bit elements lie in `a`
};
template <bool WIDE>
__device__ __forceinline__ Raw8 request8(const void* p, size_t vec, bool lo, bool hi, int type) {
    Raw8 r;
    r.a = r.b = make_uint4(0u, 0u, 0u, 0u);
    if (type == EMC2_F32) {
        if (WIDE) {
            if (lo) asm volatile("ld.global.nc.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                                 : "=r"(r.a.x), "=r"(r.a.y), "=r"(r.a.z), "=r"(r.a.w), "=r"(r.b.x), "=r"(r.b.y), "=r"(r.b.z), "=r"(r.b.w)
                                 : "l"(static_cast<const uint4*>(p) + vec));
        } else {
            if (lo) r.a = __ldg(static_cast<const uint4*>(p) + vec);
            if (hi) r.b = __ldg(static_cast<const uint4*>(p) + vec + 1);
        }
    } else if (WIDE) {
        if (lo) r.a = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint2*>(p) + vec));
    } else {
        if (lo) { const uint2 v = __ldg(static_cast<const uint2*>(p) + vec); r.a.x = v.x; r.a.y = v.y; }
        if (hi) { const uint2 v = __ldg(static_cast<const uint2*>(p) + vec + 1); r.a.z = v.x; r.a.w = v.y; }
    }
    return r;
}
__device__ __forceinline__ void floats8(float (&f)[8], const Raw8& r, int type) {
    float4 a, b;
    if (type == EMC2_F32) {
        a = make_float4(__uint_as_float(r.a.x), __uint_as_float(r.a.y), __uint_as_float(r.a.z), __uint_as_float(r.a.w));
        b = make_float4(__uint_as_float(r.b.x), __uint_as_float(r.b.y), __uint_as_float(r.b.z), __uint_as_float(r.b.w));
    } else {
        a = as_floats(make_uint2(r.a.x, r.a.y), type);
        b = as_floats(make_uint2(r.a.z, r.a.w), type);
    }
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
    f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
template <bool WIDE>
__device__ __forceinline__ void store8(void* p, size_t vec, bool hi, const float (&f)[8], int type) {
    if (type == EMC2_F32) {
        if (WIDE) {
            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(static_cast<float4*>(p) + vec),
                         "r"(__float_as_uint(f[0])), "r"(__float_as_uint(f[1])), "r"(__float_as_uint(f[2])), "r"(__float_as_uint(f[3])),
                         "r"(__float_as_uint(f[4])), "r"(__float_as_uint(f[5])), "r"(__float_as_uint(f[6])), "r"(__float_as_uint(f[7])) : "memory");
        } else {
            static_cast<float4*>(p)[vec] = make_float4(f[0], f[1], f[2], f[3]);
            if (hi) static_cast<float4*>(p)[vec + 1] = make_float4(f[4], f[5], f[6], f[7]);
        }
    } else {
        const uint4 h = make_uint4(as_halves(f[0], f[1], type), as_halves(f[2], f[3], type), as_halves(f[4], f[5], type), as_halves(f[6], f[7], type));
        if (WIDE) {
            *reinterpret_cast<uint4*>(static_cast<uint2*>(p) + vec) = h;
        } else {
            static_cast<uint2*>(p)[vec] = make_uint2(h.x, h.y);
            if (hi) static_cast<uint2*>(p)[vec + 1] = make_uint2(h.z, h.w);
        }
    }
}

#endif  // __CUDACC__

// Whether rows of `channels` in this buffer, on 16 bytes, can be accessed eight elements at once.
inline bool is_wide(int channels, int type, const void* p) { return channels % 8 == 0 && (type != EMC2_F32 || (reinterpret_cast<uintptr_t>(p) & 31) == 0); }
inline bool on_8_bytes(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 7) == 0; }

}  // namespace emc2
