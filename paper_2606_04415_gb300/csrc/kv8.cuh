// The 8-bit cache with one power-of-two scale for each block of tokens and kv head.
//
// A block of a pool: codes [kv heads][slots][d], then one fp32 scale 2^e a kv head,
// padded to 16 bytes. INT8: value (code - 128) 2^e, codes 1..255; E4M3: value of
// the e4m3 code times 2^e. Powers of two make every stored value exact in bf16 and
// every change of scale of an e4m3 row exact down to its subnormals.
#pragma once

#include <cuda_fp8.h>

#include "fp8.cuh"

namespace fnpu {
namespace kv8 {

constexpr int kMinExp = -60, kMaxExp = 60;

__host__ __device__ constexpr int64_t block_bytes(int hkv, int bs, int d) {
    return static_cast<int64_t>(hkv) * bs * d + 16 * ((hkv + 3) / 4);
}

__device__ __forceinline__ float pow2(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }
// exponent of a stored scale, held to the format's range whatever the bytes are
__device__ __forceinline__ int scale_exp(float scale) {
    return min(max(static_cast<int>(__float_as_uint(scale) >> 23 & 255u) - 127, kMinExp), kMaxExp);
}

template <int kFormat>
constexpr float kLargest = kFormat == FNPU_KV_INT8_BLOCK ? 127.f : 448.f;

// The least e with amax <= largest * 2^e, not clamped above (amax finite, >= 0).
// amax = m 2^x with m in [1, 2); largest = 1.984375 * 2^6 or 1.75 * 2^8.
template <int kFormat>
__device__ __forceinline__ int required_exp(float amax) {
    const uint32_t bits = __float_as_uint(amax), top = __float_as_uint(kLargest<kFormat>);
    const int x = static_cast<int>(bits >> 23) - static_cast<int>(top >> 23);
    return max(kMinExp, x + ((bits & 0x7FFFFFu) > (top & 0x7FFFFFu) ? 1 : 0));
}

// Codes of eight values over 2^e, of magnitude at most kLargest there: nearest, ties to
// even.
template <int kFormat>
__device__ __forceinline__ uint2 encode8(const float (&f)[8], float inv) {
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if constexpr (kFormat == FNPU_KV_INT8_BLOCK) {
            // x + 1.5 * 2^23 + 128 is rounded to an integer whose low byte is x + 128 (the
            // product is exact)
            uint32_t c[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) c[j] = __float_as_uint(__fmaf_rn(f[4 * i + j], inv, 12583040.f));
            w[i] = __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
        } else {
            const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(f[4 * i] * inv, f[4 * i + 1] * inv), __NV_SATFINITE, __NV_E4M3);
            const uint32_t hi =
                __nv_cvt_float2_to_fp8x2(make_float2(f[4 * i + 2] * inv, f[4 * i + 3] * inv), __NV_SATFINITE, __NV_E4M3);
            w[i] = lo | hi << 16;
        }
    }
    return make_uint2(w[0], w[1]);
}

// Four codes as fp32 values (before the scale).
template <int kFormat>
__device__ __forceinline__ void decode4(uint32_t w, float (&f)[4]) {
    if constexpr (kFormat == FNPU_KV_INT8_BLOCK) {
#pragma unroll
        for (int j = 0; j < 4; ++j)  // 2^23 + code, less 2^23 + 128
            f[j] = __uint_as_float(__byte_perm(w, 0x4B000000u, 0x7440 + j)) - 8388736.f;
    } else {
        uint32_t lo, hi;
        e4m3x4_to_f16x2x2(w, lo, hi);
        const float2 a = __half22float2(*reinterpret_cast<const __half2 *>(&lo));
        const float2 b = __half22float2(*reinterpret_cast<const __half2 *>(&hi));
        f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y;
    }
}

// Four codes as f16, exactly: neighbouring bytes in pairs (0, 1) and (2, 3), or with
// kAcross bytes (0, 2) and (1, 3). INT8: 1024 + code is the f16 with the code as its
// low byte; less 1152.
template <int kFormat, bool kAcross>
__device__ __forceinline__ void codes_to_f16(uint32_t w, uint32_t &a, uint32_t &b) {
    if constexpr (kFormat == FNPU_KV_INT8_BLOCK) {
        const uint32_t x = __byte_perm(w, 0x64646464u, kAcross ? 0x4240 : 0x4140);
        const uint32_t y = __byte_perm(w, 0x64646464u, kAcross ? 0x4341 : 0x4342);
        const uint32_t k = 0x64806480u;
        const __half2 u = __hsub2(*reinterpret_cast<const __half2 *>(&x), *reinterpret_cast<const __half2 *>(&k));
        const __half2 v = __hsub2(*reinterpret_cast<const __half2 *>(&y), *reinterpret_cast<const __half2 *>(&k));
        a = *reinterpret_cast<const uint32_t *>(&u);
        b = *reinterpret_cast<const uint32_t *>(&v);
    } else {
        e4m3x4_to_f16x2x2(kAcross ? __byte_perm(w, 0, 0x3120) : w, a, b);
    }
}

}  // namespace kv8
}  // namespace fnpu
