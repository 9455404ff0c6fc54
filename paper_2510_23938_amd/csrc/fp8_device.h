// fp8_device.h -- element types and the 8-bit format (OCP E4M3) on the device.
#pragma once
#include <stdint.h>
#include <hip/hip_runtime.h>

namespace hv {

constexpr int kFp8Group = 128;        // columns (and, for weights, rows) that share a scale
constexpr float kFp8Largest = 448.0f;
constexpr float kFp8SmallestScale = 0x1p-126f;  // its reciprocal is finite too

// Eight consecutive elements, at the alignment of one: gfx950 loads and stores
// them as 16-byte words at any address.
template <typename T>
struct Eight {
    T v[8];
};

template <typename T>
__device__ __forceinline__ void load_eight(const T* p, uint32_t valid, float (&f)[8]) {
    if (valid >= 8) {
        Eight<T> e;
        __builtin_memcpy(&e, p, sizeof e);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = (float)e.v[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = (uint32_t)i < valid ? (float)p[i] : 0.0f;
    }
}

template <typename T>
__device__ __forceinline__ void store_eight(T* p, uint32_t valid, const float (&f)[8]) {
    if (valid >= 8) {
        Eight<T> e;
#pragma unroll
        for (int i = 0; i < 8; ++i) e.v[i] = (T)f[i];
        __builtin_memcpy(p, &e, sizeof e);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if ((uint32_t)i < valid) p[i] = (T)f[i];
    }
}

// The largest magnitude among the finite ones (0 where there is none).
__device__ __forceinline__ float finite_largest(const float (&y)[8]) {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float a = __builtin_fabsf(y[i]);
        m = a < __builtin_inff() ? fmaxf(m, a) : m;
    }
    return m;
}

// Largest of the 16 lanes of a DPP row, in all of them.
__device__ __forceinline__ float row16_max(float m) {
    auto rotated = [](float x, auto by) {
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 + decltype(by)::value, 0xf, 0xf,
                                                          true));
    };
    m = fmaxf(m, rotated(m, std::integral_constant<int, 8>{}));
    m = fmaxf(m, rotated(m, std::integral_constant<int, 4>{}));
    m = fmaxf(m, rotated(m, std::integral_constant<int, 2>{}));
    return fmaxf(m, rotated(m, std::integral_constant<int, 1>{}));
}

__device__ __forceinline__ float fp8_scale(float largest) {
    return largest > 0.0f ? fmaxf(largest / kFp8Largest, kFp8SmallestScale) : 1.0f;
}

// Codes of eight values under a scale.  The quotient y / scale is the correctly
// rounded one: y times the scale's reciprocal, and one correction by the exact
// remainder, two instructions where a division takes ten.  (Without it ties, which are
// frequent among 16-bit values, went either way: 0.25% of a weight matrix's codes.)
// Quotients of finite values are at most 448 (1 + 2^-23), which rounds to 448, so
// nothing is clamped; a NaN and an infinity become NaN.
__device__ __forceinline__ uint2 fp8_codes(const float (&y)[8], float scale) {
    const float inv = 1.0f / scale;
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float near = y[i] * inv;
        q[i] = fmaf(-fmaf(near, scale, -y[i]), inv, near);  // with these signs a zero keeps its own
        q[i] = __builtin_fabsf(y[i]) < __builtin_inff() ? q[i] : __builtin_nanf("");
    }
    uint2 w;
    int lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
    w.x = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], lo, true);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[4], q[5], 0, false);
    w.y = __builtin_amdgcn_cvt_pk_fp8_f32(q[6], q[7], lo, true);
    return w;
}

__device__ __forceinline__ void store_codes(uint8_t* p, uint32_t valid, uint2 w) {
    if (valid >= 8) {
        __builtin_memcpy(p, &w, 8);
    } else {
        const uint64_t b = (uint64_t)w.y << 32 | w.x;
        for (uint32_t i = 0; i < valid; ++i) p[i] = (uint8_t)(b >> (8 * i));
    }
}

}  // namespace hv
