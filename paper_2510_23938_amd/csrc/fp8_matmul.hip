// fp8_matmul.hip -- the product of two matrices held in 8 bits with a scale for
// each group of 128 (hv_fp8.h has the formula).
//
// A matrix instruction (16 x 16 outputs over 128 columns) covers exactly one
// group, so its result is a group's part of the sum; the vector unit then adds
// it, times the two scales, to the 32-bit accumulators.  B's rows are the
// instruction's rows and A's its columns: a lane then holds four consecutive
// columns of one row of C, and all of them take the same a_scale.
#include <type_traits>

#include "fp8_device.h"
#include "hv_kernels.h"

namespace hv {
namespace {

using int8x = __attribute__((ext_vector_type(8))) int;
using bf16x2 = __attribute__((ext_vector_type(2))) __bf16;
using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;
using float4x = __attribute__((ext_vector_type(4))) float;

// The matrix unit adds the 16 products of a lane's 16 bytes in fixed point and
// drops what lies 14 bits or more below the largest of them (measured); between
// those it adds in 32 bits.  That is 1.5e-5 of a typical sum, far below what a
// 16-bit result rounds off.  A 32-bit result does not lose it: its codes are
// widened to bfloat16, which holds them exactly, and the bfloat16
// instruction adds in 32 bits, at half the rate.
template <typename T>
__device__ __forceinline__ float4x group_product(int8x rows, int8x cols) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(rows, cols, float4x{0, 0, 0, 0}, 0, 0, 0, 0, 0, 0);
}

__device__ __forceinline__ bf16x8 widen(int lo, int hi) {
    const bf16x2 p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
    const bf16x2 q = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
    const bf16x2 r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
    const bf16x2 s = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
    return bf16x8{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
}

template <>
__device__ __forceinline__ float4x group_product<float>(int8x rows, int8x cols) {
    float4x sum = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < 8; w += 2)
        sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(rows[w], rows[w + 1]), widen(cols[w], cols[w + 1]), sum, 0,
                                                      0, 0);
    return sum;
}

// A lane's part of a 16-row fragment over a group: 16 bytes from p and 16 from
// p + 64 (which columns a lane holds does not matter, as long as both
// operands go by the same rule).  left: bytes of the row from p on, the rest
// reads as zeros.
__device__ __forceinline__ int8x load_fragment(const uint8_t* p, int left) {
    int8x f = {0, 0, 0, 0, 0, 0, 0, 0};
    if (left >= 80) {
        __builtin_memcpy(&f, p, 16);
        __builtin_memcpy((char*)&f + 16, p + 64, 16);
    } else {
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            uint32_t v = 0;
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int at = (w >= 4 ? 64 - 16 : 0) + 4 * w + b;
                if (at < left) v |= (uint32_t)p[at] << (8 * b);
            }
            f[w] = (int)v;
        }
    }
    return f;
}

template <typename T>
__device__ __forceinline__ void store_four(T* p, int valid, float4x v) {
    T o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = (T)v[i];
    if (valid >= 4) {
        __builtin_memcpy(p, o, sizeof o);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < valid) p[i] = o[i];
    }
}

// A workgroup makes 16 x 16 outputs; its four waves take every fourth group of
// columns, straight from memory, and join their sums through LDS.
template <typename T>
__global__ void __launch_bounds__(256) stream_kernel(const uint8_t* __restrict__ a, uint64_t ld_a,
                                                     const float* __restrict__ sa, const uint8_t* __restrict__ b,
                                                     uint64_t ld_b, const float* __restrict__ sb, uint32_t m,
                                                     uint32_t n, uint32_t k, T* __restrict__ c, uint64_t ld_c) {
    __shared__ float4x part[4][64];
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const uint32_t i0 = blockIdx.y * 16, j0 = blockIdx.x * 16;
    const uint32_t groups = (k + kFp8Group - 1) / kFp8Group;
    const uint32_t i = min(i0 + lane % 16, m - 1), j = min(j0 + lane % 16, n - 1);
    const uint32_t at = lane / 16 * 16;
    const uint8_t* pa = a + i * ld_a + at;
    const uint8_t* pb = b + j * ld_b + at;
    const float* psa = sa + (uint64_t)i * groups;
    const float* psb = sb + (uint64_t)(j0 / kFp8Group) * groups;
    float4x sum = {0, 0, 0, 0};
    for (uint32_t g = wave; g < groups; g += 4) {
        const int left = (int)(k - g * kFp8Group) - (int)at;
        const float4x p = group_product<T>(load_fragment(pb + g * kFp8Group, left),
                                           load_fragment(pa + g * kFp8Group, left));
        const float s = psa[g] * psb[g];
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] = fmaf(p[e], s, sum[e]);
    }
    part[wave][lane] = sum;
    __syncthreads();
    if (wave == 0) {
        sum = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
        const uint32_t row = i0 + lane % 16, col = j0 + lane / 16 * 4;
        if (row < m && col < n) store_four(c + row * ld_c + col, (int)(n - col), sum);
    }
}

}  // namespace

hipError_t launch_fp8_matmul(int type, const MatmulArgs& a, hipStream_t s) {
    auto run = [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        const dim3 grid((uint32_t)((a.n + 15) / 16), (uint32_t)((a.m + 15) / 16));
        stream_kernel<T><<<grid, 256, 0, s>>>(a.a, a.ld_a, a.a_scales, a.b, a.ld_b, a.b_scales, (uint32_t)a.m,
                                              (uint32_t)a.n, (uint32_t)a.k, (T*)a.c, a.ld_c);
        return hipGetLastError();
    };
    switch (type) {
        case kTypeBf16: return run((__bf16*)nullptr);
        case kTypeF16: return run((_Float16*)nullptr);
        default: return run((float*)nullptr);
    }
}

}  // namespace hv
