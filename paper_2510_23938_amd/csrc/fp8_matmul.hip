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
using int4x = __attribute__((ext_vector_type(4))) int;
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

// 16 bytes of a row that has `left` bytes from p on; zeros beyond them.
__device__ __forceinline__ int4x load_16(const uint8_t* p, int left) {
    int4x f = {0, 0, 0, 0};
    if (left >= 16) {
        __builtin_memcpy(&f, p, 16);
    } else {
        uint64_t lo = 0, hi = 0;
#pragma unroll 1
        for (int b = left - 1; b >= 0; --b) {
            hi = hi << 8 | lo >> 56;
            lo = lo << 8 | p[b];
        }
        f = int4x{(int)lo, (int)(lo >> 32), (int)hi, (int)(hi >> 32)};
    }
    return f;
}

// A lane's part of a 16-row fragment over a group: 16 bytes from p and 16 from
// p + 64 (which columns a lane holds does not matter, as long as both
// operands go by the same rule).
__device__ __forceinline__ int8x load_fragment(const uint8_t* p, int left) {
    const int4x lo = load_16(p, left), hi = load_16(p + 64, left - 64);
    return int8x{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
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

// ---------------------------------------------------------------------------
// tiles in LDS

constexpr uint64_t kMaxTileLd = (1 << 23) - 1;  // offsets within a tile's 256 rows stay below 2^31

// A buffer that starts at p; its loads' offsets are in bounds by construction.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_at(const void* p) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, 0x7fffffff, 0x00020000);
}

// 16 bytes a lane from the buffer to consecutive places in LDS.
__device__ __forceinline__ void buffer_to_lds(__amdgpu_buffer_rsrc_t from, void* lds, uint32_t lane_offset,
                                              uint32_t offset) {
#ifdef __HIP_DEVICE_COMPILE__  // the host pass does not know this builtin, and would drop the kernel for it
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, lds, 16, lane_offset, offset, 0, 0);
#endif
}

// A workgroup makes TM x TN outputs, WM x WN waves a part each.  While one
// group's rows of A and B (128 bytes each) are multiplied, the next group's go
// from memory to the other half of the LDS.
template <typename T, int TM, int TN, int WM, int WN, bool kDirect>
__global__ void __launch_bounds__(WM* WN * 64)
    tile_kernel(const uint8_t* __restrict__ a, uint64_t ld_a, const float* __restrict__ sa,
                const uint8_t* __restrict__ b, uint64_t ld_b, const float* __restrict__ sb, uint32_t m, uint32_t n,
                uint32_t k, T* __restrict__ c, uint64_t ld_c, uint32_t tiles_m, uint32_t tiles) {
    constexpr int kThreads = WM * WN * 64;
    constexpr int MT = TM / WM / 16, NT = TN / WN / 16;
    constexpr int kLoadsA = TM * 8 / kThreads, kLoadsB = TN * 8 / kThreads;  // 16-byte loads of a lane
    static_assert(TN / WN <= kFp8Group && kFp8Group % (TN / WN) == 0, "a wave's columns share a scale");
    constexpr int kScales = TM + 64;  // A's, then B's
    static_assert(kScales / 64 <= WM * WN, "a wave loads 64 scales");
    static_assert(MT >= 3 && kLoadsA <= NT && kLoadsB <= (MT - 2) * NT, "a group's loads fit between its products");
    __shared__ alignas(1024) uint8_t a0[TM * 128], b0[TN * 128], a1[TM * 128], b1[TN * 128];
    __shared__ alignas(256) float4x scales[2][kScales];  // of four groups, and of the next four

    // Workgroups go to the eight XCDs in turn; each XCD gets a run of tiles, in
    // panels of 8 tiles' rows, so that the 32 it has at a time are 8 x 4 and its L2
    // serves each row of A and B several times.
    const uint32_t per_xcd = gridDim.x / 8;
    const uint32_t tile = blockIdx.x % 8 * per_xcd + blockIdx.x / 8;
    if (tile >= tiles) return;
    const uint32_t tiles_n = tiles / tiles_m;
    const uint32_t panel = tile / (8 * tiles_n), in_panel = tile - panel * 8 * tiles_n;
    const uint32_t panel_rows = min(8u, tiles_m - panel * 8);
    const uint32_t i0 = (panel * 8 + in_panel % panel_rows) * TM, j0 = in_panel / panel_rows * TN;

    const uint32_t lane = threadIdx.x % 64;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t wave_i = wave / WN * (TM / WM), wave_j = wave % WN * (TN / WN);
    const uint32_t groups = (k + kFp8Group - 1) / kFp8Group;

    // The row of LDS that a lane of load instruction l fills is 8 * (l * waves + wave) + lane / 8; its
    // 16-byte places hold the row's chunks in the order place ^ (row % 8), so that
    // the lanes of a fragment read from different banks.
    const uint32_t chunk = (lane % 8 ^ lane / 8) * 16;
    const uint8_t* const tile_a = a + i0 * ld_a;
    const uint8_t* const tile_b = b + j0 * ld_b;
    uint32_t from_a[kLoadsA], from_b[kLoadsB];
#pragma unroll
    for (int l = 0; l < kLoadsA; ++l)
        from_a[l] = min(8 * (l * WM * WN + wave) + lane / 8, m - 1 - i0) * (uint32_t)ld_a + chunk;
#pragma unroll
    for (int l = 0; l < kLoadsB; ++l)
        from_b[l] = min(8 * (l * WM * WN + wave) + lane / 8, n - 1 - j0) * (uint32_t)ld_b + chunk;
    const uint32_t part_s = wave % (kScales / 64);  // waves beyond them load a part again
    const bool scales_of_a = part_s < TM / 64;
    const float* const tile_s = scales_of_a ? sa + (uint64_t)i0 * groups : sb + (uint64_t)(j0 / kFp8Group) * groups;
    const uint32_t from_s = (scales_of_a ? min(part_s * 64 + lane, m - 1 - i0)
                                         : min(lane, (n - 1) / kFp8Group - j0 / kFp8Group)) * groups;

    // Buffer loads: a lane's offset stays, the group's is a scalar.
    const auto all_a = rows_at(tile_a), all_b = rows_at(tile_b);
    auto load_a = [&](int l, uint32_t g, uint8_t* la) {
        buffer_to_lds(all_a, la + 1024 * (l * WM * WN + wave), from_a[l], g * kFp8Group);
    };
    auto load_b = [&](int l, uint32_t g, uint8_t* lb) {
        buffer_to_lds(all_b, lb + 1024 * (l * WM * WN + wave), from_b[l], g * kFp8Group);
    };
    // Scales come four groups at a time (a load of one group's takes as many
    // requests as a load of a tile's 128-byte rows), the last four of a row where
    // there are fewer left, and are kept in LDS as [row][4].
    const uint32_t last_four = max(groups, 4u) - 4;
    float4x four;
    auto load_four = [&](uint32_t q) { __builtin_memcpy(&four, tile_s + from_s + min(4 * q, last_four), 16); };
    auto keep_four = [&](uint32_t q) { scales[q % 2][64 * part_s + lane] = four; };
    // where group g's scales stand, from a row's first one on
    auto scales_at = [&](uint32_t g) {
        return (const float*)scales + (g / 4 % 2 * kScales * 4 + g - min(g / 4 * 4, last_four));
    };
    // The columns beyond the last whole group, with zeros after them.
    auto load_rest = [&](uint32_t g, uint8_t* la, uint8_t* lb) {
        const uint32_t at = g * kFp8Group;
        const int left = (int)(k - at) - (int)chunk;
#pragma unroll
        for (int l = 0; l < kLoadsA; ++l)
            *(int4x*)(la + 1024 * (l * WM * WN + wave) + 16 * lane) = load_16(tile_a + at + from_a[l], left);
#pragma unroll
        for (int l = 0; l < kLoadsB; ++l)
            *(int4x*)(lb + 1024 * (l * WM * WN + wave) + 16 * lane) = load_16(tile_b + at + from_b[l], left);
    };

    float4x sum[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) sum[i][j] = float4x{0, 0, 0, 0};
    // Where the lane reads its fragments: 16 bytes at *_lo and 16 at *_hi, from the
    // first row of the wave's part on.  The empty asm keeps them whole, so that a read's
    // row is an offset in its instruction and takes no register.
    const uint32_t row16 = lane % 16, quarter = lane / 16;
    const uint32_t place = row16 * 128 + (quarter ^ row16 % 8) * 16;
    uint32_t a_lo = wave_i * 128 + place, a_hi = wave_i * 128 + (place ^ 64);
    uint32_t b_lo = wave_j * 128 + place, b_hi = wave_j * 128 + (place ^ 64);
    uint32_t a_scale = 4 * (wave_i + row16);
    asm("" : "+v"(a_lo), "+v"(a_hi), "+v"(b_lo), "+v"(b_hi), "+v"(a_scale));
    auto fragment = [&](const uint8_t* rows, uint32_t at_lo, uint32_t at_hi) {
        const int4x lo = *(const int4x*)(rows + at_lo), hi = *(const int4x*)(rows + at_hi);
        return int8x{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    };
    auto fragment_a = [&](const uint8_t* la, int i) { return fragment(la + 2048 * i, a_lo, a_hi); };
    auto fragment_b = [&](const uint8_t* lb, int j) { return fragment(lb + 2048 * j, b_lo, b_hi); };
    // Every wave's loads but its last kLater are in LDS, and no wave reads what it read before.
    auto meet = [&](auto later) {
        constexpr int kLater = decltype(later)::value;
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt((kLater & 15) | (kLater >> 4) << 14 | 7 << 4);  // vmcnt(kLater), lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    constexpr std::integral_constant<int, 0> kNone;
    constexpr std::integral_constant<int, kLoadsB> kOfB;

    // One group.  The fragments of A's next 16 rows come from LDS while these are
    // multiplied, and the next group's first ones while this group's last are.  By
    // then every wave has read all it needs of this half's A, so the group after
    // the next may be loaded there; of B every wave holds all it needs from the
    // start, so the group after the next is loaded over it as soon as they have met.
    // (Past the last group the last one is loaded again: nobody reads it.)  Loads are
    // issued one after each product, so that no wave stands in line for them.  A
    // product is added to its sum two instructions later, when the matrix unit has it.
    const uint32_t whole = k / kFp8Group;
    int8x fb[NT], fa;
    float scale_a, scale_b;
    const uint32_t b_scale = 4 * (TM + wave_j / kFp8Group);
    auto first = [&](const uint8_t* la, const uint8_t* lb, uint32_t g) {
#pragma unroll
        for (int j = 0; j < NT; ++j) fb[j] = fragment_b(lb, j);
        fa = fragment_a(la, 0);
        scale_a = scales_at(g)[a_scale];
        scale_b = scales_at(g)[b_scale];
    };
    auto multiply = [&](uint32_t g, uint8_t* la, uint8_t* lb, const uint8_t* next_a, const uint8_t* next_b) {
        const bool new_four = g % 4 == 1 && g / 4 * 4 + 4 < groups;
        const float* const now = scales_at(g);
        const float* const next = scales_at(g + 1);
        if (new_four) load_four(g / 4 + 1);
        const float in_b = scale_b;
        float4x p[3];
        float s[2];
        auto add = [&](int t) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                sum[t / NT][t % NT][e] = fmaf(p[t % 3][e], s[t / NT % 2], sum[t / NT][t % NT][e]);
            asm volatile("" : "+v"(sum[t / NT][t % NT]));  // here, not after a later branch
        };
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const bool last = i == MT - 1;
            if (i == 1) meet(std::integral_constant<int, 63>{});
            if (last) {
                meet(kOfB);
                if (new_four) keep_four(g / 4 + 1);
                scale_b = next[b_scale];
            }
            const int8x next_fa = last ? fragment_a(next_a, 0) : fragment_a(la, i + 1);
            const float next_scale = last ? next[a_scale] : now[a_scale + 64 * (i + 1)];
            s[i % 2] = scale_a * in_b;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const int t = i * NT + j;
                p[t % 3] = group_product<T>(fb[j], fa);
                __builtin_amdgcn_sched_barrier(0);
                if (last) {
                    fb[j] = fragment_b(next_b, j);
                    if (j < kLoadsA) load_a(j, min(g + 2, whole - 1), la);
                } else if (i >= 1 && t - NT < kLoadsB) {
                    load_b(t - NT, min(g + 2, whole - 1), lb);
                }
                if (t >= 2) add(t - 2);
                __builtin_amdgcn_sched_barrier(0);
            }
            fa = next_fa;
            scale_a = next_scale;
        }
        add(MT * NT - 2);
        add(MT * NT - 1);
    };

    for (uint32_t e = 0; e < 4; ++e) four[e] = e < groups ? tile_s[from_s + e] : 0.0f;
    keep_four(0);
    if (whole > 0) {
        const uint32_t second = min(1u, whole - 1);
#pragma unroll
        for (int l = 0; l < kLoadsA; ++l) load_a(l, 0, a0);
#pragma unroll
        for (int l = 0; l < kLoadsB; ++l) load_b(l, 0, b0);
#pragma unroll
        for (int l = 0; l < kLoadsB; ++l) load_b(l, second, b1);
        meet(kOfB);
#pragma unroll
        for (int l = 0; l < kLoadsA; ++l) load_a(l, second, a1);
        first(a0, b0, 0);
        for (uint32_t g = 0; g + 1 < whole; g += 2) {
            multiply(g, a0, b0, a1, b1);
            multiply(g + 1, a1, b1, a0, b0);
        }
        if (whole % 2 != 0) multiply(whole - 1, a0, b0, a1, b1);
        meet(kNone);
    }
    if (whole < groups) {
        load_rest(whole, a0, b0);
        __syncthreads();
        first(a0, b0, whole);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int8x rest = fragment_a(a0, i);
            const float s = scales_at(whole)[a_scale + 64 * i] * scale_b;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const float4x p = group_product<T>(fb[j], rest);
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[i][j][e] = fmaf(p[e], s, sum[i][j][e]);
            }
        }
    }
    const bool inside = i0 + TM <= m && j0 + TN <= n;
    T* const out = c + (uint64_t)(i0 + wave_i + row16) * ld_c + j0 + wave_j + quarter * 4;
    const int rows_left = (int)(m - i0 - wave_i - row16), cols_left = (int)(n - j0 - wave_j - quarter * 4);
    if (inside) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) store_four(out + 16 * i * ld_c + 16 * j, 4, sum[i][j]);
    } else {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (16 * i < rows_left && 16 * j + e < cols_left)
                        out[16 * i * ld_c + 16 * j + e] = (T)sum[i][j][e];
    }
}

}  // namespace

hipError_t launch_fp8_matmul(int type, const MatmulArgs& a, hipStream_t s) {
    auto run = [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        const bool direct = a.ld_a % 16 == 0 && a.ld_b % 16 == 0 && (uintptr_t)a.a % 16 == 0 && (uintptr_t)a.b % 16 == 0 &&
                            a.ld_a <= kMaxTileLd && a.ld_b <= kMaxTileLd;
        if (direct && a.m > 64 && a.k > 0) {
            constexpr int TM = sizeof(T) == 4 ? 128 : 256, TN = TM;
            const uint32_t tiles_m = (uint32_t)((a.m + TM - 1) / TM);
            const uint32_t tiles = tiles_m * (uint32_t)((a.n + TN - 1) / TN);
            tile_kernel<T, TM, TN, 2, TN / 64, true><<<(tiles + 7) / 8 * 8, TN / 64 * 128, 0, s>>>(
                a.a, a.ld_a, a.a_scales, a.b, a.ld_b, a.b_scales, (uint32_t)a.m, (uint32_t)a.n, (uint32_t)a.k, (T*)a.c,
                a.ld_c, tiles_m, tiles);
            return hipGetLastError();
        }
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
