// fp8_adapters.hip -- low-rank adapters of many requests beside a shared product:
//   out[t] = y[t] + f_a * (x[t] down_a^T) up_a^T,  a = index[t],
// with x in codes and scales as the product takes it.
//
// Two kernels, as the second needs a token's whole inner row: the first makes the inner
// rows x down^T (the columns in parts, whose sums lie in the workspace), the second multiplies
// them by `up` and adds y.  Both are bound by memory: x, the adapters in use, y and the
// output once each.  Tokens are taken 16 at a time as they come; for each of the different
// adapters among them one product is made, of which the tokens keep theirs.  So
// nothing is sorted, a prompt's tokens share one product, and in a batch of many requests each
// adapter is read once for 16 tokens; the matrix unit has time for the products thrown away.
//
// The inner rows stay in 32 bits: the second product is made by the 32-bit instruction,
// whose rate is enough beside reading y and writing the output.
#include <algorithm>
#include <type_traits>

#include "cache_device.h"

namespace hv {
namespace {

using bf16x2 = __attribute__((ext_vector_type(2))) __bf16;
using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;
using f16x2 = __attribute__((ext_vector_type(2))) _Float16;
using f16x8 = __attribute__((ext_vector_type(8))) _Float16;
using float4x = __attribute__((ext_vector_type(4))) float;

constexpr int kTokens = 16;    // of a product
constexpr int kWaves = 4;
constexpr int kRanks = 64;     // of a workgroup of the first kernel
constexpr uint32_t kNone = ~0u;

template <typename W>
struct Inner;

template <>
struct Inner<__bf16> {
    using Eight = bf16x8;
    static __device__ __forceinline__ Eight codes(uint32_t lo, uint32_t hi) {
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
        const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
        const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
        const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
        return Eight{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
    static __device__ __forceinline__ float4x mul(Eight a, Eight b, float4x c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};

template <>
struct Inner<_Float16> {
    using Eight = f16x8;
    static __device__ __forceinline__ Eight codes(uint32_t lo, uint32_t hi) {
        const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false);
        const f16x2 b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
        const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false);
        const f16x2 d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
        return Eight{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
    static __device__ __forceinline__ float4x mul(Eight a, Eight b, float4x c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
};

// N elements of which `left` are there; zeros for the others.
template <int N, typename E>
__device__ __forceinline__ void load_some(const E* p, int left, E (&v)[N]) {
    if (left >= N) {
        __builtin_memcpy(v, p, sizeof v);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = i < left ? p[i] : (E)0;
}

// The adapter of the tile's token lane % 16; kNone for those of none and past the last token.
__device__ __forceinline__ uint32_t adapter_of(const AdapterArgs& x, uint64_t tile) {
    const uint64_t token = tile * kTokens + lane_id() % kTokens;
    const uint32_t a = token < x.m ? (uint32_t)x.index[token] : kNone;
    return a < x.adapters ? a : kNone;
}

// ---------------------------------------------------------------------------
// inner rows: a workgroup takes 16 tokens, one of the adapters among them, up to 64 ranks and a part of the columns

template <typename W>
__global__ void __launch_bounds__(kWaves * 64) down_kernel(AdapterArgs x) {
    using Eight = typename Inner<W>::Eight;
    constexpr int RF = kRanks / 16;
    __shared__ float4x sums[kWaves][RF][64];
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t n = lane % 16, g = lane / 16;
    const uint64_t tile = (uint64_t)(blockIdx.z % x.token_rows) * kRowOfItems + blockIdx.x;
    if (tile * kTokens >= x.m) return;
    const uint32_t rank0 = blockIdx.y / x.distinct * kRanks;
    const uint32_t mine = adapter_of(x, tile);
    // the blockIdx.y-th of the different adapters
    uint64_t left = __ballot(mine != kNone);
    uint32_t adapter = kNone;
    for (uint32_t j = blockIdx.y % x.distinct; left != 0; --j) {
        const uint32_t a = __builtin_amdgcn_readlane(mine, __builtin_ctzll(left));
        if (j == 0) {
            adapter = a;
            break;
        }
        left &= ~__ballot(mine == a);
    }
    if (adapter == kNone) return;
    const uint32_t split = blockIdx.z / x.token_rows;
    const uint32_t groups = (uint32_t)((x.k + kFp8Group - 1) / kFp8Group);
    const uint32_t first = split * x.split_groups, end = min(first + x.split_groups, groups);
    const uint32_t ranks = min((uint32_t)x.rank - rank0, (uint32_t)kRanks);
    const uint64_t token = min(tile * kTokens + n, x.m - 1);  // past the last one its row again, which is not kept
    const uint8_t* const x_row = x.x + token * x.ld_x;
    const float* const s_row = x.x_scales + token * groups;
    const W* const down = (const W*)x.down + ((uint64_t)adapter * x.rank + rank0) * x.k;
    const bool keep = mine == adapter;

    float4x inner[RF];
#pragma unroll
    for (int f = 0; f < RF; ++f) inner[f] = float4x{0, 0, 0, 0};
    for (uint32_t group = first + wave; group < end; group += kWaves) {
        const float scale = s_row[group];
        float4x part[RF];
#pragma unroll
        for (int f = 0; f < RF; ++f) part[f] = float4x{0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const uint32_t col = group * kFp8Group + 64 * c + 16 * g;
            const int there = col < x.k ? (int)min((uint32_t)x.k - col, 16u) : 0;
            uint8_t codes[16];
            load_some(x_row + col, there, codes);
            uint32_t w[4];
            __builtin_memcpy(w, codes, 16);
            const Eight low = Inner<W>::codes(w[0], w[1]), high = Inner<W>::codes(w[2], w[3]);
#pragma unroll
            for (int f = 0; f < RF; ++f) {
                if (16u * f >= ranks) break;
                W a[16];
                load_some(down + (uint64_t)min(16 * f + n, ranks - 1) * x.k + col, there, a);
                Eight e[2];
                __builtin_memcpy(e, a, 32);
                part[f] = Inner<W>::mul(e[0], low, part[f]);
                part[f] = Inner<W>::mul(e[1], high, part[f]);
            }
        }
#pragma unroll
        for (int f = 0; f < RF; ++f) inner[f] += scale * part[f];
    }
#pragma unroll
    for (int f = 0; f < RF; ++f) sums[wave][f][lane] = inner[f];
    __syncthreads();
    const uint32_t f = wave;  // each wave joins one fragment of 16 ranks
    static_assert(kWaves == RF, "a fragment for each wave");
    if (!keep || 16 * f + 4 * g >= ranks) return;
    float4x sum = sums[0][f][lane];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) sum += sums[w][f][lane];
    float* const to = x.inner + ((uint64_t)split * x.m + tile * kTokens + n) * x.inner_ld + rank0 + 16 * f + 4 * g;
    *(float4x*)to = sum;
}

// ---------------------------------------------------------------------------
// outputs: a workgroup takes 64 columns and x.tiles tiles of 16 tokens, its waves in turn the adapters among them

template <typename T, typename W>
__global__ void __launch_bounds__(kWaves * 64) up_kernel(AdapterArgs x) {
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t n = lane % 16, g = lane / 16;
    const uint64_t item = item_of_block();
    const uint32_t column_blocks = (uint32_t)((x.n + 63) / 64);
    const uint64_t group = item / column_blocks, col0 = (item - group * column_blocks) * 64;
    const uint64_t tiles = (x.m + kTokens - 1) / kTokens;
    const uint64_t col = col0 + 16 * g;  // of the lane's 16 outputs
    const int there = col < x.n ? (int)min(x.n - col, (uint64_t)16) : 0;
    uint32_t job = 0;
    for (uint64_t tile = group * x.tiles; tile < min((group + 1) * x.tiles, tiles); ++tile) {
        const uint32_t mine = adapter_of(x, tile);
        const uint64_t token = tile * kTokens + n;
        uint64_t left = __ballot(token < x.m);
        while (left != 0) {
            const uint32_t a = __builtin_amdgcn_readlane(mine, __builtin_ctzll(left));
            left &= ~__ballot(mine == a);
            if (job++ % kWaves != wave) continue;
            const bool keep = mine == a && token < x.m;
            T y[16];
            load_some((const T*)x.y + token * x.ld_y + col, keep ? there : 0, y);
            float4x out[4];
#pragma unroll
            for (int f = 0; f < 4; ++f) out[f] = float4x{0, 0, 0, 0};
            if (a != kNone) {
                const W* const up = (const W*)x.up + (uint64_t)a * x.n * x.rank;
                const float factor = x.factors ? x.factors[a] : 1.0f;
                for (uint32_t r0 = 0; r0 < x.rank; r0 += 16) {
                    const uint32_t r = r0 + 4 * g;
                    const int ranks = r < x.rank ? (int)min((uint32_t)x.rank - r, 4u) : 0;
                    float4x t = {0, 0, 0, 0};
                    if (keep && ranks > 0) {
                        const float* p = x.inner + token * x.inner_ld + r;
                        for (uint32_t s = 0; s < x.splits; ++s, p += x.m * x.inner_ld) t += *(const float4x*)p;
                        t *= factor;
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) t[i] = i < ranks ? t[i] : 0.0f;
#pragma unroll
                    for (int f = 0; f < 4; ++f) {
                        // row m of fragment f is the column 16 (m / 4) + 4 f + m % 4: a lane gets 16 neighbours
                        const uint64_t c = min(col0 + 16 * (n / 4) + 4 * f + n % 4, x.n - 1);
                        W w[4];
                        load_some(up + c * x.rank + r, ranks, w);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            out[f] = __builtin_amdgcn_mfma_f32_16x16x4f32((float)w[i], t[i], out[f], 0, 0, 0);
                    }
                }
            }
            if (!keep) continue;
            T* const to = (T*)x.out + token * x.ld_out + col;
#pragma unroll
            for (int i = 0; i < 16; ++i) y[i] = (T)((float)y[i] + out[i / 4][i % 4]);
            if (there == 16) {
                __builtin_memcpy(to, y, sizeof y);
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (i < there) to[i] = y[i];
            }
        }
    }
}

template <typename T, typename W>
hipError_t launch(const AdapterArgs& a, hipStream_t s) {
    const uint64_t tiles = (a.m + kTokens - 1) / kTokens;
    if (a.adapters > 0 && a.k > 0) {
        const uint32_t rank_blocks = (uint32_t)((a.rank + kRanks - 1) / kRanks);
        dim3 grid = item_grid((uint32_t)tiles, a.distinct * rank_blocks);
        grid.z *= a.splits;
        down_kernel<W><<<grid, kWaves * 64, 0, s>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const uint64_t items = (a.n + 63) / 64 * ((tiles + a.tiles - 1) / a.tiles);
    up_kernel<T, W><<<item_grid((uint32_t)items), kWaves * 64, 0, s>>>(a);
    return hipGetLastError();
}

template <typename T>
hipError_t launch(int adapter_type, const AdapterArgs& a, hipStream_t s) {
    return adapter_type == kTypeBf16 ? launch<T, __bf16>(a, s) : launch<T, _Float16>(a, s);
}

}  // namespace

AdapterPlan fp8_adapter_plan(uint64_t m, uint64_t k, uint64_t rank, uint64_t adapters) {
    AdapterPlan p = {};
    const uint64_t tiles = (m + kTokens - 1) / kTokens, groups = (k + kFp8Group - 1) / kFp8Group;
    p.distinct = (uint32_t)std::max<uint64_t>(1, std::min({(uint64_t)kTokens, m, adapters}));
    p.inner_ld = (uint32_t)((rank + 3) / 4 * 4);
    // columns in parts until there are two workgroups for each unit, four groups a part at least
    const uint64_t wanted = 512 / std::max<uint64_t>(1, tiles * p.distinct * ((rank + kRanks - 1) / kRanks));
    const uint64_t splits = std::max<uint64_t>(1, std::min<uint64_t>({wanted, (groups + 3) / 4, 16}));
    p.split_groups = (uint32_t)std::max<uint64_t>(1, (groups + splits - 1) / splits);
    p.splits = (uint32_t)std::max<uint64_t>(1, (groups + p.split_groups - 1) / p.split_groups);
    p.tiles = m <= 1024 ? 1 : 4;
    p.token_rows = (uint32_t)((tiles + kRowOfItems - 1) / kRowOfItems);
    p.workspace = adapters > 0 && k > 0 ? (uint64_t)p.splits * m * p.inner_ld * sizeof(float) : 0;
    return p;
}

hipError_t launch_fp8_adapters(int type, int adapter_type, AdapterArgs a, const AdapterPlan& p, hipStream_t s) {
    a.distinct = p.distinct, a.splits = p.splits, a.split_groups = p.split_groups, a.tiles = p.tiles;
    a.inner_ld = p.inner_ld, a.token_rows = p.token_rows;
    if (a.k == 0) a.adapters = 0;  // nothing to add
    return type == kTypeBf16  ? launch<__bf16>(adapter_type, a, s)
           : type == kTypeF16 ? launch<_Float16>(adapter_type, a, s)
                              : launch<float>(adapter_type, a, s);
}

}  // namespace hv
