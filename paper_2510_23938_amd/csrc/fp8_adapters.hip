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
// whose rate is enough beside reading y and writing the output (2048 x 28672 of rank 16: 5 of 68 us went away with
// three quarters of it).
//
// 2048 tokens of four prompts, 8192 x 28672, rank 16: 16 and 67 us (3.6 TB/s; a copy 4.75: reading `up` anew for each
// 16 tokens costs 12 of them); 32 tokens with 16 adapters in each 16, 8192 x 8192: 6 and 6 us, three trips to memory each.
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
constexpr int kRanks = 64;     // of a workgroup of the first kernel
constexpr int kMostWaves = 16; // of a workgroup
constexpr int kStaged = 128;   // ranks of inner rows that the second kernel has in LDS
constexpr uint32_t kNone = ~0u;
constexpr float kNothingAdded = -0.0f;  // leaves zeros of either sign as they are

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

// N neighbouring elements.  kAll: all are there; otherwise `left` are, the others come back as zeros, and `last` is the
// last one that may be read.  The choice is made for whole loops, not for each load: what is loaded on one of two
// ways has to arrive before they meet.
template <bool kAll, int N, typename E>
__device__ __forceinline__ void load_some(const E* p, int left, const E* last, E (&v)[N]) {
    if constexpr (kAll) {
        __builtin_memcpy(v, p, sizeof v);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = p + i < last ? p[i] : *last;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = i < left ? v[i] : (E)0;
    }
}

// The adapter of the tile's token lane % 16; kNone for those of none and past the last token.
__device__ __forceinline__ uint32_t adapter_of(const AdapterArgs& x, uint64_t tile) {
    const uint64_t token = tile * kTokens + lane_id() % kTokens;
    const uint32_t a = token < x.m ? (uint32_t)x.index[token] : kNone;
    return a < x.adapters ? a : kNone;
}

// ---------------------------------------------------------------------------
// inner rows: a workgroup takes 16 tokens, one of the adapters among them, up to 64 ranks and a part of the columns

// Its waves take the groups of the columns in turn and add their sums through LDS: 4 of them where the columns are
// in parts for the sake of few tokens, 16 where many tokens fill the chip, which then need no parts.
template <typename W, int kWaves>
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
    auto add_group = [&](auto all, uint32_t group) {
        constexpr bool kAll = decltype(all)::value;
        const float scale = s_row[group];
        uint8_t codes[2][16];
        W a[RF][2][16];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const uint32_t col = group * kFp8Group + 64 * c + 16 * g;
            const int there = kAll ? 16 : col < x.k ? (int)min((uint32_t)x.k - col, 16u) : 0;
            load_some<kAll>(x_row + col, there, x_row + x.k - 1, codes[c]);
#pragma unroll
            for (int f = 0; f < RF; ++f) {
                if (16u * f >= ranks) break;
                const W* const row = down + (uint64_t)min(16 * f + n, ranks - 1) * x.k;
                load_some<kAll>(row + col, there, row + x.k - 1, a[f][c]);
            }
        }
        float4x part[RF];
#pragma unroll
        for (int f = 0; f < RF; ++f) part[f] = float4x{0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            uint32_t w[4];
            __builtin_memcpy(w, codes[c], 16);
            const Eight low = Inner<W>::codes(w[0], w[1]), high = Inner<W>::codes(w[2], w[3]);
#pragma unroll
            for (int f = 0; f < RF; ++f) {
                if (16u * f >= ranks) break;
                Eight e[2];
                __builtin_memcpy(e, a[f][c], 32);
                part[f] = Inner<W>::mul(e[0], low, part[f]);
                part[f] = Inner<W>::mul(e[1], high, part[f]);
            }
        }
#pragma unroll
        for (int f = 0; f < RF; ++f) inner[f] += scale * part[f];
    };
    uint32_t group = first + wave;
    const uint32_t whole = min(end, (uint32_t)(x.k / kFp8Group));
    for (; group < whole; group += kWaves) add_group(std::true_type{}, group);
    if (group < end) add_group(std::false_type{}, group);
#pragma unroll
    for (int f = 0; f < RF; ++f) sums[wave][f][lane] = inner[f];
    __syncthreads();
    const uint32_t f = wave;  // each of the first waves joins one fragment of 16 ranks
    static_assert(kWaves >= RF, "a wave for each fragment");
    if (f >= RF || !keep || 16 * f + 4 * g >= ranks) return;
    float4x sum = sums[0][f][lane];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) sum += sums[w][f][lane];
    float* const to = x.inner + ((uint64_t)split * x.m + tile * kTokens + n) * x.inner_ld + rank0 + 16 * f + 4 * g;
    *(float4x*)to = sum;
}

// ---------------------------------------------------------------------------
// outputs: a workgroup takes 64 columns and 16 tokens, its waves in turn the adapters among them

// Four elements of a token's inner row, the parts of the columns added, times its factor.
__device__ __forceinline__ float4x inner_row(const AdapterArgs& x, uint64_t token, uint32_t r, uint32_t adapter) {
    const float* p = x.inner + token * x.inner_ld + r;
    const uint64_t step = x.m * x.inner_ld;
    float4x t = {0, 0, 0, 0};
    uint32_t s = 0;
    for (; s + 4 <= x.splits; s += 4, p += 4 * step) {
        const float4x a = *(const float4x*)p, b = *(const float4x*)(p + step), c = *(const float4x*)(p + 2 * step),
                      d = *(const float4x*)(p + 3 * step);
        t = t + a + b + c + d;
    }
    for (; s < x.splits; ++s, p += step) t += *(const float4x*)p;
    return t * (x.factors ? x.factors[adapter] : 1.0f);
}

// Row m of fragment f of 64 columns is the column 16 (m / 4) + 4 f + m % 4: a lane gets 16 neighbours.
__device__ __forceinline__ uint64_t column_of(uint64_t col0, uint32_t m, int f) {
    return col0 + 16 * (m / 4) + 4 * f + m % 4;
}

// Four ranks from r on of a column of `up`, zeros for those past the last.  kQuads: the ranks are a multiple of four.
template <bool kQuads, typename W>
__device__ __forceinline__ void load_up(const AdapterArgs& x, const W* up, uint64_t column, uint32_t r, W (&w)[4]) {
    const W* const row = up + min(column, x.n - 1) * x.rank;
    const uint32_t rank = (uint32_t)x.rank;
    if constexpr (kQuads) {
        __builtin_memcpy(w, row + min(r, rank - 4), sizeof w);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) w[i] = row[min(r + i, rank - 1)];
    }
}

// out += the product of 64 columns' four ranks a lane (16 in all) and a token's.
template <bool kQuads, typename W>
__device__ __forceinline__ void multiply(const AdapterArgs& x, const W (&w)[4][4], float4x t, uint32_t r,
                                         float4x (&out)[4]) {
    const int ranks = (int)x.rank - (int)r;  // that are there; what stands for others is neither a weight nor a number
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool there = (kQuads ? 0 : i) < ranks;
#pragma unroll
        for (int f = 0; f < 4; ++f)
            out[f] = __builtin_amdgcn_mfma_f32_16x16x4f32(there ? (float)w[f][i] : 0.0f, there ? t[i] : 0.0f, out[f], 0, 0, 0);
    }
}

template <bool kAll, typename T>
__device__ __forceinline__ void add_and_store(T (&y)[16], const float4x (&out)[4], T* to, int there) {
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = (T)((float)y[i] + out[i / 4][i % 4]);
    if constexpr (kAll) {
        __builtin_memcpy(to, y, sizeof y);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (i < there) to[i] = y[i];
    }
}

// kInLds: the workgroup's inner rows (up to 128 ranks) are made once for all its waves.
template <typename T, typename W, bool kInLds, bool kQuads>
__global__ void __launch_bounds__(kMostWaves * 64) up_kernel(AdapterArgs x) {
    extern __shared__ float4x staged_rows[];  // [tokens][inner_ld + 4]: neighbouring tokens' in different banks
    float* const staged = (float*)staged_rows;
    const uint32_t pitch = x.inner_ld + 4;
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t waves = blockDim.x / 64, n = lane % 16, g = lane / 16;
    const uint32_t item = item_of_block(), group = divided(item, x.by_column_blocks);
    const uint64_t col0 = (uint64_t)(item - group * x.column_blocks) * 64;
    const uint64_t tile = group, token = tile * kTokens + n;
    if (tile * kTokens >= x.m) return;  // a workgroup past the last item
    const uint32_t mine = adapter_of(x, tile);
    const uint64_t col = col0 + 16 * g;  // of the lane's 16 outputs
    const int there = col < x.n ? (int)min(x.n - col, (uint64_t)16) : 0;
    const uint32_t vectors = x.inner_ld / 4;  // of an inner row
    auto stage = [&]() {
        const uint32_t rows = (uint32_t)min(x.m - tile * kTokens, (uint64_t)kTokens);
        for (uint32_t i = threadIdx.x; i < rows * vectors; i += blockDim.x) {
            const uint32_t row = divided(i, x.by_vectors), r = (i - row * vectors) * 4;
            const uint32_t a = (uint32_t)x.index[tile * kTokens + row];
            float4x t = {0, 0, 0, 0};
            if (a < x.adapters) t = inner_row(x, tile * kTokens + row, r, a);
            *(float4x*)&staged[row * pitch + r] = t;
        }
        __syncthreads();
    };
    auto make = [&](auto all) {
        constexpr bool kAll = decltype(all)::value;
        bool to_stage = kInLds;  // every wave does it once, the loads of its first product under way
        uint32_t job = 0;
        uint64_t left = __ballot(token < x.m);
        while (left != 0) {
            const uint32_t a = __builtin_amdgcn_readlane(mine, __builtin_ctzll(left));
            left &= ~__ballot(mine == a);
            const bool my_turn = job == wave;
            job = job + 1 == waves ? 0 : job + 1;
            if (!my_turn) continue;
            const bool keep = mine == a && token < x.m;
            const W* const up = (const W*)x.up + (a == kNone ? 0 : (uint64_t)a * x.n * x.rank);
            T y[16];
            W w[4][4];
            const T* const row = (const T*)x.y + min(token, x.m - 1) * x.ld_y;
            load_some<kAll>(row + col, there, row + x.n - 1, y);
            if (a != kNone) {
#pragma unroll
                for (int f = 0; f < 4; ++f) load_up<kQuads>(x, up, column_of(col0, n, f), 4 * g, w[f]);
            }
            if (to_stage) stage();
            to_stage = false;
            float4x out[4];
            const float start = a != kNone ? 0.0f : kNothingAdded;
#pragma unroll
            for (int f = 0; f < 4; ++f) out[f] = float4x{start, start, start, start};
            if (a != kNone) {
                for (uint32_t r0 = 0; r0 < x.rank; r0 += 16) {
                    const uint32_t r = r0 + 4 * g;
                    if (r0 > 0) {
#pragma unroll
                        for (int f = 0; f < 4; ++f) load_up<kQuads>(x, up, column_of(col0, n, f), r, w[f]);
                    }
                    float4x t = {0, 0, 0, 0};
                    if (keep && r < x.rank)
                        t = kInLds ? *(const float4x*)&staged[n * pitch + r] : inner_row(x, token, r, a);
                    multiply<kQuads>(x, w, t, r, out);
                }
            }
            if (keep) add_and_store<kAll>(y, out, (T*)x.out + token * x.ld_out + col, there);
        }
        if (to_stage) stage();
    };
    if (col0 + 64 <= x.n)
        make(std::true_type{});
    else
        make(std::false_type{});
}

// The same for many tokens: a wave takes one tile of 16 tokens and 128 columns, all the adapters among them in turn.
// What it reads is asked for at once, but for `up`, which waits for the index alone.
template <typename T, typename W, bool kQuads>
__global__ void __launch_bounds__(256) up_tiles_kernel(AdapterArgs x) {
    constexpr int CB = 2;  // blocks of 64 columns
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t n = lane % 16, g = lane / 16;
    const uint32_t item = item_of_block(), group = divided(item, x.by_column_blocks);
    const uint64_t tile = (uint64_t)group * 4 + wave, token = tile * kTokens + n;
    if (tile * kTokens >= x.m) return;
    const uint64_t col0 = (uint64_t)(item - group * x.column_blocks) * (64 * CB);
    auto make = [&](auto all) {
        constexpr bool kAll = decltype(all)::value;
        const uint32_t mine = adapter_of(x, tile);
        T y[CB][16];
        int there[CB];
        const T* const row = (const T*)x.y + min(token, x.m - 1) * x.ld_y;
#pragma unroll
        for (int b = 0; b < CB; ++b) {
            const uint64_t col = col0 + 64 * b + 16 * g;
            there[b] = kAll ? 16 : col < x.n ? (int)min(x.n - col, (uint64_t)16) : 0;
            load_some<kAll>(row + col, there[b], row + x.n - 1, y[b]);
        }
        float4x out[CB][4];
#pragma unroll
        for (int b = 0; b < CB; ++b)
#pragma unroll
            for (int f = 0; f < 4; ++f) out[b][f] = float4x{kNothingAdded, kNothingAdded, kNothingAdded, kNothingAdded};
        uint64_t left = __ballot(mine != kNone);
        while (left != 0) {
            const uint32_t a = __builtin_amdgcn_readlane(mine, __builtin_ctzll(left));
            left &= ~__ballot(mine == a);
            const bool keep = mine == a;
            const W* const up = (const W*)x.up + (uint64_t)a * x.n * x.rank;
            float4x sum[CB][4];
#pragma unroll
            for (int b = 0; b < CB; ++b)
#pragma unroll
                for (int f = 0; f < 4; ++f) sum[b][f] = float4x{0, 0, 0, 0};
            for (uint32_t r0 = 0; r0 < x.rank; r0 += 16) {
                const uint32_t r = r0 + 4 * g;
                W w[CB][4][4];
#pragma unroll
                for (int b = 0; b < CB; ++b)
#pragma unroll
                    for (int f = 0; f < 4; ++f) load_up<kQuads>(x, up, column_of(col0 + 64 * b, n, f), r, w[b][f]);
                float4x t = {0, 0, 0, 0};
                if (keep && r < x.rank) t = inner_row(x, token, r, a);
#pragma unroll
                for (int b = 0; b < CB; ++b) multiply<kQuads>(x, w[b], t, r, sum[b]);
            }
#pragma unroll
            for (int b = 0; b < CB; ++b)
#pragma unroll
                for (int f = 0; f < 4; ++f) out[b][f] = keep ? sum[b][f] : out[b][f];
        }
        if (token >= x.m) return;
#pragma unroll
        for (int b = 0; b < CB; ++b)
            add_and_store<kAll>(y[b], out[b], (T*)x.out + token * x.ld_out + col0 + 64 * b + 16 * g, there[b]);
    };
    if (col0 + 64 * CB <= x.n)
        make(std::true_type{});
    else
        make(std::false_type{});
}

template <typename T, typename W>
hipError_t launch(const AdapterArgs& a, const AdapterPlan& p, hipStream_t s) {
    const uint64_t tiles = (a.m + kTokens - 1) / kTokens;
    if (a.adapters > 0) {
        dim3 grid = item_grid((uint32_t)tiles, p.distinct * (uint32_t)((a.rank + kRanks - 1) / kRanks));
        grid.z *= a.splits;
        if (p.down_waves == 16)
            down_kernel<W, 16><<<grid, 16 * 64, 0, s>>>(a);
        else
            down_kernel<W, 4><<<grid, 4 * 64, 0, s>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const dim3 grid = item_grid((uint32_t)(a.column_blocks * (p.many ? (tiles + 3) / 4 : tiles)));
    const uint32_t staged = kTokens * (a.inner_ld + 4) * sizeof(float);
    auto up = [&](auto quads) {
        constexpr bool kQuads = decltype(quads)::value;
        if (p.many)
            up_tiles_kernel<T, W, kQuads><<<grid, 256, 0, s>>>(a);
        else if (a.rank <= kStaged)
            up_kernel<T, W, true, kQuads><<<grid, p.distinct * 64, staged, s>>>(a);
        else
            up_kernel<T, W, false, kQuads><<<grid, p.distinct * 64, 0, s>>>(a);
    };
    if (a.rank % 4 == 0)
        up(std::true_type{});
    else
        up(std::false_type{});
    return hipGetLastError();
}

template <typename T>
hipError_t launch(int adapter_type, const AdapterArgs& a, const AdapterPlan& p, hipStream_t s) {
    return adapter_type == kTypeBf16 ? launch<T, __bf16>(a, p, s) : launch<T, _Float16>(a, p, s);
}

}  // namespace

AdapterPlan fp8_adapter_plan(uint64_t m, uint64_t k, uint64_t rank, uint64_t adapters) {
    AdapterPlan p = {};
    const uint64_t tiles = (m + kTokens - 1) / kTokens, groups = (k + kFp8Group - 1) / kFp8Group;
    const uint64_t rank_blocks = (rank + kRanks - 1) / kRanks;
    p.distinct = (uint32_t)std::max<uint64_t>(1, std::min({(uint64_t)kTokens, m, adapters}));
    p.inner_ld = (uint32_t)((rank + 3) / 4 * 4);
    p.down_waves = tiles * rank_blocks >= 64 ? 16 : 4;  // 128 tiles of 8192 columns: 16 us, by four waves 33
    // columns in parts until there are two workgroups for each unit, a group for each wave at least
    const uint64_t wanted = 512 / std::max<uint64_t>(1, tiles * p.distinct * rank_blocks);
    const uint64_t splits = std::max<uint64_t>(1, std::min<uint64_t>({wanted, (groups + p.down_waves - 1) / p.down_waves, 16}));
    p.split_groups = (uint32_t)std::max<uint64_t>(1, (groups + splits - 1) / splits);
    p.splits = (uint32_t)std::max<uint64_t>(1, (groups + p.split_groups - 1) / p.split_groups);
    // More than 1024 tokens fill the chip by themselves (2048 x 28672 of rank 16: 67 us, and 94 by a wave for each adapter);
    // of fewer, each adapter has a wave (32 x 8192 with 16 in each 16 tokens: 6 us, by four waves in turn 27).
    p.many = m > 1024;
    p.token_rows = (uint32_t)((tiles + kRowOfItems - 1) / kRowOfItems);
    p.workspace = adapters > 0 && k > 0 ? (uint64_t)p.splits * m * p.inner_ld * sizeof(float) : 0;
    return p;
}

hipError_t launch_fp8_adapters(int type, int adapter_type, AdapterArgs a, const AdapterPlan& p, hipStream_t s) {
    a.distinct = p.distinct, a.splits = p.splits, a.split_groups = p.split_groups;
    a.inner_ld = p.inner_ld, a.token_rows = p.token_rows;
    a.column_blocks = (uint32_t)(p.many ? (a.n + 127) / 128 : (a.n + 63) / 64);
    a.by_column_blocks = divider(a.column_blocks), a.by_vectors = divider(a.inner_ld / 4);
    if (a.k == 0) a.adapters = 0;  // nothing to add
    return type == kTypeBf16  ? launch<__bf16>(adapter_type, a, p, s)
           : type == kTypeF16 ? launch<_Float16>(adapter_type, a, p, s)
                              : launch<float>(adapter_type, a, p, s);
}

}  // namespace hv
