// fp8_matmul.hip -- the product of two matrices held in 8 bits with a scale for
// each group of 128:
//   c[i][j] = sum over groups g of a_scales[i][g] * b_scales[j / 128][g] *
//             (sum over the group's columns t of a[i][t] * b[j][t]).
//
// A matrix instruction (16 x 16 outputs over 128 columns) covers exactly one
// group, so its result is a group's part of the sum; the vector unit then adds
// it, times the two scales, to the 32-bit accumulators.  B's rows are the
// instruction's rows and A's its columns: a lane then holds four consecutive
// columns of one row of C, and all of them take the same a_scale.
//
// Two kinds of kernels share the work, by the rows of A:
//   up to 16   (small products: 32) bound by reading B: stream_kernel.  1 x 8192 x 8192 13.7 us (4.9
//              TB/s), 8 x 28672 x 8192 45 to 48 us (5.0 TB/s, where a copy reaches 5.1).
//   more       bound by the matrix unit and its power: tile_kernel.  2048 x 28672 x
//              8192 404 us (2.4 PFLOP/s; a library's product of the same codes
//              without group scales 392).  A loop of this mix alone, products and four
//              additions each from registers, reaches 3.1 PFLOP/s on ordinary codes and
//              4.1 on equal ones: the chip lowers its clock to 1.7 GHz under it.
#include <cmath>
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
// drops what lies below 2^-13 of the largest of them (measured); between
// those it adds in 32 bits.  The 16-bit results take that for twice the rate: at worst 1.8e-3
// of the sum of the terms' magnitudes, measured 1.4e-5 of c on ordinary codes and 6.5e-5 where a few
// columns are 300 times the others, beside a rounding of 2.1e-4 (half) or 1.7e-3
// (bfloat16) of the result.  A 32-bit result does not lose it: its codes are
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

// 16 bytes of a row that has `left` bytes from p on, and k in all; zeros beyond them.
__device__ __forceinline__ int4x load_16(const uint8_t* p, int left, uint32_t k) {
    uint64_t v[2] = {0, 0};
    if (left >= 16) {
        __builtin_memcpy(v, p, 16);
    } else if (left > 0 && k >= 16) {  // the row's last 16 bytes, and down by what is before p
        __builtin_memcpy(v, p + left - 16, 16);
        const int down = 8 * (16 - left);
        v[0] = down < 64 ? v[0] >> down | v[1] << (64 - down) : v[1] >> (down - 64);
        v[1] = down < 64 ? v[1] >> down : 0;
    } else {
#pragma unroll 1
        for (int b = left - 1; b >= 0; --b) {
            v[1] = v[1] << 8 | v[0] >> 56;
            v[0] = v[0] << 8 | p[b];
        }
    }
    return int4x{(int)v[0], (int)(v[0] >> 32), (int)v[1], (int)(v[1] >> 32)};
}

// A lane's part of a 16-row fragment over a group: 16 bytes from p and 16 from
// p + 64 (which columns a lane holds does not matter, as long as both
// operands go by the same rule).
__device__ __forceinline__ int8x load_fragment(const uint8_t* p, int left, uint32_t k) {
    const int4x lo = load_16(p, left, k), hi = load_16(p + 64, left - 64, k);
    return int8x{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
}

__device__ __forceinline__ int8x load_whole(const uint8_t* p) {
    int8x f;
    __builtin_memcpy(&f, p, 16);
    __builtin_memcpy((char*)&f + 16, p + 64, 16);
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

// ---------------------------------------------------------------------------
// few rows: B straight from memory

// A workgroup makes MT x NT fragments of 16 x 16 outputs; its waves take the groups of
// columns in turn and join their sums through LDS.  Nothing is shared between
// waves but A, which the caches hold, so B goes to registers with kAhead groups on
// their way per wave.
constexpr int kStreamWaves = 8;

template <typename T, int MT, int NT, int kAhead>
__global__ void __launch_bounds__(kStreamWaves * 64)
    stream_kernel(const uint8_t* __restrict__ a, uint64_t ld_a, const float* __restrict__ sa,
                  const uint8_t* __restrict__ b, uint64_t ld_b, const float* __restrict__ sb, uint32_t m, uint32_t n,
                  uint32_t k, T* __restrict__ c, uint64_t ld_c, uint32_t tiles_m, uint64_t first) {
    __shared__ float4x part[kStreamWaves][MT * NT][64];
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint64_t tile = first + blockIdx.x;
    const uint32_t i0 = (uint32_t)(tile % tiles_m) * 16 * MT, j0 = (uint32_t)(tile / tiles_m) * 16 * NT;
    const uint32_t groups = (k + kFp8Group - 1) / kFp8Group, whole = k / kFp8Group;
    const uint32_t at = lane / 16 * 16;
    const uint8_t *row_a[MT], *row_b[NT];
    const float *scale_a[MT], *scale_b[NT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const uint32_t row = min(i0 + 16 * i + lane % 16, m - 1);
        row_a[i] = a + row * ld_a + at;
        scale_a[i] = sa + (uint64_t)row * groups;
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        row_b[j] = b + min(j0 + 16 * j + lane % 16, n - 1) * ld_b + at;
        scale_b[j] = sb + (uint64_t)(min(j0 + 16 * j, n - 1) / kFp8Group) * groups;
    }

    float4x sum[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) sum[i][j] = float4x{0, 0, 0, 0};
    int8x fa[kAhead][MT], fb[kAhead][NT];
    float in_a[kAhead][MT], in_b[kAhead][NT];
    auto load = [&](int slot, uint32_t g) {
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            fb[slot][j] = load_whole(row_b[j] + g * kFp8Group);
            in_b[slot][j] = scale_b[j][g];
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            fa[slot][i] = load_whole(row_a[i] + g * kFp8Group);
            in_a[slot][i] = scale_a[i][g];
        }
    };
    auto multiply = [&](int slot) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const float4x p = group_product<T>(fb[slot][j], fa[slot][i]);
                const float s = in_a[slot][i] * in_b[slot][j];
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[i][j][e] = fmaf(p[e], s, sum[i][j][e]);
            }
    };
    // The wave's groups are wave, wave + kStreamWaves, ...; count of the whole ones among them.
    const uint32_t count = whole > wave ? (whole - wave + kStreamWaves - 1) / kStreamWaves : 0;
    auto load_next = [&](int slot, uint32_t index) {
        if (index < count) load(slot, wave + index * kStreamWaves);
    };
#pragma unroll
    for (int d = 0; d < kAhead; ++d) load_next(d, d);
    uint32_t x = 0;
    for (; x + kAhead <= count; x += kAhead)
#pragma unroll
        for (int d = 0; d < kAhead; ++d) {
            multiply(d);
            load_next(d, x + d + kAhead);
        }
#pragma unroll
    for (int d = 0; d < kAhead - 1; ++d)
        if (x + d < count) multiply(d);
    if (whole < groups && whole % kStreamWaves == wave) {  // a last group, with zeros beyond the columns
        const int left = (int)(k - whole * kFp8Group) - (int)at;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            fb[0][j] = load_fragment(row_b[j] + whole * kFp8Group, left, k);
            in_b[0][j] = scale_b[j][whole];
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            fa[0][i] = load_fragment(row_a[i] + whole * kFp8Group, left, k);
            in_a[0][i] = scale_a[i][whole];
        }
        multiply(0);
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) part[wave][i * NT + j][lane] = sum[i][j];
    __syncthreads();
    for (uint32_t f = wave; f < MT * NT; f += kStreamWaves) {
        float4x total = part[0][f][lane];
        for (int w = 1; w < kStreamWaves; ++w) total += part[w][f][lane];
        const uint32_t row = i0 + f / NT * 16 + lane % 16, col = j0 + f % NT * 16 + lane / 16 * 4;
        if (row < m && col < n) store_four(c + row * ld_c + col, (int)(n - col), total);
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

// What a launch of tiles has besides the operands.
struct Tiles {
    uint32_t rows, count;     // of tiles, down and in all
    uint32_t splits, groups;  // the columns in `splits` parts of `groups` groups
    float* sums;              // where there are several parts: [part][m][n]
};

// Groups whose scales a lane loads at once, where the LDS holds `stages` groups.
constexpr int scale_run(int stages) { return stages == 3 ? 3 : 4; }

// A workgroup makes TM x TN outputs over one of the splits' columns, with WM x
// WN waves.  While one group's rows of A and B (128 bytes each) are multiplied, the
// next groups' go from memory to LDS, which holds S groups: directly, or where
// rows are not 16-byte aligned (kDirect = false) through registers.
//
// Sizes and stages as they fit 160 KB of LDS and 256 registers a lane: 256 x 256 with
// 2 (the least LDS traffic and loads for a product: 63% of the cycles have the matrix
// unit busy, 1.86 GHz), 256 x 128 and 192 x 128 with 3, 128 x 128 with 4.  LDS reads
// meet no bank conflicts; what is left is waiting at the meetings (30%) and for issue (34%).
template <typename T, int TM, int TN, int WM, int WN, int S, bool kDirect>
__global__ void __launch_bounds__(WM* WN * 64) tile_kernel(MatmulArgs x, Tiles tiles) {
    constexpr int kThreads = WM * WN * 64;
    constexpr int MT = TM / WM / 16, NT = TN / WN / 16;
    constexpr int kLoadsA = TM * 8 / kThreads, kLoadsB = TN * 8 / kThreads;  // 16-byte loads of a lane
    constexpr int kLoads = kLoadsA + kLoadsB;
    static_assert(TN / WN <= kFp8Group && kFp8Group % (TN / WN) == 0, "a wave's columns share a scale");
    constexpr int kScales = TM + 64;  // A's, then B's
    static_assert(kScales / 64 <= WM * WN, "a wave loads 64 scales");
    static_assert(MT >= 4 && (S > 2 || (kLoadsA <= NT && kLoadsB <= NT)) && kLoads <= (MT - 1) * NT,
                  "a group's loads fit between its products");
    constexpr int kRun = scale_run(S), kUnroll = S == 2 ? 4 : S;  // groups of a run; a multiple of S and of that
    static_assert(S >= 2 && S <= 4 && (kDirect || S == 4), "the LDS arrays and the registers' ring");
    // separate arrays: the compiler then sees that a fragment's read does not touch a stage that loads go to
    __shared__ alignas(1024) uint8_t a0[TM * 128], b0[TN * 128], a1[TM * 128], b1[TN * 128];
    __shared__ alignas(1024) uint8_t a2[S > 2 ? TM * 128 : 16], b2[S > 2 ? TN * 128 : 16];
    __shared__ alignas(1024) uint8_t a3[S > 3 ? TM * 128 : 16], b3[S > 3 ? TN * 128 : 16];
    __shared__ alignas(256) float4x scales[2][kScales];  // of kRun groups, and of the next ones
    auto stage_a = [&](auto st) {
        constexpr int i = decltype(st)::value % S;
        return i == 0 ? a0 : i == 1 ? a1 : i == 2 ? a2 : a3;
    };
    auto stage_b = [&](auto st) {
        constexpr int i = decltype(st)::value % S;
        return i == 0 ? b0 : i == 1 ? b1 : i == 2 ? b2 : b3;
    };

    // Workgroups go to the eight XCDs in turn; each XCD gets a run of tiles, in
    // panels of 8 tiles' rows, so that the 32 it has at a time are 8 x 4 and its L2
    // serves each row of A and B several times.
    const uint32_t per_xcd = gridDim.x / 8;
    const uint32_t index = blockIdx.x % 8 * per_xcd + blockIdx.x / 8;
    if (index >= tiles.count * tiles.splits) return;
    const uint32_t split = index / tiles.count, tile = index % tiles.count;
    const uint32_t panel_tiles = 8 * (tiles.count / tiles.rows);
    const uint32_t panel = tile / panel_tiles, in_panel = tile % panel_tiles;
    const uint32_t panel_rows = min(8u, tiles.rows - panel * 8);
    const uint32_t i0 = (panel * 8 + in_panel % panel_rows) * TM, j0 = in_panel / panel_rows * TN;

    const uint32_t m = (uint32_t)x.m, n = (uint32_t)x.n, k = (uint32_t)x.k;
    const uint32_t lane = threadIdx.x % 64;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t wave_i = wave / WN * (TM / WM), wave_j = wave % WN * (TN / WN);
    const uint32_t groups = (k + kFp8Group - 1) / kFp8Group;  // of a row
    // The split's groups are counted from `base`: `count` of them, `whole` of them filled by the columns.
    const uint32_t base = split * tiles.groups, count = min(tiles.groups, groups - base);
    const uint32_t whole = min(base + count, k / kFp8Group) - base, last_group = whole - 1;

    // The row of LDS that a lane of load instruction l fills is 8 * (l * waves + wave) + lane / 8; its
    // 16-byte places hold the row's chunks in the order place ^ (row % 8), so that
    // the lanes of a fragment read from different banks.
    const uint32_t chunk = (lane % 8 ^ lane / 8) * 16;
    const uint8_t* const tile_a = x.a + i0 * x.ld_a + base * kFp8Group;
    const uint8_t* const tile_b = x.b + j0 * x.ld_b + base * kFp8Group;
    uint32_t from_a[kLoadsA], from_b[kLoadsB];
#pragma unroll
    for (int l = 0; l < kLoadsA; ++l)
        from_a[l] = min(8 * (l * WM * WN + wave) + lane / 8, m - 1 - i0) * (uint32_t)x.ld_a + chunk;
#pragma unroll
    for (int l = 0; l < kLoadsB; ++l)
        from_b[l] = min(8 * (l * WM * WN + wave) + lane / 8, n - 1 - j0) * (uint32_t)x.ld_b + chunk;
    const uint32_t part_s = wave % (kScales / 64);  // waves beyond them load a part again
    const bool scales_of_a = part_s < TM / 64;
    const float* const tile_s =
        base + (scales_of_a ? x.a_scales + (uint64_t)i0 * groups : x.b_scales + (uint64_t)(j0 / kFp8Group) * groups);
    const uint32_t from_s = (scales_of_a ? min(part_s * 64 + lane, m - 1 - i0)
                                         : min(lane, (n - 1) / kFp8Group - j0 / kFp8Group)) * groups;

    // Buffer loads: a lane's offset stays, the group's is a scalar.
    const auto all_a = rows_at(tile_a), all_b = rows_at(tile_b);
    auto at = [&](int l) { return 1024 * (l * WM * WN + wave); };
    // the group's load l, of A's rows and then of B's
    int4x held[kDirect ? 1 : S][kLoads];  // on their way through registers
    auto load = [&](int l, uint32_t g, auto st) {
        constexpr int i = decltype(st)::value % S;
        if constexpr (kDirect) {
            if (l < kLoadsA)
                buffer_to_lds(all_a, stage_a(st) + at(l), from_a[l], g * kFp8Group);
            else
                buffer_to_lds(all_b, stage_b(st) + at(l - kLoadsA), from_b[l - kLoadsA], g * kFp8Group);
        } else {
            const uint8_t* const p = l < kLoadsA ? tile_a + from_a[l] : tile_b + from_b[l - kLoadsA];
            __builtin_memcpy(&held[i][l], p + g * kFp8Group, 16);
        }
    };
    auto keep = [&](int l, int4x v, auto st) {
        *(int4x*)((l < kLoadsA ? stage_a(st) + at(l) : stage_b(st) + at(l - kLoadsA)) + 16 * lane) = v;
    };
    // Scales come kRun groups at a time (a load of one group's takes as many
    // requests as a load of a tile's 128-byte rows), a row's last kRun where there
    // are fewer left, and are kept in LDS as [row][4].  A run is asked for kRun
    // groups before it goes there, at steps that the unrolled loop fixes: where a branch
    // decided, the compiler would wait there for all loads.
    const uint32_t last_run = max(count, (uint32_t)kRun) - kRun;
    const bool runs = count > kRun;
    float4x held_scales;
    auto load_run = [&](uint32_t r) { __builtin_memcpy(&held_scales, tile_s + from_s + min(kRun * r, last_run), 4 * kRun); };
    auto keep_run = [&](uint32_t r) { scales[r % 2][64 * part_s + lane] = held_scales; };
    // where group g's scales stand, from a row's first one on
    auto scales_at = [&](uint32_t g) {
        return (const float*)scales + (g / kRun % 2 * kScales * 4 + g - min(g / kRun * kRun, last_run));
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
    // loads issued after the next group's: with two stages, B's of the group after the next (see below)
    constexpr int kAfter = !kDirect ? 63 : S == 2 ? kLoadsB : (S - 2) * kLoads;
    constexpr std::integral_constant<int, kAfter> kLater;
    constexpr std::integral_constant<int, kAfter> kLaterAndRun;
    constexpr std::integral_constant<int, 0> kNone;
    constexpr std::integral_constant<int, 63> kAll;

    // One group, in LDS stage st.  The fragments of A's next 16 rows come from LDS
    // while these are multiplied, and the next group's first ones while this group's last
    // are.  By then every wave has read all it needs of this stage, so the group S
    // further on may be loaded there (past the last group the last one again: nobody
    // reads it), a load after each product so that no wave stands in line for them.
    // With two stages B's rows are asked for sooner: every wave holds all it needs
    // of them from the start, and their place is free as soon as the waves have met.
    // A product is added to its sum two instructions later, when the matrix unit has it.
    int8x fb[NT], fa;
    float scale_a, scale_b;
    const uint32_t b_scale = 4 * (TM + wave_j / kFp8Group);
    auto multiply = [&](uint32_t g, auto step) {
        constexpr int U = decltype(step)::value, ST = U % S;  // g is U modulo kUnroll
        constexpr std::integral_constant<int, ST> st;
        constexpr std::integral_constant<int, ST + 1> kNext;
        constexpr std::integral_constant<int, ST + S - 1> kLast;  // the stage before, which loads still go to
        constexpr std::integral_constant<int, ST + 2> kKept;      // through registers: the group written to LDS
        constexpr bool kAsk = U % kRun == kRun - 1, kKeep = U % kRun == kRun - 2;
        const float* const now = scales_at(g);
        const float* const next = scales_at(g + 1);
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
            if (kDirect && S == 2 && i == 1) meet(kAll);
            if (last) {
                if constexpr (kAsk) {
                    if (runs) load_run(g / kRun + 2);
                    meet(kLaterAndRun);
                } else {
                    meet(kLater);
                }
                if constexpr (kKeep)
                    if (runs) keep_run(g / kRun + 1);
                scale_b = next[b_scale];
            }
            const int8x next_fa = last ? fragment_a(stage_a(kNext), 0) : fragment_a(stage_a(st), i + 1);
            const float next_scale = last ? next[a_scale] : now[a_scale + 64 * (i + 1)];
            s[i % 2] = scale_a * in_b;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const int t = i * NT + j;
                p[t % 3] = group_product<T>(fb[j], fa);
                __builtin_amdgcn_sched_barrier(0);
                if (last) fb[j] = fragment_b(stage_b(kNext), j);
                if constexpr (!kDirect) {
                    // four groups on their way; the one after the next goes to LDS, and its place in the ring to
                    // the group four further on
                    if (i == MT - 2)
#pragma unroll
                        for (int l = j; l < kLoads; l += NT) keep(l, held[kKept.value % S][l], kKept);
                    if (last)
#pragma unroll
                        for (int l = j; l < kLoads; l += NT) load(l, min(g + 2 + S, last_group), kKept);
                } else if constexpr (S == 2) {
                    if (last && j < kLoadsA) load(j, min(g + 2, last_group), st);
                    if (i == 1 && j < kLoadsB) load(kLoadsA + j, min(g + 2, last_group), st);
                } else {
                    if (last && j < kLoads) load(j, min(g + S, last_group), st);
                    if (!last && t + NT < kLoads) load(t + NT, min(g + S - 1, last_group), kLast);
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
    constexpr std::integral_constant<int, 0> kStage0;
    constexpr std::integral_constant<int, 1> kStage1;
    constexpr std::integral_constant<int, 2> kStage2;
    constexpr std::integral_constant<int, 3> kStage3;

    if (whole > 0) {
        auto load_all = [&](uint32_t ahead, auto st, int first, int end) {
#pragma unroll
            for (int l = first; l < end; ++l) load(l, min(ahead, last_group), st);
        };
        // the first scales before all else: LDS waits for them, and loads end in their order
#pragma unroll
        for (uint32_t e = 0; e < kRun; ++e) held_scales[e] = tile_s[from_s + min(e, count - 1)];
        asm volatile("" ::: "memory");
        if constexpr (!kDirect) {
            load_all(0, kStage0, 0, kLoads);
            load_all(1, kStage1, 0, kLoads);
            load_all(2, kStage2, 0, kLoads);
            load_all(3, kStage3, 0, kLoads);
#pragma unroll
            for (int l = 0; l < kLoads; ++l) {
                keep(l, held[0][l], kStage0);
                keep(l, held[1][l], kStage1);
            }
            load_all(4, kStage0, 0, kLoads);
            load_all(5, kStage1, 0, kLoads);
        } else if constexpr (S == 2) {
            load_all(0, kStage0, 0, kLoads);
            load_all(1, kStage1, kLoadsA, kLoads);
        } else {
            load_all(0, kStage0, 0, kLoads);
            load_all(1, kStage1, 0, kLoads);
            if constexpr (S > 3) load_all(2, kStage2, 0, kLoads);
        }
        keep_run(0);
        if (runs) load_run(1);
        meet(kLater);
        if constexpr (kDirect && S == 2) load_all(1, kStage1, 0, kLoadsA);
        if constexpr (kDirect && S == 3) load_all(2, kStage2, 0, NT < kLoads ? NT : kLoads);
        if constexpr (kDirect && S == 4) load_all(3, kStage3, 0, NT < kLoads ? NT : kLoads);
#pragma unroll
        for (int j = 0; j < NT; ++j) fb[j] = fragment_b(b0, j);
        fa = fragment_a(a0, 0);
        scale_a = scales_at(0)[a_scale];
        scale_b = scales_at(0)[b_scale];
        uint32_t g = 0;
        for (; g + kUnroll <= whole; g += kUnroll) {
            multiply(g, kStage0);
            multiply(g + 1, kStage1);
            multiply(g + 2, kStage2);
            if constexpr (kUnroll > 3) multiply(g + 3, kStage3);
        }
        if (g < whole) multiply(g, kStage0);
        if (g + 1 < whole) multiply(g + 1, kStage1);
        if constexpr (kUnroll > 3)
            if (g + 2 < whole) multiply(g + 2, kStage2);
    }
    if (whole < count) {  // a last group, with zeros beyond the columns
        meet(kNone);
        const int left = (int)(k - (base + whole) * kFp8Group) - (int)chunk;
#pragma unroll
        for (int l = 0; l < kLoads; ++l) {
            const uint8_t* const p = l < kLoadsA ? tile_a + from_a[l] : tile_b + from_b[l - kLoadsA];
            keep(l, load_16(p + whole * kFp8Group, left, k), kStage0);
        }
        scales[0][64 * part_s + lane][0] = tile_s[from_s + whole];
        __syncthreads();
#pragma unroll
        for (int j = 0; j < NT; ++j) fb[j] = fragment_b(b0, j);
        const float in_b = ((const float*)scales)[b_scale];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int8x rows = fragment_a(a0, i);
            const float s = ((const float*)scales)[a_scale + 64 * i] * in_b;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const float4x p = group_product<T>(fb[j], rows);
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[i][j][e] = fmaf(p[e], s, sum[i][j][e]);
            }
        }
    }

    // A lane has four columns of a row; to store whole lines a wave turns 16 rows at a
    // time in LDS, so that neighbouring lanes have 16 bytes each of one row (stores
    // of the lanes' own columns, 32 bytes of a row, took 7 us of a 256 x 256
    // tile's 50).
    meet(kNone);  // nobody reads stages any more
    auto store = [&](auto* out, uint64_t ld) {  // out: the matrix
        using O = std::remove_pointer_t<decltype(out)>;
        constexpr int kSize = sizeof(O), kRow = TN / WN * kSize, kPlaces = kRow / 16, kElements = 16 / kSize;
        static_assert(WM * WN * 16 * kRow <= TM * 128, "the waves' 16 rows fit a stage");
        uint8_t* const area = a0 + wave * 16 * kRow;
        auto place = [&](uint32_t row, uint32_t chunk) { return area + row * kRow + (chunk ^ row % kPlaces) * 16; };
#pragma unroll
        for (int i = 0; i < MT; ++i) {
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                O four[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) four[e] = (O)sum[i][j][e];
                const uint32_t byte = (16 * j + 4 * quarter) * kSize;
                __builtin_memcpy(place(row16, byte / 16) + byte % 16, four, sizeof four);
            }
            asm volatile("" ::: "memory");  // a wave's LDS accesses stay in order
#pragma unroll
            for (int r = 0; r < 16; r += 64 / kPlaces) {
                const uint32_t in_16 = r + lane / kPlaces, chunk_of = lane % kPlaces;
                const int4x v = *(const int4x*)place(in_16, chunk_of);
                const uint32_t row = i0 + wave_i + 16 * i + in_16, col = j0 + wave_j + chunk_of * kElements;
                if (row >= m || col >= n) continue;
                O* const to = out + row * ld + col;
                if (col + kElements <= n) {
                    __builtin_memcpy(to, &v, 16);
                } else {
                    O elements[kElements];
                    __builtin_memcpy(elements, &v, 16);
#pragma unroll
                    for (int e = 0; e < kElements; ++e)
                        if (col + e < n) to[e] = elements[e];
                }
            }
            asm volatile("" ::: "memory");
        }
    };
    if (tiles.splits > 1)
        store(tiles.sums + (uint64_t)split * m * n, (uint64_t)n);
    else
        store((T*)x.c, x.ld_c);
}

// A's or B's rows, 16 bytes a lane, to aligned ones of ld_to >= k bytes (a multiple of
// 16; zeros beyond the columns).
__global__ void __launch_bounds__(256) pack_kernel(const uint8_t* __restrict__ from, uint64_t ld, uint32_t rows,
                                                   uint32_t k, uint8_t* __restrict__ to, uint64_t ld_to) {
    const uint32_t chunks = (uint32_t)(ld_to / 16);
    const uint64_t count = (uint64_t)rows * chunks;
    for (uint64_t c = (uint64_t)blockIdx.x * 256 + threadIdx.x; c < count; c += (uint64_t)gridDim.x * 256) {
        const uint64_t row = c / chunks;
        const uint32_t at = (uint32_t)(c % chunks) * 16;
        *(int4x*)(to + row * ld_to + at) = load_16(from + row * ld + at, (int)(k - at), k);
    }
}

// Adds the splits' sums, in their order (no splits: zeros); eight at a time are on
// their way (one at a time, 77 x 5001 of six splits took 5.2 us, 4.1 so).
template <typename T>
__global__ void __launch_bounds__(256) join_kernel(const float* __restrict__ sums, uint32_t splits, uint32_t m,
                                                   uint32_t n, T* __restrict__ c, uint64_t ld_c) {
    const uint32_t fours = (n + 3) / 4;
    const uint64_t size = (uint64_t)m * n, count = (uint64_t)m * fours;
    for (uint64_t f = (uint64_t)blockIdx.x * 256 + threadIdx.x; f < count; f += (uint64_t)gridDim.x * 256) {
        const uint64_t row = f / fours;
        const uint32_t col = (uint32_t)(f % fours) * 4, valid = min(n - col, 4u);
        const float* p = sums + row * n + col;
        float4x total = {0, 0, 0, 0};
        for (uint32_t s = 0; s < splits; s += 8) {
            float4x v[8];
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) {
                const float* const from = p + min(s + i, splits - 1) * size;
                if (valid == 4)
                    __builtin_memcpy(&v[i], from, 16);
                else
#pragma unroll
                    for (uint32_t e = 0; e < 4; ++e) v[i][e] = from[min(e, valid - 1)];
            }
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i)
                if (s + i < splits) total += v[i];
        }
        store_four(c + row * ld_c + col, (int)valid, total);
    }
}

}  // namespace

namespace {

template <typename T>
hipError_t launch_join(const float* sums, uint32_t splits, const MatmulArgs& x, hipStream_t s) {
    const uint64_t blocks = (x.m * ((x.n + 3) / 4) + 255) / 256;
    join_kernel<T><<<(uint32_t)(blocks < 2048 ? blocks : 2048), 256, 0, s>>>(sums, splits, (uint32_t)x.m,
                                                                            (uint32_t)x.n, (T*)x.c, x.ld_c);
    return hipGetLastError();
}

template <typename T, int TM, int TN, int WM, int WN, int S, bool kDirect>
hipError_t launch_tiles(const MatmulArgs& x, uint32_t splits, hipStream_t s) {
    const uint32_t groups = (uint32_t)((x.k + kFp8Group - 1) / kFp8Group);
    Tiles tiles;
    tiles.rows = (uint32_t)((x.m + TM - 1) / TM);
    tiles.count = tiles.rows * (uint32_t)((x.n + TN - 1) / TN);
    tiles.groups = (groups + splits - 1) / splits;
    tiles.splits = (groups + tiles.groups - 1) / tiles.groups;
    tiles.sums = (float*)x.workspace;
    const uint32_t grid = (tiles.count * tiles.splits + 7) / 8 * 8;
    tile_kernel<T, TM, TN, WM, WN, S, kDirect><<<grid, WM * WN * 64, 0, s>>>(x, tiles);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess || tiles.splits == 1 ? e : launch_join<T>(tiles.sums, tiles.splits, x, s);
}

template <typename T, int MT, int NT, int kAhead>
hipError_t launch_stream(const MatmulArgs& x, hipStream_t s) {
    const uint32_t tiles_m = (uint32_t)((x.m + 16 * MT - 1) / (16 * MT));
    const uint64_t tiles = tiles_m * ((x.n + 16 * NT - 1) / (16 * NT));
    constexpr uint64_t kMost = 1u << 22;  // workgroups of a launch: 2^31 lanes
    for (uint64_t first = 0; first < tiles; first += kMost) {
        const uint64_t count = tiles - first < kMost ? tiles - first : kMost;
        stream_kernel<T, MT, NT, kAhead><<<(uint32_t)count, kStreamWaves * 64, 0, s>>>(
            x.a, x.ld_a, x.a_scales, x.b, x.ld_b, x.b_scales, (uint32_t)x.m, (uint32_t)x.n, (uint32_t)x.k, (T*)x.c,
            x.ld_c, tiles_m, first);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// ---------------------------------------------------------------------------
// which kernels a product takes

enum Shape { k256x256, k256x128, k192x128, k128x128, kUnaligned, kShapes };
static_assert(kMatmul256x256 - k256x256 == kMatmulUnaligned - kUnaligned, "tile kinds in the shapes' order");

// What a tile takes, in us: `fixed`, and a group's `full` where every compute unit
// has a tile and `lone` where few have.  Measured at 8 and 64 groups with 256 tiles, half of that and one; one
// tile of 256 x 256 over 64 groups takes 128 us on a full chip, two of 256 x 128 take 140,
// four of 128 x 128 164.
struct Cost {
    uint32_t rows, cols;
    float fixed, full, lone;
};
constexpr Cost kCost[2][kShapes] = {
    {{256, 256, 8.8f, 1.86f, 1.17f},
     {256, 128, 7.2f, 0.98f, 0.63f},
     {192, 128, 6.3f, 0.77f, 0.53f},
     {128, 128, 5.4f, 0.56f, 0.38f},
     {128, 128, 10.0f, 0.95f, 0.78f}},
    {{256, 256, 0, 0, 0},  // 32-bit results: the widened codes leave no registers for it
     {256, 128, 8.5f, 2.03f, 1.35f},
     {192, 128, 7.8f, 1.60f, 1.13f},
     {128, 128, 8.0f, 1.10f, 0.88f},
     {128, 128, 12.7f, 1.35f, 1.10f}}};
constexpr uint64_t kUnits = 256;  // compute units: one tile each at a time
constexpr uint32_t kMaxSplits = 64;
// Adding up the splits' sums: a launch, and 4 bytes of each sum that the tiles write
// besides and that are read again (the join alone, three splits of 128 x 8192, 4.4 us; a constant
// from it alone, 2.5 and 5.5e6, takes too many splits: 333 x 2048 x 2048 14.0 us, 10.6 so).
float join_cost(uint64_t m, uint64_t n, uint32_t splits) {
    return splits == 1 ? 0.0f : 3.0f + (float)m * (float)n * 4.0f * (float)splits / 3.1e6f;
}

uint64_t tiles_of(const Cost& c, uint64_t m, uint64_t n) {
    return (m + c.rows - 1) / c.rows * ((n + c.cols - 1) / c.cols);
}

// Whole rounds of a tile on every unit, and a last one that fewer units share.
float rounds_cost(const Cost& c, uint64_t tiles, uint64_t groups) {
    const float full = c.fixed + c.full * (float)groups, rest = (float)(tiles % kUnits) / (float)kUnits;
    return (float)(tiles / kUnits) * full +
           (rest > 0 ? c.fixed + (c.lone + (c.full - c.lone) * rest) * (float)groups : 0.0f);
}

// The cheapest single shape, with the columns of A and B in parts where that
// pays: few tiles or a last round of few, many groups.
struct Choice {
    Shape shape;
    uint32_t splits;
    float cost;
};
Choice choose(bool wide, bool aligned, uint64_t m, uint64_t n, uint64_t groups) {
    Choice best = {kShapes, 1, 0};
    for (int s = aligned ? (wide ? k256x128 : k256x256) : kUnaligned; s < (aligned ? kUnaligned : kShapes); ++s) {
        const Cost& c = kCost[wide][s];
        const uint64_t tiles = tiles_of(c, m, n);
        const uint32_t most = c.rows != 128 || tiles >= 4 * kUnits ? 1 : kMaxSplits;
        for (uint32_t p = 1; p <= most && (p == 1 || groups / p >= 4); ++p) {
            const uint64_t each = (groups + p - 1) / p;
            const uint32_t parts = (uint32_t)((groups + each - 1) / each);
            const float cost = rounds_cost(c, tiles * parts, each) + join_cost(m, n, parts);
            if (best.shape == kShapes || cost < best.cost) best = {(Shape)s, parts, cost};
        }
    }
    return best;
}

// A product by tiles: `main` over its first rows and columns, and where the largest tiles
// would leave a last round mostly empty, the rest by smaller ones (2048 x 28672
// over 64 groups: 768 of 896 tiles of 256 x 256, then 256 of 256 x 128).
struct Plan {
    Choice main, rest;
    uint64_t rows, cols;  // main's
};
Plan plan_of(bool wide, bool aligned, uint64_t m, uint64_t n, uint64_t groups) {
    Plan plan = {choose(wide, aligned, m, n, groups), {}, m, n};
    if (wide || !aligned) return plan;
    const Cost& c = kCost[0][k256x256];
    const uint64_t down = (m + 255) / 256, across = (n + 255) / 256, rounds = down * across / kUnits;
    if (rounds == 0 || down * across % kUnits == 0) return plan;
    const uint64_t less = across >= down ? rounds * kUnits / down : rounds * kUnits / across;
    if (less == 0) return plan;
    const uint64_t rows = across >= down ? m : less * 256, cols = across >= down ? less * 256 : n;
    const Choice rest = choose(false, true, across >= down ? m : m - rows, across >= down ? n - cols : n, groups);
    const float main_cost = rounds_cost(c, tiles_of(c, rows, cols), groups);
    if (main_cost + rest.cost + 2.0f < plan.main.cost) plan = {{k256x256, 1, main_cost}, rest, rows, cols};
    return plan;
}

// Up to 16 rows of A (or 32, as two fragments) straight from memory.  A workgroup's
// fragments of B share those of A, whose rows take as many loads as theirs, and a unit
// with one workgroup more than others is the last to end: the fewest loads of a unit
// that has the most (8 x 20480 x 4096: 23.2 us by single fragments, 18.4 by 5; 8 x 11008 x
// 4096 14.6, 11.7 by 3; 16 x 8192 x 28672 71, 57 by 2, 78 by 4).  Of up to five fragments a
// unit holds two workgroups at once; more leave room for one, so seven only where each unit
// has but one (16 x 28672 x 8192: 45.9 us by 7, 49.3 by 4; 8 x 28672 x 8192 45.2 and 46.7; but 8
// x 57344 x 4096 49.1 and 46.0 by 5), and six and eight never: three and four then do as
// much in two rounds (16 x 24576 x 4096 24.3 us by 6, 22.9 by 3; 16 x 32768 x 8192 56.4 by 8,
// 51.5 by 4).  Rows at odd addresses wait for their requests, however many workgroups there
// are (11 x 57344 x 1023: 34.9 us by 7, 45.3 by 5), and of equal loads the higher count ends
// sooner (16 x 36864 x 2047: 61.9 us by 3, 46.8 by 5).  Up to four rows of A take next to
// nothing (2 x 28672 x 8192: 44.6 us by single fragments, 55.9, 49.0 and 49.4 by 2, 4 and 7).
// Two fragments of A only where one workgroup on each unit is enough (17 x 28672 x 8192 58
// us, 49 by tiles).
//
// The cost, in us: a launch, and a row of 128 bytes at a time or all of B from memory (two
// fragments of A, by four of B 17 x 16384 x 8192 31.1 us, by two 17 x 8192 x 8192 20.5).
// Rows that are not 16-byte aligned take three times as long (16 x 1000 x 8191 32 us, 17.5 by
// tiles; 16 x 1025 x 1023 5.9 and 14.1).
struct Stream {
    int kind;
    float cost;
};
Stream stream_of(bool aligned, uint64_t m, uint64_t n, uint64_t k, uint64_t groups) {
    struct Kind {
        int kind;
        uint32_t each;  // fragments of B
        bool alone;     // only where a unit has one workgroup (single fragments of A: of aligned rows)
    };
    constexpr Kind kFew[] = {{kMatmulStream1, 1, false}, {kMatmulStream2, 2, false}, {kMatmulStream3, 3, false},
                             {kMatmulStream4, 4, false}, {kMatmulStream5, 5, false}, {kMatmulStream7, 7, true}};
    constexpr Kind kTwo[] = {{kMatmulStreamTwo1, 1, true}, {kMatmulStreamTwo2, 2, true}, {kMatmulStreamTwo4, 4, true}};
    const bool two = m > 16 && m <= 32;
    const uint64_t fragments = (n + 15) / 16;
    Stream best = {kMatmulStream1, INFINITY};
    uint64_t least = 0;
    for (int i = 0; i < (m <= 4 ? 1 : two ? 3 : 6); ++i) {
        const Kind& c = two ? kTwo[i] : kFew[i];
        const uint64_t workgroups = (fragments + c.each - 1) / c.each, rounds = (workgroups + kUnits - 1) / kUnits;
        const uint64_t loads = rounds * (16 * c.each + m);
        if ((c.alone && rounds > 1 && (two || aligned)) || (least > 0 && loads + aligned > least)) continue;
        least = loads;
        best = {c.kind,
                3.0f + fmaxf((float)(loads * groups) * (aligned ? 0.0043f : 0.014f),
                             (float)n * (float)k / (two && c.each == 4 ? 4.7e6f : 3.9e6f))};
    }
    return best;
}

// What tiles take for 17 to 32 rows of A, in us, where `cost` is what full ones take: less
// for the rows that are not there, which at odd addresses are a request each, but all of B from
// memory, by workgroups that mostly wait.  By tiles and by two fragments of A: 17 x 16384 x 4096
// 23.5 and 17.5 us, x 2047 19.3 and 22.0, 24 x 4096 x 4095 in 32 bits 19.7 and 22.6, 32 x 8192 x 1023
// 17.3 and 10.7.  Over 465 sizes from 17 x 500 x 259 to 32 x 8192 x 28672 the choice by these costs
// is within 6% of the faster one, but for 8192 x 8192 of B, which tiles take 18.5 us for or 23.6,
// from one run to another, and fragments 20.5; without this correction 20 of them lost 5% to 34%.
float two_rows_cost(float cost, bool wide, bool aligned, uint64_t m, uint64_t n, uint64_t k) {
    const float absent = !aligned ? 1.0f + 0.15f * (float)(32 - m) : wide ? 4.0f : 1.0f;
    return fmaxf(cost - absent, 6.0f + (float)n * (float)k / 5.0e6f);
}

// Copying rows to aligned ones, in us: two launches (a small product waits for the
// host to make them), and each byte there and back.
float pack_cost(uint64_t m, uint64_t n, uint64_t k) { return 12.0f + (float)(m + n) * (float)k * 2.0f / 4.5e6f; }

}  // namespace

// Tiles serve more rows: a workgroup then reads B's rows for 128 of A's at once (64 x
// 4096 x 4096 14.6 us, 15.2 by four fragments of 16 rows; 64 x 8192 x 8192 18.5 and 31).
int fp8_matmul_parts(bool wide, bool aligned, bool tiles, uint64_t m, uint64_t n, uint64_t k,
                     MatmulPart parts[kMatmulMostParts]) {
    const uint64_t groups = (k + kFp8Group - 1) / kFp8Group;
    if (groups == 0) {
        parts[0] = {kMatmulZeros, 1, m, n};
        return 1;
    }
    const Stream stream = stream_of(aligned, m, n, k, groups);
    if (!tiles || (aligned && m <= 16)) {
        parts[0] = {stream.kind, 1, m, n};
        return 1;
    }
    int count = 0;
    Plan plan = plan_of(wide, true, m, n, groups);
    float cost = plan.main.cost + (plan.rows < m || plan.cols < n ? plan.rest.cost : 0.0f);
    if (!aligned) {
        // Rows at any address go through registers to LDS in tiles of 128 x 128 alone;
        // where there is much to multiply a copy of them is paid for by the larger tiles
        // (866 x 16640 x 9809: 384 us, 250 with the copy).
        const Plan direct = plan_of(wide, false, m, n, groups);
        if (cost + pack_cost(m, n, k) < direct.main.cost) {
            cost += pack_cost(m, n, k);
            parts[count++] = {kMatmulPack, 1, m, n};
        } else {
            cost = direct.main.cost;
            plan = direct;
        }
    }
    if (m > 16 && m <= 32) cost = two_rows_cost(cost, wide, aligned, m, n, k);
    if (m <= 32 && stream.cost < cost) {
        parts[0] = {stream.kind, 1, m, n};
        return 1;
    }
    parts[count++] = {kMatmul256x256 + plan.main.shape, plan.main.splits, plan.rows, plan.cols};
    if (plan.rows < m || plan.cols < n)
        parts[count++] = {kMatmul256x256 + plan.rest.shape, plan.rest.splits, plan.rows < m ? m - plan.rows : m,
                          plan.cols < n ? n - plan.cols : n};
    return count;
}

namespace {

template <typename T>
hipError_t launch_part(const MatmulPart& p, const MatmulArgs& x, hipStream_t s) {
    switch (p.kind) {
        case kMatmulZeros: return launch_join<T>(nullptr, 0, x, s);
        case kMatmulStream1: return launch_stream<T, 1, 1, 2>(x, s);
        case kMatmulStream2: return launch_stream<T, 1, 2, 2>(x, s);
        case kMatmulStream3: return launch_stream<T, 1, 3, 1>(x, s);
        case kMatmulStream4: return launch_stream<T, 1, 4, 1>(x, s);
        case kMatmulStream5: return launch_stream<T, 1, 5, 1>(x, s);
        case kMatmulStream7: return launch_stream<T, 1, 7, 1>(x, s);
        case kMatmulStreamTwo1: return launch_stream<T, 2, 1, 1>(x, s);
        case kMatmulStreamTwo2: return launch_stream<T, 2, 2, 1>(x, s);
        case kMatmulStreamTwo4: return launch_stream<T, 2, 4, 1>(x, s);
        case kMatmul256x256:
            if constexpr (sizeof(T) == 2) return launch_tiles<T, 256, 256, 2, 4, 2, true>(x, p.splits, s);
            return hipErrorInvalidValue;  // not among a 32-bit result's shapes
        case kMatmul256x128: return launch_tiles<T, 256, 128, 4, 2, 3, true>(x, p.splits, s);
        case kMatmul192x128: return launch_tiles<T, 192, 128, 2, 4, 3, true>(x, p.splits, s);
        case kMatmul128x128: return launch_tiles<T, 128, 128, 2, 4, 4, true>(x, p.splits, s);
        case kMatmulUnaligned: return launch_tiles<T, 128, 128, 2, 4, 4, false>(x, p.splits, s);
        default: return hipErrorInvalidValue;
    }
}

// Where the copies of A and B and the splits' sums stand in the workspace.
struct Scratch {
    uint64_t ld, a, b, sums, bytes;
};
Scratch scratch_of(const MatmulPart* parts, int count, uint64_t m, uint64_t n, uint64_t k) {
    auto up = [](uint64_t v) { return (v + 255) / 256 * 256; };
    Scratch s = {(k + 15) / 16 * 16, 0, 0, 0, 0};
    for (int i = 0; i < count; ++i) {
        if (parts[i].kind == kMatmulPack) {
            s.b = up(m * s.ld);
            s.sums = s.b + up(n * s.ld);
            s.bytes = s.sums;
        }
        const uint64_t sums = parts[i].splits > 1 ? parts[i].splits * parts[i].rows * parts[i].cols * 4 : 0;
        if (s.sums + sums > s.bytes) s.bytes = s.sums + sums;
    }
    return s;
}

hipError_t launch_pack(const uint8_t* from, uint64_t ld, uint64_t rows, uint64_t k, uint8_t* to, uint64_t ld_to,
                       hipStream_t s) {
    const uint64_t blocks = (rows * (ld_to / 16) + 255) / 256;
    pack_kernel<<<(uint32_t)(blocks < 8192 ? blocks : 8192), 256, 0, s>>>(from, ld, (uint32_t)rows, (uint32_t)k, to,
                                                                        ld_to);
    return hipGetLastError();
}

bool rows_aligned(const uint8_t* p, uint64_t ld) { return ld % 16 == 0 && (uintptr_t)p % 16 == 0; }

template <typename T>
hipError_t launch(MatmulArgs x, hipStream_t s) {
    const bool tiles = fp8_matmul_tiles(x.ld_a, x.ld_b);
    const bool a_aligned = rows_aligned(x.a, x.ld_a), b_aligned = rows_aligned(x.b, x.ld_b);
    MatmulPart parts[kMatmulMostParts];
    const int count = fp8_matmul_parts(sizeof(T) == 4, a_aligned && b_aligned, tiles, x.m, x.n, x.k, parts);
    const Scratch scratch = scratch_of(parts, count, x.m, x.n, x.k);
    uint8_t* const workspace = (uint8_t*)x.workspace;
    x.workspace = workspace + scratch.sums;
    const uint64_t groups = (x.k + kFp8Group - 1) / kFp8Group;
    const MatmulPart whole = {0, 1, x.m, x.n};
    for (int i = 0; i < count; ++i) {
        hipError_t e;
        if (parts[i].kind == kMatmulPack) {
            // only an operand whose own rows are at odd addresses: aligned ones, such as verified
            // weights, are read where they lie
            e = hipSuccess;
            if (!a_aligned) {
                e = launch_pack(x.a, x.ld_a, x.m, x.k, workspace + scratch.a, scratch.ld, s);
                x.a = workspace + scratch.a;
                x.ld_a = scratch.ld;
            }
            if (e == hipSuccess && !b_aligned) {
                e = launch_pack(x.b, x.ld_b, x.n, x.k, workspace + scratch.b, scratch.ld, s);
                x.b = workspace + scratch.b;
                x.ld_b = scratch.ld;
            }
        } else {  // its first rows and columns, or (a second one) the last
            const bool last = i > 0 && parts[i - 1].kind != kMatmulPack;
            const uint64_t row = last ? whole.rows - parts[i].rows : 0, col = last ? whole.cols - parts[i].cols : 0;
            MatmulArgs part = x;
            part.m = parts[i].rows;
            part.n = parts[i].cols;
            part.a += row * x.ld_a;
            part.a_scales += row * groups;
            part.b += col * x.ld_b;
            part.b_scales += col / kFp8Group * groups;
            part.c = (T*)x.c + row * x.ld_c + col;
            e = launch_part<T>(parts[i], part, s);
        }
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

bool fp8_matmul_tiles(uint64_t ld_a, uint64_t ld_b) { return ld_a <= kMaxTileLd && ld_b <= kMaxTileLd; }

uint64_t fp8_matmul_workspace(bool wide, bool aligned, uint64_t m, uint64_t n, uint64_t k) {
    MatmulPart parts[kMatmulMostParts];
    const int count = fp8_matmul_parts(wide, aligned, true, m, n, k, parts);
    return scratch_of(parts, count, m, n, k).bytes;
}

hipError_t launch_fp8_matmul(int type, const MatmulArgs& x, hipStream_t s) {
    switch (type) {
        case kTypeBf16: return launch<__bf16>(x, s);
        case kTypeF16: return launch<_Float16>(x, s);
        default: return launch<float>(x, s);
    }
}

}  // namespace hv
