// fp8_cache.hip -- new tokens' keys and values into the 8-bit cache.
//
// A wave takes one block of 16 tokens of one head, keys and values: it has the
// block's new elements in registers, takes their largest magnitude, and writes
// codes under the power of two that this asks for (or the larger one that the block
// had).  The division by a power of two is exact, so each code is rounded once.
//
// Keys are written as they come, eight elements a lane.  Of the values a lane has
// neighbouring dimensions of all 16 tokens, which in the cache lie side by side
// for each dimension: 16 loads of two elements a lane turn the block without LDS or
// exchanges between lanes, and the stores are whole lines.
//
// Bound by memory: 16384 tokens of 8 heads of 128 dimensions in bfloat16 (101 MB) 26 us, 3.8 TB/s, where a copy
// reaches 4.75: 1.6 rounds of the waves that the chip holds, each with three trips to memory (the sequences,
// the page beside the elements, the stores).  A token of each of 8 sequences takes 6 us, those trips and a launch.
#include <algorithm>
#include <type_traits>

#include "cache_device.h"

namespace hv {
namespace {

// The largest magnitude of a wave's 64 lanes, in all of them.
__device__ __forceinline__ float wave_max(float m) {
    m = row16_max(m);
    m = fmaxf(m, __shfl_xor(m, 16));
    return fmaxf(m, __shfl_xor(m, 32));
}

// The smallest power of two, at least 2^-126, under which magnitudes up to `largest` are at most 448 = 1.75 * 2^8.
__device__ __forceinline__ float power_scale(float largest) {
    const uint32_t bits = __float_as_uint(largest);
    const int e = (int)(bits >> 23) - 8 + ((bits & 0x7fffff) > 0x600000);
    return __uint_as_float((uint32_t)max(e, 1) << 23);
}

__device__ __forceinline__ float finite_or_zero(float x) {
    const float a = __builtin_fabsf(x);
    return a < __builtin_inff() ? a : 0.0f;
}

// Two codes in the low half, of values divided by a power of two whose reciprocal is `inverse`.
__device__ __forceinline__ uint32_t two_codes(float a, float b, float inverse) {
    const float nan = __builtin_nanf("");
    a = __builtin_fabsf(a) < __builtin_inff() ? a * inverse : nan;
    b = __builtin_fabsf(b) < __builtin_inff() ? b * inverse : nan;
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xffff;
}

// Four codes under a scale that is 1 / ratio of theirs.
__device__ __forceinline__ uint32_t rescaled(uint32_t codes, float ratio) {
    const float a = __builtin_amdgcn_cvt_f32_fp8(codes, 0) * ratio, b = __builtin_amdgcn_cvt_f32_fp8(codes, 1) * ratio;
    const float c = __builtin_amdgcn_cvt_f32_fp8(codes, 2) * ratio, d = __builtin_amdgcn_cvt_f32_fp8(codes, 3) * ratio;
    const int low = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, low, true);
}

// The scale of a block, from its new values' largest magnitude and, where it has earlier tokens, its old scale.
__device__ __forceinline__ float block_scale(float largest, bool has_old, float old) {
    const float need = power_scale(largest);
    return has_old ? fmaxf(need, old) : need;
}

// Bytes 0 to count - 1 of a word set.
__device__ __forceinline__ uint32_t low_bytes(int count) {
    return count <= 0 ? 0u : count >= 4 ? ~0u : (1u << 8 * count) - 1;
}

constexpr int kWaves = 4;

// KI: groups of eight elements of a lane's share of the keys; VI: pairs of dimensions of the values.
template <typename T, int KI, int VI>
__global__ void __launch_bounds__(kWaves * 64) write_kernel(WriteArgs x) {
    const uint32_t lane = threadIdx.x % 64;
    const uint32_t head = blockIdx.y * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    if (head >= x.cache.heads) return;
    auto first_written = [&](const Sequence& s) { return max(s.position, 0); };
    auto end_written = [&](const Sequence& s) { return min(s.position + s.rows, x.batch.capacity); };
    const ItemPlace place = find_item(x.batch, item_of_block(), [&](const Sequence& s) -> uint32_t {
        const int p0 = first_written(s), p1 = end_written(s);
        return s.rows > 0 && p1 > p0 ? (p1 - 1) / 16 - p0 / 16 + 1 : 0;
    });
    if (!place.found) return;
    const Sequence s = place.sequence;
    const int p0 = first_written(s), p1 = end_written(s);
    const uint32_t block = p0 / 16 + place.within, column = page_column(block, x.cache.divide);
    const int32_t page = x.batch.table[place.index * x.batch.ld_table + column];
    const uint32_t in_page = block - column * x.cache.page_blocks;
    // slots [a, b) of the block get new tokens, those before a hold earlier ones
    const int a = max(p0 - (int)block * 16, 0), b = min(p1 - (int)block * 16, 16);
    const int64_t row0 = s.row + ((int)block * 16 - s.position);  // of slot 0

    const uint32_t dims = x.cache.head_dim;
    const T* const k_from = (const T*)x.k + head * x.k_head;
    const T* const v_from = (const T*)x.v + head * x.v_head;

    // keys: eights of the block's elements, token by token
    float k[KI][8];
    int slot[KI];
    const uint32_t eights = dims / 8;
#pragma unroll
    for (int i = 0; i < KI; ++i) {
        const uint32_t at = i * 64 + lane, t = at / eights;
        slot[i] = (int)t;
        const bool fresh = (int)t >= a && (int)t < b;
        if (fresh) {
            load_eight(k_from + (row0 + t) * (int64_t)x.k_token + (at - t * eights) * 8, 8, k[i]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) k[i][e] = 0.0f;
        }
    }
    // values: two neighbouring dimensions of each token
    using Two = T __attribute__((ext_vector_type(2)));
    float v[VI][16][2];
    uint4 held[VI][2];
#pragma unroll
    for (int i = 0; i < VI; ++i) {
        const uint32_t d = (i * 64 + lane) * 2;
        const bool inside = d < dims;
#pragma unroll
        for (int t = 0; t < 16; ++t) {
            Two two = {(T)0.0f, (T)0.0f};
            if (t >= a && t < b && inside) __builtin_memcpy(&two, v_from + (row0 + t) * (int64_t)x.v_token + d, sizeof two);
            v[i][t][0] = (float)two.x;
            v[i][t][1] = (float)two.y;
        }
    }

    // the page and what the block holds, with those loads under way
    if (page < 0 || (uint32_t)page >= x.cache.pages) return;
    const uint64_t scale_at = ((uint64_t)page * x.cache.heads + head) * x.cache.page_blocks + in_page;
    uint8_t* const k_to = x.cache.k_codes + page * x.cache.k_page + head * x.cache.k_head + (uint64_t)in_page * 16 * dims;
    uint8_t* const v_to = x.cache.v_codes + page * x.cache.v_page + head * x.cache.v_head + (uint64_t)in_page * 16 * dims;
    float k_old = 0.0f, v_old = 0.0f;
    if (a > 0) {
        k_old = cache_scale(x.cache.k_scales[scale_at]);
        v_old = cache_scale(x.cache.v_scales[scale_at]);
    }
#pragma unroll
    for (int i = 0; i < VI; ++i) {
        const uint32_t d = (i * 64 + lane) * 2;
        held[i][0] = held[i][1] = uint4{0, 0, 0, 0};
        if ((a > 0 || b < 16) && d < dims) __builtin_memcpy(held[i], v_to + d * 16, 32);
    }

    float k_most = 0.0f, v_most = 0.0f;
#pragma unroll
    for (int i = 0; i < KI; ++i) k_most = fmaxf(k_most, finite_largest(k[i]));
#pragma unroll
    for (int i = 0; i < VI; ++i)
#pragma unroll
        for (int t = 0; t < 16; ++t) v_most = fmaxf(v_most, fmaxf(finite_or_zero(v[i][t][0]), finite_or_zero(v[i][t][1])));
    const float k_scale = block_scale(wave_max(k_most), a > 0, k_old);
    const float v_scale = block_scale(wave_max(v_most), a > 0, v_old);
    const float k_inverse = 1.0f / k_scale, v_inverse = 1.0f / v_scale;

#pragma unroll
    for (int i = 0; i < KI; ++i) {
        uint8_t* const to = k_to + (uint32_t)(i * 64 + lane) * 8;
        if (slot[i] >= a && slot[i] < b) {
            const uint2 w = {two_codes(k[i][0], k[i][1], k_inverse) | two_codes(k[i][2], k[i][3], k_inverse) << 16,
                             two_codes(k[i][4], k[i][5], k_inverse) | two_codes(k[i][6], k[i][7], k_inverse) << 16};
            __builtin_memcpy(to, &w, 8);
        } else if (slot[i] < a && k_scale != k_old) {
            uint2 w;
            __builtin_memcpy(&w, to, 8);
            w = {rescaled(w.x, k_old * k_inverse), rescaled(w.y, k_old * k_inverse)};
            __builtin_memcpy(to, &w, 8);
        }
    }
    const float v_ratio = v_old * v_inverse;
#pragma unroll
    for (int i = 0; i < VI; ++i) {
        const uint32_t d = (i * 64 + lane) * 2;
        if (d >= dims) continue;
        uint32_t w[2][4];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint32_t before[4] = {held[i][e].x, held[i][e].y, held[i][e].z, held[i][e].w};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t fresh = two_codes(v[i][4 * q][e], v[i][4 * q + 1][e], v_inverse) |
                                       two_codes(v[i][4 * q + 2][e], v[i][4 * q + 3][e], v_inverse) << 16;
                const uint32_t old_bytes = low_bytes(a - 4 * q), new_bytes = low_bytes(b - 4 * q) & ~old_bytes;
                uint32_t kept = before[q];
                if (a > 0 && v_scale != v_old) kept = (rescaled(kept, v_ratio) & old_bytes) | (kept & ~old_bytes);
                w[e][q] = (fresh & new_bytes) | (kept & ~new_bytes);
            }
        }
        __builtin_memcpy(v_to + d * 16, w, 32);
    }
    if (lane == 0) {
        x.cache.k_scales[scale_at] = k_scale;
        x.cache.v_scales[scale_at] = v_scale;
    }
}

template <typename T>
hipError_t launch(const WriteArgs& a, hipStream_t s) {
    // Blocks that new tokens touch: a sequence of n rows touches (n + 14) / 16 + 1 at most and n at most.
    const uint64_t tokens = a.batch.tokens;
    const uint64_t blocks = std::min<uint64_t>(tokens, tokens / 16 + 2 * std::min<uint64_t>(a.batch.count, tokens));
    const dim3 grid = item_grid((uint32_t)blocks, (a.cache.heads + kWaves - 1) / kWaves);
    const uint32_t d = a.cache.head_dim;
    auto run = [&](auto ki, auto vi) {
        write_kernel<T, decltype(ki)::value, decltype(vi)::value><<<grid, kWaves * 64, 0, s>>>(a);
        return hipGetLastError();
    };
    using std::integral_constant;
    integral_constant<int, 1> one;
    integral_constant<int, 2> two;
    // 2 * d eights of keys and d / 2 pairs of values, 64 at a time
    if (d <= 32) return run(one, one);
    if (d <= 64) return run(two, one);
    if (d <= 128) return run(integral_constant<int, 4>{}, one);
    return run(integral_constant<int, 8>{}, two);
}

}  // namespace

hipError_t launch_fp8_cache_write(int type, const WriteArgs& a, hipStream_t s) {
    return type == kTypeBf16 ? launch<__bf16>(a, s) : type == kTypeF16 ? launch<_Float16>(a, s) : launch<float>(a, s);
}

}  // namespace hv
