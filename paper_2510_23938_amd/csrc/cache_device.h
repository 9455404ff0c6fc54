// cache_device.h -- the 8-bit cache and a batch's sequences on the device.
#pragma once
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include <hip/hip_runtime.h>

#include "fp8_device.h"
#include "hv_kernels.h"

namespace hv {

constexpr uint32_t kCacheBlock = 16;  // tokens of a head that share a scale

// The power of two that a scale stands for: its exponent, as a number from 2^-126 to 2^127.
__device__ __forceinline__ float cache_scale(float s) {
    const uint32_t e = __float_as_uint(s) & 0x7f800000;
    return __uint_as_float(min(max(e, 0x00800000u), 0x7f000000u));
}

// b / blocks_per_page of a block number below 2^26 and up to 2^12 blocks a page: with divide = ceil(2^38 /
// blocks_per_page) the product stays below 2^64, and its quotient is above the true one by less than 2^26 / 2^38,
// which is less than a whole number's fraction by 2^12 lacks to the next.
__device__ __forceinline__ uint32_t page_column(uint32_t block, uint64_t divide) {
    return (uint32_t)(block * divide >> 38);
}

// With l the bits of d - 1, mul = floor(2^(31 + l) / d) + 1 is off by at most 2^l / 2^(31 + l) of itself: too little to
// change the quotient of a number below 2^31.
inline Divider divider(uint32_t d) {
    if (d <= 1) return {0, 0};
    uint32_t l = 1;
    while (((uint64_t)1 << l) < d) ++l;
    return {(uint32_t)(((uint64_t)1 << (31 + l)) / d + 1), l - 1};
}
__device__ __forceinline__ uint32_t divided(uint32_t n, Divider d) {
    return d.mul != 0 ? __umulhi(n, d.mul) >> d.shift : n;
}

// Sum of x over this lane and those before it, by DPP: within rows of 16, then across them.
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
    auto moved = [](uint32_t v, auto ctrl, auto rows) {
        return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
    };
    using std::integral_constant;
    integral_constant<int, 0xf> all;
    x += moved(x, integral_constant<int, 0x111>{}, all);  // row_shr:1
    x += moved(x, integral_constant<int, 0x112>{}, all);
    x += moved(x, integral_constant<int, 0x114>{}, all);
    x += moved(x, integral_constant<int, 0x118>{}, all);
    x += moved(x, integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});  // row_bcast:15
    x += moved(x, integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});  // row_bcast:31
    return x;
}

__device__ __forceinline__ uint32_t lane_id() { return __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0)); }

// A sequence's rows of the call, and the position of the first; no rows where the batch does not describe a
// valid sequence.
struct Sequence {
    int32_t row, rows, position;
};

__device__ __forceinline__ Sequence sequence_at(const BatchArgs& b, uint32_t i) {
    const int32_t first = b.starts[i], end = b.starts[i + 1];
    const int32_t rows = first >= 0 && end > first && end <= b.tokens ? end - first : 0;
    return {first, rows, max(b.lengths[i], 0) - rows};
}

__device__ __forceinline__ Sequence sequence_in_lane(const Sequence& s, uint32_t lane) {
    return {__builtin_amdgcn_readlane(s.row, lane), __builtin_amdgcn_readlane(s.rows, lane),
            __builtin_amdgcn_readlane(s.position, lane)};
}

// A workgroup for each of more items than a launch's first dimension holds (2^32 threads): the rest in the third.
constexpr uint32_t kRowOfItems = 1u << 20;
inline dim3 item_grid(uint32_t items, uint32_t y = 1) {
    return dim3(std::min(items, kRowOfItems), y, (items + kRowOfItems - 1) / kRowOfItems);
}
__device__ __forceinline__ uint32_t item_of_block() { return blockIdx.z * kRowOfItems + blockIdx.x; }

// Which sequence an item belongs to, where sequence i has items(sequence) of them, and the item's
// number there.  Every wave looks for itself; all its lanes take part.
struct ItemPlace {
    bool found;
    uint32_t index, within;
    Sequence sequence;
};

template <typename Items>
__device__ __forceinline__ ItemPlace find_item(const BatchArgs& b, uint32_t item, Items items) {
    const uint32_t lane = lane_id();
    for (uint32_t base = 0; base < b.count; base += 64) {
        const Sequence s = base + lane < b.count ? sequence_at(b, base + lane) : Sequence{0, 0, 0};
        const uint32_t n = items(s), upto = wave_scan(n);
        const uint64_t at = __ballot(upto > item);
        if (at != 0) {
            const uint32_t l = __builtin_ctzll(at);
            return {true, base + l, item - __builtin_amdgcn_readlane(upto - n, l), sequence_in_lane(s, l)};
        }
        item -= __builtin_amdgcn_readlane(upto, 63);
    }
    return {false, 0, 0, {0, 0, 0}};
}

}  // namespace hv
