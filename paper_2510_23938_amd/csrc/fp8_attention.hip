// fp8_attention.hip -- attention of new tokens over the 8-bit cache:
//   out = sum_j w_j v_j,  w = softmax_j(scale * q . k_j) over the positions that a token sees.
//
// One pass over the keys, 64 at a time, with the running maximum m and sum l of
// each row's weights: p = exp2(s - m), l = sum p, o = sum p v, and where m grows by more
// than 2^8 the sums so far are scaled down.  A "row" is one head of one new token; the
// heads that share a key head and the tokens of a sequence are rows of one problem,
// so each key is read once for all of them.
//
// Codes are widened to the 16-bit type, which holds them exactly, and multiplied by
// its matrix instruction, whose sums are in 32 bits.  The product of keys and queries
// is made transposed (keys down, rows across): its result leaves a lane with
// weights of one row only, and the keys are taken in such an order that they are
// those of one block of 16 tokens (or of two), all of them, in order.  That is the layout in which
// the second product wants its weights, so they never leave the lane; a lane has one key
// scale, which joins the softmax's own multiplication, and one value scale,
// which the conversion of codes applies; and values lie in the cache by dimensions so that
// their 16 bytes are those 16 tokens.
//
// Two kernels: up to 32 rows (a token or a few each of many sequences), bound by reading
// the cache, take it from memory to registers (666 MB of 64 sequences 133 us, 5.0 TB/s; one of 131072 tokens 56 us, 4.8,
// where a copy reaches 4.75); more rows, bound by the matrix and vector units, which
// take turns more than they overlap (33% and 44% of the cycles), share it in LDS (4 prompts of 2048 tokens, 64 heads
// on 8 of 128 dimensions, 350 us, 0.79 PFLOP/s; one of 16384 tokens 1.0, where a library's product reaches 1.3 to 1.5).
// In both, a sequence's keys are cut into segments where there are too few rows to fill the
// chip; the parts' sums are joined by another kernel, in order.  A call whose sequences can have no more than 1536
// tokens is never cut: its one launch (777 tokens: 11 us) is shorter than two (13.6, with room for 8192).
#include <algorithm>
#include <cfloat>
#include <type_traits>

#include "cache_device.h"

namespace hv {
namespace {

using bf16x2 = __attribute__((ext_vector_type(2))) __bf16;
using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;
using f16x2 = __attribute__((ext_vector_type(2))) _Float16;
using f16x8 = __attribute__((ext_vector_type(8))) _Float16;
using float4x = __attribute__((ext_vector_type(4))) float;
using float16x = __attribute__((ext_vector_type(16))) float;

constexpr int kTile = 64;         // keys of a step
constexpr int kMatrix = 0x8, kDsRead = 0x100;  // instruction groups of the scheduler
constexpr int kWaitAll = 0;       // s_waitcnt: nothing outstanding
constexpr float kLazy = 8.0f;     // binary orders that a row's weights may grow before its sums are scaled
// What turns scores into exponents, at least: the smallest positive number, as what is not seen is minus infinity times it.
// Sums of a query and codes are below 2^128, so what this changes is less than 2^-21 of an exponent.
constexpr float kLeastBy = 0x1p-149f;
constexpr float kNothing = -FLT_MAX;  // the maximum of a row that has seen nothing
// Half precision: binary orders that weights are raised by, so that those of blocks with small scales lose less.  With
// kLazy and half of a score's last place, which is worth less than one there (kCoarse), they stay below 2^13.
constexpr int kRaised = 4;

// ---------------------------------------------------------------------------
// the 16-bit types

template <typename T>
struct Wide;

template <>
struct Wide<__bf16> {
    using Eight = bf16x8;
    // The exponents are those of 32 bits: a block's scale goes into its values as it is.
    static constexpr bool kRelative = false;
    template <bool kHigh>
    static __device__ __forceinline__ bf16x2 two(uint32_t w, float scale) {
        return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, kHigh);
    }
    static __device__ __forceinline__ Eight codes(uint32_t lo, uint32_t hi, float scale) {
        const bf16x2 a = two<false>(lo, scale), b = two<true>(lo, scale), c = two<false>(hi, scale), d = two<true>(hi, scale);
        return Eight{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
    // sum and the weights of eight, as they are after their rounding
    static __device__ __forceinline__ float add(Eight p, float sum) {
        const bf16x2 one = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
        for (int i = 0; i < 8; i += 2) sum = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{p[i], p[i + 1]}, one, sum, false);
        return sum;
    }
    static __device__ __forceinline__ float4x mul16(Eight a, Eight b, float4x c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
    static __device__ __forceinline__ float16x mul32(Eight a, Eight b, float16x c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
};

template <>
struct Wide<_Float16> {
    using Eight = f16x8;
    // Values times their scale may leave the type: the scale goes into the weights, relative to the largest scale of
    // what the row sees.
    static constexpr bool kRelative = true;
    template <bool kHigh>
    static __device__ __forceinline__ f16x2 two(uint32_t w, float scale) {
        return __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, kHigh);
    }
    static __device__ __forceinline__ Eight codes(uint32_t lo, uint32_t hi, float scale) {
        const f16x2 a = two<false>(lo, scale), b = two<true>(lo, scale), c = two<false>(hi, scale), d = two<true>(hi, scale);
        return Eight{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
    static __device__ __forceinline__ float4x mul16(Eight a, Eight b, float4x c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
    static __device__ __forceinline__ float16x mul32(Eight a, Eight b, float16x c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    }
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// A weight's exponent is s * by - m, by one instruction that rounds once, while m is a rounded product: of the largest score
// that leaves m's rounding error, half of its last place, which all of a row's weights have in common.  Where m's last place
// is worth one or more the product is rounded before the subtraction, as m was, so that the largest weight stays what it
// has to be: at 2^31 half of a last place is 2^7 binary orders, which no sum would hold.
constexpr float kCoarse = 0x1p23f;
__device__ __forceinline__ float coarse_exponent(float s, float by, float m) {
#pragma clang fp contract(off)
    const float scaled = s * by;
    return scaled - m;
}

// 2^e as the conversions' scale, at least 2^-126.
__device__ __forceinline__ float power_of(int e) { return __uint_as_float((uint32_t)max(e + 127, 1) << 23); }
__device__ __forceinline__ int exponent_of(float power) { return (int)(__float_as_uint(power) >> 23) - 127; }

// Codes that a weight of zero does not hide: NaN, and in bfloat16 those whose value under the block's scale is 2^128 or
// more, an infinity.  Such a code's magnitude, as a byte, is the limit or more: 0x7f, or that of 2^(128 - e).  What is
// added to a byte's low seven bits makes its high bit of that.
template <typename T>
__device__ __forceinline__ uint32_t lost_codes(float power) {
    const int e = Wide<T>::kRelative ? 0 : exponent_of(power), limit = e < 120 ? 0x7f : (135 - e) << 3;
    return (0x80 - limit) * 0x01010101u;
}
// The high bit of each byte that is one of them.
__device__ __forceinline__ uint32_t lost_bytes(uint32_t w, uint32_t lost) { return ((w & 0x7f7f7f7f) + lost) & 0x80808080; }
// Zero codes in their place; whether there were any.
__device__ __forceinline__ uint32_t take_lost(uint32_t& w, uint32_t lost) {
    const uint32_t m = lost_bytes(w, lost);
    w &= ~(m | (m - (m >> 7)));
    return m;
}
__device__ __forceinline__ uint32_t take_lost(uint4& w, uint32_t lost) {
    return take_lost(w.x, lost) | take_lost(w.y, lost) | take_lost(w.z, lost) | take_lost(w.w, lost);
}
// The code of 1 in their place, and of zero elsewhere.
__device__ __forceinline__ uint32_t ones_at_lost(uint32_t w, uint32_t lost) {
    const uint32_t m = lost_bytes(w, lost);
    return m >> 2 | m >> 3 | m >> 4;
}

// ---------------------------------------------------------------------------
// which keys, and who takes them

// The first key that a position's window has, if not negative.  A position before the first, which sees nothing, is taken
// for the first: its distance to a window's start may not fit.
__device__ __forceinline__ int window_from(const AttentionArgs& x, int position) {
    return x.window ? max(position, 0) - x.window + 1 : 0;
}

// Tiles of 64 keys that the positions p_min to p_max see: the first `sinks` of them from 0 on, the others from `first`.
struct Range {
    int first, sinks, count;
    __device__ __forceinline__ int tile(int t) const { return t < sinks ? t : first + t - sinks; }
};

__device__ __forceinline__ Range range_of(const AttentionArgs& x, int p_min, int p_max) {
    const int hi = min(p_max, x.batch.capacity - 1);
    if (hi < 0 || x.cache.pages == 0) return {0, 0, 0};
    const int lo = max(window_from(x, p_min), 0);
    const int lo_tile = lo / kTile, hi_tile = hi / kTile;
    const int sinks = x.window ? min(lo_tile, (min(x.sinks, hi + 1) + kTile - 1) / kTile) : 0;
    return {lo_tile, sinks, sinks + max(hi_tile - lo_tile + 1, 0)};
}

// A workgroup's work.
struct Job {
    bool found;
    Sequence sequence;
    uint32_t index, row_tile, head, segment, segments, part;
};

// A sequence's work: row tiles of R rows for each key head, and the key tiles that each of them may see.
struct Work {
    Sequence sequence;
    uint32_t row_tiles, units, tiles;
};

template <int R>
__device__ __forceinline__ Work work_at(const AttentionArgs& x, uint32_t i) {
    Work w = {{0, 0, 0}, 0, 0, 0};
    if (i >= x.batch.count) return w;
    w.sequence = sequence_at(x.batch, i);
    if (w.sequence.rows == 0) return w;
    w.row_tiles = ((uint32_t)w.sequence.rows * x.share + R - 1) / R;
    w.units = w.row_tiles * x.cache.heads;
    w.tiles = (uint32_t)range_of(x, w.sequence.position, w.sequence.position + w.sequence.rows - 1).count;
    return w;
}

// All lanes' units times tiles.  Each is cut at 2^40, so that 64 of them add in two pieces: one of those is enough for a share
// of 2^30 tiles (2^9 slots), and no sequence has more than 2^24.
__device__ __forceinline__ uint64_t total_tiles(const Work& w) {
    const uint64_t mine = min((uint64_t)w.units * w.tiles, (uint64_t)1 << 40);
    const uint32_t low = wave_scan((uint32_t)mine & 0xffff), high = wave_scan((uint32_t)(mine >> 16));
    return ((uint64_t)(uint32_t)__builtin_amdgcn_readlane(high, 63) << 16) + (uint32_t)__builtin_amdgcn_readlane(low, 63);
}

// Segments of a unit's tiles, `share` of them each.  A quarter of a segment more does not cost another, so the
// segments of all units that are cut in two or more are fewer than 2 * slots: s < c / share + 3/4 with c / share > 5/4.
__device__ __forceinline__ uint32_t segments_of(uint32_t tiles, uint32_t share) {
    const uint32_t slack = share / 4;
    return tiles <= share + slack ? 1 : (tiles - slack + share - 1) / share;
}

// The job of number `item`; or, for the join, that of the item-th unit which is cut (its first segment's).
template <int R, bool kJoin>
__device__ __forceinline__ Job find_job(const AttentionArgs& x, uint32_t item) {
    const uint32_t lane = lane_id();
    Work w = work_at<R>(x, lane);
    // tiles of a segment: an even share of all for each of the slots, at least `least`
    uint32_t share = ~0u;
    if (x.log2_slots != 0) {
        uint64_t total = total_tiles(w);
        for (uint32_t base = 64; base < x.batch.count; base += 64) total += total_tiles(work_at<R>(x, base + lane));
        const uint64_t even = (total + ((uint64_t)1 << x.log2_slots) - 1) >> x.log2_slots;
        share = (uint32_t)min(max(even, (uint64_t)x.least), (uint64_t)1 << 30);
    }
    uint32_t part = 0;
    for (uint32_t base = 0;;) {
        const bool cut = w.tiles > share + share / 4 && share != ~0u;
        uint32_t segments = 1;
        if (__ballot(cut) != 0) segments = cut ? segments_of(w.tiles, share) : 1;
        const uint32_t parts = cut ? w.units * segments : 0;
        const uint32_t items = kJoin ? (cut ? w.units : 0) : w.units * segments;
        const uint32_t upto = wave_scan(items), parts_upto = wave_scan(parts);
        const uint64_t at = __ballot(upto > item);
        if (at != 0) {
            const uint32_t l = __builtin_ctzll(at);
            const uint32_t within = item - __builtin_amdgcn_readlane(upto - items, l);
            const uint32_t n = __builtin_amdgcn_readlane(segments, l), all = __builtin_amdgcn_readlane(items, l);
            const uint32_t unit = kJoin || n == 1 ? within : within / n, segment = kJoin ? 0 : within - unit * n;
            const uint32_t row_tiles = __builtin_amdgcn_readlane(w.row_tiles, l);
            const uint32_t row_tile = divided(unit, x.by_heads);
            part += __builtin_amdgcn_readlane(parts_upto - parts, l) + unit * n + segment;
            // the last rows, which see the most, first; what a batch without order may ask for stays in bounds
            const bool ok = within < all && (n == 1 || part + (kJoin ? n - 1 : 0) < x.parts_limit);
            return {ok, sequence_in_lane(w.sequence, l), base + l, row_tiles - 1 - row_tile, unit - row_tile * x.cache.heads,
                    segment, n, part};
        }
        item -= __builtin_amdgcn_readlane(upto, 63);
        part += __builtin_amdgcn_readlane(parts_upto, 63);
        base += 64;
        if (base >= x.batch.count) return {};
        w = work_at<R>(x, base + lane);
    }
}

// Whether a position sees some of the block's 16 tokens from `key` on.
__device__ __forceinline__ bool block_seen(const AttentionArgs& x, int key, int position) {
    return key <= position && (key + (int)kCacheBlock > window_from(x, position) || key < x.sinks);
}

// `from`: the first key that a position's window has.
__device__ __forceinline__ bool sees(const AttentionArgs& x, int position, int from, int key) {
    return (key <= position) & ((key >= from) | (key < x.sinks));
}
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Whether some of the positions p_min to p_max does not see some key of the tile from key0 on.
__device__ __forceinline__ bool is_edge(const AttentionArgs& x, int key0, int p_min, int p_max) {
    return key0 + kTile - 1 > p_min || (x.window && p_max - key0 >= x.window && key0 + kTile > x.sinks);
}

// The pages of a sequence's blocks of 16 tokens.  The table's last column stands in for those behind it, so that
// nothing has to be decided before it is read.
struct Places {
    const int32_t* table;
    uint32_t last, pages, page_blocks;  // last: block that the table has a column for
    uint64_t divide;
    struct Block {
        uint32_t page, block;  // and the number in the page
        bool listed;
        uint32_t pages;        // of the cache
        __device__ __forceinline__ bool there() const { return listed & (page < pages); }
    };
    __device__ __forceinline__ Places(const AttentionArgs& x, uint32_t sequence)
        : table(x.batch.table + sequence * x.batch.ld_table), last((uint32_t)x.batch.capacity / kCacheBlock - 1),
          pages(x.cache.pages), page_blocks(x.cache.page_blocks), divide(x.cache.divide) {}
    __device__ __forceinline__ Block of(uint32_t block, bool wanted = true) const {
        const uint32_t inside = min(block, last), column = page_column(inside, divide);
        return {(uint32_t)table[column], inside - column * page_blocks, wanted && block == inside, pages};
    }
    __device__ __forceinline__ Block first_if_none(const Block& b) const {
        return {b.there() ? b.page : 0, b.there() ? b.block : 0, b.listed, pages};
    }
};

// Parts' sums: [part][R][DP] sums, then [part][R] pairs of maximum and sum of weights.
template <int R, int DP>
__device__ __forceinline__ float* part_rows(const AttentionArgs& x, uint32_t part) {
    return x.parts + (uint64_t)part * R * DP;
}
template <int R, int DP>
__device__ __forceinline__ float2* part_weights(const AttentionArgs& x, uint32_t part) {
    return (float2*)(x.parts + (uint64_t)x.parts_limit * R * DP) + (uint64_t)part * R;
}

// Four neighbouring dimensions of a row's output.
template <typename T>
__device__ __forceinline__ void store_four(T* p, float4x v) {
    struct Four {
        T v[4];
    } four = {{(T)v[0], (T)v[1], (T)v[2], (T)v[3]}};
    __builtin_memcpy(p, &four, sizeof four);
}

template <typename T>
__device__ __forceinline__ T* out_at(const AttentionArgs& x, const Job& job, uint32_t row) {
    const uint32_t token = divided(row, x.by_share);
    return (T*)x.out + (uint64_t)(job.sequence.row + token) * x.out_token +
           (uint64_t)(job.head * x.share + (row - token * x.share)) * x.out_head;
}

// 16 neighbouring dimensions of a row's query; zeros where there are none.
template <typename T>
__device__ __forceinline__ void load_query(const AttentionArgs& x, const Job& job, uint32_t row, uint32_t rows, uint32_t d,
                                           typename Wide<T>::Eight (&q)[2]) {
    uint32_t zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (row < rows && d < x.cache.head_dim) {
        const uint32_t token = divided(row, x.by_share);
        const T* const p = (const T*)x.q + (uint64_t)(job.sequence.row + token) * x.q_token +
                           (uint64_t)(job.head * x.share + (row - token * x.share)) * x.q_head + d;
        __builtin_memcpy(zero, p, 32);
    }
    __builtin_memcpy(&q[0], zero, 16);
    __builtin_memcpy(&q[1], zero + 4, 16);
}

// ---------------------------------------------------------------------------
// few rows: the cache from memory to registers

// A workgroup takes 16 * F rows and one segment of their keys, its NW waves a tile of 64 keys in turn: a tile's 16 KB (of
// 128 dimensions) are asked for a tile ahead, 128 KB for each unit, which is what its share of HBM's rate
// times its latency asks for.  In a
// tile, a lane (row n = lane % 16, group g = lane / 16) has the weights of block g.  For that, fragment f of four has
// as its key m the token 4 f + m % 4 of block m / 4.
template <typename T, int DP, int F, int NW>
__global__ void __launch_bounds__(NW * 64) stream_attention(AttentionArgs x) {
    constexpr int R = 16 * F, NC = DP / 64, ND = DP / 16;
    constexpr int CE = std::min(ND, 64 / (NW * F));  // 16 dimensions each of all waves' sums that LDS holds at once
    static_assert(CE >= 1, "LDS holds a fragment of each wave");
    using W = Wide<T>;
    using Eight = typename W::Eight;
    __shared__ float4x sums[NW][F][CE][64];
    __shared__ float2 weights[NW][R];
    const Job job = find_job<R, false>(x, item_of_block());
    if (!job.found) return;
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t n = lane % 16, g = lane / 16, dims = x.cache.head_dim;
    const uint32_t rows_all = job.sequence.rows * x.share, row0 = job.row_tile * R, rows = min(rows_all - row0, (uint32_t)R);

    int pos[F], from[F];
#pragma unroll
    for (int fr = 0; fr < F; ++fr) {
        const uint32_t row = 16 * fr + n;
        pos[fr] = job.sequence.position + (int)divided(row0 + min(row, rows - 1), x.by_share);
        from[fr] = window_from(x, pos[fr]);
    }
    const int p_min = uniform(job.sequence.position + (int)divided(row0, x.by_share));
    const int p_max = uniform(job.sequence.position + (int)divided(row0 + rows - 1, x.by_share));
    const Range range = range_of(x, p_min, p_max);
    const int first = (int)((int64_t)range.count * job.segment / job.segments);
    const int end = (int)((int64_t)range.count * (job.segment + 1) / job.segments);

    const Places places(x, job.index);
    const uint8_t* const k_head = x.cache.k_codes + job.head * x.cache.k_head + (n % 4) * dims;
    const uint8_t* const v_head = x.cache.v_codes + job.head * x.cache.v_head;
    // Dimensions past the last are read as others of the same key, against zeros of the query, and of the values
    // into rows of sums that nobody stores.
    uint32_t k_from[NC], v_from[ND];
#pragma unroll
    for (int c = 0; c < NC; ++c) k_from[c] = 64 * c + 16 * g < dims ? 64 * c + 16 * g : 0;
#pragma unroll
    for (int e = 0; e < ND; ++e) v_from[e] = 16 * e + n < dims ? 16 * (16 * e + n) : 0;

    float4x o[F][ND];
    float m[F], l[F];
    int v_most[F];  // kRelative: the exponent of the largest value scale that the row has met
#pragma unroll
    for (int fr = 0; fr < F; ++fr) {
        v_most[fr] = -126;
        m[fr] = kNothing;
        l[fr] = 0.0f;
#pragma unroll
        for (int e = 0; e < ND; ++e) o[fr][e] = float4x{0, 0, 0, 0};
    }
    bool poisoned = false;  // whether a tile that some row does not see all of had a lost code among its values

    // Nothing is decided around these loads, so that the compiler knows which are under way and waits for no others:
    // what has no place is read at the cache's first block, and hidden afterwards.
    uint4 k[4][NC], v[ND];
    float k_scale = 0.0f, v_scale = 0.0f;
    // a tile's places: of the block that a lane reads keys of, and of the one that it has values and weights of
    Places::Block k_next = {0, 0, false, 0}, v_next = {0, 0, false, 0};
    auto look = [&](int t, Places::Block& k_place, Places::Block& v_place) {
        const uint32_t block = (uint32_t)range.tile(min(t, end - 1)) * 4;
        k_place = places.of(block + n / 4, t < end);
        v_place = places.of(block + g, t < end);
    };
    auto load_keys = [&](const Places::Block& b) {
        const Places::Block at = places.first_if_none(b);
        const uint8_t* const p = k_head + at.page * x.cache.k_page + at.block * (16 * dims);
#pragma unroll
        for (int f = 0; f < 4; ++f)
#pragma unroll
            for (int c = 0; c < NC; ++c) k[f][c] = *(const uint4*)(p + 4 * f * dims + k_from[c]);
    };
    auto load_values = [&](const Places::Block& b) {
        const Places::Block at = places.first_if_none(b);
        const uint8_t* const p = v_head + at.page * x.cache.v_page + at.block * (16 * dims);
#pragma unroll
        for (int e = 0; e < ND; ++e) v[e] = *(const uint4*)(p + v_from[e]);
    };
    auto load_scales = [&](const Places::Block& b) {
        const Places::Block at = places.first_if_none(b);
        const uint64_t i = ((uint64_t)at.page * x.cache.heads + job.head) * x.cache.page_blocks + at.block;
        k_scale = x.cache.k_scales[i];
        v_scale = x.cache.v_scales[i];
    };

    int t = first + (int)wave;
    bool here = false;  // whether the block that a lane has weights of is in the cache
    if (t < end) {
        look(t, k_next, v_next);
        here = v_next.there();
        load_keys(k_next);
        load_scales(v_next);
        load_values(v_next);
        look(t + NW, k_next, v_next);
    }
    __builtin_amdgcn_sched_barrier(0);
    Eight q[F][NC][2];
#pragma unroll
    for (int fr = 0; fr < F; ++fr)
#pragma unroll
        for (int c = 0; c < NC; ++c)
            load_query<T>(x, job, row0 + 16 * fr + n, row0 + rows, 64 * c + 16 * g, q[fr][c]);
    // The queries are here before the loop, as far as the compiler knows too, which would wait for them in it, and by
    // that for what was asked for after them.
    __builtin_amdgcn_s_waitcnt(kWaitAll);
    for (; t < end; t += NW) {
        const int tile = range.tile(t), key0 = tile * kTile;
        // asked for before the next tile's codes, so that it is there a tile later without waiting for them
        Places::Block k_then, v_then;
        look(t + 2 * NW, k_then, v_then);
        __builtin_amdgcn_sched_barrier(0);
        float4x s[F][4];
#pragma unroll
        for (int f = 0; f < 4; ++f) {
#pragma unroll
            for (int fr = 0; fr < F; ++fr) s[fr][f] = float4x{0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const Eight a = W::codes(k[f][c].x, k[f][c].y, 1.0f), b = W::codes(k[f][c].z, k[f][c].w, 1.0f);
#pragma unroll
                for (int fr = 0; fr < F; ++fr) {
                    s[fr][f] = W::mul16(a, q[fr][c][0], s[fr][f]);
                    s[fr][f] = W::mul16(b, q[fr][c][1], s[fr][f]);
                }
            }
        }
        const float to_log2 = fmaxf(cache_scale(k_scale) * x.scale, kLeastBy);
        const float v_power = cache_scale(v_scale);
        load_keys(k_next);

        const bool edge = is_edge(x, key0, p_min, p_max) || __ballot(!here) != 0;
        if (edge) {
            asm volatile("");  // a branch: the comparisons are not made for other tiles
#pragma unroll
            for (int fr = 0; fr < F; ++fr)
#pragma unroll
                for (int f = 0; f < 4; ++f)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        s[fr][f][r] = (here & sees(x, pos[fr], from[fr], key0 + 16 * (int)g + 4 * f + r)) ? s[fr][f][r] : -__builtin_inff();
            uint32_t any = 0;
            const uint32_t lost = lost_codes<T>(v_power);
#pragma unroll
            for (int e = 0; e < ND; ++e) any |= take_lost(v[e], lost);
            poisoned |= __ballot(any != 0) != 0;
        }
        const float widen_by = W::kRelative ? 1.0f : v_power;
        Eight p[F][2];
#pragma unroll
        for (int fr = 0; fr < F; ++fr) {
            float top = s[fr][0][0];
#pragma unroll
            for (int f = 0; f < 4; ++f)
#pragma unroll
                for (int r = 0; r < 4; ++r) top = fmaxf(top, s[fr][f][r]);
            top *= to_log2;
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            if (__ballot(top > m[fr] + kLazy) != 0) {  // for those rows: no row's rounding depends on another
                const float grown = top > m[fr] + kLazy ? top : m[fr], down = exp2_fast(m[fr] - grown);
                m[fr] = grown;
                l[fr] *= down;
#pragma unroll
                for (int e = 0; e < ND; ++e) o[fr][e] *= down;
            }
            float by = 1.0f;
            if constexpr (W::kRelative) {
                const int e = here && block_seen(x, key0 + 16 * (int)g, pos[fr]) ? exponent_of(v_power) : -126;
                int most = max(e, __shfl_xor(e, 16));
                most = max(most, __shfl_xor(most, 32));
                if (__ballot(most > v_most[fr]) != 0) {
                    const int grown = max(most, v_most[fr]);
                    const float down = exp2_fast((float)(v_most[fr] - grown));
#pragma unroll
                    for (int d = 0; d < ND; ++d) o[fr][d] *= down;
                    v_most[fr] = grown;
                }
                by = power_of(e - v_most[fr] + kRaised);
            }
            float score_by = to_log2, less = m[fr];
            if (__builtin_fabsf(less) >= kCoarse) {  // for those rows alone
#pragma unroll
                for (int f = 0; f < 4; ++f)
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[fr][f][r] = coarse_exponent(s[fr][f][r], to_log2, less);
                score_by = 1.0f;
                less = 0.0f;
            }
#pragma unroll
            for (int f = 0; f < 4; ++f)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float w = exp2_fast(fmaf(s[fr][f][r], score_by, -less));
                    l[fr] += w;
                    p[fr][f / 2][f % 2 * 4 + r] = (T)(W::kRelative ? w * by : w);
                }
        }
#pragma unroll
        for (int e = 0; e < ND; ++e) {
            const Eight a = W::codes(v[e].x, v[e].y, widen_by), b = W::codes(v[e].z, v[e].w, widen_by);
#pragma unroll
            for (int fr = 0; fr < F; ++fr) {
                o[fr][e] = W::mul16(a, p[fr][0], o[fr][e]);
                o[fr][e] = W::mul16(b, p[fr][1], o[fr][e]);
            }
        }
        here = v_next.there();
        load_scales(v_next);
        load_values(v_next);
        k_next = k_then;
        v_next = v_then;
    }

    if (poisoned) {  // such a value makes NaN of the rows that see it, and of no others
        for (t = first + (int)wave; t < end; t += NW) {
            const int key0 = range.tile(t) * kTile;
            look(t, k_next, v_next);
            here = v_next.there();
            if (!is_edge(x, key0, p_min, p_max) && __ballot(!here) == 0) continue;
            load_scales(v_next);
            load_values(v_next);
            const uint32_t lost = lost_codes<T>(cache_scale(v_scale));
#pragma unroll
            for (int fr = 0; fr < F; ++fr) {
                Eight seen[2];
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    seen[i / 8][i % 8] = (here & sees(x, pos[fr], from[fr], key0 + 16 * (int)g + i)) ? (T)1.0f : (T)0.0f;
#pragma unroll
                for (int e = 0; e < ND; ++e) {
                    float4x hits = {0, 0, 0, 0};
                    hits = W::mul16(W::codes(ones_at_lost(v[e].x, lost), ones_at_lost(v[e].y, lost), 1.0f), seen[0], hits);
                    hits = W::mul16(W::codes(ones_at_lost(v[e].z, lost), ones_at_lost(v[e].w, lost), 1.0f), seen[1], hits);
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[fr][e][r] = hits[r] > 0 ? __builtin_nanf("") : o[fr][e][r];
                }
            }
        }
    }

    // the waves' sums, to their common maximum
#pragma unroll
    for (int fr = 0; fr < F; ++fr) {
        l[fr] += __shfl_xor(l[fr], 16);
        l[fr] += __shfl_xor(l[fr], 32);
        if (g == 0) weights[wave][16 * fr + n] = float2{m[fr], l[fr]};
    }
    __syncthreads();
    float down[F];
#pragma unroll
    for (int fr = 0; fr < F; ++fr) {
        float most = kNothing;
#pragma unroll
        for (int w = 0; w < NW; ++w) most = fmaxf(most, weights[w][16 * fr + n].x);
        l[fr] = 0.0f;
#pragma unroll
        for (int w = 0; w < NW; ++w) l[fr] += exp2_fast(weights[w][16 * fr + n].x - most) * weights[w][16 * fr + n].y;
        down[fr] = exp2_fast(m[fr] - most);
        if constexpr (W::kRelative) down[fr] *= power_of(v_most[fr] - kRaised);
        m[fr] = most;
    }
    const bool whole = job.segments == 1;
    if (!whole && wave == 0 && g == 0) {
#pragma unroll
        for (int fr = 0; fr < F; ++fr) part_weights<R, DP>(x, job.part)[16 * fr + n] = float2{m[fr], l[fr]};
    }
#pragma unroll
    for (int e0 = 0; e0 < ND; e0 += CE) {
        if (16u * e0 >= dims) break;
        if (e0 > 0) __syncthreads();
#pragma unroll
        for (int fr = 0; fr < F; ++fr)
#pragma unroll
            for (int e = 0; e < CE; ++e)
                if (e0 + e < ND) sums[wave][fr][e][lane] = o[fr][e0 + e < ND ? e0 + e : 0] * down[fr];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < (F * CE + NW - 1) / NW; ++i) {
            const uint32_t at = i * NW + wave;  // uniform
            const uint32_t fr = at / CE, e = at % CE, d = 16 * (e0 + e) + 4 * g, row = 16 * fr + n;
            if (at >= F * CE || d >= dims || row >= rows) continue;
            float4x sum = sums[0][fr][e][lane];
#pragma unroll
            for (int w = 1; w < NW; ++w) sum += sums[w][fr][e][lane];
            if (!whole) {
                *(float4x*)(part_rows<R, DP>(x, job.part) + row * DP + d) = sum;
                continue;
            }
            float total = 0.0f;
#pragma unroll
            for (int k = 0; k < F; ++k) total = (uint32_t)k == fr ? l[k] : total;
            store_four(out_at<T>(x, job, row0 + row) + d, total == 0.0f ? float4x{0, 0, 0, 0} : sum / total);
        }
    }
}

// ---------------------------------------------------------------------------
// many rows: tiles of keys and values in LDS

constexpr int kManyRows = 128;  // of a workgroup: four waves of 32

// Where LDS has the chunk of 8 elements of a key's row, of CP of them: 16 lanes that read the same chunk of
// neighbouring rows find them in different banks (16 times 16 bytes before banks repeat).
template <int CP>
__device__ __forceinline__ uint32_t chunk_place(uint32_t row, uint32_t chunk) {
    return CP % 16 == 0 ? chunk ^ (row & 15) : CP % 8 == 0 ? chunk ^ (row >> 1 & 7) : chunk ^ (row >> 2 & 3);
}

// Lane (row n = lane % 32, half h = lane / 32) of a wave has the weights of the blocks h and 2 + h of a tile.  For
// that, fragment f of two has as its key m the token 4 (m / 8) + m % 4 of block 2 f + m / 4 % 2, and LDS holds the keys in
// that order.  Each of the four waves brings one of a tile's blocks and widens it once for all: LDS holds what the
// matrix unit reads, two tiles of keys and values (64 KB for 128 dimensions), so that two workgroups share a unit and one
// computes while the other waits.
template <typename T, int DP>
__global__ void __launch_bounds__(256, DP <= 128 ? 2 : 1) tile_attention(AttentionArgs x) {
    constexpr int R = kManyRows, NC = DP / 32, NO = DP / 32;
    constexpr int CP = DP / 8;  // chunks of 8 elements of a key
    constexpr int L = (DP + 63) / 64;  // loads of a lane, of its wave's block of keys, and of values
    using W = Wide<T>;
    using Eight = typename W::Eight;
    __shared__ Eight keys[2][64 * CP];
    __shared__ Eight vals[2][4 * 2 * DP];  // [block][its halves of 8 tokens][dimension]
    // a block's key scale in the softmax's exponents, or -1 where it is not in the cache, and its value scale
    __shared__ float2 scales[2][4];
    __shared__ int poisoned;  // whether a tile that some row does not see all of had a lost code among its values
    const Job job = find_job<R, false>(x, item_of_block());
    if (!job.found) return;
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t n = lane % 32, h = lane / 32, dims = x.cache.head_dim;
    const uint32_t rows_all = job.sequence.rows * x.share, row0 = job.row_tile * R, rows = min(rows_all - row0, (uint32_t)R);
    const uint32_t my_row0 = row0 + wave * 32;
    const bool idle = wave * 32 >= rows;  // a wave without rows loads and meets the others, no more
    const uint32_t my_rows = idle ? 1 : min(rows - wave * 32, 32u);

    Eight q[NC][2];
#pragma unroll
    for (int c = 0; c < NC; ++c) load_query<T>(x, job, my_row0 + n, row0 + rows, 32 * c + 16 * h, q[c]);
    const int base = job.sequence.position;
    const int pos = base + (int)divided(min(my_row0 + n, row0 + rows - 1), x.by_share);
    const int from = window_from(x, pos);
    const int p_min = uniform(base + (int)divided(min(my_row0, row0 + rows - 1), x.by_share));
    const int p_max = uniform(idle ? -1 : base + (int)divided(min(my_row0 + my_rows - 1, row0 + rows - 1), x.by_share));
    const int all_min = uniform(base + (int)divided(row0, x.by_share)), all_max = uniform(base + (int)divided(row0 + rows - 1, x.by_share));
    const Range range = range_of(x, all_min, all_max);
    const int first = (int)((int64_t)range.count * job.segment / job.segments);
    const int end = (int)((int64_t)range.count * (job.segment + 1) / job.segments);

    // Loads at an address that is the same for all lanes go by the vector unit all the same: one by the scalar unit
    // comes back out of order with LDS reads, which would all wait for it.
    uint32_t nothing = 0;
    asm volatile("" : "+v"(nothing));
    const int32_t* const table = x.batch.table + job.index * x.batch.ld_table + nothing;
    const float* const k_scales = x.cache.k_scales + nothing;
    const float* const v_scales = x.cache.v_scales + nothing;
    const uint8_t* const k_head = x.cache.k_codes + job.head * x.cache.k_head;
    const uint8_t* const v_head = x.cache.v_codes + job.head * x.cache.v_head;

    // what a lane brings of its wave's block: chunks of keys, and dimensions of values
    uint32_t k_from[L], k_to[L][2];
    bool k_there[L], v_there[L];
    uint4 k_in[L], v_in[L];  // zeros stay where no dimensions are
#pragma unroll
    for (int i = 0; i < L; ++i) {
        const uint32_t id = 64 * i + lane, token = id / (DP / 16), d = id % (DP / 16) * 16;
        const uint32_t row = 32 * (wave / 2) + token / 4 * 8 + wave % 2 * 4 + token % 4;
        k_there[i] = id < DP && d < dims;
        k_from[i] = token * dims + d;
#pragma unroll
        for (int e = 0; e < 2; ++e) k_to[i][e] = row * CP + chunk_place<CP>(row, d / 8 + e);
        v_there[i] = id < dims;
        k_in[i] = v_in[i] = uint4{0, 0, 0, 0};
    }
    float2 scale_in = {0, 0};
    // The wave's block of the next tile to be loaded: its page, negative for none, and its place there.  The table's
    // last column stands in for those behind it, so that nothing has to be decided before the load.
    int next_page = -1;
    uint32_t in_page = 0;
    bool listed = false;
    bool here = false;      // whether the block under way is in the cache
    const uint32_t last_block = (uint32_t)x.batch.capacity / kCacheBlock - 1;
    auto look = [&](int t) {
        const uint32_t block = (uint32_t)range.tile(t) * 4 + wave, inside = min(block, last_block);
        const uint32_t column = page_column(inside, x.cache.divide);
        listed = block == inside;
        in_page = inside - column * x.cache.page_blocks;
        next_page = table[column];
    };
    // Loads tile t - 1, whose place is known by now, and looks for that of tile t.
    auto load = [&](int t) {
        const uint32_t page = (uint32_t)uniform(next_page), in_page_now = in_page;
        here = listed & (page < x.cache.pages);
        if (t < end) look(t);
        if (!here) {  // its keys are not seen; no NaN stays among its values
#pragma unroll
            for (int i = 0; i < L; ++i) v_in[i] = uint4{0, 0, 0, 0};
            return;
        }
        const uint8_t* const k = k_head + page * x.cache.k_page + in_page_now * (16 * dims);
        const uint8_t* const v = v_head + page * x.cache.v_page + in_page_now * (16 * dims);
        const uint64_t at = ((uint64_t)page * x.cache.heads + job.head) * x.cache.page_blocks + in_page_now;
        scale_in = float2{k_scales[at], v_scales[at]};
#pragma unroll
        for (int i = 0; i < L; ++i)
            if (k_there[i]) k_in[i] = *(const uint4*)(k + k_from[i]);
#pragma unroll
        for (int i = 0; i < L; ++i)
            if (v_there[i]) v_in[i] = *(const uint4*)(v + (64 * i + lane) * 16);
    };
    auto hand_over = [&](int t) {
        const int stage = (t - first) & 1;
        if (is_edge(x, range.tile(t) * kTile, all_min, all_max)) {
            uint32_t any = 0;
            const uint32_t lost = lost_codes<T>(cache_scale(scale_in.y));
#pragma unroll
            for (int i = 0; i < L; ++i) any |= take_lost(v_in[i], lost);
            if (any != 0) poisoned = 1;
        }
        const float widen_by = W::kRelative ? 1.0f : cache_scale(scale_in.y);
#pragma unroll
        for (int i = 0; i < L; ++i) {
            if (64 * (i + 1) > DP && 64 * i + lane >= DP) break;
            keys[stage][k_to[i][0]] = W::codes(k_in[i].x, k_in[i].y, 1.0f);
            keys[stage][k_to[i][1]] = W::codes(k_in[i].z, k_in[i].w, 1.0f);
            vals[stage][(2 * wave) * DP + 64 * i + lane] = W::codes(v_in[i].x, v_in[i].y, widen_by);
            vals[stage][(2 * wave + 1) * DP + 64 * i + lane] = W::codes(v_in[i].z, v_in[i].w, widen_by);
        }
        if (lane == 0)
            scales[stage][wave] = float2{here ? fmaxf(cache_scale(scale_in.x) * x.scale, kLeastBy) : -1.0f,
                                         cache_scale(scale_in.y)};
    };

    float16x o[NO];
#pragma unroll
    for (int e = 0; e < NO; ++e)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[e][i] = 0.0f;
    float m = kNothing, l = 0.0f;
    int v_most = -126;

    // One tile for the wave's rows.
    auto step = [&](int stage, int key0) {
        const float2 scale[2] = {scales[stage][h], scales[stage][2 + h]};
        const bool edge = is_edge(x, key0, p_min, p_max) || __ballot(fminf(scale[0].x, scale[1].x) < 0.0f) != 0;
        const float to_log2[2] = {__builtin_fabsf(scale[0].x), __builtin_fabsf(scale[1].x)};
        float16x s[2];
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[f][i] = 0.0f;
        Eight k[2 * NC][2];
#pragma unroll
        for (int c = 0; c < 2 * NC; ++c)
#pragma unroll
            for (int f = 0; f < 2; ++f)
                k[c][f] = keys[stage][(32 * f + n) * CP + chunk_place<CP>(n, 4 * (c / 2) + 2 * h + c % 2)];
#pragma unroll
        for (int c = 0; c < 2 * NC; ++c)
#pragma unroll
            for (int f = 0; f < 2; ++f) s[f] = W::mul32(k[c][f], q[c / 2][c % 2], s[f]);
        // eight reads ahead of the products, which the compiler would make two at a time
        constexpr int kAhead = std::min(8, 4 * NC);
        __builtin_amdgcn_sched_group_barrier(kDsRead, kAhead, 0);
#pragma unroll
        for (int i = 0; i < (4 * NC - kAhead) / 2; ++i) {
            __builtin_amdgcn_sched_group_barrier(kMatrix, 2, 0);
            __builtin_amdgcn_sched_group_barrier(kDsRead, 2, 0);
        }
        __builtin_amdgcn_sched_group_barrier(kMatrix, kAhead, 0);
        Eight v[2][NO];  // of the half block at work, and the next one
        auto read_values = [&](int i) {  // half a of the wave's block f, i = 2 f + a
#pragma unroll
            for (int e = 0; e < NO; ++e) v[i % 2][e] = vals[stage][(4 * (i / 2) + 2 * h + i % 2) * DP + 32 * e + n];
        };
        read_values(0);
        if (edge) {
            asm volatile("");  // a branch: the comparisons are not made for other tiles
#pragma unroll
            for (int f = 0; f < 2; ++f)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    s[f][i] = ((scale[f].x > 0.0f) & sees(x, pos, from, key0 + 32 * f + 16 * (int)h + i)) ? s[f][i] : -__builtin_inff();
        }
        float top[2];
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            top[f] = s[f][0];
#pragma unroll
            for (int i = 1; i < 16; ++i) top[f] = fmaxf(top[f], s[f][i]);
        }
        float most = fmaxf(top[0] * to_log2[0], top[1] * to_log2[1]);
        most = fmaxf(most, __shfl_xor(most, 32));
        if (__ballot(most > m + kLazy) != 0) {  // for those rows: no row's rounding depends on another
            const float grown = most > m + kLazy ? most : m, down = exp2_fast(m - grown);
            m = grown;
            l *= down;
#pragma unroll
            for (int e = 0; e < NO; ++e) o[e] *= down;
        }
        float raise[2] = {1.0f, 1.0f};  // by the values' scales, relative to the largest that the row has met
        if constexpr (W::kRelative) {
            int e[2];
#pragma unroll
            for (int f = 0; f < 2; ++f) {
                const bool counts = scale[f].x > 0.0f && block_seen(x, key0 + 32 * f + 16 * (int)h, pos);
                e[f] = counts ? exponent_of(scale[f].y) : -126;
            }
            int largest = max(e[0], e[1]);
            largest = max(largest, __shfl_xor(largest, 32));
            if (__ballot(largest > v_most) != 0) {
                const int grown = max(largest, v_most);
                const float by = exp2_fast((float)(v_most - grown));
#pragma unroll
                for (int d = 0; d < NO; ++d) o[d] *= by;
                v_most = grown;
            }
#pragma unroll
            for (int f = 0; f < 2; ++f) raise[f] = power_of(e[f] - v_most + kRaised);
        }
        float score_by[2] = {to_log2[0], to_log2[1]}, less = m;
        if (__builtin_fabsf(less) >= kCoarse) {  // for those rows alone
#pragma unroll
            for (int f = 0; f < 2; ++f) {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[f][i] = coarse_exponent(s[f][i], to_log2[f], less);
                score_by[f] = 1.0f;
            }
            less = 0.0f;
        }
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            Eight p[2];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float w = exp2_fast(fmaf(s[f][i], score_by[f], -less));
                if constexpr (W::kRelative) {
                    l += w;
                    w *= raise[f];
                }
                p[i / 8][i % 8] = (T)w;
            }
#pragma unroll
            for (int a = 0; a < 2; ++a) {
                if (2 * f + a < 3) read_values(2 * f + a + 1);
                if constexpr (!W::kRelative) l = W::add(p[a], l);
#pragma unroll
                for (int e = 0; e < NO; ++e) o[e] = W::mul32(v[a][e], p[a], o[e]);
            }
        }
    };

    if (threadIdx.x == 0) poisoned = 0;
    __syncthreads();
    if (first < end) {
        look(first);
        load(first + 1);
        hand_over(first);
    }
    // The queries have arrived, as far as the compiler knows too: it would wait for them within the loop, and by that
    // for the tile that was asked for last.
    __builtin_amdgcn_s_waitcnt(kWaitAll);
    __syncthreads();
    for (int t = first; t < end; ++t) {
        const int key0 = range.tile(t) * kTile;
        if (t + 1 < end) load(t + 2);
        if (key0 <= p_max) step((t - first) & 1, key0);
        if (t + 1 < end) hand_over(t + 1);
        __syncthreads();
    }
    if (poisoned && !idle) {  // such a value makes NaN of the rows that see it, and of no others
        const Places places(x, job.index);
        for (int t = first; t < end; ++t) {
            const int key0 = range.tile(t) * kTile;
            if (!is_edge(x, key0, all_min, all_max)) continue;
            for (int f = 0; f < 2; ++f) {
                const Places::Block place = places.of((uint32_t)key0 / kCacheBlock + 2 * f + h);
                const bool here = place.there();
                Eight seen[2];
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    seen[i / 8][i % 8] = (here & sees(x, pos, from, key0 + 32 * f + 16 * (int)h + i)) ? (T)1.0f : (T)0.0f;
                const uint8_t* const block = v_head + (here ? place.page * x.cache.v_page + place.block * (16 * dims) : 0);
                const uint64_t at = ((uint64_t)place.page * x.cache.heads + job.head) * x.cache.page_blocks + place.block;
                const uint32_t lost = lost_codes<T>(cache_scale(here ? x.cache.v_scales[at] : 1.0f));
#pragma unroll
                for (int e = 0; e < NO; ++e) {
                    uint4 w = {0, 0, 0, 0};
                    if (here && 32 * e + n < dims) w = *(const uint4*)(block + 16 * (32 * e + n));
                    float16x hits;
#pragma unroll
                    for (int i = 0; i < 16; ++i) hits[i] = 0.0f;
                    hits = W::mul32(W::codes(ones_at_lost(w.x, lost), ones_at_lost(w.y, lost), 1.0f), seen[0], hits);
                    hits = W::mul32(W::codes(ones_at_lost(w.z, lost), ones_at_lost(w.w, lost), 1.0f), seen[1], hits);
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[e][i] = hits[i] > 0 ? __builtin_nanf("") : o[e][i];
                }
            }
        }
    }

    l += __shfl_xor(l, 32);
    if constexpr (W::kRelative) {
#pragma unroll
        for (int e = 0; e < NO; ++e) o[e] *= power_of(v_most - kRaised);
    }
    if (idle || n >= my_rows) return;
    const uint32_t row = wave * 32 + n;
    if (job.segments > 1 && h == 0) part_weights<R, DP>(x, job.part)[row] = float2{m, l};
    const float inverse = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int e = 0; e < NO; ++e)
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            const uint32_t d = 32 * e + 8 * a + 4 * h;
            if (d >= dims) continue;
            const float4x four = {o[e][4 * a], o[e][4 * a + 1], o[e][4 * a + 2], o[e][4 * a + 3]};
            if (job.segments > 1)
                *(float4x*)(part_rows<R, DP>(x, job.part) + row * DP + d) = four;
            else
                store_four(out_at<T>(x, job, row0 + row) + d, l == 0.0f ? float4x{0, 0, 0, 0} : four * inverse);
        }
}

// ---------------------------------------------------------------------------
// the parts' sums joined, in order: workgroups of 16 rows of each unit that is cut

template <typename T, int DP, int R>
__device__ __forceinline__ void join_row(const AttentionArgs& x, const Job& job, uint32_t row, uint32_t d) {
    const float2* const weights = part_weights<R, DP>(x, job.part) + row;
    const float* const from = part_rows<R, DP>(x, job.part) + row * DP + d;
    // Eight parts at a time are on their way; the maximum of those so far scales the sums, as in a segment.
    constexpr uint32_t kStep = 8;
    float most = kNothing, total = 0.0f;
    float4x sum = {0, 0, 0, 0};
    for (uint32_t i = 0; i < job.segments; i += kStep) {
        float2 w[kStep];
        float4x part[kStep];
#pragma unroll
        for (uint32_t k = 0; k < kStep; ++k) {
            const uint32_t at = min(i + k, job.segments - 1);
            w[k] = weights[at * R];
            part[k] = *(const float4x*)(from + (uint64_t)at * R * DP);
            if (i + k >= job.segments) w[k] = float2{kNothing, 0.0f};
        }
        float top = most;
#pragma unroll
        for (uint32_t k = 0; k < kStep; ++k) top = fmaxf(top, w[k].x);
        const float down = exp2_fast(most - top);
        total *= down;
        sum *= down;
        most = top;
#pragma unroll
        for (uint32_t k = 0; k < kStep; ++k) {
            const float up = i + k < job.segments ? exp2_fast(w[k].x - top) : 0.0f;
            total += up * w[k].y;
            sum += i + k < job.segments ? up * part[k] : float4x{0, 0, 0, 0};
        }
    }
    store_four(out_at<T>(x, job, job.row_tile * R + row) + d, total == 0.0f ? float4x{0, 0, 0, 0} : sum / total);
}

template <typename T, int DP, int R>
__global__ void __launch_bounds__(16 * (DP / 4)) join_attention(AttentionArgs x) {
    constexpr uint32_t kLanes = DP / 4;
    const Job job = find_job<R, true>(x, blockIdx.x);
    if (!job.found) return;
    const uint32_t rows = min(job.sequence.rows * x.share - job.row_tile * R, (uint32_t)R);
    const uint32_t d = threadIdx.x % kLanes * 4;
    if (d >= x.cache.head_dim) return;
    for (uint32_t row = blockIdx.y * 16 + threadIdx.x / kLanes; row < rows; row += gridDim.y * 16)
        join_row<T, DP, R>(x, job, row, d);
}

 // ---------------------------------------------------------------------------
// launches

template <typename T, int DP, int R, typename Main>
hipError_t run(const AttentionArgs& a, const AttentionPlan& plan, uint32_t threads, Main main, hipStream_t s) {
    main<<<item_grid(plan.jobs), threads, 0, s>>>(a);
    if (plan.join == 0) return hipGetLastError();
    // where there are many units few of them are cut
    join_attention<T, DP, R><<<dim3(plan.join, plan.join >= 256 ? 1 : R / 16), 16 * (DP / 4), 0, s>>>(a);
    return hipGetLastError();
}

template <typename T, int DP>
hipError_t launch(const AttentionArgs& a, const AttentionPlan& plan, hipStream_t s) {
    // Eight waves as long as they have the registers; with 256 of them a lane (8 sequences of 8000 tokens): 16 rows of 256
    // dimensions took 153 us by eight waves and 54 by four, 32 of 128 45 and 33.
    constexpr int NW = DP <= 128 ? 8 : 4, NW2 = DP <= 64 ? 8 : 4;
    switch (plan.rows) {
        case 16: return run<T, DP, 16>(a, plan, NW * 64, stream_attention<T, DP, 1, NW>, s);
        case 32: return run<T, DP, 32>(a, plan, NW2 * 64, stream_attention<T, DP, 2, NW2>, s);
        default: return run<T, DP, kManyRows>(a, plan, 256, tile_attention<T, DP>, s);
    }
}

template <typename T>
hipError_t launch(const AttentionArgs& a, const AttentionPlan& plan, hipStream_t s) {
    switch (plan.dims) {
        case 64: return launch<T, 64>(a, plan, s);
        case 96: return run<T, 96, kManyRows>(a, plan, 256, tile_attention<T, 96>, s);
        case 128: return launch<T, 128>(a, plan, s);
        case 192: return launch<T, 192>(a, plan, s);
        default: return launch<T, 256>(a, plan, s);
    }
}

}  // namespace

AttentionPlan fp8_attention_plan(uint64_t sequences, uint64_t capacity, uint64_t tokens, uint64_t heads, uint64_t kv_heads,
                                 uint64_t head_dim, uint64_t window, uint64_t sinks) {
    AttentionPlan plan = {};
    plan.dims = (uint32_t)((head_dim + 63) / 64 * 64);
    const uint64_t share = heads / kv_heads;
    const uint64_t rows = (tokens + sequences - 1) / sequences * share;  // of a sequence, on the average
    // (8 sequences of 8000 tokens, 64 rows of 128 dimensions: straight from memory 79 us, by tiles 46; 32 rows 33 and 41)
    plan.rows = rows <= 16 ? 16 : rows <= 32 ? 32 : kManyRows;
    if (plan.rows == kManyRows && head_dim > 64 && head_dim <= 96) plan.dims = 96;  // products and LDS of three quarters
    const uint64_t units = kv_heads * (tokens * share / plan.rows + std::min(sequences, tokens));
    // tiles that one row tile may see at most
    const uint64_t reach = window == 0 ? capacity : std::min(capacity, window + sinks + tokens + 2 * kTile);
    const uint64_t tiles = (reach + kTile - 1) / kTile;
    plan.least = 4;
    // Up to 1536 tokens a workgroup's eight waves take three tiles each, which costs less than the join's launch.  Shares:
    // as many as run at a time, one workgroup a unit of few rows (131072 tokens: 256 shares 56 us, 512 65, 1024 84; 64
    // sequences 136, 140, 137), two of many (777 tokens after 30,000 with a window of 4095: 256 63 us, 512 55, 1024 63).
    // At least four tiles (one sequence of 2000 tokens: 13.2 us, at least eight 14.3, sixteen 15.7).
    plan.log2_slots = tiles <= 24 ? 0 : plan.rows == kManyRows ? 9 : 8;
    const uint32_t slots = plan.log2_slots ? 1u << plan.log2_slots : 0;
    plan.jobs = (uint32_t)(units + 2 * slots);
    plan.join = (uint32_t)std::min<uint64_t>(units, slots);
    plan.parts = 2 * slots;
    plan.workspace = (uint64_t)plan.parts * plan.rows * (plan.dims + 2) * sizeof(float);
    return plan;
}

hipError_t launch_fp8_attention(int type, AttentionArgs a, const AttentionPlan& plan, hipStream_t s) {
    a.log2_slots = plan.log2_slots;
    a.by_share = divider(a.share);
    a.by_heads = divider(a.cache.heads);
    a.least = plan.least;
    a.parts_limit = plan.parts;
    return type == kTypeBf16 ? launch<__bf16>(a, plan, s) : launch<_Float16>(a, plan, s);
}

}  // namespace hv
