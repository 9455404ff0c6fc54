// hv_fp8_cache.cpp -- C ABI of the 8-bit cache and the attention over it: argument checks and launches.
#include "hv_fp8_cache.h"

#include <algorithm>
#include <cfloat>
#include <cmath>

#include "fp8_host.h"

using namespace hvh;

namespace {

constexpr uint64_t kMaxPages = ((uint64_t)1 << 31) - 1, kMaxHeads = 65535, kMaxPageTokens = 65536;
constexpr uint64_t kMaxCount = 65536, kMaxCapacity = (uint64_t)1 << 30, kMaxRows = (uint64_t)1 << 30;
constexpr uint64_t kMaxStride = (uint64_t)1 << 40;
static_assert(HV_FP8_CACHE_BLOCK == 16, "the kernels' block");

#define HV_LIMIT(what, value, limit)                                                                             \
    do {                                                                                                         \
        if ((value) > (limit))                                                                                   \
            return fail(HV_ERR_INVALID_ARG, "%s = %llu exceeds the limit of %llu", what, (unsigned long long)(value), \
                        (unsigned long long)(limit));                                                            \
    } while (0)

hv_status check_head_dim(uint64_t head_dim) {
    if (head_dim < 16 || head_dim > 256 || head_dim % 16 != 0)
        return fail(HV_ERR_INVALID_ARG, "head_dim = %llu is no multiple of 16 from 16 to 256", (unsigned long long)head_dim);
    return HV_OK;
}

// Whether `outer` things, each of `inner` things of `size`, lie apart by these strides without overlap, all of them
// within what can be addressed.
bool nested(uint64_t size, uint64_t inner, uint64_t inner_stride, uint64_t outer, uint64_t outer_stride) {
    using Wide = unsigned __int128;
    const Wide span = (Wide)(inner - 1) * inner_stride + size;
    return (inner <= 1 || inner_stride >= size) && (outer <= 1 || outer_stride >= span) &&
           (Wide)(outer - 1) * outer_stride + span <= (Wide)1 << 62;
}

// Pages and heads of `bytes` bytes each, apart by the two strides: one nested in the other.
hv_status check_places(const char* what, uint64_t bytes, uint64_t pages, uint64_t page, uint64_t heads, uint64_t head) {
    if (page % 16 != 0 || head % 16 != 0)
        return fail(HV_ERR_INVALID_ARG, "%s: pages or heads are not a multiple of 16 bytes apart", what);
    HV_LIMIT(what, page, kMaxStride);
    HV_LIMIT(what, head, kMaxStride);
    if (!nested(bytes, heads, head, pages, page) && !nested(bytes, pages, page, heads, head))
        return fail(HV_ERR_INVALID_ARG, "%s: pages or heads overlap (%llu and %llu bytes apart, %llu each)", what,
                    (unsigned long long)page, (unsigned long long)head, (unsigned long long)bytes);
    return HV_OK;
}

hv_status check_cache(const hv_fp8_cache* c) {
    if (c == nullptr) return fail(HV_ERR_INVALID_ARG, "cache is NULL");
    HV_LIMIT("pages", c->pages, kMaxPages);
    if (c->kv_heads == 0) return fail(HV_ERR_INVALID_ARG, "kv_heads is 0");
    HV_LIMIT("kv_heads", c->kv_heads, kMaxHeads);
    if (c->page_tokens == 0 || c->page_tokens % 16 != 0 || c->page_tokens > kMaxPageTokens)
        return fail(HV_ERR_INVALID_ARG, "page_tokens = %llu is no multiple of 16 from 16 to 65536",
                    (unsigned long long)c->page_tokens);
    HV_TRY(check_head_dim(c->head_dim));
    if (c->pages == 0) return HV_OK;  // nothing of it is read or written
    HV_TRY(check_pointer("k_codes", c->k_codes, 16));
    HV_TRY(check_pointer("v_codes", c->v_codes, 16));
    HV_TRY(check_pointer("k_scales", c->k_scales, sizeof(float)));
    HV_TRY(check_pointer("v_scales", c->v_scales, sizeof(float)));
    const uint64_t bytes = c->page_tokens * c->head_dim;
    HV_TRY(check_places("k_codes", bytes, c->pages, c->k_page, c->kv_heads, c->k_head));
    return check_places("v_codes", bytes, c->pages, c->v_page, c->kv_heads, c->v_head);
}

hv_status check_batch(const hv_fp8_batch* b, uint64_t page_tokens) {
    if (b == nullptr) return fail(HV_ERR_INVALID_ARG, "batch is NULL");
    HV_LIMIT("sequences", b->count, kMaxCount);
    HV_LIMIT("columns", b->columns, kMaxCapacity);
    HV_LIMIT("columns * page_tokens", b->columns * page_tokens, kMaxCapacity);
    if (b->count == 0) return HV_OK;
    HV_TRY(check_pointer("starts", b->starts, sizeof(int32_t)));
    HV_TRY(check_pointer("lengths", b->lengths, sizeof(int32_t)));
    if (b->columns == 0) return HV_OK;
    HV_TRY(check_pointer("pages", b->pages, sizeof(int32_t)));
    if (b->ld_pages < b->columns && b->count > 1)
        return fail(HV_ERR_INVALID_ARG, "ld_pages = %llu is below the table's %llu columns", (unsigned long long)b->ld_pages,
                    (unsigned long long)b->columns);
    HV_LIMIT("ld_pages", b->ld_pages, kMaxStride);
    return HV_OK;
}

// [tokens][heads][dim] with the dimensions adjacent: tokens and heads nested either way.
hv_status check_rows(const char* what, const void* p, size_t element, uint64_t tokens, uint64_t token, uint64_t heads,
                     uint64_t head, uint64_t dim) {
    HV_TRY(check_pointer(what, p, element));
    HV_LIMIT(what, token, kMaxStride);
    HV_LIMIT(what, head, kMaxStride);
    if (!nested(dim, heads, head, tokens, token) && !nested(dim, tokens, token, heads, head))
        return fail(HV_ERR_INVALID_ARG, "%s: rows overlap (tokens %llu and heads %llu elements apart, %llu each)", what,
                    (unsigned long long)token, (unsigned long long)head, (unsigned long long)dim);
    return HV_OK;
}

hv_status check_attention(uint64_t sequences, uint64_t capacity, uint64_t tokens, uint64_t heads, uint64_t kv_heads,
                          uint64_t head_dim) {
    HV_LIMIT("sequences", sequences, kMaxCount);
    HV_LIMIT("capacity", capacity, kMaxCapacity);
    HV_LIMIT("kv_heads", kv_heads, kMaxHeads);
    HV_TRY(check_head_dim(head_dim));
    if (kv_heads == 0 || heads == 0 || heads % kv_heads != 0)
        return fail(HV_ERR_INVALID_ARG, "heads = %llu is no multiple of the %llu key heads", (unsigned long long)heads,
                    (unsigned long long)kv_heads);
    HV_LIMIT("heads", heads, kMaxRows);
    HV_LIMIT("tokens * heads", tokens, kMaxRows / heads);
    return HV_OK;
}

hv::CacheArgs cache_args(const hv_fp8_cache& c) {
    const uint64_t blocks = c.page_tokens / 16;
    return {c.k_codes, c.k_scales, c.v_codes, c.v_scales, c.k_page, c.k_head, c.v_page, c.v_head,
            (uint32_t)c.pages, (uint32_t)c.kv_heads, (uint32_t)blocks, (uint32_t)c.head_dim,
            (((uint64_t)1 << 38) + blocks - 1) / blocks};
}

hv::BatchArgs batch_args(const hv_fp8_batch& b, uint64_t page_tokens, uint64_t tokens) {
    return {b.starts, b.lengths, b.pages, b.ld_pages, (uint32_t)b.count, (int32_t)(b.columns * page_tokens),
            (int32_t)tokens};
}

}  // namespace

extern "C" {

hv_status hv_fp8_cache_write(const hv_fp8_cache* cache, const hv_fp8_batch* batch, hv_type type, const void* k,
                             uint64_t k_token, uint64_t k_head, const void* v, uint64_t v_token, uint64_t v_head,
                             uint64_t tokens, hipStream_t stream) {
    HV_TRY(check_type(type));
    HV_TRY(check_cache(cache));
    HV_TRY(check_batch(batch, cache->page_tokens));
    HV_LIMIT("tokens * heads", tokens, kMaxRows / cache->kv_heads);
    if (tokens == 0 || batch->count == 0 || batch->columns == 0 || cache->pages == 0) return HV_OK;
    HV_TRY(check_rows("k", k, size_of(type), tokens, k_token, cache->kv_heads, k_head, cache->head_dim));
    HV_TRY(check_rows("v", v, size_of(type), tokens, v_token, cache->kv_heads, v_head, cache->head_dim));
    const hv::WriteArgs args = {cache_args(*cache), batch_args(*batch, cache->page_tokens, tokens), k, k_token, k_head, v,
                                v_token, v_head};
    return done(hv::launch_fp8_cache_write(type, args, stream), "cache write kernel");
}

size_t hv_fp8_attention_workspace_bytes(uint64_t sequences, uint64_t capacity, uint64_t tokens, uint64_t heads,
                                        uint64_t kv_heads, uint64_t head_dim, uint32_t window, uint32_t sinks) {
    if (sequences == 0 || capacity == 0 || tokens == 0 ||
        check_attention(sequences, capacity, tokens, heads, kv_heads, head_dim) != HV_OK)
        return 0;
    return round_up(hv::fp8_attention_plan(sequences, capacity, tokens, heads, kv_heads, head_dim, window, sinks).workspace);
}

hv_status hv_fp8_attention(const hv_fp8_cache* cache, const hv_fp8_batch* batch, hv_type type, const void* q,
                           uint64_t q_token, uint64_t q_head, uint64_t tokens, uint64_t heads, float scale,
                           uint32_t window, uint32_t sinks, void* out, uint64_t out_token, uint64_t out_head,
                           void* workspace, size_t workspace_bytes, hipStream_t stream) {
    if (type != HV_BF16 && type != HV_F16)
        return fail(HV_ERR_INVALID_ARG, "element type %d is neither HV_BF16 nor HV_F16", (int)type);
    HV_TRY(check_cache(cache));
    HV_TRY(check_batch(batch, cache->page_tokens));
    const uint64_t capacity = batch->columns * cache->page_tokens;
    HV_TRY(check_attention(batch->count, capacity, tokens, heads, cache->kv_heads, cache->head_dim));
    const float log2_scale = scale * 1.44269504088896341f;
    if (!(scale > 0.0f) || !std::isfinite(log2_scale) || log2_scale < FLT_MIN)
        return fail(HV_ERR_INVALID_ARG, "scale = %g is not positive and finite", (double)scale);
    if (tokens == 0 || batch->count == 0) return HV_OK;
    HV_TRY(check_rows("q", q, 2, tokens, q_token, heads, q_head, cache->head_dim));
    HV_TRY(check_rows("out", out, 2, tokens, out_token, heads, out_head, cache->head_dim));
    const hv::AttentionPlan plan = hv::fp8_attention_plan(batch->count, capacity, tokens, heads, cache->kv_heads,
                                                          cache->head_dim, window, sinks);
    HV_TRY(check_workspace(workspace, workspace_bytes, round_up(plan.workspace)));
    // Positions are below 2^31, so a longer window leaves nothing out; those that the table has, below kMaxCapacity.
    const bool windowed = window < 1u << 31;
    hv::AttentionArgs args = {};
    args.cache = cache_args(*cache);
    args.batch = batch_args(*batch, cache->page_tokens, tokens);
    args.q = q, args.q_token = q_token, args.q_head = q_head;
    args.out = out, args.out_token = out_token, args.out_head = out_head;
    args.share = (uint32_t)(heads / cache->kv_heads);
    args.scale = log2_scale;
    args.window = windowed ? (int)window : 0;
    args.sinks = (int)std::min<uint64_t>(sinks, kMaxCapacity);
    args.parts = static_cast<float*>(workspace);
    return done(hv::launch_fp8_attention(type, args, plan, stream), "attention kernels");
}

}  // extern "C"
