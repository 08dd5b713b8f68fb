// C ABI of the key-value cache and of attention (see include/any4.h): argument validation, plans, launches.
#include "any4_attn.h"
#include "any4_internal.h"

using namespace any4;

namespace {

bool aligned(const void* p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
bool aligned16(const void* p) { return aligned(p, 16); }
bool strides_ok(int64_t token, int64_t head) { return token >= 0 && head >= 0; }
bool strides_aligned(int64_t token, int64_t head) { return token % 8 == 0 && head % 8 == 0; }
bool scale_ok(float s) { return s > 0.0f && s < __builtin_inff(); }
constexpr int64_t kMaxStride = (int64_t)1 << 23;             // any4_attn_prompt: 64 rows' offsets in 32 bits
constexpr int kMaxKvHeads = 4095, kMaxHeads = 65535;
constexpr int64_t kMaxRequests = 65535, kMaxTokens = 0x7FFFFFFF - 2047;
constexpr int64_t kMaxChunkRequests = (int64_t)1 << 29;      // any4_attn_chunk: what a first launch finds out, four words a request, has 32-bit places

// the units of work of one request are counted in 32 bits
bool tokens_ok(int64_t max_tokens, int heads, int kv_heads) {
    return max_tokens >= 1 && max_tokens <= kMaxTokens && (max_tokens / 128 + 1) * kv_heads * ((heads / kv_heads + 15) / 16) <= 0x7FFFFFFF;
}
bool heads_ok(int heads, int kv_heads) {
    return kv_heads >= 1 && kv_heads <= kMaxKvHeads && heads >= 1 && heads <= kMaxHeads && heads % kv_heads == 0;
}

// the rows of a call (queries of the heads that share a KV head) are counted in 32 bits
bool rows_ok(int64_t q_tokens, int heads, int kv_heads) { return q_tokens * (heads / kv_heads) <= kMaxTokens; }

int cache_check(const any4_kv_cache* c) {
    if (!c || !c->k || !c->v) return ANY4_ERR_NULL;
    if (c->bits != 16 && c->bits != 8 && c->bits != 4) return ANY4_ERR_BITS;
    if (c->bits != 16 && !c->scales) return ANY4_ERR_NULL;
    if (c->pages < 1 || c->pages > 0x7FFFFFFF || c->kv_heads < 1 || c->kv_heads > kMaxKvHeads) return ANY4_ERR_SHAPE;
    if (c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1))) return ANY4_ERR_SHAPE;
    if (c->head_dim != 64 && c->head_dim != 128) return ANY4_ERR_SHAPE;
    if (!aligned16(c->k) || !aligned16(c->v) || (c->bits != 16 && !aligned16(c->scales))) return ANY4_ERR_ALIGN;
    return ANY4_OK;
}

int rotation_check(const any4_rotation* r, int head_dim) {
    if (!r || !r->positions || !r->freqs) return ANY4_ERR_NULL;
    if (r->axes < 1 || r->axes > 4 || r->axis_stride < 0 || r->rotary_dim < 8 || r->rotary_dim % 8 || r->rotary_dim > head_dim || !(r->eps >= 0.0f) ||
        !(r->eps < __builtin_inff()))
        return ANY4_ERR_SHAPE;
    if (!aligned(r->positions, 8) || !aligned(r->freqs, 8) || !aligned16(r->q_norm) || !aligned16(r->k_norm)) return ANY4_ERR_ALIGN;
    return ANY4_OK;
}

int launched(hipError_t e) { return e == hipSuccess ? ANY4_OK : ANY4_ERR_HIP; }

// more tokens than a request may have are as good as all
int at_most(int64_t tokens) { return (int)(tokens < kMaxTokens ? tokens : kMaxTokens); }

int decode(const uint16_t* q, int64_t q_request_stride, int64_t q_head_stride, const any4_kv_cache* cache, const int32_t* page_table,
           int64_t table_stride, int64_t table_width, const int32_t* lengths, int64_t requests, int heads, int window, int sinks, float softmax_scale,
           uint16_t* out, void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = cache_check(cache)) return rc;
    if (requests < 0 || requests > kMaxRequests || !heads_ok(heads, cache->kv_heads) || !scale_ok(softmax_scale) ||
        !strides_ok(q_request_stride, q_head_stride) || table_width < 1 || table_width > kMaxTokens / cache->page_size || table_stride < 0 ||
        !tokens_ok(table_width * cache->page_size, heads, cache->kv_heads))
        return ANY4_ERR_SHAPE;
    if (requests == 0) return ANY4_OK;
    if (!q || !page_table || !lengths || !out) return ANY4_ERR_NULL;
    if (!aligned16(q) || !aligned(page_table, 4) || !aligned(lengths, 4) || !aligned16(out) || !aligned16(workspace) ||
        !strides_aligned(q_request_stride, q_head_stride))
        return ANY4_ERR_ALIGN;
    const DecodePlan pl = plan_attn_decode(requests, heads, cache->kv_heads, cache->head_dim, table_width * cache->page_size, device_compute_units());
    if (pl.workspace > 0 && (!workspace || workspace_bytes < pl.workspace)) return ANY4_ERR_WORKSPACE;
    return launched(launch_attn_decode({q, q_request_stride, q_head_stride}, *cache, page_table, table_stride, table_width, lengths, requests, heads,
                                       window, sinks, softmax_scale, out, pl, workspace, static_cast<hipStream_t>(stream)));
}

}  // namespace

extern "C" {

int any4_kv_write(const uint16_t* k, int64_t k_token_stride, int64_t k_head_stride, const uint16_t* v, int64_t v_token_stride,
                  int64_t v_head_stride, int64_t tokens, const int64_t* slots, const any4_kv_cache* cache, void* stream) {
    if (int rc = cache_check(cache)) return rc;
    if (tokens < 0 || tokens > kMaxTokens || !strides_ok(k_token_stride, k_head_stride) || !strides_ok(v_token_stride, v_head_stride))
        return ANY4_ERR_SHAPE;
    if (tokens == 0) return ANY4_OK;
    if (!k || !v || !slots) return ANY4_ERR_NULL;
    if (!aligned16(k) || !aligned16(v) || !aligned(slots, 8) || !strides_aligned(k_token_stride, k_head_stride) ||
        !strides_aligned(v_token_stride, v_head_stride))
        return ANY4_ERR_ALIGN;
    return launched(launch_kv_write({k, k_token_stride, k_head_stride}, {v, v_token_stride, v_head_stride}, tokens, slots, *cache,
                                    static_cast<hipStream_t>(stream)));
}

int any4_kv_read(const any4_kv_cache* cache, const int64_t* slots, int64_t tokens, uint16_t* k, uint16_t* v, void* stream) {
    if (int rc = cache_check(cache)) return rc;
    if (tokens < 0 || tokens > kMaxTokens) return ANY4_ERR_SHAPE;
    if (tokens == 0) return ANY4_OK;
    if (!k || !v || !slots) return ANY4_ERR_NULL;
    if (!aligned16(k) || !aligned16(v) || !aligned(slots, 8)) return ANY4_ERR_ALIGN;
    return launched(launch_kv_read(*cache, slots, tokens, k, v, static_cast<hipStream_t>(stream)));
}

int any4_rope(const uint16_t* q, int64_t q_token_stride, int64_t q_head_stride, const uint16_t* k, int64_t k_token_stride, int64_t k_head_stride,
              int64_t tokens, int heads, int kv_heads, int head_dim, int f16, const any4_rotation* turn, uint16_t* q_out, int64_t q_out_token_stride,
              int64_t q_out_head_stride, uint16_t* k_out, int64_t k_out_token_stride, int64_t k_out_head_stride, void* stream) {
    if (tokens < 0 || tokens > kMaxTokens || heads < 1 || heads > kMaxHeads || kv_heads < 1 || kv_heads > kMaxKvHeads || (head_dim != 64 && head_dim != 128) ||
        !strides_ok(q_token_stride, q_head_stride) || !strides_ok(k_token_stride, k_head_stride) || !strides_ok(q_out_token_stride, q_out_head_stride) ||
        !strides_ok(k_out_token_stride, k_out_head_stride))
        return ANY4_ERR_SHAPE;
    if (tokens == 0) return ANY4_OK;
    if (int rc = rotation_check(turn, head_dim)) return rc;
    if (!q || !k || !q_out || !k_out) return ANY4_ERR_NULL;
    if (!aligned16(q) || !aligned16(k) || !aligned16(q_out) || !aligned16(k_out) || !strides_aligned(q_token_stride, q_head_stride) ||
        !strides_aligned(k_token_stride, k_head_stride) || !strides_aligned(q_out_token_stride, q_out_head_stride) ||
        !strides_aligned(k_out_token_stride, k_out_head_stride))
        return ANY4_ERR_ALIGN;
    const RopeArgs r{{q, q_token_stride, q_head_stride}, {k, k_token_stride, k_head_stride}, {nullptr, 0, 0}, q_out, k_out, q_out_token_stride, q_out_head_stride,
                     k_out_token_stride, k_out_head_stride, tokens, nullptr, heads, kv_heads, head_dim, f16 != 0};
    return launched(launch_rope(r, *turn, nullptr, device_compute_units(), static_cast<hipStream_t>(stream)));
}

int any4_rope_kv_write(const uint16_t* q, int64_t q_token_stride, int64_t q_head_stride, const uint16_t* k, int64_t k_token_stride, int64_t k_head_stride,
                       const uint16_t* v, int64_t v_token_stride, int64_t v_head_stride, int64_t tokens, int heads, const any4_rotation* turn,
                       const int64_t* slots, const any4_kv_cache* cache, uint16_t* q_out, int64_t q_out_token_stride, int64_t q_out_head_stride,
                       uint16_t* k_out, int64_t k_out_token_stride, int64_t k_out_head_stride, void* stream) {
    if (int rc = cache_check(cache)) return rc;
    if (tokens < 0 || tokens > kMaxTokens || heads < 1 || heads > kMaxHeads || !strides_ok(q_token_stride, q_head_stride) ||
        !strides_ok(k_token_stride, k_head_stride) || !strides_ok(v_token_stride, v_head_stride) || !strides_ok(q_out_token_stride, q_out_head_stride) ||
        (k_out && !strides_ok(k_out_token_stride, k_out_head_stride)))
        return ANY4_ERR_SHAPE;
    if (tokens == 0) return ANY4_OK;
    if (int rc = rotation_check(turn, cache->head_dim)) return rc;
    if (!q || !k || !v || !slots || !q_out) return ANY4_ERR_NULL;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out) || !aligned16(k_out) || !aligned(slots, 8) ||
        !strides_aligned(q_token_stride, q_head_stride) || !strides_aligned(k_token_stride, k_head_stride) || !strides_aligned(v_token_stride, v_head_stride) ||
        !strides_aligned(q_out_token_stride, q_out_head_stride) || (k_out && !strides_aligned(k_out_token_stride, k_out_head_stride)))
        return ANY4_ERR_ALIGN;
    const RopeArgs r{{q, q_token_stride, q_head_stride}, {k, k_token_stride, k_head_stride}, {v, v_token_stride, v_head_stride}, q_out, k_out,
                     q_out_token_stride, q_out_head_stride, k_out_token_stride, k_out_head_stride, tokens, slots, heads, cache->kv_heads, cache->head_dim,
                     cache->f16 != 0};
    return launched(launch_rope(r, *turn, cache, device_compute_units(), static_cast<hipStream_t>(stream)));
}

size_t any4_attn_decode_workspace_bytes(int64_t requests, int heads, int kv_heads, int head_dim, int64_t max_tokens) {
    if (requests < 1 || requests > kMaxRequests || !heads_ok(heads, kv_heads) || (head_dim != 64 && head_dim != 128) ||
        !tokens_ok(max_tokens, heads, kv_heads))
        return 0;
    return plan_attn_decode(requests, heads, kv_heads, head_dim, max_tokens, device_compute_units()).workspace;
}

int any4_attn_decode(const uint16_t* q, int64_t q_request_stride, int64_t q_head_stride, const any4_kv_cache* cache,
                     const int32_t* page_table, int64_t table_stride, int64_t table_width, const int32_t* lengths, int64_t requests,
                     int heads, float softmax_scale, uint16_t* out, void* workspace, size_t workspace_bytes, void* stream) {
    return decode(q, q_request_stride, q_head_stride, cache, page_table, table_stride, table_width, lengths, requests, heads, 0, 0, softmax_scale, out,
                  workspace, workspace_bytes, stream);
}

int any4_attn_decode_window(const uint16_t* q, int64_t q_request_stride, int64_t q_head_stride, const any4_kv_cache* cache,
                            const int32_t* page_table, int64_t table_stride, int64_t table_width, const int32_t* lengths, int64_t requests,
                            int heads, int64_t window, int64_t sinks, float softmax_scale, uint16_t* out, void* workspace, size_t workspace_bytes,
                            void* stream) {
    if (window < 1 || sinks < 0) return cache_check(cache) ? cache_check(cache) : ANY4_ERR_SHAPE;
    return decode(q, q_request_stride, q_head_stride, cache, page_table, table_stride, table_width, lengths, requests, heads, at_most(window),
                  at_most(sinks), softmax_scale, out, workspace, workspace_bytes, stream);
}

int any4_attn_prompt(const uint16_t* q, int64_t q_token_stride, int64_t q_head_stride, const uint16_t* k, int64_t k_token_stride,
                     int64_t k_head_stride, const uint16_t* v, int64_t v_token_stride, int64_t v_head_stride, int64_t q_tokens,
                     int64_t k_tokens, const int32_t* q_starts, const int32_t* k_starts, int64_t requests, int heads, int kv_heads,
                     int head_dim, int f16, int causal, float softmax_scale, uint16_t* out, void* stream) {
    if (requests < 0 || requests > kMaxTokens || q_tokens < 0 || q_tokens > kMaxTokens || k_tokens < 0 || k_tokens > kMaxTokens ||
        !heads_ok(heads, kv_heads) || (head_dim != 64 && head_dim != 128) || !scale_ok(softmax_scale) ||
        !strides_ok(q_token_stride, q_head_stride) || !strides_ok(k_token_stride, k_head_stride) || !strides_ok(v_token_stride, v_head_stride) ||
        k_token_stride >= kMaxStride || v_token_stride >= kMaxStride)
        return ANY4_ERR_SHAPE;
    if (prompt_blocks(q_tokens, requests, heads) > 0x7FFFFFFF) return ANY4_ERR_SHAPE;
    if (requests == 0 || q_tokens == 0) return ANY4_OK;
    // (without a single key k and v are not read)
    if (!q || !q_starts || !k_starts || !out || (k_tokens > 0 && (!k || !v))) return ANY4_ERR_NULL;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned(q_starts, 4) || !aligned(k_starts, 4) || !aligned16(out) ||
        !strides_aligned(q_token_stride, q_head_stride) || !strides_aligned(k_token_stride, k_head_stride) ||
        !strides_aligned(v_token_stride, v_head_stride))
        return ANY4_ERR_ALIGN;
    const PromptArgs a{{q, q_token_stride, q_head_stride}, {k, k_token_stride, k_head_stride}, {v, v_token_stride, v_head_stride},
                       q_tokens, k_tokens, q_starts, k_starts, (int)requests, heads, kv_heads, head_dim, f16 != 0, causal != 0, softmax_scale, out};
    return launched(launch_attn_prompt(a, static_cast<hipStream_t>(stream)));
}

int any4_attn_prompt_window(const uint16_t* q, int64_t q_token_stride, int64_t q_head_stride, const uint16_t* k, int64_t k_token_stride,
                            int64_t k_head_stride, const uint16_t* v, int64_t v_token_stride, int64_t v_head_stride, int64_t q_tokens,
                            int64_t k_tokens, const int32_t* q_starts, const int32_t* k_starts, int64_t requests, int heads, int kv_heads,
                            int head_dim, int f16, int64_t window, int64_t sinks, float softmax_scale, uint16_t* out, void* stream) {
    if (requests < 0 || requests > kMaxTokens || q_tokens < 0 || q_tokens > kMaxTokens || k_tokens < 0 || k_tokens > kMaxTokens ||
        !heads_ok(heads, kv_heads) || (head_dim != 64 && head_dim != 128) || !scale_ok(softmax_scale) || window < 1 || sinks < 0 ||
        !strides_ok(q_token_stride, q_head_stride) || !strides_ok(k_token_stride, k_head_stride) || !strides_ok(v_token_stride, v_head_stride) ||
        k_token_stride >= kMaxStride || v_token_stride >= kMaxStride || !rows_ok(q_tokens, heads, kv_heads))
        return ANY4_ERR_SHAPE;
    const ChunkPlan pl = plan_attn_chunk(requests, q_tokens, heads, kv_heads, head_dim, k_tokens, false, device_compute_units());
    if (pl.blocks > 0x7FFFFFFF) return ANY4_ERR_SHAPE;
    if (requests == 0 || q_tokens == 0) return ANY4_OK;
    // (without a single key k and v are not read)
    if (!q || !q_starts || !k_starts || !out || (k_tokens > 0 && (!k || !v))) return ANY4_ERR_NULL;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned(q_starts, 4) || !aligned(k_starts, 4) || !aligned16(out) ||
        !strides_aligned(q_token_stride, q_head_stride) || !strides_aligned(k_token_stride, k_head_stride) ||
        !strides_aligned(v_token_stride, v_head_stride))
        return ANY4_ERR_ALIGN;
    const ChunkArgs a{{q, q_token_stride, q_head_stride}, {k, k_token_stride, k_head_stride}, {v, v_token_stride, v_head_stride}, q_tokens, k_tokens, q_starts,
                      k_starts, nullptr, 0, 0, nullptr, (int)requests, heads, kv_heads, head_dim, at_most(window), at_most(sinks), f16 != 0, softmax_scale, out};
    return launched(launch_attn_chunk(a, nullptr, pl, nullptr, static_cast<hipStream_t>(stream)));
}

size_t any4_attn_chunk_workspace_bytes(int64_t requests, int64_t q_tokens, int heads, int kv_heads, int head_dim, int64_t max_tokens) {
    if (requests < 1 || requests > kMaxChunkRequests || q_tokens < 1 || q_tokens > kMaxTokens || !heads_ok(heads, kv_heads) || (head_dim != 64 && head_dim != 128) ||
        max_tokens < 1 || max_tokens > kMaxTokens || !rows_ok(q_tokens, heads, kv_heads))
        return 0;
    return plan_attn_chunk(requests, q_tokens, heads, kv_heads, head_dim, max_tokens, true, device_compute_units()).workspace;
}

int any4_attn_chunk(const uint16_t* q, int64_t q_token_stride, int64_t q_head_stride, const any4_kv_cache* cache, const int32_t* page_table,
                    int64_t table_stride, int64_t table_width, const int32_t* q_starts, const int32_t* lengths, int64_t q_tokens, int64_t requests,
                    int heads, int64_t window, int64_t sinks, float softmax_scale, uint16_t* out, void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = cache_check(cache)) return rc;
    if (requests < 0 || requests > kMaxChunkRequests || q_tokens < 0 || q_tokens > kMaxTokens || !heads_ok(heads, cache->kv_heads) || !scale_ok(softmax_scale) ||
        !strides_ok(q_token_stride, q_head_stride) || table_width < 1 || table_width > kMaxTokens / cache->page_size || table_stride < 0 || window < 0 ||
        sinks < 0 || !rows_ok(q_tokens, heads, cache->kv_heads))
        return ANY4_ERR_SHAPE;
    const ChunkPlan pl = plan_attn_chunk(requests, q_tokens, heads, cache->kv_heads, cache->head_dim, table_width * cache->page_size, true, device_compute_units());
    if (pl.blocks > 0x7FFFFFFF) return ANY4_ERR_SHAPE;
    if (requests == 0 || q_tokens == 0) return ANY4_OK;
    if (!q || !page_table || !q_starts || !lengths || !out) return ANY4_ERR_NULL;
    if (!aligned16(q) || !aligned(page_table, 4) || !aligned(q_starts, 4) || !aligned(lengths, 4) || !aligned16(out) || !aligned16(workspace) ||
        !strides_aligned(q_token_stride, q_head_stride))
        return ANY4_ERR_ALIGN;
    if (pl.workspace > 0 && (!workspace || workspace_bytes < pl.workspace)) return ANY4_ERR_WORKSPACE;
    const ChunkArgs a{{q, q_token_stride, q_head_stride}, {nullptr, 0, 0}, {nullptr, 0, 0}, q_tokens, 0, q_starts, nullptr, page_table, table_stride, table_width,
                      lengths, (int)requests, heads, cache->kv_heads, cache->head_dim, at_most(window), at_most(sinks), cache->f16 != 0, softmax_scale, out};
    return launched(launch_attn_chunk(a, cache, pl, workspace, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
