// What the kernels of the key-value cache and of attention share.
//
// The cache is paged: [pages][KV heads][page_size][head_dim] for k and for v, so that the tokens of a page and head are
// one contiguous piece, which is what a wavefront of decode attention reads.  16 bits a value, or a code of 8 or 4 bits with a
// bf16 scale and offset for each (token, KV head) of k and of v: value = scale * code + offset.  scales holds the four of a token
// and head side by side (k scale, k offset, v scale, v offset; 8 bytes), one load for whoever needs them.
#pragma once
#include "any4.h"
#include "any4_device.h"
#include <type_traits>

namespace any4 {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// The cache as a kernel sees it.
struct KvPages {
    uint8_t* k;
    uint8_t* v;
    uint16_t* scales;         // 16 bits: NULL
    int64_t slots;            // pages * page_size
    int pages, page_shift, kv_heads;
    // bytes of the tokens of one page and head, and where (page, head) starts: ((page * kv_heads + head) << page_shift) tokens
    __device__ __forceinline__ int64_t first_token(int page, int head) const { return ((int64_t)page * kv_heads + head) << page_shift; }
};

inline KvPages kv_pages(const any4_kv_cache& c) {
    KvPages p{static_cast<uint8_t*>(c.k), static_cast<uint8_t*>(c.v), c.scales, c.pages * c.page_size, (int)c.pages, 0, c.kv_heads};
    while ((1 << p.page_shift) < c.page_size) ++p.page_shift;
    return p;
}

// largest / smallest over the 16 (or 8) lanes of a head's vector; every lane gets it
template <int LANES, class F> __device__ __forceinline__ float lanes_reduce(float v, F f) {
    v = f(v, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0xB1 /*quad_perm 1 0 3 2*/, 0xF, 0xF, false)));
    v = f(v, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x4E /*quad_perm 2 3 0 1*/, 0xF, 0xF, false)));
    v = f(v, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x141 /*row_half_mirror*/, 0xF, 0xF, false)));
    if constexpr (LANES == 16) v = f(v, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x140 /*row_mirror*/, 0xF, 0xF, false)));
    return v;
}

// each lane gets the sum of the lanes up to its own
__device__ __forceinline__ int lanes_scan(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111 /*row_shr:1*/, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x112 /*row_shr:2*/, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114 /*row_shr:4*/, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118 /*row_shr:8*/, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142 /*row_bcast:15*/, 0xA, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x143 /*row_bcast:31*/, 0xC, 0xF, false);
    return v;
}

// Strides in values: from a token (or request) to the next, from a head to the next.  A head's values lie side by side.
struct Rows {
    const uint16_t* p;
    int64_t token, head;
};

// Matrix instructions in the two 16-bit types.  Operand lane l of 16x16x32: row (A) or column (B) l % 16, the 8 values 8 * (l / 16) ..
// along k; result lane l: column l % 16, rows 4 * (l / 16) + register.  Of 32x32x16: row or column l % 32, values 8 * (l / 32) ..;
// result: column l % 32, rows 8 * (register / 4) + 4 * (l / 32) + register % 4.
template <bool F16> __device__ __forceinline__ f32x4 mma16(const u32x4& a, const u32x4& b, const f32x4& c) {
    if constexpr (F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
template <bool F16> __device__ __forceinline__ f32x16 mma32(const u32x4& a, const u32x4& b, const f32x16& c) {
    if constexpr (F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
constexpr float kLog2e = 1.44269504088896340736f;

hipError_t launch_kv_write(const Rows& k, const Rows& v, int64_t tokens, const int64_t* slots, const any4_kv_cache& c, hipStream_t stream);
hipError_t launch_kv_read(const any4_kv_cache& c, const int64_t* slots, int64_t tokens, uint16_t* k, uint16_t* v, hipStream_t stream);

// Rows of q, k and v (without a cache no v) and where the turned ones go.
struct RopeArgs {
    Rows q, k, v;
    uint16_t *q_out, *k_out;
    int64_t qo_token, qo_head, ko_token, ko_head;
    int64_t tokens;
    const int64_t* slots;
    int heads, kv_heads, head_dim;
    bool f16;
};
hipError_t launch_rope(const RopeArgs& r, const any4_rotation& turn, const any4_kv_cache* c, int cus, hipStream_t stream);

// How a decode call is shared out.
struct DecodePlan {
    int shared, head_tiles;   // query heads of a KV head, and in how many parts of at most 16
    int at_once;              // requests of a launch
    int waves, blocks, cus;   // wavefronts of a block, most blocks, compute units
    size_t words_bytes, workspace;      // arrival words, and all with the pieces' results
};
DecodePlan plan_attn_decode(int64_t requests, int heads, int kv_heads, int head_dim, int64_t max_tokens, int cus);
hipError_t launch_attn_decode(const Rows& q, const any4_kv_cache& c, const int32_t* table, int64_t table_stride, int64_t table_width,
                              const int32_t* lengths, int64_t requests, int heads, int window, int sinks, float softmax_scale, uint16_t* out,
                              const DecodePlan& pl, void* workspace, hipStream_t stream);          // window 0: all tokens are seen

// Packed prompts: rows of q, k and v, where each request's rows start.
struct PromptArgs {
    Rows q, k, v;
    int64_t q_tokens, k_tokens;
    const int32_t* q_starts;
    const int32_t* k_starts;
    int requests, heads, kv_heads, head_dim;
    bool f16, causal;
    float softmax_scale;
    uint16_t* out;
};
constexpr int kPromptRows = 128;          // queries of a block
// a tile of each request may be short; blocks that no request has end at once
inline int64_t prompt_blocks(int64_t q_tokens, int64_t requests, int heads) {
    return (q_tokens / kPromptRows + (requests < q_tokens ? requests : q_tokens)) * heads;
}
hipError_t launch_attn_prompt(const PromptArgs& a, hipStream_t stream);

// The newest tokens of requests over the cache, or packed prompts over packed keys (k, v, k_starts; no cache), with or without a window.
struct ChunkArgs {
    Rows q, k, v;
    int64_t q_tokens, k_tokens;
    const int32_t* q_starts;
    const int32_t* k_starts;
    const int32_t* table;
    int64_t table_stride, table_width;
    const int32_t* lengths;
    int requests, heads, kv_heads, head_dim, window, sinks;      // window 0: all tokens are seen
    bool f16;
    float softmax_scale;
    uint16_t* out;
};
// How a call is shared out: blocks (some have nothing to do), how many of them would fill the chip (0: no keys are cut into pieces), pieces that
// the workspace has room for, tiles of rows that may be cut.
struct ChunkPlan {
    int64_t blocks;
    int target, slots, cut_tiles;
    bool small;               // whether it may be one that takes 32 rows at a time
    size_t plan_bytes, workspace;      // of these in front: what a first launch finds out for more than 64 requests
};
ChunkPlan plan_attn_chunk(int64_t requests, int64_t q_tokens, int heads, int kv_heads, int head_dim, int64_t max_tokens, bool cut, int cus);
hipError_t launch_attn_chunk(const ChunkArgs& a, const any4_kv_cache* cache, const ChunkPlan& pl, void* workspace, hipStream_t stream);

}  // namespace any4
