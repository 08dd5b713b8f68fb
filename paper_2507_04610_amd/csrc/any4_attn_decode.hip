// any4_attn_decode: one new token for each request attends to its tokens in the paged cache.
//
// For a KV head and the up to 16 query heads that share it, tokens j:
//     s_j = scale q . k_j,   o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),   m = max_j s_j
// in one pass over the cache with a running maximum.  The cache is read once, and that bounds the operator: a few
// floating-point operations for each byte at up to 16 heads.  Everything else is arranged so that no byte takes a detour.
//
// A wavefront takes 32 tokens a step, for all heads of the KV head.  S^T = K Q^T with v_mfma_f32_16x16x32, k's rows as the A
// operand straight from memory (lane: token l % 16, 8 values along the head); the scores of a head then lie in the 4 lanes l % 16 =
// head, 8 tokens in each, and that is already the B operand of O^T = V^T P^T over 32 tokens, the tokens of lane l / 16 = g being
// 4 g .. 4 g + 3 of either 16.  V^T's lanes hold 8 tokens of one place along the head, which 8 loads of D / 16 places each give after
// half a v_perm a value: no LDS, no exchange between lanes but a head's maximum.
//
// Codes c of 8 or 4 bits go to the matrix cores as 16-bit floats that hold them exactly (c + kBias: 1024 + c in fp16 and 128 + c in
// bf16 take two bits set in place; c itself for 8 bits in bf16), scale and offset are applied to sums:
//     q . k_j = ks_j (q . c'_j - kBias sum(q)) + ko_j sum(q)
//     o = sum_j (p_j vs_j) (c_j - kCentre) + sum_j p_j (vo_j + kCentre vs_j)
// where the first sum has p_j vs_j rounded to 16 bits and is taken as sum(.. c'_j) - (kBias + kCentre) sum(..) with the same
// rounded weights, so that their rounding meets values around 0 as it does without codes.
//
// Rounding: scores, maxima, sums and accumulators are fp32; p (times vs) is rounded to 16 bits for the matrix cores, once.
#include "any4_attn.h"
#include "any4_internal.h"
#include "any4_splitk.h"

namespace any4 {

namespace {

constexpr int kWaves = 8, kThreads = 64 * kWaves, kStep = 32;

struct DecodeArgs {
    Rows q;
    KvPages c;
    const int32_t* table;
    int64_t table_stride;
    int table_width;
    const int32_t* lengths;
    int heads, shared, head_tiles;
    float scale_log2;                  // softmax scale * log2(e)
    uint16_t* out;
    int splits, chunk;
    float* partial;                    // [request][KV head][head tile][split][query head][D + 2]: sums, then maximum and sum of weights
    uint8_t* words;
};

template <int N> __device__ __forceinline__ void load_words(const uint8_t* p, uint32_t (&w)[N]) {
    if constexpr (N >= 4) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const u32x4 x = reinterpret_cast<const u32x4*>(p)[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[4 * i + j] = x[j];
        }
    } else if constexpr (N == 2) {
        const u32x2 x = *reinterpret_cast<const u32x2*>(p);
        w[0] = x[0];
        w[1] = x[1];
    } else {
        w[0] = *reinterpret_cast<const uint32_t*>(p);
    }
}

__device__ __forceinline__ float ubyte(uint32_t w, int j) { return (float)((w >> (8 * j)) & 0xFFu); }
// high halves of two fp32 values: their bf16 where nothing is lost
__device__ __forceinline__ uint32_t high_halves(float lo, float hi) {
    return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}

template <int BITS, bool F16> struct Codes {
    static constexpr int kBias = BITS == 16 ? 0 : F16 ? 1024 : BITS == 4 ? 128 : 0;
    static constexpr int kCentre = BITS == 16 ? 0 : 1 << (BITS - 1);
    static constexpr uint32_t kMagic = F16 ? 0x64006400u : 0x43004300u;
};

// A operand of S^T from a token's words: matrix instruction i
template <int BITS, bool F16, int N> __device__ __forceinline__ u32x4 k_operand(const uint32_t (&w)[N], int i) {
    using C = Codes<BITS, F16>;
    if constexpr (BITS == 16) return u32x4{w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
    if constexpr (BITS == 8 && F16) {
        return u32x4{__builtin_amdgcn_perm(0x64646464u, w[2 * i], 0x04010400u), __builtin_amdgcn_perm(0x64646464u, w[2 * i], 0x04030402u),
                     __builtin_amdgcn_perm(0x64646464u, w[2 * i + 1], 0x04010400u), __builtin_amdgcn_perm(0x64646464u, w[2 * i + 1], 0x04030402u)};
    }
    if constexpr (BITS == 8 && !F16) {
        const uint32_t a = w[2 * i], b = w[2 * i + 1];
        return u32x4{high_halves(ubyte(a, 0), ubyte(a, 1)), high_halves(ubyte(a, 2), ubyte(a, 3)), high_halves(ubyte(b, 0), ubyte(b, 1)),
                     high_halves(ubyte(b, 2), ubyte(b, 3))};
    }
    if constexpr (BITS == 4) {
        const uint32_t a = w[i];                               // pairs (code x, code x + 4)
        return u32x4{(a & 0x000F000Fu) | C::kMagic, ((a >> 4) & 0x000F000Fu) | C::kMagic, ((a >> 8) & 0x000F000Fu) | C::kMagic,
                     ((a >> 12) & 0x000F000Fu) | C::kMagic};
    }
}

// two tokens' values of place m, the first in the low half
template <int BITS, bool F16, int N> __device__ __forceinline__ uint32_t v_pair(const uint32_t (&a)[N], const uint32_t (&b)[N], int m) {
    using C = Codes<BITS, F16>;
    if constexpr (BITS == 16) return __builtin_amdgcn_perm(b[m >> 1], a[m >> 1], m & 1 ? 0x07060302u : 0x05040100u);
    if constexpr (BITS == 8 && F16) {
        const uint32_t sel = 0x0C000C00u | (uint32_t)(4 + (m & 3)) << 16 | (uint32_t)(m & 3);
        return __builtin_amdgcn_perm(b[m >> 2], a[m >> 2], sel) | C::kMagic;
    }
    if constexpr (BITS == 8 && !F16) return high_halves(ubyte(a[m >> 2], m & 3), ubyte(b[m >> 2], m & 3));
    if constexpr (BITS == 4) {
        const uint32_t w = __builtin_amdgcn_perm(b[0], a[0], m < 4 ? 0x05040100u : 0x07060302u);
        return ((w >> (4 * (m & 3))) & 0x000F000Fu) | C::kMagic;
    }
}

// over the four lanes that hold a head's tokens
template <class F> __device__ __forceinline__ float head_reduce(float v, F f) {
    v = f(v, __shfl_xor(v, 16));
    return f(v, __shfl_xor(v, 32));
}

template <int BITS, int D, bool F16>
__global__ __launch_bounds__(kThreads) void attn_decode_kernel(DecodeArgs a) {
    using C = Codes<BITS, F16>;
    constexpr int KM = D / 32, VM = D / 16;                     // matrix instructions of S^T (16 tokens) and of O^T (32 tokens)
    constexpr int ROW = D * BITS / 8;                           // bytes of a token
    constexpr int KW = D * BITS / 128;                          // words of a lane: k of one token
    constexpr int VB = VM * BITS / 8, VW = VB < 4 ? 1 : VB / 4; // bytes and words of a lane: v of one token
    constexpr bool QUANT = BITS != 16;
    extern __shared__ float lds[];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int split = blockIdx.x, request = blockIdx.z;
    const int kv_head = a.head_tiles == 1 ? (int)blockIdx.y : (int)blockIdx.y / a.head_tiles;
    const int head_tile = (int)blockIdx.y - kv_head * a.head_tiles;
    const int first_head = kv_head * a.shared + head_tile * 16, here = min(16, a.shared - head_tile * 16);

    int len = max(a.lengths[request], 0);
    if ((int64_t)len > (int64_t)a.table_width << a.c.page_shift) len = (int)((int64_t)a.table_width << a.c.page_shift);
    const int active = max(1, (int)(((int64_t)len + a.chunk - 1) / a.chunk));
    if (split >= active) return;
    const int t0 = split * a.chunk, t1 = (int)min((int64_t)len, (int64_t)t0 + a.chunk);
    const int32_t* table = a.table + (int64_t)request * a.table_stride;

    // Q^T, columns past `here` are zeros
    u32x4 q[KM];
    float sum_q = 0.0f;
    {
        const uint16_t* qp = a.q.p + (int64_t)request * a.q.token + (int64_t)(first_head + min(col, here - 1)) * a.q.head;
#pragma unroll
        for (int i = 0; i < KM; ++i) {
            q[i] = *reinterpret_cast<const u32x4*>(qp + (QUANT ? (D / 4) * g + 8 * i : 32 * i + 8 * g));
            if (col >= here) q[i] = u32x4{0u, 0u, 0u, 0u};
            if constexpr (QUANT) {
#pragma unroll
                for (int j = 0; j < 4; ++j) sum_q += h16lo_to_f32<F16>(q[i][j]) + h16hi_to_f32<F16>(q[i][j]);
            }
            if constexpr (BITS == 4) {                          // pairs (x, x + 4), as the codes come
                const u32x4 r = q[i];
                q[i] = u32x4{__builtin_amdgcn_perm(r[2], r[0], 0x05040100u), __builtin_amdgcn_perm(r[2], r[0], 0x07060302u),
                             __builtin_amdgcn_perm(r[3], r[1], 0x05040100u), __builtin_amdgcn_perm(r[3], r[1], 0x07060302u)};
            }
        }
    }
    if constexpr (QUANT) sum_q = head_reduce(sum_q, [](float x, float y) { return x + y; }) * a.scale_log2;

    float m_ref = -__builtin_inff(), l = 0.0f, vo_sum = 0.0f;
    f32x4 o[VM], ones_sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int m = 0; m < VM; ++m) o[m] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    // fp16 weights p * vs: held as p * (vs * 2^-exponent), with the largest vs so far between 1 and 2, or small scales would leave fp16's range
    int exponent = -126;

    const int page_mask = (1 << a.c.page_shift) - 1;
    for (int t = t0 + kStep * wave; t < t1; t += kStep * kWaves) {
        // tokens of the two 16s that exist; a page that does not has none
        int there[2];
        int64_t tok[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int th = t + 16 * h < len ? t + 16 * h : t;
            const int page = __builtin_amdgcn_readfirstlane(table[th >> a.c.page_shift]);
            const bool ok = page >= 0 && page < a.c.pages;
            there[h] = ok ? min(max(len - (t + 16 * h), 0), 16) : 0;
            tok[h] = a.c.first_token(ok ? page : 0, kv_head) + (th & page_mask);
        }
        uint32_t kw[2][KW], vw[8][VW];
        u32x4 so[2][2 * 2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint8_t* kp = a.c.k + tok[h] * ROW;
            if constexpr (BITS == 16) {
#pragma unroll
                for (int i = 0; i < KM; ++i) {
                    const u32x4 x = *reinterpret_cast<const u32x4*>(kp + col * ROW + 64 * i + 16 * g);
#pragma unroll
                    for (int j = 0; j < 4; ++j) kw[h][4 * i + j] = x[j];
                }
            } else {
                load_words(kp + col * ROW + (ROW / 4) * g, kw[h]);
                const u32x4* sp = reinterpret_cast<const u32x4*>(a.c.scales + tok[h] * 4) + 2 * g;
                so[h][0] = sp[0];
                so[h][1] = sp[1];
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint8_t* vp = a.c.v + tok[j >> 2] * ROW + (4 * g + (j & 3)) * ROW + VB * col;
            if constexpr (VB == 2) vw[j][0] = *reinterpret_cast<const uint16_t*>(vp);
            else load_words(vp, vw[j]);
        }

        f32x4 s[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            s[h] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < KM; ++i) s[h] = mma16<F16>(k_operand<BITS, F16>(kw[h], i), q[i], s[h]);
        }
        float x[8], vs[8], vo[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int h = j >> 2, r = j & 3;
            if constexpr (QUANT) {
                const uint32_t kk = so[h][r >> 1][2 * (r & 1)], vv = so[h][r >> 1][2 * (r & 1) + 1];
                const float u = fmaf(s[h][r], a.scale_log2, -(float)C::kBias * sum_q);
                x[j] = fmaf(bf16lo_to_f32(kk), u, bf16hi_to_f32(kk) * sum_q);
                vs[j] = bf16lo_to_f32(vv);
                vo[j] = fmaf((float)C::kCentre, vs[j], bf16hi_to_f32(vv));
            } else {
                x[j] = s[h][r] * a.scale_log2;
            }
        }
        if (there[0] + there[1] < 32) {
            // what lies behind the last token, or in a page that does not exist, may be anything: none of it comes near a sum
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool ok = 4 * g + (j & 3) < there[j >> 2];
                x[j] = ok ? x[j] : -__builtin_inff();
                if constexpr (QUANT) {
                    vs[j] = ok ? vs[j] : 0.0f;
                    vo[j] = ok ? vo[j] : 0.0f;
                } else {
#pragma unroll
                    for (int w = 0; w < VW; ++w) vw[j][w] = ok ? vw[j][w] : 0u;
                }
            }
        }

        float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
        top = head_reduce(top, [](float u, float v) { return fmaxf(u, v); });
        float factor = 1.0f;
        bool moved = top > m_ref;
        if constexpr (QUANT && F16) {
            float big = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) big = fmaxf(big, fabsf(vs[j]));
            big = head_reduce(big, [](float u, float v) { return fmaxf(u, v); });
            const int e = min(max((int)(__float_as_uint(big) >> 23) - 127, -126), 126);
            if (e > exponent) {
                factor = __builtin_ldexpf(1.0f, max(exponent - e, -126));
                exponent = e;
                moved = true;
            }
        }
        if (__builtin_amdgcn_ballot_w64(moved)) {
            const float m_new = fmaxf(m_ref, top);
            const float alpha = m_new > m_ref ? exp2_fast(m_ref - m_new) : 1.0f;
            m_ref = m_new;
            l *= alpha;
            vo_sum *= alpha;
            const float f = alpha * factor;
            ones_sum *= f;
#pragma unroll
            for (int m = 0; m < VM; ++m) o[m] *= f;
        }
        const float m_use = m_ref == -__builtin_inff() ? 0.0f : m_ref;
        const float unit = __builtin_ldexpf(1.0f, -exponent);
        u32x4 p;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x[j] = exp2_fast(x[j] - m_use);
            l += x[j];
            if constexpr (QUANT) {
                vo_sum = fmaf(x[j], vo[j], vo_sum);
                x[j] *= F16 ? vs[j] * unit : vs[j];
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) p[j] = f32x2_to_h16x2<F16>(x[2 * j], x[2 * j + 1]);
        if constexpr (QUANT) {
            constexpr uint32_t kOnes = F16 ? 0x3C003C00u : 0x3F803F80u;
            ones_sum = mma16<F16>(u32x4{kOnes, kOnes, kOnes, kOnes}, p, ones_sum);
        }
#pragma unroll
        for (int m = 0; m < VM; ++m) {
            u32x4 v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = v_pair<BITS, F16>(vw[2 * j], vw[2 * j + 1], m);
            o[m] = mma16<F16>(v, p, o[m]);
        }
    }

    // The wavefronts' results meet in LDS: [wave][head][D], then [wave][head] maximum and sum of weights.
    auto add = [](float u, float v) { return u + v; };
    l = head_reduce(l, add);
    if constexpr (QUANT) vo_sum = head_reduce(vo_sum, add);
    float* ml = lds + kWaves * here * D;
    if (col < here) {
        const float back = QUANT && F16 ? __builtin_ldexpf(1.0f, exponent) : 1.0f;
        float* to = lds + (wave * here + col) * D;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int m = 0; m < VM; ++m) {
                float v = o[m][r];
                if constexpr (QUANT) v = fmaf(back, v - (float)(C::kBias + C::kCentre) * ones_sum[0], vo_sum);
                to[VM * (4 * g + r) + m] = v;
            }
        if (g == 0) {
            ml[2 * (wave * here + col)] = m_ref;
            ml[2 * (wave * here + col) + 1] = l;
        }
    }
    __syncthreads();
    const int64_t pair = ((int64_t)request * gridDim.y + blockIdx.y);
    uint16_t* out = a.out + ((int64_t)request * a.heads + first_head) * D;
    const int room = min(16, a.shared) * (D + 2);               // of a piece (the last head tile may have fewer heads)
    float* mine = a.partial + (pair * a.splits + split) * room;
    for (int i = threadIdx.x; i < here * D; i += kThreads) {
        const int n = i / D;
        float top = -__builtin_inff();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, ml[2 * (w * here + n)]);
        const float use = top == -__builtin_inff() ? 0.0f : top;
        float sum = 0.0f, v = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float f = exp2_fast(ml[2 * (w * here + n)] - use);
            sum = fmaf(f, ml[2 * (w * here + n) + 1], sum);
            v = fmaf(f, lds[w * here * D + i], v);
        }
        if (active == 1) {
            out[i] = (uint16_t)f32_to_h16<F16>(sum == 0.0f ? 0.0f : v / sum);
        } else {
            splitk_store(mine + i, v);
            if (i - n * D < 2) splitk_store(mine + here * D + 2 * n + (i - n * D), i == n * D ? top : sum);
        }
    }
    if (active == 1) return;

    // The last piece of a request and head to come adds all of them, in their order.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    int* last = reinterpret_cast<int*>(lds);
    if (threadIdx.x == 0) *last = arrive_one(reinterpret_cast<unsigned long long*>(a.words + pair * kWordBytes), active);
    __syncthreads();
    const bool joins = *last != 0;
    __syncthreads();
    if (!joins) return;
    const float* all = a.partial + pair * a.splits * room;
    for (int i = threadIdx.x; i < active * here * 2; i += kThreads) {
        const int w = i / (here * 2);
        lds[i] = splitk_load(all + (int64_t)w * room + here * D + (i - w * here * 2));
    }
    __syncthreads();
    for (int i = threadIdx.x; i < here * D; i += kThreads) {
        const int n = i / D;
        float top = -__builtin_inff(), sum = 0.0f, v = 0.0f;
        for (int w = 0; w < active; ++w) top = fmaxf(top, lds[2 * (w * here + n)]);
        const float use = top == -__builtin_inff() ? 0.0f : top;
#pragma unroll 8
        for (int w = 0; w < active; ++w) {
            const float f = exp2_fast(lds[2 * (w * here + n)] - use);
            sum = fmaf(f, lds[2 * (w * here + n) + 1], sum);
            v = fmaf(f, splitk_load(all + (int64_t)w * room + i), v);
        }
        out[i] = (uint16_t)f32_to_h16<F16>(sum == 0.0f ? 0.0f : v / sum);
    }
}

template <int BITS, int D, bool F16> hipError_t launch(const DecodeArgs& a, const dim3& grid, int here, hipStream_t stream) {
    constexpr auto kernel = attn_decode_kernel<BITS, D, F16>;
    const int most = kWaves * 16 * (D + 2) * (int)sizeof(float);
    if (hipError_t e = ensure_lds<kernel>(most); e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, grid, dim3(kThreads), kWaves * here * (D + 2) * sizeof(float), stream, a);
    return hipGetLastError();
}

}  // namespace

constexpr int kMaxSplits = 128, kMinChunk = kStep * kWaves, kMaxChunk = 2048;

DecodePlan plan_attn_decode(int64_t requests, int heads, int kv_heads, int head_dim, int64_t max_tokens, int cus) {
    DecodePlan p{};
    p.shared = heads / kv_heads;
    p.head_tiles = (p.shared + 15) / 16;
    const int64_t pairs = requests * kv_heads * p.head_tiles;
    const int64_t want = pairs > 0 ? (2 * (int64_t)cus + pairs - 1) / pairs : 1;
    int64_t chunk = (max_tokens + want - 1) / want;
    if (chunk > kMaxChunk) chunk = kMaxChunk;
    if (chunk < kMinChunk) chunk = kMinChunk;
    if (chunk * kMaxSplits < max_tokens) chunk = (max_tokens + kMaxSplits - 1) / kMaxSplits;
    chunk = (chunk + kStep - 1) / kStep * kStep;
    p.chunk = (int)chunk;
    p.splits = (int)((max_tokens + chunk - 1) / chunk);
    if (p.splits < 1) p.splits = 1;
    if (p.splits > 1) {
        const int here = p.shared < 16 ? p.shared : 16;
        p.words_bytes = (size_t)pairs * kWordBytes;
        p.workspace = p.words_bytes + (size_t)pairs * p.splits * here * (head_dim + 2) * sizeof(float);
    }
    return p;
}

hipError_t launch_attn_decode(const Rows& q, const any4_kv_cache& c, const int32_t* table, int64_t table_stride, int64_t table_width,
                              const int32_t* lengths, int64_t requests, int heads, float softmax_scale, uint16_t* out, const DecodePlan& pl,
                              void* workspace, hipStream_t stream) {
    DecodeArgs a{q, kv_pages(c), table, table_stride, (int)table_width, lengths, heads, pl.shared, pl.head_tiles, softmax_scale * kLog2e, out,
                 pl.splits, pl.chunk, nullptr, static_cast<uint8_t*>(workspace)};
    a.partial = reinterpret_cast<float*>(a.words + pl.words_bytes);
    const dim3 grid((unsigned)pl.splits, (unsigned)(c.kv_heads * pl.head_tiles), (unsigned)requests);
    const int here = pl.shared < 16 ? pl.shared : 16;
    auto dims = [&](auto bits, auto f16) {
        return c.head_dim == 128 ? launch<decltype(bits)::value, 128, decltype(f16)::value>(a, grid, here, stream)
                                 : launch<decltype(bits)::value, 64, decltype(f16)::value>(a, grid, here, stream);
    };
    auto types = [&](auto bits) { return c.f16 ? dims(bits, std::true_type{}) : dims(bits, std::false_type{}); };
    return c.bits == 16 ? types(std::integral_constant<int, 16>{}) : c.bits == 8 ? types(std::integral_constant<int, 8>{}) : types(std::integral_constant<int, 4>{});
}

}  // namespace any4
