// any4_rope / any4_rope_kv_write: queries and keys of a list of tokens are normalised and turned by their positions, in one pass, the latter
// into the paged cache with v beside them.
//
//     y = x / sqrt(mean(x^2) + eps) * w,    (y_a, y_b) -> (y_a cos - y_b sin, y_b cos + y_a sin),    angle_i = position[axis_i] * freq_i
// A lane has eight values of a head, four pairs of them where they are turned: values 4 i .. and half a turned part further, or eight that
// lie side by side (interleaved, and what is not turned).  So no value changes lanes, and a sum of squares is all that lanes exchange.
//
// A block takes four tokens and goes over their heads, a few at a time (4, with heads of 64 values 8): 256 angles at most, one for a thread,
// lie in LDS for all of them.  Memory bounds it: q, k and v are read once and written once.
//
// Rounding: norm, angles' sine and cosine and the turn are fp32, the result is rounded once; the angles themselves are fp64 until whole turns
// are off them (position 10^6 in fp32 would be off by 0.06).  A key that goes into the cache as codes is rounded to 16 bits first, so that the cache holds what
// any4_rope and any4_kv_write one after the other would have put there, bit for bit.
//
// Measured, 32 query and 8 KV heads of 128 unless said otherwise, us:
//     16384 tokens with norms into a cache of 8 bits             82   (4.9 TB/s, as a copy; vector units busy 73 %.  Loads when a head is worked on 98)
//     the same into a cache of 4 bits, and read back             98  (into 8 bits 103, 82 of it the write)
//     5001 tokens, three axes, norms, fp16, q and k alone        20 in the kernel, 25 with the call's gaps (5.1 and 4.0 TB/s)
//     45 tokens, 16 and 2 heads, no norms; 16 tokens, 16 bits    3 and 4 in the kernel, 5 with the call (loads that wait for each other: position, frequency)
#include "any4_attn.h"
#include "any4_kv_encode.h"
#include "any4_launches.h"

namespace any4 {

namespace {

constexpr int kThreads = 256, kTokens = 4;

struct Args {
    Rows q, k, v;
    uint16_t *q_out, *k_out;
    int64_t qo_token, qo_head, ko_token, ko_head;
    int64_t tokens;
    const int64_t* slots;
    const int64_t* positions;
    int64_t axis_stride;
    const uint8_t* axis_of;
    const double* freqs;
    const uint16_t *q_norm, *k_norm;
    int heads, kv_heads, axes, rotary, per_block;     // per_block: heads of a block
    float eps;
    bool interleaved;
    KvPages c;
};

__device__ __forceinline__ u32x2 load_four(const uint16_t* p) { return *reinterpret_cast<const u32x2*>(p); }
__device__ __forceinline__ void store_four(uint16_t* p, uint32_t a, uint32_t b) { *reinterpret_cast<u32x2*>(p) = u32x2{a, b}; }

// BITS 0: no cache.  (16 bits in either type are the same cache, but not the same keys.)
template <int BITS, int D, bool F16>
__global__ __launch_bounds__(kThreads) void rope_kernel(Args a) {
    constexpr int LANES = D / 8, AT_ONCE = kThreads / (kTokens * LANES);
    __shared__ f32x2 table[kTokens][D / 2 + 2];                // cosine and sine
    __shared__ u32x2 norms[2][D / 4];                          // weights (from memory they would be waited for together with the next head's values)
    const int part = threadIdx.x % LANES, vec = threadIdx.x / LANES, mine = vec / AT_ONCE;
    const int64_t t0 = (int64_t)blockIdx.x * kTokens, t = t0 + mine;
    const int half = a.rotary / 2;
    // this lane's values of a head of q or k: four from `lo`, four from `hi`
    const bool turned = part * 8 < a.rotary, split = turned && !a.interleaved;
    const int lo = split ? 4 * part : 8 * part, hi = split ? half + 4 * part : 8 * part + 4;
    const int first = blockIdx.y * a.per_block + vec % AT_ONCE, all = a.heads + (BITS != 0 ? 2 : 1) * a.kv_heads;   // heads of this block
    const int end = min(all, (int)(blockIdx.y + 1) * a.per_block);
    struct Eight {
        u32x2 lo, hi;
    };
    auto fetch = [&](int h) -> Eight {
        const int j = h - a.heads;
        const uint16_t* from = j < 0 ? a.q.p + t * a.q.token + h * a.q.head
                             : BITS == 0 || j < a.kv_heads ? a.k.p + t * a.k.token + j * a.k.head : a.v.p + t * a.v.token + (j - a.kv_heads) * a.v.head;
        const bool is_v = BITS != 0 && j >= a.kv_heads;
        return Eight{load_four(from + (is_v ? 8 * part : lo)), load_four(from + (is_v ? 8 * part + 4 : hi))};
    };
    // (a head's values are asked for before those of the head in front of it are worked on, the first before the angles)
    Eight next{};
    if (t < a.tokens && first < end) next = fetch(first);
    if (threadIdx.x < D / 2) {
        const uint16_t* const from = threadIdx.x < D / 4 ? a.q_norm : a.k_norm;
        if (from) norms[threadIdx.x / (D / 4)][threadIdx.x % (D / 4)] = load_four(from + 4 * (threadIdx.x % (D / 4)));
    }
    for (int i = threadIdx.x; i < kTokens * half; i += kThreads) {
        const int tok = i / half, j = i - tok * half;
        if (t0 + tok >= a.tokens) break;
        const int axis = a.axis_of ? min((int)a.axis_of[j], a.axes - 1) : 0;
        const double turns = (double)a.positions[axis * a.axis_stride + t0 + tok] * a.freqs[j] * 0.15915494309189533577;
        const float x = 2.0f * (float)(turns - rint(turns));
        f32x2 cs;
        float s, c;
        sincospif(x, &s, &c);
        cs[0] = c;
        cs[1] = s;
        table[tok][j] = cs;
    }
    __syncthreads();
    if (t >= a.tokens) return;

    f32x2 cs[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) cs[i] = turned ? table[mine][4 * part + i] : f32x2{1.0f, 0.0f};

    auto turn = [&](const Eight& in, int of_k, uint32_t (&y)[4]) {
        const u32x2 p = in.lo, r = in.hi;
        float x[8];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            x[2 * j] = h16lo_to_f32<F16>(p[j]);
            x[2 * j + 1] = h16hi_to_f32<F16>(p[j]);
            x[4 + 2 * j] = h16lo_to_f32<F16>(r[j]);
            x[4 + 2 * j + 1] = h16hi_to_f32<F16>(r[j]);
        }
        if (of_k ? a.k_norm : a.q_norm) {
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = fmaf(x[j], x[j], sum);
            sum = lanes_reduce<LANES>(sum, [](float u, float v) { return u + v; });
            const float by = rsqrtf(fmaf(sum, 1.0f / D, a.eps));
            const u32x2 wp = norms[of_k][lo / 4], wr = norms[of_k][hi / 4];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                x[2 * j] *= by * h16lo_to_f32<F16>(wp[j]);
                x[2 * j + 1] *= by * h16hi_to_f32<F16>(wp[j]);
                x[4 + 2 * j] *= by * h16lo_to_f32<F16>(wr[j]);
                x[4 + 2 * j + 1] *= by * h16hi_to_f32<F16>(wr[j]);
            }
        }
        if (turned) {
            if (a.interleaved) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float u = x[2 * j], v = x[2 * j + 1];
                    x[2 * j] = fmaf(u, cs[j][0], -(v * cs[j][1]));
                    x[2 * j + 1] = fmaf(v, cs[j][0], u * cs[j][1]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float u = x[j], v = x[4 + j];
                    x[j] = fmaf(u, cs[j][0], -(v * cs[j][1]));
                    x[4 + j] = fmaf(v, cs[j][0], u * cs[j][1]);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = f32x2_to_h16x2<F16>(x[2 * j], x[2 * j + 1]);
    };
    int64_t slot = -1;
    if constexpr (BITS != 0) slot = a.slots[t];
    const bool kept = BITS != 0 && slot >= 0 && slot < a.c.slots;
    const int page = kept ? (int)(slot >> a.c.page_shift) : 0, place = (int)(slot & ((1 << a.c.page_shift) - 1));

    for (int h = first; h < end; h += AT_ONCE) {
        const Eight in = next;
        if (h + AT_ONCE < end) next = fetch(h + AT_ONCE);
        if (h < a.heads) {
            uint32_t y[4];
            turn(in, 0, y);
            uint16_t* to = a.q_out + t * a.qo_token + h * a.qo_head;
            store_four(to + lo, y[0], y[1]);
            store_four(to + hi, y[2], y[3]);
            continue;
        }
        const bool is_v = h >= a.heads + a.kv_heads;
        const int j = h - a.heads - (is_v ? a.kv_heads : 0);
        uint32_t y[4];
        int at_lo = lo, at_hi = hi;
        if (is_v) {
            at_lo = 8 * part;
            at_hi = 8 * part + 4;
            y[0] = in.lo[0];
            y[1] = in.lo[1];
            y[2] = in.hi[0];
            y[3] = in.hi[1];
        } else {
            turn(in, 1, y);
            if (a.k_out) {
                uint16_t* to = a.k_out + t * a.ko_token + j * a.ko_head;
                store_four(to + lo, y[0], y[1]);
                store_four(to + hi, y[2], y[3]);
            }
        }
        if constexpr (BITS != 0) {
            if (!kept) continue;                               // (a whole vector's lanes alike)
            const int64_t at = a.c.first_token(page, j) + place;
            uint8_t* held = is_v ? a.c.v : a.c.k;
            if constexpr (BITS == 16) {
                uint16_t* to = reinterpret_cast<uint16_t*>(held) + at * D;
                store_four(to + at_lo, y[0], y[1]);
                store_four(to + at_hi, y[2], y[3]);
            } else {
                float x[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[2 * i] = h16lo_to_f32<F16>(y[i]);
                    x[2 * i + 1] = h16hi_to_f32<F16>(y[i]);
                }
                uint32_t so;
                const u32x2 w = encode<BITS, LANES>(x, so);
                if constexpr (BITS == 8) {
                    *reinterpret_cast<uint32_t*>(held + at * D + at_lo) = w[0];
                    *reinterpret_cast<uint32_t*>(held + at * D + at_hi) = w[1];
                } else {
                    *reinterpret_cast<uint16_t*>(held + at * (D / 2) + at_lo / 2) = (uint16_t)w[0];
                    *reinterpret_cast<uint16_t*>(held + at * (D / 2) + at_hi / 2) = (uint16_t)(w[0] >> 16);
                }
                if (part == 0) reinterpret_cast<uint32_t*>(a.c.scales)[2 * at + (is_v ? 1 : 0)] = so;
            }
        }
    }
}

template <int BITS, int D, bool F16> hipError_t launch(const Args& given, int cus, hipStream_t stream) {
    constexpr int AT_ONCE = kThreads / (kTokens * (D / 8));
    const int all = given.heads + (BITS != 0 ? 2 : 1) * given.kv_heads, passes = (all + AT_ONCE - 1) / AT_ONCE;
    const int64_t blocks = (given.tokens + kTokens - 1) / kTokens;
    // few tokens: their heads are shared out over blocks, up to two for a compute unit
    const int64_t most = 2 * (int64_t)cus / blocks;
    const int parts = (int)(most < 1 ? 1 : most < passes ? most : passes);
    return launch_blocks(blocks, kThreads, hipSuccess, [&](int64_t first, int64_t count) {
        Args a = given;
        const int64_t at = first * kTokens, left = given.tokens - at;
        a.tokens = left < count * kTokens ? left : count * kTokens;
        a.q.p += at * a.q.token;
        a.k.p += at * a.k.token;
        if (BITS != 0) {
            a.v.p += at * a.v.token;
            a.slots += at;
        }
        a.q_out += at * a.qo_token;
        if (a.k_out) a.k_out += at * a.ko_token;
        a.positions += at;
        a.per_block = (passes + parts - 1) / parts * AT_ONCE;
        hipLaunchKernelGGL((rope_kernel<BITS, D, F16>), dim3((unsigned)count, (unsigned)((all + a.per_block - 1) / a.per_block)), dim3(kThreads), 0, stream, a);
        return hipGetLastError();
    });
}

}  // namespace

hipError_t launch_rope(const RopeArgs& r, const any4_rotation& turn, const any4_kv_cache* c, int cus, hipStream_t stream) {
    Args a{r.q, r.k, r.v, r.q_out, r.k_out, r.qo_token, r.qo_head, r.ko_token, r.ko_head, r.tokens, r.slots, turn.positions, turn.axis_stride, turn.axis_of,
           turn.freqs, turn.q_norm, turn.k_norm, r.heads, r.kv_heads, turn.axes, turn.rotary_dim, 0, turn.eps, turn.interleaved != 0, {}};
    if (c) a.c = kv_pages(*c);
    auto types = [&](auto bits, auto dim) {
        return r.f16 ? launch<decltype(bits)::value, decltype(dim)::value, true>(a, cus, stream)
                     : launch<decltype(bits)::value, decltype(dim)::value, false>(a, cus, stream);
    };
    auto dims = [&](auto bits) {
        return r.head_dim == 128 ? types(bits, std::integral_constant<int, 128>{}) : types(bits, std::integral_constant<int, 64>{});
    };
    const int bits = c ? c->bits : 0;
    return bits == 16 ? dims(std::integral_constant<int, 16>{}) : bits == 8 ? dims(std::integral_constant<int, 8>{})
         : bits == 4 ? dims(std::integral_constant<int, 4>{}) : dims(std::integral_constant<int, 0>{});
}

}  // namespace any4
