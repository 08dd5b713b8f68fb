// any4_attn_prompt: attention of packed prompts, causal or not, query heads sharing KV heads.
//
//     s_ij = scale q_i . k_j,   o_i = sum_j exp(s_ij - m_i) v_j / sum_j exp(s_ij - m_i)
// in one pass over the keys with a running maximum m_i; neither scores nor weights leave the registers.
// Two matrix products of 2 D operations a score bound it, beside the exponential and its sums on the vector units.
//
// A block takes 128 queries of one head, a wavefront 32 of them, and walks over the keys 64 at a time.  k and v are copied to
// LDS without passing registers, the next 64 while these are worked on.  S^T = K Q^T with v_mfma_f32_32x32x16: a query's
// scores then lie in two lanes, a maximum is one exchange, and the weights are at once the B operand of O^T = V^T P^T, whose keys are
// taken in the order in which the lanes have them (lane half g: keys 4 g .. 4 g + 3 and 8 + 4 g .. of every 16).  V^T's operand comes
// out of the row-major tile by transposing LDS reads.  Tiles are swizzled in pieces of 16 bytes so that 16 (k) or 4 (v)
// neighbouring rows' pieces lie in different banks.
//
// The matrix cores make a tile's scores while the vector units turn the ones of the tile in front of it into weights: one after the other
// 2 x 8192 causal tokens took 1140 us, like this 1050.  So k is copied two tiles ahead, v one.
//
// Measured, 32 query heads on 8 KV heads of 128, bf16, causal:
//     2 prompts of 8192 tokens            1050 us, 1.05 PFLOP/s (a product of 8192^3 in the library: 1.28 .. 1.36)
//         in fp16                         1150 us (two conversions and a pack for each pair of weights, one instruction in bf16)
//         heads of 64                      630 us (half the matrix work, as many exponentials)
//     12 of 65 .. 2048 behind contexts of up to 1024    370 us, 0.81 PFLOP/s
//     one of 77                            9.3 us (starts, q, k and v wait for each other; 32 blocks)
// Of the long ones' time the matrix cores are busy 54 %, the vector units 53 % (packed: 41 and 49), beside each other, at 1.8 .. 1.9 GHz; a wavefront
// waits 30 % of its time.  For each score of a lane the matrix cores take 32 cycles, the exponential 9 and its scaling, maximum, sum and rounding
// about 14 on the vector units; the rest is waiting for LDS and for the block's other wavefronts.
// Prescribing the order of LDS reads, matrix and vector instructions changed nothing (1046 .. 1061 us), 64 queries a wavefront do not fit
// the registers (85 spilled, 1600 us).
//
// The maximum in use is raised only when a score exceeds it by 2^kSlack, which spares nearly all rescaling of o: weights of
// up to 2^kSlack lose nothing in floating point.
//
// Rounding: scores, maxima, sums and accumulators are fp32; the weights are rounded to 16 bits for the matrix cores, once.
#include "any4_attn.h"
#include "any4_internal.h"
#include "any4_launches.h"
#include "any4_lds_copy.h"

namespace any4 {

namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves, kKeys = 64;
constexpr float kSlack = 8.0f;
constexpr float kFar = 1048576.0f;        // 2^20: up to there a maximum's rounding moves the exponents by 2^-4 at most, for all keys of a query alike

#pragma clang diagnostic ignored "-Wint-to-pointer-cast"          // LDS offsets as pointers
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) u32x4* lds_u4;
typedef __attribute__((address_space(3))) u32x2* lds_u2;
typedef __attribute__((address_space(3))) s16x4* lds_s4;

struct Args {
    Rows q, k, v;
    const int32_t* q_starts;
    const int32_t* k_starts;
    int q_tokens, k_tokens, requests, heads, kv_heads, shared, causal;
    unsigned first_block;              // of this launch
    float scale_log2;
    uint16_t* out;
};

// 4 rows x 16 columns: lane i of 16 gives the address of row i / 4, columns 4 * (i % 4) .., and gets column i of the four rows
__device__ __forceinline__ u32x2 lds_read_transposed(uint32_t at) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(at)));
}

// the part of a tile that a wavefront copies: 16-byte pieces, 64 an instruction
template <int D> struct Tile {
    static constexpr int kRow = 2 * D, kBytes = kKeys * kRow, kPieces = D / 8, kRows = 64 / kPieces;     // rows an instruction
    static constexpr int kCopies = kKeys / kRows / kWaves;                                                // of a wavefront
    __device__ static __forceinline__ int swizzle_k(int row) { return D == 128 ? row & 15 : (row >> 1) & 7; }
    __device__ static __forceinline__ int swizzle_v(int row) { return D == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2; }
};

template <int D, bool F16>
__global__ __launch_bounds__(kThreads, 2) void attn_prompt_kernel(Args a) {
    using T = Tile<D>;
    constexpr int QM = D / 16, OM = D / 32, ROWS = 32 * kWaves;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, g = lane >> 5;

    // KV heads fastest: blocks that read the same keys tend to share an XCD and its L2
    const unsigned block = a.first_block + blockIdx.x, rest = block / (unsigned)a.kv_heads, kv_head = block - rest * (unsigned)a.kv_heads;
    const unsigned place = rest / (unsigned)a.shared;
    const int head = (int)(kv_head * (unsigned)a.shared + (rest - place * (unsigned)a.shared));

    // which request's tile this is
    int request = -1, tile = 0, lq = 0, q_at = 0;
    for (int r0 = 0, before = 0; r0 < a.requests && request < 0; r0 += 64) {
        const int r = min(r0 + lane, a.requests - 1);
        const int s0 = min(max(a.q_starts[r], 0), a.q_tokens), s1 = min(max(a.q_starts[r + 1], 0), a.q_tokens);
        const int rows = r0 + lane < a.requests ? max(s1 - s0, 0) : 0, tiles = (rows + ROWS - 1) / ROWS;
        int sum = tiles;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int u = __shfl_up(sum, d);
            if (lane >= d) sum += u;
        }
        const unsigned long long past = __builtin_amdgcn_ballot_w64(before + sum > (int)place);
        if (past) {
            const int f = __builtin_ctzll(past);
            request = r0 + f;
            lq = __builtin_amdgcn_readlane(rows, f);
            q_at = __builtin_amdgcn_readlane(s0, f);
            const int all = __builtin_amdgcn_readlane(tiles, f);
            tile = (int)place - (before + __builtin_amdgcn_readlane(sum, f) - all);
            if (a.causal) tile = all - 1 - tile;               // the most keys first
        }
        before += __builtin_amdgcn_readlane(sum, 63);
    }
    if (request < 0) return;
    const int k_at = min(max(a.k_starts[request], 0), a.k_tokens);
    const int lk = max(min(max(a.k_starts[request + 1], 0), a.k_tokens) - k_at, 0);
    const int q0 = tile * ROWS, q_wave = q0 + 32 * wave, query = q_wave + n;
    const int ahead = lk - lq;                                  // query i sees keys 0 .. i + ahead
    const int end = a.causal ? min(lk, min(q0 + ROWS, lq) + ahead) : lk;          // of the block's keys
    const int tiles = end > 0 ? (end + kKeys - 1) / kKeys : 0;
    const int lim = a.causal ? min(query + ahead, lk - 1) : lk - 1;                // last key of this lane's query

    u32x4 q[QM];
    {
        const uint16_t* qp = a.q.p + (int64_t)(q_at + min(query, lq - 1)) * a.q.token + (int64_t)head * a.q.head + 8 * g;
#pragma unroll
        for (int i = 0; i < QM; ++i) q[i] = *reinterpret_cast<const u32x4*>(qp + 16 * i);
    }

    // copies: lane -> row and piece of each instruction; LDS has piece c of row r at c ^ swizzle(r).  LDS: two tiles of k, two of v.
    const char* k_base = reinterpret_cast<const char*>(a.k.p + (int64_t)k_at * a.k.token + (int64_t)kv_head * a.k.head);
    const char* v_base = reinterpret_cast<const char*>(a.v.p + (int64_t)k_at * a.v.token + (int64_t)kv_head * a.v.head);
    const uint32_t k_step = (uint32_t)a.k.token * 2u, v_step = (uint32_t)a.v.token * 2u;
    const int copy_row = T::kCopies * wave * T::kRows + lane / T::kPieces, copy_piece = lane % T::kPieces;
    uint32_t k_from[T::kCopies], v_from[T::kCopies];
#pragma unroll
    for (int j = 0; j < T::kCopies; ++j) {
        const int row = copy_row + j * T::kRows;
        k_from[j] = (uint32_t)row * k_step + 16u * (uint32_t)(copy_piece ^ T::swizzle_k(row));
        v_from[j] = (uint32_t)row * v_step + 16u * (uint32_t)(copy_piece ^ T::swizzle_v(row));
    }
    auto copy_rows = [&](const char* base, uint32_t step, const uint32_t (&from)[T::kCopies], int t, uint32_t to) {
        const int k0 = t * kKeys;
        const char* tile_base = base + (int64_t)k0 * step;
#pragma unroll
        for (int j = 0; j < T::kCopies; ++j) {
            uint32_t off = from[j];
            // (rows past the last are copies of it; they are masked)
            if (k0 + kKeys > lk) off -= (uint32_t)max(copy_row + j * T::kRows - (lk - 1 - k0), 0) * step;
            copy_to_lds(to + (uint32_t)(T::kCopies * wave + j) * 1024u, tile_base, off);
        }
    };
    auto copy_k = [&](int t, uint32_t parity) { copy_rows(k_base, k_step, k_from, t, parity * T::kBytes); };
    auto copy_v = [&](int t, uint32_t parity) { copy_rows(v_base, v_step, v_from, t, (2 + parity) * T::kBytes); };

    // operand addresses within a tile
    uint32_t k_lane[QM], v_lane[OM];
    {
        const int i16 = lane & 15, v_row = 4 * g + (i16 >> 2);
#pragma unroll
        for (int i = 0; i < QM; ++i) k_lane[i] = (uint32_t)(n * T::kRow + (((2 * i + g) ^ T::swizzle_k(n)) << 4));
#pragma unroll
        for (int m = 0; m < OM; ++m)
            v_lane[m] = (uint32_t)(2 * T::kBytes + v_row * T::kRow + 8 * (i16 & 1) +
                                   (((4 * m + 2 * ((lane >> 4) & 1) + ((i16 >> 1) & 1)) ^ T::swizzle_v(v_row)) << 4));
    }

    float m_ref = -__builtin_inff(), l = 0.0f;
    f32x16 o[OM], s[2];
#pragma unroll
    for (int m = 0; m < OM; ++m)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[m][r] = 0.0f;

    auto scores = [&](uint32_t buf, f32x16 (&to)[2]) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int r = 0; r < 16; ++r) to[u][r] = 0.0f;
#pragma unroll
            for (int i = 0; i < QM; ++i) {
                const u32x4 k = *(lds_u4)(k_lane[i] + (buf + (uint32_t)(u * 32 * T::kRow)));
                to[u] = mma32<F16>(k, q[i], to[u]);
            }
        }
    };
    auto mask = [&](int t, f32x16 (&x)[2]) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int r = 0; r < 16; ++r) x[u][r] = t * kKeys + 32 * u + 8 * (r >> 2) + 4 * g + (r & 3) <= lim ? x[u][r] : -__builtin_inff();
    };
    auto highest = [&](const f32x16 (&x)[2]) -> float {
        float top = x[0][0];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, x[u][r]);
        const u32x2 both = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false));
        return fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])) * a.scale_log2;
    };
    // The maximum in use follows the scores x, whose weights' exponents are then scale x - m_sub: a product that is not rounded, less a maximum that
    // is.  Beyond 2^31 that rounding alone would leave the exponents' range: where some query's maximum lies beyond kFar, the scores are
    // replaced by their distance from it, both rounded alike.
    float m_sub = 0.0f;
    unsigned long long far = 0ull;                              // queries whose maximum lies beyond kFar
    auto raise = [&](f32x16 (&x)[2]) {
        const float top = highest(x);
        if ((__builtin_amdgcn_ballot_w64(top > m_ref + kSlack) | far) != 0ull) {
            const float m_new = fmaxf(m_ref, top);
            const float alpha = m_new > m_ref ? exp2_fast(m_ref - m_new) : 1.0f;
            m_ref = m_new;
            m_sub = m_ref == -__builtin_inff() ? 0.0f : m_ref;
            l *= alpha;
#pragma unroll
            for (int m = 0; m < OM; ++m) o[m] *= alpha;
            far = __builtin_amdgcn_ballot_w64(fabsf(m_sub) > kFar);
            if (far) {
                const float back = 1.0f / a.scale_log2;
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
#pragma clang fp contract(off)
                        const float scaled = x[u][r] * a.scale_log2;
                        x[u][r] = (scaled - m_sub) * back;
                    }
                m_sub = 0.0f;
            }
        }
    };
    auto weigh = [&](const f32x16 (&x)[2], u32x4 (&p)[4]) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int r = 0; r < 16; r += 2) {
                const float e = exp2_fast(fmaf(x[u][r], a.scale_log2, -m_sub)), f = exp2_fast(fmaf(x[u][r + 1], a.scale_log2, -m_sub));
                l += e + f;
                p[2 * u + (r >> 3)][(r >> 1) & 3] = f32x2_to_h16x2<F16>(e, f);
            }
    };
    auto v_operand = [&](uint32_t buf, int c, int m) -> u32x4 {
        const uint32_t at = v_lane[m] + (buf + (uint32_t)(c * 16 * T::kRow));
        const u32x2 lo = lds_read_transposed(at), hi = lds_read_transposed(at + 8 * T::kRow);
        return u32x4{lo[0], lo[1], hi[0], hi[1]};
    };

    // Tile t, whose scores are there: its weights and its part of o, while the matrix cores make the next tile's scores.  THIS, NEXT: its
    // parity, the next one's.  All queries see all keys of both tiles.
    auto step = [&](int t, uint32_t even) {
        loads_left<0>();
        lds_barrier();                                          // k of t + 1 and v of t are there, and nobody reads the other tiles any more
        if (t + 2 < tiles) copy_k(t + 2, even);
        copy_v(t + 1, even ^ 1u);
        f32x16 next[2];
        u32x4 p[4];
        scores((even ^ 1u) * T::kBytes, next);
        weigh(s, p);
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int m = 0; m < OM; ++m) o[m] = mma32<F16>(v_operand(even * T::kBytes, c, m), p[c], o[m]);
        s[0] = next[0];
        s[1] = next[1];
        raise(s);
    };
    // The same where some query may not see some key of t or t + 1, or t is the last.
    auto last_step = [&](int t, uint32_t even) {
        const int k0 = t * kKeys;
        const uint32_t buf = even * T::kBytes;
        loads_left<0>();
        lds_barrier();
        if (t + 2 < tiles) copy_k(t + 2, even);
        if (t + 1 < tiles) copy_v(t + 1, even ^ 1u);
        if (!(a.causal && k0 > q_wave + 31 + ahead)) {          // (else no query of this wavefront sees a key of t or behind it)
            u32x4 p[4];
            weigh(s, p);
            // A key that some query does not see has weight 0 for it, and 0 times what is not finite would be NaN: keys with such
            // values are taken out of the product and added one by one to the queries that see them.
            constexpr uint32_t kExp = F16 ? 0x7C007C00u : 0x7F807F80u, kOne = F16 ? 0x04000400u : 0x00800080u;
            unsigned long long bad = 0ull;                      // bit 16 c + 8 half + slot
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
                uint32_t bits[4] = {0u, 0u, 0u, 0u};
#pragma unroll
                for (int m = 0; m < OM; ++m) {
                    const u32x4 v = v_operand(buf, c, m);
#pragma unroll
                    for (int w = 0; w < 4; ++w) bits[w] |= (v[w] & kExp) + kOne;       // (an exponent of all ones carries into the half's top bit)
                }
                if (__builtin_amdgcn_ballot_w64(((bits[0] | bits[1] | bits[2] | bits[3]) & 0x80008000u) != 0u) == 0ull) continue;
                uint32_t some = 0u;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const unsigned long long lanes = __builtin_amdgcn_ballot_w64((bits[j >> 1] >> (16 * (j & 1) + 15)) & 1u);
                    some |= ((uint32_t)lanes != 0u ? 1u : 0u) << j | ((uint32_t)(lanes >> 32) != 0u ? 1u : 0u) << (8 + j);
                }
                bad |= (unsigned long long)some << (16 * c);
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint32_t mine = (uint32_t)(bad >> (16 * c)) >> (8 * g);
                u32x4 keep;
#pragma unroll
                for (int w = 0; w < 4; ++w) keep[w] = ((mine >> (2 * w)) & 1u ? 0u : 0xFFFFu) | ((mine >> (2 * w + 1)) & 1u ? 0u : 0xFFFF0000u);
#pragma unroll
                for (int m = 0; m < OM; ++m) o[m] = mma32<F16>(v_operand(buf, c, m) & keep, p[c], o[m]);
            }
#pragma unroll 1
            while (bad) {
                const int b = __builtin_ctzll(bad), c = b >> 4, half = (b >> 3) & 1, slot = b & 7;
                bad &= bad - 1;
                const int row = 16 * c + (slot < 4 ? 4 * half + slot : 4 + 4 * half + slot);
                uint32_t pair = 0u;
#pragma unroll
                for (int x = 0; x < 16; ++x) pair = x == 4 * c + (slot >> 1) ? p[x >> 2][x & 3] : pair;
                const float mine = slot & 1 ? h16hi_to_f32<F16>(pair) : h16lo_to_f32<F16>(pair), other = __shfl_xor(mine, 32);
                const float weight = g == half ? mine : other;
                const bool seen = k0 + row <= lim;
#pragma unroll
                for (int m = 0; m < OM; ++m)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const uint32_t piece = (uint32_t)((4 * m + r) ^ T::swizzle_v(row));
                        const u32x2 v = *(lds_u2)(buf + 2u * T::kBytes + (uint32_t)(row * T::kRow) + 16u * piece + 8u * (uint32_t)g);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float x = e & 1 ? h16hi_to_f32<F16>(v[e >> 1]) : h16lo_to_f32<F16>(v[e >> 1]);
                            o[m][4 * r + e] = seen ? fmaf(weight, x, o[m][4 * r + e]) : o[m][4 * r + e];
                        }
                    }
            }
            if (t + 1 < tiles) {
                scores((even ^ 1u) * T::kBytes, s);
                mask(t + 1, s);
                raise(s);
            }
        }
    };
    const int whole = min(tiles, max(a.causal ? min(lk, q0 + ahead + 1) : lk, 0) / kKeys);      // tiles of which all queries see all keys
    if (tiles > 0) {
        copy_k(0, 0);
        copy_v(0, 0);
        if (tiles > 1) copy_k(1, 1);
        loads_left<0>();
        lds_barrier();
        scores(0, s);
        if (whole == 0) mask(0, s);
        raise(s);
    }
    int t = 0;
    for (; t + 2 < whole; t += 2) {
        step(t, 0u);
        step(t + 1, 1u);
    }
#pragma unroll 1
    for (; t < tiles; ++t) last_step(t, (uint32_t)(t & 1));

    l += __shfl_xor(l, 32);
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;              // (no key seen: o is 0 as well)
    if (query < lq) {
        uint16_t* out = a.out + ((int64_t)(q_at + query) * a.heads + head) * D + 4 * g;
#pragma unroll
        for (int m = 0; m < OM; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                *reinterpret_cast<u32x2*>(out + 32 * m + 8 * r) =
                    u32x2{f32x2_to_h16x2<F16>(o[m][4 * r] * inv, o[m][4 * r + 1] * inv), f32x2_to_h16x2<F16>(o[m][4 * r + 2] * inv, o[m][4 * r + 3] * inv)};
    }
}

template <int D, bool F16> hipError_t launch(Args a, int64_t blocks, hipStream_t stream) {
    constexpr auto kernel = attn_prompt_kernel<D, F16>;
    constexpr int bytes = 4 * Tile<D>::kBytes;
    if (hipError_t e = ensure_lds<kernel>(bytes); e != hipSuccess) return e;
    return launch_blocks(blocks, kThreads, hipSuccess, [&](int64_t first, int64_t count) {
        a.first_block = (unsigned)first;
        hipLaunchKernelGGL(kernel, dim3((unsigned)count), dim3(kThreads), bytes, stream, a);
        return hipGetLastError();
    });
}

}  // namespace

hipError_t launch_attn_prompt(const PromptArgs& p, hipStream_t stream) {
    Args a{p.q, p.k, p.v, p.q_starts, p.k_starts, (int)p.q_tokens, (int)p.k_tokens, p.requests, p.heads, p.kv_heads, p.heads / p.kv_heads,
           p.causal, 0u, p.softmax_scale * kLog2e, p.out};
    static_assert(kPromptRows == 32 * kWaves, "prompt_blocks() counts tiles of a block's queries");
    const int64_t blocks = prompt_blocks(p.q_tokens, p.requests, p.heads);
    if (p.head_dim == 128) return p.f16 ? launch<128, true>(a, blocks, stream) : launch<128, false>(a, blocks, stream);
    return p.f16 ? launch<64, true>(a, blocks, stream) : launch<64, false>(a, blocks, stream);
}

}  // namespace any4
