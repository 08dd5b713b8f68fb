// any4_kv_write / any4_kv_read: k and v of a list of tokens into the paged cache and back.
//
// A block does 16 tokens (32 with heads of 64) of one KV head: a head's vector is 8 values each for 16 (8) lanes, 16 bytes a load.
// The inputs of a block are pieces of 256 bytes a token, its cache side is one contiguous piece where the tokens are
// neighbours: with 4 bits 1 KB rather than the 64-byte pieces that a block of one token and all heads would write.  Both
// kernels read every byte once and write every byte once; memory bounds all but the writes of codes.
//
// Measured, 8 KV heads of 128, us of the kernel: 16384 tokens into 16 bits 30 (134 MB, 4.5 TB/s), 65536 out of it 102 (537 MB, 5.3 TB/s),
// 16384 into 8 bits 29 (102 MB, 3.5 TB/s) and out of it 16 (6.2), into 4 bits 28 (85 MB, 3.1 TB/s) and out of it 14 (6.0), 2047 into 8 bits 6.7 and
// out of it 4.0, 16 into 16 bits 2.  Writes of codes are bound by their arithmetic rather than by memory: the vector units are busy 72 % of the time
// (16384 tokens, 8 bits; 480 instructions a wavefront, about 170 of them for the 16 quotients of a lane).
#include "any4_attn.h"
#include "any4_kv_encode.h"
#include "any4_launches.h"

namespace any4 {

namespace {

constexpr int kThreads = 256;

template <int BITS, int D, bool F16>
__global__ __launch_bounds__(kThreads) void kv_write_kernel(Rows k, Rows v, int64_t tokens, const int64_t* __restrict__ slots, KvPages c) {
    constexpr int LANES = D / 8, TOKENS = kThreads / LANES;
    const int part = threadIdx.x % LANES, head = blockIdx.y;
    const int64_t t = (int64_t)blockIdx.x * TOKENS + threadIdx.x / LANES;
    if (t >= tokens) return;
    const int64_t slot = slots[t];
    const u32x4 kw = *reinterpret_cast<const u32x4*>(k.p + t * k.token + head * k.head + 8 * part);
    const u32x4 vw = *reinterpret_cast<const u32x4*>(v.p + t * v.token + head * v.head + 8 * part);
    if (slot < 0 || slot >= c.slots) return;                // (a whole vector's lanes leave together)
    const int64_t at = c.first_token((int)(slot >> c.page_shift), head) + (slot & ((1 << c.page_shift) - 1));
    if constexpr (BITS == 16) {
        reinterpret_cast<u32x4*>(c.k)[at * LANES + part] = kw;
        reinterpret_cast<u32x4*>(c.v)[at * LANES + part] = vw;
    } else {
        float x[8];
        uint32_t ks, vs;
        widen<F16>(kw, x);
        const u32x2 kc = encode<BITS, LANES>(x, ks);
        widen<F16>(vw, x);
        const u32x2 vc = encode<BITS, LANES>(x, vs);
        if constexpr (BITS == 8) {
            reinterpret_cast<u32x2*>(c.k)[at * LANES + part] = kc;
            reinterpret_cast<u32x2*>(c.v)[at * LANES + part] = vc;
        } else {
            reinterpret_cast<uint32_t*>(c.k)[at * LANES + part] = kc[0];
            reinterpret_cast<uint32_t*>(c.v)[at * LANES + part] = vc[0];
        }
        if (part == 0) reinterpret_cast<u32x2*>(c.scales)[at] = u32x2{ks, vs};
    }
}

// value = scale * code + offset in fp32 (the product is exact), rounded once, within the type's range
template <int BITS, bool F16> __device__ __forceinline__ u32x4 decode(const u32x2& w, uint32_t scale_offset) {
    const float s = bf16lo_to_f32(scale_offset), o = bf16hi_to_f32(scale_offset);
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t c = BITS == 8 ? (w[j >> 2] >> (8 * (j & 3))) & 0xFFu : (w[0] >> (4 * j)) & 0xFu;
        x[j] = fmaf((float)c, s, o);
        if (F16 && fabsf(x[j]) > 65504.0f) x[j] = copysignf(65504.0f, x[j]);       // (a bf16 offset may lie outside of fp16's range)
    }
    return u32x4{f32x2_to_h16x2<F16>(x[0], x[1]), f32x2_to_h16x2<F16>(x[2], x[3]), f32x2_to_h16x2<F16>(x[4], x[5]),
                 f32x2_to_h16x2<F16>(x[6], x[7])};
}

template <int BITS, int D, bool F16>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(KvPages c, const int64_t* __restrict__ slots, int64_t tokens, uint16_t* __restrict__ k,
                                                           uint16_t* __restrict__ v) {
    constexpr int LANES = D / 8, TOKENS = kThreads / LANES;
    const int part = threadIdx.x % LANES, head = blockIdx.y;
    const int64_t t = (int64_t)blockIdx.x * TOKENS + threadIdx.x / LANES;
    if (t >= tokens) return;
    const int64_t slot = slots[t];
    u32x4 kw = {0u, 0u, 0u, 0u}, vw = kw;
    if (slot >= 0 && slot < c.slots) {
        const int64_t at = c.first_token((int)(slot >> c.page_shift), head) + (slot & ((1 << c.page_shift) - 1));
        if constexpr (BITS == 16) {
            kw = reinterpret_cast<const u32x4*>(c.k)[at * LANES + part];
            vw = reinterpret_cast<const u32x4*>(c.v)[at * LANES + part];
        } else {
            const u32x2 so = reinterpret_cast<const u32x2*>(c.scales)[at];
            u32x2 kc = {0u, 0u}, vc = kc;
            if constexpr (BITS == 8) {
                kc = reinterpret_cast<const u32x2*>(c.k)[at * LANES + part];
                vc = reinterpret_cast<const u32x2*>(c.v)[at * LANES + part];
            } else {
                kc[0] = reinterpret_cast<const uint32_t*>(c.k)[at * LANES + part];
                vc[0] = reinterpret_cast<const uint32_t*>(c.v)[at * LANES + part];
            }
            kw = decode<BITS, F16>(kc, so[0]);
            vw = decode<BITS, F16>(vc, so[1]);
        }
    }
    const int64_t to = (t * c.kv_heads + head) * LANES + part;
    reinterpret_cast<u32x4*>(k)[to] = kw;
    reinterpret_cast<u32x4*>(v)[to] = vw;
}

// launch(first token, tokens, grid) until one is refused: one launch below 2^28 tokens (heads of 64: 2^29)
template <class F> hipError_t launch_tokens(const any4_kv_cache& c, int64_t tokens, F launch) {
    const int per_block = kThreads / (c.head_dim / 8);
    return launch_blocks((tokens + per_block - 1) / per_block, kThreads, hipSuccess, [&](int64_t first, int64_t count) {
        const int64_t at = first * per_block, left = tokens - at;
        launch(at, left < count * per_block ? left : count * per_block, dim3((unsigned)count, (unsigned)c.kv_heads));
        return hipGetLastError();
    });
}

}  // namespace

hipError_t launch_kv_write(const Rows& k, const Rows& v, int64_t tokens, const int64_t* slots, const any4_kv_cache& c, hipStream_t stream) {
    return launch_tokens(c, tokens, [&](int64_t at, int64_t n, dim3 grid) {
        const Rows kr{k.p + at * k.token, k.token, k.head}, vr{v.p + at * v.token, v.token, v.head};
        with_variant(c, [&](auto bits, auto dim, auto f16) {
            hipLaunchKernelGGL((kv_write_kernel<decltype(bits)::value, decltype(dim)::value, decltype(f16)::value>), grid, dim3(kThreads), 0,
                               stream, kr, vr, n, slots + at, kv_pages(c));
        });
    });
}

hipError_t launch_kv_read(const any4_kv_cache& c, const int64_t* slots, int64_t tokens, uint16_t* k, uint16_t* v, hipStream_t stream) {
    return launch_tokens(c, tokens, [&](int64_t at, int64_t n, dim3 grid) {
        const int64_t to = at * c.kv_heads * c.head_dim;
        with_variant(c, [&](auto bits, auto dim, auto f16) {
            hipLaunchKernelGGL((kv_read_kernel<decltype(bits)::value, decltype(dim)::value, decltype(f16)::value>), grid, dim3(kThreads), 0,
                               stream, kv_pages(c), slots + at, n, k + to, v + to);
        });
    });
}

}  // namespace any4
