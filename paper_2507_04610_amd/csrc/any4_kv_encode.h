// How a cache of 8 or 4 bits holds a head's vector, for the kernels that write into it.
#pragma once
#include "any4_attn.h"

namespace any4 {

// Scale and offset of the values x[0 .. 7] of LANES lanes, and this lane's codes: section 2.5.1's asymmetric grid, with the
// scale and offset that the readers will use (rounded to bf16 first), as any4_quantize scales its groups.  The quotient is
// the IEEE one: the code nearest to (x - offset) / scale, ties to even.
template <int BITS, int LANES>
__device__ __forceinline__ u32x2 encode(const float (&x)[8], uint32_t& scale_offset) {
    constexpr float kTop = (float)((1 << BITS) - 1);
    float lo = x[0], hi = x[0];
    bool finite = true;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        lo = fminf(lo, x[j]);
        hi = fmaxf(hi, x[j]);
        finite &= fabsf(x[j]) < __builtin_inff();
    }
    // (a value that is not finite reaches all lanes of the vector as hi = inf)
    lo = lanes_reduce<LANES>(lo, [](float a, float b) { return fminf(a, b); });
    hi = lanes_reduce<LANES>(finite ? hi : __builtin_inff(), [](float a, float b) { return fmaxf(a, b); });
    uint32_t sb = f32_to_bf16((hi - lo) / kTop);
    const uint32_t ob = f32_to_bf16(lo);
    if ((sb & 0x7F80u) == 0x7F80u) {                        // nothing to hold such a vector in: it reads back as NaN
        scale_offset = 0x7FC07FC0u;
        return u32x2{0u, 0u};
    }
    if (sb == 0u) sb = 0x3F80u;                             // a constant vector: any scale will do
    scale_offset = sb | (ob << 16);
    const float s = bf16_to_f32(sb), o = bf16_to_f32(ob);
    u32x2 w = {0u, 0u};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t c = (uint32_t)fminf(fmaxf(rintf((x[j] - o) / s), 0.0f), kTop);
        if constexpr (BITS == 8) w[j >> 2] |= c << (8 * (j & 3));
        else w[0] |= c << (4 * j);
    }
    return w;
}

template <bool F16> __device__ __forceinline__ void widen(const u32x4& a, float (&x)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[2 * j] = h16lo_to_f32<F16>(a[j]);
        x[2 * j + 1] = h16hi_to_f32<F16>(a[j]);
    }
}

// calls f with the variant's bits, head_dim and type as compile-time values; 16 bits are the same words in either type
template <class F> inline void with_variant(const any4_kv_cache& c, F f) {
    auto dims = [&](auto bits, auto f16) {
        if (c.head_dim == 128) f(bits, std::integral_constant<int, 128>{}, f16);
        else f(bits, std::integral_constant<int, 64>{}, f16);
    };
    auto types = [&](auto bits) {
        if (c.f16) dims(bits, std::true_type{});
        else dims(bits, std::false_type{});
    };
    if (c.bits == 16) dims(std::integral_constant<int, 16>{}, std::false_type{});
    else if (c.bits == 8) types(std::integral_constant<int, 8>{});
    else types(std::integral_constant<int, 4>{});
}

}  // namespace any4
