// What the kernels share that attend to tiles of 64 keys in LDS: how a tile lies there and how it is read, and the running maximum's constants.
#pragma once
#include "any4_attn.h"

namespace any4 {

constexpr int kKeys = 64;
constexpr float kSlack = 8.0f;            // a maximum in use may be exceeded by 2^kSlack
constexpr float kFar = 1048576.0f;        // 2^20: up to there a maximum's rounding moves the exponents by 2^-4 at most, for all keys of a query alike

#pragma clang diagnostic ignored "-Wint-to-pointer-cast"          // LDS offsets as pointers
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) u32x4* lds_u4;
typedef __attribute__((address_space(3))) u32x2* lds_u2;
typedef __attribute__((address_space(3))) s16x4* lds_s4;

// 4 rows x 16 columns: lane i of 16 gives the address of row i / 4, columns 4 * (i % 4) .., and gets column i of the four rows
__device__ __forceinline__ u32x2 lds_read_transposed(uint32_t at) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(at)));
}

// the part of a tile that a wavefront copies: 16-byte pieces, 64 an instruction
template <int D, int WAVES> struct Tile {
    static constexpr int kRow = 2 * D, kBytes = kKeys * kRow, kPieces = D / 8, kRows = 64 / kPieces;     // rows an instruction
    static constexpr int kCopies = kKeys / kRows / WAVES;                                                // of a wavefront
    __device__ static __forceinline__ int swizzle_k(int row) { return D == 128 ? row & 15 : (row >> 1) & 7; }
    __device__ static __forceinline__ int swizzle_v(int row) { return D == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2; }
};

}  // namespace any4
