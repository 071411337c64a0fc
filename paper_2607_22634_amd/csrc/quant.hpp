// The 4-bit cache format: 32 values of a row share an exponent byte E and are
// e2m1 codes times 2^(E - 127).  gfx950 converts both ways, two values per
// instruction, with the shared exponent as the exponent field of an fp32 scale.
#pragma once

#include "common.hpp"

namespace presto {
namespace quant {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kNanExp = 255;  // a group that is not finite
constexpr int kLeastExp = 7, kMostExp = 252;  // (6 * 2^126 would not be an fp32 or bf16)

// A block is 16 positions of one KV head: codes, then exponents.
__host__ __device__ constexpr int block_bytes(int dim) { return 17 * dim / 2; }
__host__ __device__ constexpr int code_bytes(int dim) { return 8 * dim; }

// Offsets in a block.  K: the codes of a position are in order; V: position
// 4 g + i and value x = (dim / 16) n + y have their code in [g][n][i][y / 2].
template <int D>
__device__ __forceinline__ int k_code_at(int r, int x) { return r * (D / 2) + x / 2; }
template <int D>
__device__ __forceinline__ int k_exp_at(int r, int x) { return 8 * D + r * (D / 32) + x / 32; }
template <int D>
__device__ __forceinline__ int v_code_at(int r, int x) {
    constexpr int PER = D / 16;
    return (((r >> 2) * 16 + x / PER) * 4 + (r & 3)) * (PER / 2) + (x % PER) / 2;
}
template <int D>
__device__ __forceinline__ int v_exp_at(int r, int x) { return 8 * D + ((r >> 2) * (D / 32) + x / 32) * 4 + (r & 3); }

// The exponent byte of a group with this largest magnitude: the least from
// kLeastExp on with 7 * 2^(E - 127) >= top, kMostExp at most.  7 = 1.75 * 2^2.
__device__ __forceinline__ int group_exp(float top) {
    const uint32_t u = __float_as_uint(top);
    const int e = (int)(u >> 23), m = (int)(u & 0x7fffffu);
    if (e == 255) return kNanExp;
    return min(max(e - (m <= 0x600000 ? 2 : 1), kLeastExp), kMostExp);
}

__device__ __forceinline__ float exp_scale(int e) { return __uint_as_float((uint32_t)e << 23); }

// Eight values as codes, the first in the low nibble.
__device__ __forceinline__ uint32_t encode8(const float v[8], int e) {
    if (e == kNanExp) return 0;
    const float s = exp_scale(e);
    uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[0], v[1], s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], s, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], s, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], s, 3);
}

// The other way: values as pairs of bf16, which holds them exactly.
template <int B>
__device__ __forceinline__ uint32_t decode2(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, B));
}

}  // namespace quant
}  // namespace presto
