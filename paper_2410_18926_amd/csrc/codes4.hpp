// Codes of the 4-bit store (include/lorann_states4.h) and what they become on the way to the matrix cores.
//
// A row is held as step * r_g * code: a float step for the row, for each 32 values a factor r_g = (1 + m / 8) 2^e <= 1 in a byte (a binary16 number without its sign and
// its last seven bits), and codes of a sign and the magnitudes 0, 1/2, 1, 3/2, 2, 3, 4, 6.  r_g * code has at most six significant bits and lies within 2^-14 .. 6, so it is
// formed exactly in binary16; the step is applied to the products, in float, as the 8-bit store's is.
#pragma once
#include "states_store.hpp"

namespace lorann {

// Eight codes as binary16, in the order of their nibbles.
__device__ __forceinline__ f16x8 codes4_to_half(uint32_t w) {
    union { f16x2 p[4]; f16x8 h; } x;
    x.p[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 0);
    x.p[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 1);
    x.p[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 2);
    x.p[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 3);
    return x.h;
}

// Byte `g` of a row's factors as binary16, in both halves of a register.  A factor's top bit is 0: it is cleared, so that memory that was never written gives finite numbers too (a weight
// of 0 times one is 0; the masked keys' steps are not used).
__device__ __forceinline__ uint32_t factor_pair(uint32_t factors, uint32_t g) {
    factors &= 0x7f7f7f7fu;
    return __builtin_amdgcn_perm(0u, factors, 0x000c000cu | g << 8 | g << 24) >> 1;          // (the byte at bits 8 .. 15 of each half, then moved down by one)
}
__device__ __forceinline__ f16x8 spread(uint32_t pair) {
    union { uint32_t u; f16x2 h; } x;
    x.u = pair;
    return f16x8{x.h[0], x.h[1], x.h[0], x.h[1], x.h[0], x.h[1], x.h[0], x.h[1]};
}
__device__ __forceinline__ _Float16 factor_half(uint32_t factors, int g) {
    union { uint16_t u; _Float16 h; } x;
    x.u = (uint16_t)((factors >> (8 * g) & 127u) << 7);
    return x.h;
}

// A row of the values' codes holds two components of a token in a byte.  Eight tokens, w0 the first four: the two components' codes, tokens in the order of token_place.
__device__ __forceinline__ void split_values4(uint32_t w0, uint32_t w1, uint32_t& low, uint32_t& high) {
    low = (w0 & 0x0f0f0f0fu) | (w1 << 4 & 0xf0f0f0f0u);
    high = (w0 >> 4 & 0x0f0f0f0fu) | (w1 & 0xf0f0f0f0u);
}
// Where token t of eight comes to lie: 0, 4, 1, 5, 2, 6, 3, 7.
__device__ __forceinline__ constexpr int token_place(int t) { return 2 * (t & 3) + (t >> 2); }

}  // namespace lorann
