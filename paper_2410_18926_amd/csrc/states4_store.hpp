// Quantising a token's keys and values into a slot of the 4-bit store, and reading them back.  Format in codes4.hpp.
#pragma once
#include "codes4.hpp"

namespace lorann {

// The largest of four lanes (a quarter of a row of 16) in each of them.
__device__ __forceinline__ uint32_t quad_max_u32(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, true));       // quad_perm 1 0 3 2
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, true));       // quad_perm 2 3 0 1
    return v;
}
__device__ __forceinline__ uint32_t other_pair(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, true); }

// The smallest r = (1 + m / 8) 2^e >= 2^-13 with r * top >= group, as a float's bits; inv = 1 / top within a few units of the last place.  A quotient surely not above the exact one is
// rounded upwards to four bits: that is r or the number below it, which the product shows (the sign of a fused sum is exact).
__device__ __forceinline__ uint32_t factor_bits(float group, float top, float inv) {
    const uint32_t q = max(__float_as_uint(group * inv * (1.0f - 0x1p-20f)), 0x39000000u);
    const uint32_t r = (q + 0xfffffu) & 0xfff00000u;
    return fmaf(__uint_as_float(r), top, -group) < 0.0f ? r + 0x100000u : r;
}

// top / 6, rounded as a division rounds: the product with the rounded reciprocal, corrected by its remainder once (top is 2^-100 or more).
__device__ __forceinline__ float sixth(float top) {
    const float q = top * (1.0f / 6.0f);
    return fmaf(fmaf(-q, 6.0f, top), 1.0f / 6.0f, q);
}

// Eight consecutive elements of a row, and the bits of the largest magnitude among them as a float: infinities and NaN are above every number.  16-bit elements are compared two at a time as
// they stand.
template <typename T>
struct Row8 {                                  // 16-bit elements, two to a register
    i32x4 raw;
    __device__ __forceinline__ void load(const T* p, bool wide) { raw = load8_raw(p, 0, wide); }
    __device__ __forceinline__ void clear() { raw = i32x4{0, 0, 0, 0}; }
    __device__ __forceinline__ uint32_t largest() const {
        typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
        u16x2 m = {0, 0};
#pragma unroll
        for (int j = 0; j < 4; ++j) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, (uint32_t)raw[j] & 0x7fff7fffu));
        return __float_as_uint(Bits16<T>::widen(max(m[0], m[1])));
    }
    __device__ __forceinline__ void values(float (&f)[8]) const { widen8<T>(raw, f); }
};
template <>
struct Row8<float> {
    float f[8];
    __device__ __forceinline__ void load(const float* p, bool wide) { Eight<float>::load(p, wide, f); }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = 0.0f;
    }
    __device__ __forceinline__ uint32_t largest() const {
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(f[j]) & 0x7fffffffu);
        return m;
    }
    __device__ __forceinline__ void values(float (&to)[8]) const {
#pragma unroll
        for (int j = 0; j < 8; ++j) to[j] = f[j];
    }
};

// Eight codes of a row: nearest to 6 x / (r top), halfway to the even code, exactly.
//   16-bit elements: 6 x (14 bits) and r top (15 bits) are exact floats.  The quotient is corrected by its remainder once, so that it is off by at most 2^-23 relative and is
//   the halfway point itself where the exact quotient is: other quotients lie 2^-19 away from those (of 3 bits) or more.
//   float: a quotient within 2^-21 of a halfway point is decided by the exact products 24 |x| and n r top in double.
template <typename T>
__device__ __forceinline__ uint32_t codes4_of(const float (&x)[8], float r, float top) {
    uint32_t c = 0;
    if constexpr (sizeof(T) == 2) {
        const float keep = top > kHugeRow ? kHugeDown : 1.0f, unit = r * (top * keep), inv = __builtin_amdgcn_rcpf(unit);
        float q[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float y = x[j] * (6.0f * keep), q0 = y * inv;
            q[j] = fmaf(-fmaf(q0, unit, -y), inv, q0);          // (the remainder's signs so that -0 stays -0: -0 unit + 0 = +0, and -0 inv - 0 = -0)
        }
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, q[0], q[1], 1.0f, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, q[2], q[3], 1.0f, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, q[4], q[5], 1.0f, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, q[6], q[7], 1.0f, 3);
    } else {
        const float keep = top > kHugeRow ? kHugeDown : 1.0f, scale = 6.0f / (r * (top * keep)) * keep;
        float lo[8], hi[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float q = x[j] * scale;
            lo[j] = q * (1.0f - 0x1p-21f);
            hi[j] = q * (1.0f + 0x1p-21f);
        }
        uint32_t d = 0;
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, lo[0], lo[1], 1.0f, 0);
        d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(d, hi[0], hi[1], 1.0f, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, lo[2], lo[3], 1.0f, 1);
        d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(d, hi[2], hi[3], 1.0f, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, lo[4], lo[5], 1.0f, 2);
        d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(d, hi[4], hi[5], 1.0f, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, lo[6], lo[7], 1.0f, 3);
        d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(d, hi[6], hi[7], 1.0f, 3);
        if (c != d) {
            const double unit = (double)r * (double)top;
            c = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const double t = 24.0 * fabs((double)x[j]);
                const uint32_t n = (t > unit) + (t >= 3 * unit) + (t > 5 * unit) + (t >= 7 * unit) + (t > 10 * unit) + (t >= 14 * unit) + (t > 20 * unit);
                c |= (n | (__float_as_uint(x[j]) >> 28 & 8u)) << (4 * j);
            }
        }
    }
    return c;
}

// Four nibbles of the low half of a word as four bytes, and back.
__device__ __forceinline__ uint32_t nibbles_apart(uint32_t x) {
    x &= 0xffffu;
    x = (x | x << 8) & 0x00ff00ffu;
    return (x | x << 4) & 0x0f0f0f0fu;
}
__device__ __forceinline__ uint32_t nibbles_together(uint32_t x) {
    x &= 0x0f0f0f0fu;
    x = (x | x >> 4) & 0x00ff00ffu;
    return (x | x >> 8) & 0xffffu;
}

// Of the 16 lanes of a row, lane l holds the codes of components 8 l .. 8 l + 7 (one nibble each); as rows of the values' codes (components 32 g + n and 32 g + 16 + n in byte 16 g + n)
// the same lane holds the four bytes from value_row(l) on: its quad's other pair has the other nibbles.
__device__ __forceinline__ int value_row(int l) { return (l >> 2) * 16 + (l & 1) * 8 + (l >> 1 & 1) * 4; }
__device__ __forceinline__ uint32_t to_value_rows(uint32_t own, int l) {
    const uint32_t other = other_pair(own);
    return l & 2 ? nibbles_apart(other >> 16) | nibbles_apart(own >> 16) << 4 : nibbles_apart(own) | nibbles_apart(other) << 4;
}
__device__ __forceinline__ uint32_t from_value_rows(uint32_t own, int l) {
    const uint32_t other = other_pair(own);
    return l & 2 ? nibbles_together(other >> 4) | nibbles_together(own >> 4) << 16 : nibbles_together(own) | nibbles_together(other) << 16;
}

// Blocks, runs of slots and the turning of the values are those of the 8-bit store's kernels (states_store.hpp); a row of the values has dim / 2 bytes.  Two rows of a thread (16 tokens
// apart) are turned together: afterwards lane L holds, for the first of them in the lower half of the wavefront and for the second in the upper, the four tokens' bytes of two rows.
__device__ __forceinline__ int turned_row(int lane) { return value_row(lane & 15) + (lane >> 4 & 1) * 2; }

// Blocks: the heads' keys, then their values, of 64 tokens, then those of the next tokens: rows of a token lie side by side in the caller's projection (50000 tokens of 8 heads of 128, slices of
// one of 48 heads: 93 us with the token blocks first, 73 so; reading back, where whole rows are written, 60 and 65).
template <typename T>
__global__ void __launch_bounds__(256) k_states4_write(Store st, TokenRows k, TokenRows v, const int64_t* __restrict__ slots, int64_t tokens, int dim) {
    __shared__ BlockSlots bs;
    __shared__ __align__(16) uint8_t lds[64 * kTokenStride + 16];
    const int64_t token0 = ((int64_t)blockIdx.z * gridDim.y + blockIdx.y) * kBlockTokens;
    const bool values = blockIdx.x >= (unsigned)st.heads;
    const int head = blockIdx.x - (values ? st.heads : 0);
    if (token0 >= tokens) return;
    const TokenRows in = values ? v : k;
    const int lane = threadIdx.x & 15, d = lane * 8, P = 1 << st.shift, half = dim / 2;
    const int last = (int)min(tokens - 1 - token0, (int64_t)kBlockTokens - 1);
    // a group of 16 lanes per row, 16 rows at a time: all rows are requested first, without regard to their slots
    Row8<T> f[4];
    {
        const T* x = (const T*)in.p + token0 * in.token + head * in.head + (d < dim ? d : 0);
        const int t = threadIdx.x >> 4;
        if (last >= 16) {
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i].load(x + min(i * 16 + t, last) * in.token, in.wide);
        } else {                                               // (a few tokens: one row a group)
            f[0].load(x + min(t, last) * in.token, in.wide);
#pragma unroll
            for (int i = 1; i < 4; ++i) f[i].clear();
        }
    }
    load_slots(bs, st, slots, token0, tokens, values);
    if (d >= dim) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i].clear();
    }
    uint32_t code[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        code[i] = 0;
        if (i > 0 && last < 16) continue;
        const int t = i * 16 + (threadIdx.x >> 4);
        const uint32_t group = quad_max_u32(f[i].largest()), most = row_max_u32(group);
        const bool bad = most >= 0x7f800000u, zero = bad || __uint_as_float(most) < kTinyRow;
        const float top = zero ? 1.0f : __uint_as_float(most);
        // (above 2^126 the reciprocal would not be a normal float: both are scaled down by the same power of two, which leaves their ratio; a group that this makes inexact is below every factor)
        const float keep = top > kHugeRow ? kHugeDown : 1.0f, low = top * keep;
        const uint32_t r = factor_bits(zero ? 0.0f : __uint_as_float(group) * keep, low, __builtin_amdgcn_rcpf(low));
        float x[8];
        f[i].values(x);
        code[i] = zero ? 0u : codes4_of<T>(x, __uint_as_float(r), top);
        uint32_t factors = d < dim ? ((r >> 20) - 896u) << (8 * (lane >> 2)) : 0u;            // (the exponent moves from a float's offset to binary16's)
        factors |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)factors, 0x128, 0xf, 0xf, true);
        factors |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)factors, 0x124, 0xf, 0xf, true);
        const int64_t slot = bs.slot[t];
        if (slot >= 0) {
            const int64_t base = st.row(slot >> st.shift, head);
            const int off = (int)(slot & (P - 1));
            if (lane == 0) {
                (values ? st.vs : st.ks)[base + off] = bad ? __int_as_float(0x7fc00000) : zero ? 0.0f : sixth(top);
                (values ? st.vf : st.kf)[base + off] = factors;
            }
            if (!values && d < dim) *(uint32_t*)(st.kc + (base + off) * half + d / 2) = code[i];
        }
    }
    if (!values) return;
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
        uint32_t lo = to_value_rows(code[i], lane), hi = to_value_rows(code[i + 1], lane);
        turn(lo, hi);
        const int wl = threadIdx.x & 63, row = turned_row(wl), t0 = (i + (wl >> 5)) * 16 + (threadIdx.x >> 6) * 4;
        if (row < half) {
            *(uint32_t*)&lds[row * kTokenStride + t0] = lo;
            *(uint32_t*)&lds[(row + 1) * kTokenStride + t0] = hi;
        }
    }
    __syncthreads();
    auto place = [&](int t, int row) {
        const int64_t slot = bs.slot[t];
        return st.vc + st.row(slot >> st.shift, head) * half + ((int64_t)row << st.shift) + (slot & (P - 1));
    };
    for (int i = threadIdx.x; i < bs.n16 * half; i += 256) {
        const int row = i / bs.n16, t = bs.first[i - row * bs.n16];
        const uint8_t* p = &lds[row * kTokenStride + t];
        *(i32x4*)place(t, row) = i32x4{(int)any_word(p), (int)any_word(p + 4), (int)any_word(p + 8), (int)any_word(p + 12)};
    }
    for (int i = threadIdx.x; i < bs.n4 * half; i += 256) {
        const int row = i / bs.n4, t = bs.first[bs.n16 + i - row * bs.n4];
        *(uint32_t*)place(t, row) = any_word(&lds[row * kTokenStride + t]);
    }
    for (int i = threadIdx.x; i < bs.n1 * half; i += 256) {
        const int row = i / bs.n1, t = bs.first[bs.n16 + bs.n4 + i - row * bs.n1];
        *place(t, row) = (int8_t)lds[row * kTokenStride + t];
    }
}

template <typename T>
__global__ void __launch_bounds__(256) k_states4_read(Store st, const int64_t* __restrict__ slots, int64_t tokens, TokenRows k, TokenRows v, int dim) {
    __shared__ BlockSlots bs;
    __shared__ __align__(16) uint8_t lds[64 * kTokenStride + 16];
    const int64_t token0 = (int64_t)blockIdx.x * kBlockTokens;
    const int head = blockIdx.y;
    const bool values = blockIdx.z;
    const TokenRows to = values ? v : k;
    if (!to.p) return;
    load_slots(bs, st, slots, token0, tokens, values);
    const int lane = threadIdx.x & 15, d = lane * 8, P = 1 << st.shift, half = dim / 2;
    if (values) {
        auto place = [&](int t, int row) {
            const int64_t slot = bs.slot[t];
            return st.vc + st.row(slot >> st.shift, head) * half + ((int64_t)row << st.shift) + (slot & (P - 1));
        };
        for (int i = threadIdx.x; i < bs.n16 * half; i += 256) {
            const int row = i / bs.n16, t = bs.first[i - row * bs.n16];
            union { i32x4 w; uint8_t b[16]; } x;
            x.w = *(const i32x4*)place(t, row);
            uint8_t* p = &lds[row * kTokenStride + t];
            if ((t & 3) == 0) {
#pragma unroll
                for (int j = 0; j < 4; ++j) ((uint32_t*)p)[j] = (uint32_t)x.w[j];
            } else {
#pragma unroll
                for (int j = 0; j < 16; ++j) p[j] = x.b[j];
            }
        }
        for (int i = threadIdx.x; i < bs.n4 * half; i += 256) {
            const int row = i / bs.n4, t = bs.first[bs.n16 + i - row * bs.n4];
            union { uint32_t w; uint8_t b[4]; } x;
            x.w = *(const uint32_t*)place(t, row);
            uint8_t* p = &lds[row * kTokenStride + t];
#pragma unroll
            for (int j = 0; j < 4; ++j) p[j] = x.b[j];
        }
        for (int i = threadIdx.x; i < bs.n1 * half; i += 256) {
            const int row = i / bs.n1, t = bs.first[bs.n16 + bs.n4 + i - row * bs.n1];
            lds[row * kTokenStride + t] = (uint8_t)*place(t, row);
        }
        __syncthreads();
    }
    T* x = (T*)to.p + token0 * to.token + head * to.head;
    const int last = (int)min(tokens - 1 - token0, (int64_t)kBlockTokens - 1);
    uint32_t code[4], factors[4];
    float step[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        code[i] = factors[i] = 0;
        step[i] = 0.0f;
        if (i * 16 > last) continue;
        const int t = i * 16 + (threadIdx.x >> 4);
        const int64_t slot = bs.slot[t];
        const int64_t base = slot < 0 ? 0 : st.row(slot >> st.shift, head);
        const int off = slot < 0 ? 0 : (int)(slot & (P - 1));
        step[i] = (values ? st.vs : st.ks)[base + off];         // (of some token where there is none)
        factors[i] = (values ? st.vf : st.kf)[base + off];
        if (!values && d < dim) code[i] = *(const uint32_t*)(st.kc + (base + off) * half + d / 2);
    }
    if (values) {
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            const int wl = threadIdx.x & 63, row = turned_row(wl), t0 = (i + (wl >> 5)) * 16 + (threadIdx.x >> 6) * 4;
            uint32_t lo = 0, hi = 0;
            if (row < half) {
                lo = *(const uint32_t*)&lds[row * kTokenStride + t0];
                hi = *(const uint32_t*)&lds[(row + 1) * kTokenStride + t0];
            }
            turn_back(lo, hi);
            code[i] = from_value_rows(lo, lane);
            code[i + 1] = from_value_rows(hi, lane);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = i * 16 + (threadIdx.x >> 4);
        if (d >= dim || t > last) break;
        const f16x8 c = codes4_to_half(code[i]);
        const float r = (float)factor_half(factors[i], lane >> 2);
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            f[j] = bs.slot[t] < 0 ? 0.0f : step[i] * (r * (float)c[j]);          // (r times a code is exact)
            asm("" : "+v"(f[j]));          // rounded to float here: product and conversion in one instruction would round once, from the exact product
        }
        Eight<T>::store(x + t * to.token + d, to.wide, f);
    }
}

}  // namespace lorann
