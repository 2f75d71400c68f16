// The paged 8-bit state store: layout, element types, quantising a token's keys and values into its slot, reading them back.
//
// A row x (one token, one head, keys or values) is held as codes rint(127 x / a), a = max|x|, with the step a / 127 in float.
#pragma once
#include "common.hpp"

namespace lorann {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// Device view of the store (include/lorann_states.h).  Offsets are formed in 64 bits: a store may pass 2^31 codes.
struct Store {
    int8_t *kc, *vc;
    float *ks, *vs;
    int64_t pages;
    int32_t heads, shift;      // page size = 1 << shift

    __device__ __forceinline__ int64_t row(int64_t page, int head) const { return (page * heads + head) << shift; }   // first token's place in the scales
};

// Rows below this are held as zeros (the reciprocal of their maximum would not be a normal float).
constexpr float kTinyRow = 0x1p-100f;
// Rows above this are scaled down by a power of two before they are multiplied by 127 (which would overflow); their codes are the same.
constexpr float kHugeRow = 0x1p100f, kHugeDown = 0x1p-30f;

struct TokenRows {             // rows of `dim` consecutive elements, distances in elements
    void* p;
    int64_t token, head;
    bool wide;                 // every row starts at a multiple of 16 bytes
};

// Eight consecutive elements as floats, and back (each rounded once).
template <typename T> struct Eight;
template <> struct Eight<float> {
    static __device__ __forceinline__ void load(const float* p, bool wide, float (&f)[8]) {
        if (wide) {
            const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) { f[j] = a[j]; f[4 + j] = b[j]; }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = p[j];
        }
    }
    static __device__ __forceinline__ void store(float* p, bool wide, const float (&f)[8]) {
        if (wide) {
            *(f32x4*)p = f32x4{f[0], f[1], f[2], f[3]};
            *(f32x4*)(p + 4) = f32x4{f[4], f[5], f[6], f[7]};
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] = f[j];
        }
    }
};
template <typename T> struct Eight {
    typedef T T8 __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ void load(const T* p, bool wide, float (&f)[8]) {
        if (wide) {
            const T8 v = *(const T8*)p;
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = (float)v[j];
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = (float)p[j];
        }
    }
    static __device__ __forceinline__ void store(T* p, bool wide, const float (&f)[8]) {
        if (wide) {
            T8 v;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = (T)f[j];
            *(T8*)p = v;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] = (T)f[j];
        }
    }
};

// A block of the two kernels below has 64 consecutive tokens of one head, keys (blockIdx.z 0) or values (1).  Rows are handled 8 elements to a thread; keys
// go straight between the caller's rows and the store's.  Values change places in LDS, [component][token]: in the store the tokens of a component lie
// together, so tokens whose slots follow each other are moved together - 16 at a time where 16 tokens fill an aligned 16-slot group, else 4 at a
// time, else one by one.  `follows`, bit t: token t + 1 has the slot after token t's.
constexpr int kBlockTokens = 64;

struct SlotRuns {
    uint64_t by16, by4, by1;       // first tokens of groups of 16 and of 4, and single tokens
};
__device__ __forceinline__ SlotRuns find_runs(int64_t slot, bool have, uint64_t follows) {
    // bit t of r2, r4, ...: the slots of 2, 4, ... tokens from t on follow each other
    const uint64_t r2 = follows, r4 = r2 & r2 >> 1 & r2 >> 2, r8 = r4 & r4 >> 4 & r2 >> 3, r16 = r8 & r8 >> 8 & r2 >> 7;
    SlotRuns r;
    r.by16 = __ballot(have && (slot & 15) == 0) & r16;
    uint64_t taken = r.by16;
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) taken |= taken << o;
    r.by4 = __ballot(have && (slot & 3) == 0) & r4 & ~taken;
    uint64_t four = r.by4;
    four |= four << 1;
    four |= four << 2;
    r.by1 = __ballot(have) & ~taken & ~four;
    return r;
}

constexpr int kTokenStride = kBlockTokens + 4;     // bytes between components in LDS: 17 words, so that neither walk meets one bank

// Slots of the block's tokens, their runs, and the list of groups to move; every thread of the block calls it.
struct BlockSlots {
    int64_t slot[kBlockTokens];    // -1: none
    uint8_t first[kBlockTokens];   // first token of each group: the groups of 16, of 4, the single tokens
    int n16, n4, n1;
};
__device__ __forceinline__ void load_slots(BlockSlots& b, const Store& st, const int64_t* __restrict__ slots, int64_t token0, int64_t tokens, bool runs) {
    if (threadIdx.x < 64) {
        const int t = threadIdx.x;
        int64_t s = token0 + t < tokens ? slots[token0 + t] : -1;
        const bool have = (uint64_t)s < (uint64_t)(st.pages << st.shift);
        if (!have) s = -1;
        b.slot[t] = s;
        if (runs) {
            const int64_t after = __shfl_down(s, 1, 64);
            const SlotRuns r = find_runs(s, have, __ballot(t < 63 && have && after == s + 1));
            const uint64_t below = (1ull << t) - 1;
            b.n16 = __popcll(r.by16);
            b.n4 = __popcll(r.by4);
            b.n1 = __popcll(r.by1);
            if (r.by16 >> t & 1) b.first[__popcll(r.by16 & below)] = t;
            if (r.by4 >> t & 1) b.first[b.n16 + __popcll(r.by4 & below)] = t;
            if (r.by1 >> t & 1) b.first[b.n16 + b.n4 + __popcll(r.by1 & below)] = t;
        }
    }
    __syncthreads();
}

// A word of four bytes from any byte address in LDS (two aligned words, shifted).
__device__ __forceinline__ uint32_t any_word(const uint8_t* p) {
    const uint32_t a = (uint32_t)(uintptr_t)p & 3;
    const uint32_t* w = (const uint32_t*)(p - a);
    return __builtin_amdgcn_alignbyte(w[1], w[0], a);
}

// One rounded division per value would be most of the kernel's time: rint(127 x / top) is formed as rint(q) with q = 127 x * (1 / top), and the quotient is
// divided only where q lies within 2^-10 of a half, where an error of q (below 2^-15: three roundings of 2^-24 relative, |q| <= 127) could decide.
__device__ __forceinline__ float code_of(float x, float top, float inverse) {
    const float p = x * 127.0f, q = p * inverse, r = rintf(q);
    return fabsf(fabsf(q - r) - 0.5f) < 0x1p-10f ? rintf(p / top) : r;
}

template <typename T>
__global__ void __launch_bounds__(256) k_states_write(Store st, TokenRows k, TokenRows v, const int64_t* __restrict__ slots, int64_t tokens, int dim) {
    __shared__ BlockSlots bs;
    __shared__ __align__(16) uint8_t lds[128 * kTokenStride + 16];
    const int64_t token0 = (int64_t)blockIdx.x * kBlockTokens;
    const int head = blockIdx.y;
    const bool values = blockIdx.z;
    load_slots(bs, st, slots, token0, tokens, values);
    const TokenRows in = values ? v : k;
    const int lane = threadIdx.x & 15, d = lane * 8, P = 1 << st.shift;
    // a group of 16 lanes per row, 16 rows at a time: all rows are requested before the first is used
    float f[4][8];
    const T* x = (const T*)in.p + token0 * in.token + head * in.head;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = i * 16 + (threadIdx.x >> 4);
        if (d < dim && bs.slot[t] >= 0) Eight<T>::load(x + t * in.token + d, in.wide, f[i]);
        else {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[i][j] = 0.0f;
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = i * 16 + (threadIdx.x >> 4);
        float top = 0.0f;
        bool bad = false;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            bad |= !(fabsf(f[i][j]) <= 3.4028235e38f);
            top = fmaxf(top, fabsf(f[i][j]));
        }
        if (bad) top = INFINITY;                               // (the maximum of the row, unless a value of it is no number: then infinity)
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 16));
        bad = top == INFINITY;
        const bool zero = bad || top < kTinyRow;
        const float keep = top > kHugeRow ? kHugeDown : 1.0f, low = top * keep, inverse = zero ? 0.0f : 1.0f / low;
        union { int8_t c[8]; uint2 u; } code;
#pragma unroll
        for (int j = 0; j < 8; ++j) code.c[j] = zero ? (int8_t)0 : (int8_t)code_of(f[i][j] * keep, low, inverse);
        const int64_t slot = bs.slot[t];
        if (slot < 0) continue;
        const int64_t base = st.row(slot >> st.shift, head);
        const int off = (int)(slot & (P - 1));
        if (lane == 0) (values ? st.vs : st.ks)[base + off] = bad ? __int_as_float(0x7fc00000) : zero ? 0.0f : top / 127.0f;
        if (d >= dim) continue;
        if (!values) *(uint2*)(st.kc + (base + off) * dim + d) = code.u;
        else {
#pragma unroll
            for (int j = 0; j < 8; ++j) lds[(d + j) * kTokenStride + t] = (uint8_t)code.c[j];
        }
    }
    if (!values) return;
    __syncthreads();
    auto place = [&](int t, int comp) {
        const int64_t slot = bs.slot[t];
        return st.vc + st.row(slot >> st.shift, head) * dim + ((int64_t)comp << st.shift) + (slot & (P - 1));
    };
    for (int i = threadIdx.x; i < bs.n16 * dim; i += 256) {
        const int comp = i / bs.n16, t = bs.first[i - comp * bs.n16];
        const uint8_t* p = &lds[comp * kTokenStride + t];
        *(i32x4*)place(t, comp) = i32x4{(int)any_word(p), (int)any_word(p + 4), (int)any_word(p + 8), (int)any_word(p + 12)};
    }
    for (int i = threadIdx.x; i < bs.n4 * dim; i += 256) {
        const int comp = i / bs.n4, t = bs.first[bs.n16 + i - comp * bs.n4];
        *(uint32_t*)place(t, comp) = any_word(&lds[comp * kTokenStride + t]);
    }
    for (int i = threadIdx.x; i < bs.n1 * dim; i += 256) {
        const int comp = i / bs.n1, t = bs.first[bs.n16 + bs.n4 + i - comp * bs.n1];
        *place(t, comp) = (int8_t)lds[comp * kTokenStride + t];
    }
}

template <typename T>
__global__ void __launch_bounds__(256) k_states_read(Store st, const int64_t* __restrict__ slots, int64_t tokens, TokenRows k, TokenRows v, int dim) {
    __shared__ BlockSlots bs;
    __shared__ __align__(16) uint8_t lds[128 * kTokenStride + 16];
    const int64_t token0 = (int64_t)blockIdx.x * kBlockTokens;
    const int head = blockIdx.y;
    const bool values = blockIdx.z;
    const TokenRows to = values ? v : k;
    if (!to.p) return;
    load_slots(bs, st, slots, token0, tokens, values);
    const int lane = threadIdx.x & 15, d = lane * 8, P = 1 << st.shift;
    if (values) {
        auto place = [&](int t, int comp) {
            const int64_t slot = bs.slot[t];
            return st.vc + st.row(slot >> st.shift, head) * dim + ((int64_t)comp << st.shift) + (slot & (P - 1));
        };
        for (int i = threadIdx.x; i < bs.n16 * dim; i += 256) {
            const int comp = i / bs.n16, t = bs.first[i - comp * bs.n16];
            union { i32x4 w; uint8_t b[16]; } x;
            x.w = *(const i32x4*)place(t, comp);
            uint8_t* p = &lds[comp * kTokenStride + t];
            if ((t & 3) == 0) {
#pragma unroll
                for (int j = 0; j < 4; ++j) ((uint32_t*)p)[j] = (uint32_t)x.w[j];
            } else {
#pragma unroll
                for (int j = 0; j < 16; ++j) p[j] = x.b[j];
            }
        }
        for (int i = threadIdx.x; i < bs.n4 * dim; i += 256) {
            const int comp = i / bs.n4, t = bs.first[bs.n16 + i - comp * bs.n4];
            union { uint32_t w; uint8_t b[4]; } x;
            x.w = *(const uint32_t*)place(t, comp);
            uint8_t* p = &lds[comp * kTokenStride + t];
#pragma unroll
            for (int j = 0; j < 4; ++j) p[j] = x.b[j];
        }
        for (int i = threadIdx.x; i < bs.n1 * dim; i += 256) {
            const int comp = i / bs.n1, t = bs.first[bs.n16 + bs.n4 + i - comp * bs.n1];
            lds[comp * kTokenStride + t] = (uint8_t)*place(t, comp);
        }
        __syncthreads();
    }
    if (d >= dim) return;
    T* x = (T*)to.p + token0 * to.token + head * to.head;
    uint2 code[4];
    float step[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = i * 16 + (threadIdx.x >> 4);
        const int64_t slot = bs.slot[t];
        const int64_t base = slot < 0 ? 0 : st.row(slot >> st.shift, head);
        const int off = slot < 0 ? 0 : (int)(slot & (P - 1));
        step[i] = (values ? st.vs : st.ks)[base + off];         // (of some token where there is none)
        code[i] = uint2{0, 0};
        if (!values) code[i] = *(const uint2*)(st.kc + (base + off) * dim + d);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = i * 16 + (threadIdx.x >> 4);
        if (token0 + t >= tokens) break;
        union { int8_t c[8]; uint2 u; } c;
        c.u = code[i];
        if (values) {
#pragma unroll
            for (int j = 0; j < 8; ++j) c.c[j] = (int8_t)lds[(d + j) * kTokenStride + t];
        }
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            f[j] = bs.slot[t] < 0 ? 0.0f : step[i] * (float)c.c[j];
            asm("" : "+v"(f[j]));          // rounded to float here: product and conversion in one instruction would round once, from the exact product
        }
        Eight<T>::store(x + t * to.token + d, to.wide, f);
    }
}

}  // namespace lorann
