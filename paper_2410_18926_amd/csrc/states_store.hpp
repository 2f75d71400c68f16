// The paged 8-bit state store: layout, element types, quantising a token's keys and values into its slot, reading them back.
//
// A row x (one token, one head, keys or values) is held as codes rint(127 x / a), a = max|x|, with the step a / 127 in float.
//
// Writing reads 2 D elements per token and head and writes 2 D + 8 bytes, reading the other way round: both are bound by memory.  Measured: 50000 tokens
// of 8 heads of 128, bfloat16, slots in order within passages of 411 (311 MB): written in 81 us (3.8 TB/s), read back in 72 us (4.3 TB/s); 8 tokens: 4.7 and
// 4.2 us, the latency of slots -> rows -> store.
// Values are stored turned, [component][token]: the second product of the attention contracts over tokens, so 16 tokens of a component are one
// 16-byte load there.  The price is paid here, by writes whose slots do not follow each other: a token alone writes a byte to each of D lines (20000
// tokens in runs of 1 to 5 slots, 8 heads of 128: 663 us, 0.2 TB/s).  Prompts and passages are written in order; a decoding step writes few tokens.
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

// The largest of 16 lanes (a row of the wavefront) in each of them.
__device__ __forceinline__ uint32_t row_max_u32(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xf, 0xf, true));      // rotated by 8, 4, 2, 1 lanes
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xf, 0xf, true));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x122, 0xf, 0xf, true));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x121, 0xf, 0xf, true));
    return v;
}

// Four rows of 16 lanes hold four tokens t .. t + 3, lane l of a row the bytes 8 l .. 8 l + 7 of its token in `lo`, `hi`.  Afterwards `lo`, `hi` hold the four
// tokens' bytes of components turned_component(lane) and the next one; turn_back undoes it.
__device__ __forceinline__ void turn(uint32_t& lo, uint32_t& hi) {
    const auto a = __builtin_amdgcn_permlane32_swap(lo, hi, false, false);     // lower half: bytes 0-3 of tokens r, r + 2; upper half: bytes 4-7
    const uint32_t x = __builtin_amdgcn_perm(a[1], a[0], 0x05010400u), y = __builtin_amdgcn_perm(a[1], a[0], 0x07030602u);
    const auto b = __builtin_amdgcn_permlane16_swap(x, y, false, false);       // even rows: the first two components, of tokens 0, 2 and 1, 3; odd rows: the others
    lo = __builtin_amdgcn_perm(b[1], b[0], 0x05010400u);
    hi = __builtin_amdgcn_perm(b[1], b[0], 0x07030602u);
}
__device__ __forceinline__ void turn_back(uint32_t& lo, uint32_t& hi) {
    const uint32_t x = __builtin_amdgcn_perm(hi, lo, 0x06040200u), y = __builtin_amdgcn_perm(hi, lo, 0x07050301u);
    const auto b = __builtin_amdgcn_permlane16_swap(x, y, false, false);
    const uint32_t p = __builtin_amdgcn_perm(b[1], b[0], 0x06040200u), q = __builtin_amdgcn_perm(b[1], b[0], 0x07050301u);
    const auto a = __builtin_amdgcn_permlane32_swap(p, q, false, false);
    lo = a[0];
    hi = a[1];
}
__device__ __forceinline__ int turned_component(int lane) { return (lane & 15) * 8 + (lane >> 5) * 4 + (lane >> 4 & 1) * 2; }

// Eight codes of a row whose largest magnitude is `top` (finite, not tiny).  The definition divides: rint(127 x / top).  Here q = x * (127 / top), rounded by
// adding 1.5 * 2^23, whose low byte then is the code; where a q lies within 2^-14 of a half, the eight are divided (one wavefront in twenty).  Before rounding, q and the
// definition's quotient are each off by at most two roundings of 2^-24 relative of at most 127: 2^-15 in all.
__device__ __forceinline__ uint2 codes_of(const float (&x)[8], float top) {
    const float scale = 127.0f / top;
    float t[8], worst = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float q = x[j] * scale;
        t[j] = q + 12582912.0f;
        worst = fmaxf(worst, fabsf(q - (t[j] - 12582912.0f)));
    }
    if (worst > 0.5f - 0x1p-14f) {
        const float keep = top > kHugeRow ? kHugeDown : 1.0f, low = top * keep;
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = rintf(x[j] * keep * 127.0f / low) + 12582912.0f;
    }
    uint32_t c[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) c[j] = __builtin_amdgcn_perm(__float_as_uint(t[2 * j + 1]), __float_as_uint(t[2 * j]), 0x0c0c0400u);
    return uint2{c[0] | c[1] << 16, c[2] | c[3] << 16};
}

template <typename T>
__global__ void __launch_bounds__(256) k_states_write(Store st, TokenRows k, TokenRows v, const int64_t* __restrict__ slots, int64_t tokens, int dim) {
    __shared__ BlockSlots bs;
    __shared__ __align__(16) uint8_t lds[128 * kTokenStride + 16];
    const int64_t token0 = (int64_t)blockIdx.x * kBlockTokens;
    const int head = blockIdx.y;
    const bool values = blockIdx.z;
    const TokenRows in = values ? v : k;
    const int lane = threadIdx.x & 15, d = lane * 8, P = 1 << st.shift;
    const int last = (int)min(tokens - 1 - token0, (int64_t)kBlockTokens - 1);
    // a group of 16 lanes per row, 16 rows at a time: all rows are requested first, without regard to their slots
    float f[4][8];
    {
        const T* x = (const T*)in.p + token0 * in.token + head * in.head + (d < dim ? d : 0);
        const int t = threadIdx.x >> 4;
        if (last >= 16) {
#pragma unroll
            for (int i = 0; i < 4; ++i) Eight<T>::load(x + min(i * 16 + t, last) * in.token, in.wide, f[i]);
        } else {                                               // (a few tokens: one row a group)
            Eight<T>::load(x + min(t, last) * in.token, in.wide, f[0]);
#pragma unroll
            for (int i = 1; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) f[i][j] = 0.0f;
        }
    }
    load_slots(bs, st, slots, token0, tokens, values);
    if (d >= dim) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) f[i][j] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (i > 0 && last < 16) break;
        const int t = i * 16 + (threadIdx.x >> 4);
        uint32_t most = 0;                                     // bits of the largest magnitude: infinities and NaN are above every number
#pragma unroll
        for (int j = 0; j < 8; ++j) most = max(most, __float_as_uint(f[i][j]) & 0x7fffffffu);
        most = row_max_u32(most);
        const float top = __uint_as_float(most);
        const bool bad = most >= 0x7f800000u, zero = bad || top < kTinyRow;
        uint2 code = codes_of(f[i], zero ? 1.0f : top);
        if (zero) code = uint2{0, 0};
        const int64_t slot = bs.slot[t];
        if (slot >= 0) {
            const int64_t base = st.row(slot >> st.shift, head);
            const int off = (int)(slot & (P - 1));
            if (lane == 0) (values ? st.vs : st.ks)[base + off] = bad ? __int_as_float(0x7fc00000) : zero ? 0.0f : top / 127.0f;
            if (!values && d < dim) *(uint2*)(st.kc + (base + off) * dim + d) = code;
        }
        if (values) {
            turn(code.x, code.y);
            const int comp = turned_component(threadIdx.x & 63), t0 = i * 16 + (threadIdx.x >> 6) * 4;
            if (comp < dim) {
                *(uint32_t*)&lds[comp * kTokenStride + t0] = code.x;
                *(uint32_t*)&lds[(comp + 1) * kTokenStride + t0] = code.y;
            }
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
    T* x = (T*)to.p + token0 * to.token + head * to.head;
    const int last = (int)min(tokens - 1 - token0, (int64_t)kBlockTokens - 1);
    uint2 code[4];
    float step[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (i * 16 > last) break;
        const int t = i * 16 + (threadIdx.x >> 4);
        const int64_t slot = bs.slot[t];
        const int64_t base = slot < 0 ? 0 : st.row(slot >> st.shift, head);
        const int off = slot < 0 ? 0 : (int)(slot & (P - 1));
        step[i] = (values ? st.vs : st.ks)[base + off];         // (of some token where there is none)
        code[i] = uint2{0, 0};
        if (values) {
            const int comp = turned_component(threadIdx.x & 63), t0 = i * 16 + (threadIdx.x >> 6) * 4;
            if (comp < dim) code[i] = uint2{*(const uint32_t*)&lds[comp * kTokenStride + t0], *(const uint32_t*)&lds[(comp + 1) * kTokenStride + t0]};
            turn_back(code[i].x, code[i].y);
        } else if (d < dim) code[i] = *(const uint2*)(st.kc + (base + off) * dim + d);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = i * 16 + (threadIdx.x >> 4);
        if (d >= dim || t > last) break;
        union { int8_t c[8]; uint2 u; } c;
        c.u = code[i];
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
