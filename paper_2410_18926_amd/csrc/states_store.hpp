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
};

// One group of 16 lanes per row, 8 values a lane.
template <typename T>
__global__ void __launch_bounds__(256) k_states_write(Store st, TokenRows k, TokenRows v, const int64_t* __restrict__ slots, int64_t tokens, int dim) {
    const int64_t row = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 4;
    const int lane = threadIdx.x & 15;
    const int64_t t = row / st.heads;
    const int h = (int)(row - t * st.heads);
    const bool values = blockIdx.y;
    if (t >= tokens) return;
    const int64_t slot = slots[t];
    if ((uint64_t)slot >= (uint64_t)(st.pages << st.shift)) return;
    const TokenRows in = values ? v : k;
    const T* x = (const T*)in.p + t * in.token + h * in.head;
    float f[8], top = 0.0f;
    bool bad = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int d = lane * 8 + j;
        f[j] = d < dim ? (float)x[d] : 0.0f;
        bad |= !(fabsf(f[j]) <= 3.4028235e38f);
        top = fmaxf(top, fabsf(f[j]));
    }
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) {
        top = fmaxf(top, __shfl_xor(top, o, 16));
        bad |= __shfl_xor((int)bad, o, 16) != 0;
    }
    const bool zero = bad || top < kTinyRow;
    const float keep = top > kHugeRow ? kHugeDown : 1.0f;
    const int64_t page = slot >> st.shift;
    const int off = (int)(slot & ((1 << st.shift) - 1));
    const int64_t base = st.row(page, h);
    if (lane == 0) (values ? st.vs : st.ks)[base + off] = bad ? __int_as_float(0x7fc00000) : zero ? 0.0f : top / 127.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int d = lane * 8 + j;
        if (d >= dim) break;
        const int8_t c = zero ? (int8_t)0 : (int8_t)rintf(f[j] * keep * 127.0f / (top * keep));
        if (values) st.vc[base * dim + ((int64_t)d << st.shift) + off] = c;
        else st.kc[(base + off) * dim + d] = c;
    }
}

template <typename T>
__global__ void __launch_bounds__(256) k_states_read(Store st, const int64_t* __restrict__ slots, int64_t tokens, TokenRows k, TokenRows v, int dim) {
    const int64_t row = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 4;
    const int lane = threadIdx.x & 15;
    const int64_t t = row / st.heads;
    const int h = (int)(row - t * st.heads);
    const bool values = blockIdx.y;
    const TokenRows to = values ? v : k;
    if (t >= tokens || !to.p) return;
    const int64_t slot = slots[t];
    const bool have = (uint64_t)slot < (uint64_t)(st.pages << st.shift);
    const int64_t page = slot >> st.shift;
    const int off = (int)(slot & ((1 << st.shift) - 1));
    const int64_t base = have ? st.row(page, h) : 0;
    const float step = have ? (values ? st.vs : st.ks)[base + off] : 0.0f;
    T* x = (T*)to.p + t * to.token + h * to.head;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int d = lane * 8 + j;
        if (d >= dim) break;
        int8_t c = 0;
        if (have) c = values ? st.vc[base * dim + ((int64_t)d << st.shift) + off] : st.kc[(base + off) * dim + d];
        float value = step * (float)c;
        asm("" : "+v"(value));         // rounded to float here: product and conversion in one instruction would round once, from the exact product
        x[d] = (T)value;
    }
}

}  // namespace lorann
