// Softmax attention over the paged 8-bit state store (states_store.hpp).
//
// For query q and key j with codes K_j, V_j and steps sk_j, sv_j, in units of log2:
//   x_j = <q, K_j> (scale sk_j log2 e) + bias;   y_j = x_j + log2 sv_j;   M = max_j y_j (running);
//   w_j = 2^(y_j - M);   out = (sum_j w_j V_j) / (sum_j w_j / sv_j).
// The steps of the values are folded into the exponent, so the operand w of the second product lies in [0, 1] whatever the steps are and the codes stay
// integers: both products are binary16 matrix products whose codes are exact, and the only rounding before the answer's is w's to 11 bits
// (2^-12 relative per weight; the answer's own rounding to bfloat16 is 2^-9).  Queries become binary16 with a power of two per row, which
// loses nothing of their 8 or 11 bits down to 2^-28 of the row's largest.
#pragma once
#include "states_store.hpp"

namespace lorann {

constexpr int kTileKeys = 64;          // keys a wavefront takes at a time
constexpr int kRows = 32;              // query rows (token, head of the group) of a block
constexpr int kAttendWaves = 4;

struct AttendArgs {
    Store st;
    const void* q;
    void* out;
    int64_t q_token, q_head, out_token, out_head;
    int64_t tokens;
    int32_t sequences, group;          // group: query heads per head of the store
    const int32_t* q_start;            // NULL: tokens / sequences each
    float c;                           // scale * log2 e
    const int32_t* tables;
    int32_t width;
    const int32_t* lengths;
    const int64_t* ids;                // NULL: sequence s reads its own table and is causal
    int32_t found;                     // passages per sequence (1 without ids)
    int64_t passages;
    const float* scores;
    float weight;                      // score_weight * log2 e
    int32_t unit, units;               // a table's keys are taken in `units` units of `unit` keys
    int32_t splits, per_split;         // units (over all passages of the sequence) per split
    float *part_acc, *part_m, *part_l; // [splits][tokens * query heads][dim], and [splits][tokens * query heads] (splits > 1)
    bool q_wide, out_wide;             // rows are aligned to 16 / 8 bytes
};

// Which tile of query rows a block has.
struct RowTile {
    int32_t s;             // sequence
    int32_t first, count;  // its tokens
    int32_t row0;          // first row of the tile: row = token * group + head of the group
};

// Tile `x` of the sequences' row tiles in order.  With q_start the tiles are counted by every wavefront, 64 sequences at a time.  false: none left.
template <int ROWS>
__device__ __forceinline__ bool find_tile(const AttendArgs& a, int x, RowTile& t) {
    if (!a.q_start) {
        const int each = (int)(a.tokens / a.sequences);
        const int per = (each * a.group + ROWS - 1) / ROWS;
        t.s = x / per;
        t.first = t.s * each;
        t.count = each;
        t.row0 = (x - t.s * per) * ROWS;
        return t.s < a.sequences;
    }
    const int lane = threadIdx.x & 63;
    int base = 0;
    for (int s0 = 0; s0 < a.sequences; s0 += 64) {
        const int s = s0 + lane;
        int first = 0, count = 0;
        if (s < a.sequences) {
            first = min(max(a.q_start[s], 0), (int)a.tokens);
            count = max(min(a.q_start[s + 1], (int)a.tokens) - first, 0);
        }
        const int n = (count * a.group + ROWS - 1) / ROWS;
        int upto = n;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int w = __shfl_up(upto, o, 64);
            if (lane >= o) upto += w;
        }
        const unsigned long long past = __ballot(base + upto > x);
        if (past) {
            const int src = __ffsll((long long)past) - 1;
            t.s = s0 + src;
            t.first = __builtin_amdgcn_readlane(first, src);         // (scalar, so that everything that follows from them is)
            t.count = __builtin_amdgcn_readlane(count, src);
            t.row0 = (x - base - (__builtin_amdgcn_readlane(upto, src) - __builtin_amdgcn_readlane(n, src))) * ROWS;
            return true;
        }
        base += __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

// Sixteen codes as binary16, two registers' worth of eight: a code with its sign bit flipped, under the exponent of 1024, is 1024 + 128 + code.
__device__ __forceinline__ void codes_to_half(const i32x4 c, f16x8& lo, f16x8& hi) {
    union { uint32_t u[4]; f16x8 h; } a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t x = (uint32_t)c[i] ^ 0x80808080u;
        const uint32_t p = __builtin_amdgcn_perm(0x64646464u, x, 0x04010400u), q = __builtin_amdgcn_perm(0x64646464u, x, 0x04030402u);
        if (i < 2) { a.u[2 * i] = p; a.u[2 * i + 1] = q; }
        else       { b.u[2 * i - 4] = p; b.u[2 * i - 3] = q; }
    }
    const _Float16 o = (_Float16)1152.0f;
    const f16x8 off = {o, o, o, o, o, o, o, o};
    lo = a.h - off;
    hi = b.h - off;
}

template <typename T> struct Bits16;
template <> struct Bits16<_Float16> {
    static __device__ __forceinline__ float widen(uint16_t u) { union { uint16_t u; _Float16 h; } x; x.u = u; return (float)x.h; }
    static __device__ __forceinline__ uint16_t narrow(float f) { union { uint16_t u; _Float16 h; } x; x.h = (_Float16)f; return x.u; }
};
template <> struct Bits16<__bf16> {
    static __device__ __forceinline__ float widen(uint16_t u) { return __uint_as_float((uint32_t)u << 16); }
    static __device__ __forceinline__ uint16_t narrow(float f) { union { uint16_t u; __bf16 h; } x; x.h = (__bf16)f; return x.u; }
};

// Eight consecutive 16-bit elements, two to a register.
__device__ __forceinline__ i32x4 load8_raw(const void* base, int64_t at, bool wide) {
    const uint16_t* p = (const uint16_t*)base + at;
    if (wide) return *(const i32x4*)p;
    i32x4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = (int)((uint32_t)p[2 * j] | (uint32_t)p[2 * j + 1] << 16);
    return v;
}
template <typename T>
__device__ __forceinline__ void widen8(const i32x4 v, float (&f)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = Bits16<T>::widen((uint16_t)((uint32_t)v[j >> 1] >> (16 * (j & 1))));
}

template <typename T>
__device__ __forceinline__ void store4(void* base, int64_t at, bool wide, const f32x4 f) {
    uint16_t* p = (uint16_t*)base + at;
    if (wide) {
        uint2 v;
        v.x = (uint32_t)Bits16<T>::narrow(f[0]) | (uint32_t)Bits16<T>::narrow(f[1]) << 16;
        v.y = (uint32_t)Bits16<T>::narrow(f[2]) | (uint32_t)Bits16<T>::narrow(f[3]) << 16;
        *(uint2*)p = v;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) p[j] = Bits16<T>::narrow(f[j]);
    }
}

// The largest finite magnitude as a power of two that brings it to [2^14, 2^15), and its inverse (1 for rows of zeros and rows below 2^-100).
__device__ __forceinline__ void row_power(float top, float& to_half, float& back) {
    const int e = top < kTinyRow ? 14 : (int)((__float_as_uint(top) >> 23) & 255) - 127;
    to_half = ldexpf(1.0f, 14 - e);
    back = ldexpf(1.0f, e - 14);
}

// What a key's steps become: y = product * <q, K> + add, and the sum's term w * inverse.
//   - A key that is not there has add = -inf: its weight is 0 in every row.
//   - A step of 0 stands beside codes of 0, so any step may be taken in its place: 1.
//   - A NaN step of the values acts through add alone: rows that do not see the key multiply `inverse` by 0.
// While all steps of the values are within 2^+-45 ("tame"), a weight w of 2^-24 of the row's largest is still a normal float and w * inverse
// is the sum's term.  Beyond that the terms are computed by an exponential of their own (sum_term).
constexpr float kTameLog2 = 45.0f;
struct KeySteps { float product, add, inverse; bool wild; };
__device__ __forceinline__ KeySteps key_steps(float ks, float vs, float c, float bias, bool have) {
    vs = vs == 0.0f ? 1.0f : vs < 0x1p-120f ? 0x1p-120f : vs;
    const float lg = __log2f(vs);
    KeySteps k;
    k.product = have ? ks * c : 0.0f;
    k.add = have ? lg + bias : -INFINITY;
    k.inverse = have && vs == vs ? __builtin_amdgcn_rcpf(vs) : 1.0f;       // (1 ulp)
    k.wild = have && fabsf(lg) > kTameLog2;
    return k;
}

// The sum's term of a key in units of 2^M, where steps span more than a float's exponent.
__device__ __forceinline__ float sum_term(float y, float m, float inverse) {
    return y == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(y - m + __log2f(inverse));
}

// x * 2^d where 2^d may be below the normal floats and the product is not.
__device__ __forceinline__ float times_exp2(float x, float d) {
    const float h = __builtin_amdgcn_exp2f(0.5f * d);
    return x * h * h;
}

// LDS is served in a wavefront's order; this keeps the compiler from moving accesses that other lanes depend on.
__device__ __forceinline__ void wave_lds_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Few query rows: bound by reading the states.  A block has up to 32 rows of one head and a range of keys; its wavefronts take tiles of 64 keys in turn,
// codes straight from memory into registers in the order of the matrix operands (no LDS: the order of the contracted axis is free), and
// their sums are joined in LDS at the end.  The first product is formed transposed (keys x rows), so a lane holds 32 scores of ONE row: statistics are
// in-lane but for one exchange between the halves of the wavefront, and the weights are the second product's operand as they stand.
template <typename T, int D>
__global__ void __launch_bounds__(64 * kAttendWaves) k_attend_rows(AttendArgs a) {
    constexpr int C = D / 32;                                   // 16-byte pieces of a lane's half of a key row; 32-value tiles of the answer
    __shared__ __align__(16) float lds_step[kAttendWaves][3][kTileKeys];
    __shared__ __align__(16) float lds_acc[kAttendWaves][kRows][D + 4];
    __shared__ float lds_m[kAttendWaves][kRows], lds_l[kAttendWaves][kRows];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, half = lane >> 5;
    const int head = blockIdx.y, split = blockIdx.z;
    RowTile tile;
    if (!find_tile<kRows>(a, blockIdx.x, tile)) return;
    const int rows = tile.count * a.group;
    const int row = tile.row0 + n;
    const bool live = row < rows;
    const int tok = live ? row / a.group : 0;
    const int qh = head * a.group + (live ? row - tok * a.group : 0);

    // queries, normalised to binary16 by a power of two per row
    f16x8 qf[2 * C];
    float q_back;
    {
        float f[2 * C][8], top = 0.0f;
#pragma unroll
        for (int i = 0; i < 2 * C; ++i) {
            const int d = 32 * (i >> 1) + 16 * half + 8 * (i & 1);
            if (live) widen8<T>(load8_raw(a.q, (int64_t)(tile.first + tok) * a.q_token + (int64_t)qh * a.q_head + d, a.q_wide), f[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (!live) f[i][j] = 0.0f;
                const float m = fabsf(f[i][j]);
                if (m <= 3.4028235e38f) top = fmaxf(top, m);
            }
        }
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        float up;
        row_power(top, up, q_back);
#pragma unroll
        for (int i = 0; i < 2 * C; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) qf[i][j] = (_Float16)(f[i][j] * up);
    }

    f32x16 acc[C];
#pragma unroll
    for (int i = 0; i < C; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) acc[i][j] = 0.0f;
    float M = -INFINITY, L = 0.0f;
    bool wild = false;                                           // some step so far is not tame

    const int P = 1 << a.st.shift;
    const int all_units = a.found * a.units;
    const int u_begin = split * a.per_split, u_end = min(all_units, u_begin + a.per_split);
    int turn = 0;
    for (int u = u_begin; u < u_end; ++u) {
        const int r = u / a.units, sub = u - r * a.units;
        int64_t table = tile.s;
        float bias = 0.0f;
        int see = 0x7fffffff, last_see = 0x7fffffff;             // keys the lane's row sees, and the tile's last row
        if (a.ids) {
            const int64_t id = a.ids[(int64_t)tile.s * a.found + r];
            if ((uint64_t)id >= (uint64_t)a.passages) continue;
            table = id;
            if (a.scores) bias = a.weight * a.scores[(int64_t)tile.s * a.found + r];
            if (bias == -INFINITY) continue;
        }
        const int length = min(max(a.lengths[table], 0), a.width << a.st.shift);
        if (!a.ids) {
            see = length - tile.count + tok + 1;
            const int last = min(rows, tile.row0 + kRows) - 1;
            last_see = length - tile.count + last / a.group + 1;
        }
        const int k_begin = sub * a.unit, k_end = min(min(length, last_see), k_begin + a.unit);
        const int32_t* pages = a.tables + table * a.width;
        for (int k0 = k_begin; k0 < k_end; k0 += kTileKeys) {
            if ((turn++ & (kAttendWaves - 1)) != wave) continue;
            wave_lds_order();                                    // the previous tile's steps have been read
            // lane = key of the tile: its page, its steps
            const int key = k0 + lane;
            int32_t page = key < length ? pages[key >> a.st.shift] : -1;
            const bool have = (uint32_t)page < (uint64_t)a.st.pages;
            if (!have) page = 0;
            {
                const int64_t at = a.st.row(page, head) + (key & (P - 1));
                const KeySteps ks = key_steps(a.st.ks[at], a.st.vs[at], a.c, bias, have);
                lds_step[wave][0][lane] = ks.product;
                lds_step[wave][1][lane] = ks.add;
                lds_step[wave][2][lane] = ks.inverse;
                wild = wild || __ballot(ks.wild);
                wave_lds_order();
            }
            // operands: row i of the first product's tile b is key 32 (i >> 2 & 1) + 16 b + 4 (i >> 3) + (i & 3), so that a half's 16 results of a
            // tile are 16 consecutive keys - the 16 consecutive bytes of a component in the transposed values
            i32x4 kr[2][C], vr[2][C];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int kk = 32 * (n >> 2 & 1) + 16 * b + 4 * (n >> 3) + (n & 3), kv = 32 * half + 16 * b;
                const int64_t pk = __shfl(page, kk, 64), pv = __shfl(page, kv, 64);
                const int8_t* kp = a.st.kc + (a.st.row(pk, head) + ((k0 + kk) & (P - 1))) * D + 16 * half;
                const int8_t* vp = a.st.vc + a.st.row(pv, head) * D + ((int64_t)n << a.st.shift) + ((k0 + kv) & (P - 1));
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    kr[b][i] = *(const i32x4*)(kp + 32 * i);
                    vr[b][i] = *(const i32x4*)(vp + ((int64_t)(32 * i) << a.st.shift));
                }
            }
            f32x16 s[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
#pragma unroll
                for (int j = 0; j < 16; ++j) s[b][j] = 0.0f;
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    f16x8 lo, hi;
                    codes_to_half(kr[b][i], lo, hi);
                    s[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lo, qf[2 * i], s[b], 0, 0, 0);
                    s[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(hi, qf[2 * i + 1], s[b], 0, 0, 0);
                }
            }
            float top = -INFINITY;
            const bool cut = k0 + kTileKeys > length - tile.count;          // some row may not see all of it
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f32x4 sk = *(const f32x4*)&lds_step[wave][0][32 * half + 16 * b + 4 * g], lv = *(const f32x4*)&lds_step[wave][1][32 * half + 16 * b + 4 * g];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float y = fmaf(s[b][4 * g + j] * q_back, sk[j], lv[j]);
                        if (cut) y = k0 + 32 * half + 16 * b + 4 * g + j < see ? y : -INFINITY;
                        s[b][4 * g + j] = y;
                        top = fmaxf(top, y);
                    }
                }
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float m_new = fmaxf(M, top), m_use = m_new == -INFINITY ? 0.0f : m_new;
            const float shrink = __builtin_amdgcn_exp2f(M - m_use);
            L = wild ? times_exp2(L, M - m_use) : L * shrink;
            M = m_new;
#pragma unroll
            for (int i = 0; i < C; ++i)
#pragma unroll
                for (int j = 0; j < 16; ++j) acc[i][j] *= shrink;
            if (wild) {
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int j = 0; j < 16; ++j) L += sum_term(s[b][j], m_use, lds_step[wave][2][32 * half + 16 * b + j]);
            }
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                f16x8 w[2];
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f32x4 iv = *(const f32x4*)&lds_step[wave][2][32 * half + 16 * b + 4 * g];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float e = __builtin_amdgcn_exp2f(s[b][4 * g + j] - m_use);
                        if (!wild) L = fmaf(e, iv[j], L);
                        w[g >> 1][4 * (g & 1) + j] = (_Float16)e;
                    }
                }
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    f16x8 lo, hi;
                    codes_to_half(vr[b][i], lo, hi);
                    acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lo, w[0], acc[i], 0, 0, 0);
                    acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(hi, w[1], acc[i], 0, 0, 0);
                }
            }
        }
    }
    L += __shfl_xor(L, 32, 64);

    // join the wavefronts
    if (half == 0) { lds_m[wave][n] = M; lds_l[wave][n] = L; }
    __syncthreads();
    float m_all = lds_m[0][n];
#pragma unroll
    for (int w = 1; w < kAttendWaves; ++w) m_all = fmaxf(m_all, lds_m[w][n]);
    {
        const float f = __builtin_amdgcn_exp2f(M - (m_all == -INFINITY ? 0.0f : m_all));
#pragma unroll
        for (int i = 0; i < C; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f32x4 o;
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] = acc[i][4 * g + j] * f;
                *(f32x4*)&lds_acc[wave][n][32 * i + 8 * g + 4 * half] = o;
            }
    }
    __syncthreads();
    constexpr int Q = D / 4;
    const int heads = a.st.heads * a.group;
    for (int i = threadIdx.x; i < kRows * Q; i += 64 * kAttendWaves) {
        const int rr = i / Q, d = (i - rr * Q) * 4;
        const int grow = tile.row0 + rr;
        if (grow >= rows) break;
        float m = lds_m[0][rr];
#pragma unroll
        for (int w = 1; w < kAttendWaves; ++w) m = fmaxf(m, lds_m[w][rr]);
        const float m_use = m == -INFINITY ? 0.0f : m;
        float l = 0.0f;
        f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < kAttendWaves; ++w) {
            l += times_exp2(lds_l[w][rr], lds_m[w][rr] - m_use);
            o += *(const f32x4*)&lds_acc[w][rr][d];
        }
        const int t = tile.first + grow / a.group, hq = head * a.group + grow % a.group;
        if (a.splits == 1) {
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
            store4<T>(a.out, (int64_t)t * a.out_token + (int64_t)hq * a.out_head + d, a.out_wide, o * inv);
        } else {
            const int64_t at = ((int64_t)split * a.tokens + t) * heads + hq;
            *(f32x4*)&a.part_acc[at * D + d] = o;
            if (d == 0) { a.part_m[at] = m; a.part_l[at] = l; }
        }
    }
}

// Joins the splits of each row: a block per row, D / 4 threads for the row's values and as many splits side by side as the block has room for.
template <typename T, int D>
__global__ void __launch_bounds__(256) k_attend_join(AttendArgs a) {
    constexpr int Q = D / 4, SIDE = 256 / Q;
    __shared__ __align__(16) f32x4 lds_o[SIDE][Q];
    __shared__ float lds_l[SIDE], lds_m[4];
    const int heads = a.st.heads * a.group;
    const int64_t all = a.tokens * heads, row = blockIdx.x, t = row / heads;
    if (a.q_start && (t < a.q_start[0] || t >= a.q_start[a.sequences])) return;      // no sequence's: nothing was computed
    float m = -INFINITY;
    for (int s = threadIdx.x; s < a.splits; s += 256) m = fmaxf(m, a.part_m[(int64_t)s * all + row]);
    m = wave_max_f32(m);
    if ((threadIdx.x & 63) == 0) lds_m[threadIdx.x >> 6] = m;
    __syncthreads();
    m = fmaxf(fmaxf(lds_m[0], lds_m[1]), fmaxf(lds_m[2], lds_m[3]));
    const float m_use = m == -INFINITY ? 0.0f : m;
    const int side = threadIdx.x / Q, d = threadIdx.x - side * Q;
    if (side < SIDE) {
        float l = 0.0f;
        f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
        for (int s = side; s < a.splits; s += SIDE) {
            const int64_t at = (int64_t)s * all + row;
            const float dm = a.part_m[at] - m_use;
            l += times_exp2(a.part_l[at], dm);
            o += *(const f32x4*)&a.part_acc[at * D + 4 * d] * __builtin_amdgcn_exp2f(dm);
        }
        lds_o[side][d] = o;
        if (d == 0) lds_l[side] = l;
    }
    __syncthreads();
    if (threadIdx.x >= Q) return;
    float l = 0.0f;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < SIDE; ++i) {
        l += lds_l[i];
        o += lds_o[i][d];
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    store4<T>(a.out, t * a.out_token + (row - t * heads) * a.out_head + 4 * d, a.out_wide, o * inv);
}

}  // namespace lorann
