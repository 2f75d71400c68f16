// The weight that causal attention gives each key, added up over the queries of a sequence and the query heads of a head (include/lorann_evict.h).
//
//   y_ij = <q_i, K_j> (scale log2 e) step_j;   m_i = max_j y_ij;   l_i = sum_j 2^(y_ij - m_i);   sums_j += sum_i 2^(y_ij - m_i) / l_i
//
// A weight needs its row's sum, so the scores are needed twice.  Few rows: k_weights_scores forms them once, bound by reading the keys, and keeps them in the workspace (4 bytes a score
// where a key and head has D + 4 or D / 2 + 8), from which k_weights_add takes them.  Many rows: they are formed twice on the matrix cores, first with a block's rows held
// and the keys passing by (k_weights_rows: m and l), then with a block's keys held and the rows passing by (k_weights_keys: the sums stay in registers, no atomics, one order).
// Products are exact in binary16 as in attend.hpp; everything after them is float.
#pragma once
#include "attend.hpp"

namespace lorann {

struct WeightArgs {
    AttendArgs a;              // out, part_acc, scores: not used
    float* y;                  // few rows: [heads][tokens * group][row_keys]
    int64_t row_keys;          // keys of a table, rounded up to whole tiles
    const float* before;       // [sequences][heads][keys], or NULL
    float* sums;
    int64_t keys;              // of a table
    // many rows: rows of a sequence begin at a multiple of 32 (padded_row)
    float step_c, back_c;      // scale log2 e = step_c back_c, the second a power of two that leaves `back` a normal float
    int64_t padded;            // rows of a head
    f16x8* q16;                // [heads][padded / 32][D / 16][64]: operands of the matrix instructions, as the lanes hold them
    float* back;               // [heads][padded]: what a product of such a row, times a key's step and step_c, is to be multiplied by: a power of two
    float *row_m, *row_inv;    // [heads][padded]: m, 1 / l
};

// Many rows: while keys' steps (times step_c) are up to this, a product (below 2^29) times one is no infinity.  Where a block meets a larger one, steps take the row's factor first, a power of
// two: the same bits where both are finite.  (Always first, a score takes one instruction more; chosen tile by tile inside the loop, 300 tokens after 60000 keys took 489 us instead of 476.)
constexpr float kMostStep = 0x1p98f;

// Sequence s's rows begin here: ru(x) + ru(y) <= ru(x + y) + 32, so no two sequences' tiles of 32 overlap.
__device__ __forceinline__ int64_t padded_row(int64_t first_row, int s) { return (first_row + 31) / 32 * 32 + 32 * (int64_t)s; }

// (m, l) of two parts of a row; l = 0 where a part has no key.
__device__ __forceinline__ void join_sums(float& m, float& l, float m2, float l2) {
    const float top = fmaxf(m, m2), use = top == -INFINITY ? 0.0f : top;
    l = l * __builtin_amdgcn_exp2f(m - use) + l2 * __builtin_amdgcn_exp2f(m2 - use);
    m = top;
}

// Eight codes of a key from component `at` on (a multiple of 8), as binary16 operands: code, or r_g * code.
template <int D, int BITS>
__device__ __forceinline__ f16x8 key_operand(const int8_t* row, int at, uint32_t factors) {
    if constexpr (BITS == 4) return codes4_to_half(*(const uint32_t*)(row + at / 2)) * spread(factor_pair(factors, (uint32_t)at / 32));
    else {
        const i32x2 c = *(const i32x2*)(row + at);
        f16x8 lo, hi;
        codes_to_half(i32x4{c[0], c[1], 0, 0}, lo, hi);
        return lo;
    }
}

// The largest finite magnitude of a lane's elements: of 16-bit magnitudes as they stand, two at a time; element by element only where one is an infinity or NaN.  (All of them as floats took 350
// instructions of a wavefront of k_weights_rows, which has some 2500 in all where a block has 8 tiles of keys: 41.9 us, 41.3 so.)
template <typename T, int N>
__device__ __forceinline__ float largest_finite(const i32x4 (&raw)[N]) {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    constexpr uint32_t infinity = std::is_same_v<T, _Float16> ? 0x7c00 : 0x7f80;
    u16x2 m = {0, 0};
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, (uint32_t)raw[i][j] & 0x7fff7fffu));
    uint32_t most = max((uint32_t)m[0], (uint32_t)m[1]);
    if (__ballot(most >= infinity)) {
        most = 0;
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t u = (uint32_t)raw[i][j >> 1] >> (16 * (j & 1)) & 0x7fffu;
                most = u < infinity ? max(most, u) : most;
            }
    }
    return Bits16<T>::widen((uint16_t)most);
}

// Few rows.  A block has up to 16 rows of one head and a range of keys; its wavefronts take tiles of 64 keys in turn, codes straight from memory into registers, the next tile's in flight
// (as k_attend_rows).  A lane keeps a maximum and a sum of its own until the end.  64 single tokens after up to 8192 keys, 32 heads on 8 of 128, 8 bits: 89 us for 352 MB of keys and 43 of
// scores, 4.4 TB/s.
template <typename T, int D, int BITS>
__global__ void __launch_bounds__(64 * kAttendWaves, 3) k_weights_scores(WeightArgs wa) {
    const AttendArgs& a = wa.a;
    constexpr int S32 = D / 32, ROW = D * BITS / 8;
    constexpr int PIECE = BITS == 8 ? 8 : 4;                    // bytes of a lane's eight codes
    __shared__ __align__(16) float lds_step[kAttendWaves][2][kTileKeys];
    __shared__ float lds_m[kAttendWaves][kRows], lds_l[kAttendWaves][kRows];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, quarter = lane >> 4;
    const BlockWork work = block_work(a);
    const int head = work.head, split = work.split;
    RowTile tile;
    if (!find_tile<kRows, false>(a, work.tile, tile)) return;
    const int rows = tile.count * a.group;
    const int row = tile.row0 + n;
    const bool live = row < rows;
    const int tok = live ? row / a.group : 0;
    const int see_after = tile.count - 1 - tok;
    const int behind = tile.count - 1 - (min(rows, tile.row0 + kRows) - 1) / a.group, first_behind = tile.count - 1 - tile.row0 / a.group;
    const int P = 1 << a.st.shift;

    const int qh = head * a.group + (live ? row - tok * a.group : 0);
    const int64_t q_at = (int64_t)(tile.first + tok) * a.q_token + (int64_t)qh * a.q_head;
    auto component = [&](int i) { return (D / 4) * quarter + 8 * i; };         // first of the lane's 8 in step i
    i32x4 raw[S32];
#pragma unroll
    for (int i = 0; i < S32; ++i) raw[i] = load8_raw(a.q, q_at + component(i), a.q_wide);
    int page = 0;
    KeyTiles it;
    it.start(a, tile.s, split);
    auto find_page = [&](const KeyTile& kt) {
        if (kt.have) page = kt.pages[min(kt.k + lane, kt.length - 1) >> a.st.shift];
    };
    const uint32_t page_bytes = (uint32_t)ROW << a.st.shift;
    uint32_t kr[4][S32][PIECE / 4], rkf[4];
    float rks = 0.0f;
    bool rhave = false;
    auto fetch_keys = [&](const KeyTile& kt) {
        if (!kt.have) return;
        const bool known = (uint32_t)page < (uint64_t)a.st.pages;
        rhave = known && kt.k + lane < kt.length;
        const int row_of_key = (known ? page : 0) * a.st.heads + head, place = (kt.k + lane) & (P - 1);
        rks = a.st.ks[((uint64_t)(uint32_t)row_of_key << a.st.shift) + (uint32_t)place];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int key = 16 * b + n;                         // (results: key 16 b + 4 quarter + j, so that a store of the four quarters fills 64 bytes of a row)
            const uint64_t r = (uint32_t)__shfl(row_of_key, key, 64);
            const uint32_t at = (uint32_t)((kt.k + key) & (P - 1));
            const int8_t* kp = a.st.kc + r * page_bytes + at * ROW + component(0) * BITS / 8;
#pragma unroll
            for (int i = 0; i < S32; ++i)
#pragma unroll
                for (int j = 0; j < PIECE / 4; ++j) kr[b][i][j] = *(const uint32_t*)(kp + PIECE * i + 4 * j);
            if constexpr (BITS == 4) rkf[b] = a.st.kf[(r << a.st.shift) + at];
        }
    };
    it.skip(a, tile.s, behind, 1 + wave);
    KeyTile cur = it.t;
    find_page(cur);
    fetch_keys(cur);
    it.skip(a, tile.s, behind, kAttendWaves);
    find_page(it.t);

    f16x8 qf[S32];
    float q_back;
    {
#pragma unroll
        for (int i = 0; i < S32; ++i)
            if (!live) raw[i] = i32x4{0, 0, 0, 0};
        float top = largest_finite<T>(raw);
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        float up;
        row_power(top, up, q_back);
#pragma unroll
        for (int i = 0; i < S32; ++i) {
            float f[8];
            widen8<T>(raw[i], f);
#pragma unroll
            for (int j = 0; j < 8; ++j) qf[i][j] = (_Float16)(f[j] * up);
        }
    }

    // The block's rows of scores as a buffer: what a row that is not there would store lies behind its end and is dropped, without a branch that the loads' waits would have to
    // take into account.
    const uint32_t row_bytes = (uint32_t)(wa.row_keys * 4);      // (16 rows of at most 2^30 bytes would not fit: kMostScores)
    const auto y_rows = __builtin_amdgcn_make_buffer_rsrc(wa.y + ((int64_t)head * a.tokens * a.group + (int64_t)tile.first * a.group + tile.row0) * wa.row_keys, 0,
                                                          min(rows - tile.row0, kRows) * row_bytes, 0x00027000);
    const uint32_t y_at = live ? n * row_bytes + 16 * quarter : 0xffffe000u;
    float M = -INFINITY, L = 0.0f;
    while (cur.have) {
        wave_lds_order();                                       // the previous tile's steps have been read
        lds_step[wave][0][lane] = rhave ? rks * a.c : 0.0f;
        lds_step[wave][1][lane] = rhave ? 0.0f : -INFINITY;
        wave_lds_order();
        f32x4 s[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            s[b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < S32; ++i) {
                f16x8 k;
                if constexpr (BITS == 4) k = codes4_to_half(kr[b][i][0]) * spread(factor_pair(rkf[b], (uint32_t)component(i) / 32));
                else {
                    f16x8 hi;
                    codes_to_half(i32x4{(int)kr[b][i][0], (int)kr[b][i][PIECE / 4 - 1], 0, 0}, k, hi);
                }
                s[b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, qf[i], s[b], 0, 0, 0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        const KeyTile nxt = it.t;
        fetch_keys(nxt);
        it.skip(a, tile.s, behind, kAttendWaves);
        find_page(it.t);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const f32x4 sk = *(const f32x4*)&lds_step[wave][0][16 * b + 4 * quarter], lv = *(const f32x4*)&lds_step[wave][1][16 * b + 4 * quarter];
#pragma unroll
            for (int j = 0; j < 4; ++j) s[b][j] = fmaf(s[b][j], sk[j] * q_back, lv[j]);          // (in this order: as in k_attend_rows)
        }
        if (cur.k + kTileKeys > cur.length - first_behind) {    // some row may not see all of it
            const int see = cur.length - see_after - cur.k - 4 * quarter;
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int j = 0; j < 4; ++j) s[b][j] = 16 * b + j < see ? s[b][j] : -INFINITY;
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(i32x4, s[b]), y_rows, live ? y_at + 4 * cur.k : y_at, 64 * b, 0);
        float top = M;
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int j = 0; j < 4; ++j) top = fmaxf(top, s[b][j]);
        const float use = top == -INFINITY ? 0.0f : top;
        float l = L * __builtin_amdgcn_exp2f(M - use);
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int j = 0; j < 4; ++j) l += __builtin_amdgcn_exp2f(s[b][j] - use);
        L = l;
        M = top;
        cur = nxt;
    }
    join_sums(M, L, __shfl_xor(M, 32, 64), __shfl_xor(L, 32, 64));
    join_sums(M, L, __shfl_xor(M, 16, 64), __shfl_xor(L, 16, 64));
    if (quarter == 0) { lds_m[wave][n] = M; lds_l[wave][n] = L; }
    __syncthreads();
    if (threadIdx.x < kRows && live) {
#pragma unroll
        for (int w = 1; w < kAttendWaves; ++w) join_sums(M, L, lds_m[w][n], lds_l[w][n]);
        const int64_t all = (int64_t)a.tokens * a.group, at = ((int64_t)split * a.st.heads + head) * all + (int64_t)tile.first * a.group + row;
        a.part_m[at] = M;
        a.part_l[at] = L;
    }
}

// Tokens of sequence s.
__device__ __forceinline__ void tokens_of(const AttendArgs& a, int s, int& first, int& count) {
    const int each = (int)(a.tokens / a.sequences);
    first = a.q_start ? min(max(a.q_start[s], 0), (int)a.tokens) : s * each;
    count = a.q_start ? max(min(a.q_start[s + 1], (int)a.tokens) - first, 0) : each;
}

constexpr int kAddKeys = 1024;         // keys of a block: four a thread
constexpr int kAddRows = 32;           // rows whose sums are joined at a time

// Few rows, second half: bound by reading the scores (the same case: 16 us).  Blocks: (chunk of keys, head, sequence).
__global__ void __launch_bounds__(256) k_weights_add(WeightArgs wa) {
    const AttendArgs& a = wa.a;
    __shared__ float lds_m[kAddRows], lds_inv[kAddRows];
    const int head = blockIdx.y, s = blockIdx.z, tid = threadIdx.x;
    const int64_t j0 = (int64_t)blockIdx.x * kAddKeys + 4 * tid;
    int first, count;
    tokens_of(a, s, first, count);
    const int length = a.found ? min(max(a.lengths[s], 0), a.width << a.st.shift) : 0;
    const int rows = (int64_t)blockIdx.x * kAddKeys < length ? count * a.group : 0;
    const int64_t at = ((int64_t)s * a.st.heads + head) * wa.keys + j0;
    const bool mine = j0 < wa.keys;                             // (keys of a table are a multiple of 16)
    float sum[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) sum[j] = mine && wa.before ? wa.before[at + j] : 0.0f;
    const int64_t all = (int64_t)a.tokens * a.group, row_at = (int64_t)first * a.group;
    float more[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int r0 = 0; r0 < rows; r0 += kAddRows) {
        const int many = min(kAddRows, rows - r0);
        {
            // eight threads a row join its splits
            const int r = tid >> 3, part = tid & 7;
            float m = -INFINITY, l = 0.0f;
            if (r < many)
                for (int p = part; p < a.splits; p += 8) {
                    const int64_t i = ((int64_t)p * a.st.heads + head) * all + row_at + r0 + r;
                    join_sums(m, l, a.part_m[i], a.part_l[i]);
                }
#pragma unroll
            for (int o = 1; o < 8; o <<= 1) join_sums(m, l, __shfl_xor(m, o, 64), __shfl_xor(l, o, 64));
            if (r < many && part == 0) {
                lds_m[r] = m == -INFINITY ? 0.0f : m;
                lds_inv[r] = l == 0.0f ? 0.0f : 1.0f / l;
            }
        }
        __syncthreads();
        if (mine) {
            const float* y = wa.y + ((int64_t)head * all + row_at + r0) * wa.row_keys + j0;
            for (int r = 0; r < many; ++r) {
                const int see = length - count + (r0 + r) / a.group + 1 - (int)j0;       // keys that the row sees from j0 on
                if (see <= 0) continue;
                const f32x4 v = *(const f32x4*)(y + r * wa.row_keys);
                const float m = lds_m[r], inv = lds_inv[r];
                if (inv != inv) {                               // (a row whose sum is no number: keys that are there, logits of -infinity among them, get none)
                    if ((uint32_t)a.tables[(int64_t)s * a.width + (j0 >> a.st.shift)] < (uint64_t)a.st.pages)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (j < see) more[j] = inv;
                    continue;
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j < see && v[j] != -INFINITY) more[j] = fmaf(__builtin_amdgcn_exp2f(v[j] - m), inv, more[j]);
            }
        }
        __syncthreads();
    }
    if (!mine) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) wa.sums[at + j] = sum[j] + more[j];
}

// Many rows: m and l.  A block has 128 rows of one head, a wavefront 32; keys pass by, 64 at a time, converted once for the block into LDS.  The maximum is taken over x = product * step,
// which the row's factor (a power of two: m = x back is exact, and no term is above 1 however large logits are) is applied to together with it: y - m = fma(x, back, -m), so a score costs five instructions and its exponential.
// A block that has met a key above kMostStep begins again, x = product * (step * back), y - m = fma(x, 1, -m).
// 4 x 32 tokens after 16000 keys, 32 heads on 8 of 128, 4 bits: 42 us, the matrix instructions alone 7; some 40 % of the cycles are vector instructions, a third of those convert codes and find addresses.
// (Four wavefronts a SIMD instead of three: 17 registers spill, 92 us for the call instead of 86.)
template <typename T, int D, int BITS>
__global__ void __launch_bounds__(256, 3) k_weights_rows(WeightArgs wa) {
    const AttendArgs& a = wa.a;
    constexpr int N = D / 16, KS = D + 8, ROW = D * BITS / 8;
    constexpr int PIECES = kTileKeys * D / 16, PER = (PIECES + 255) / 256;      // pieces of 16 codes
    typedef std::conditional_t<BITS == 4, i32x2, i32x4> Piece;
    __shared__ __align__(16) _Float16 lds_k[2][kTileKeys * KS];
    __shared__ __align__(16) float lds_step[2][2][kTileKeys];
    __shared__ int lds_large;                                   // a key is above kMostStep
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, half = lane >> 5;
    const BlockWork work = block_work(a);
    const int head = work.head, split = work.split;
    RowTile tile;
    if (!find_tile<128, true>(a, work.tile, tile)) return;
    const int rows = tile.count * a.group, row = tile.row0 + wave * 32 + n, P = 1 << a.st.shift;
    const bool live = row < rows;
    const int see_after = tile.count - 1 - (live ? row / a.group : 0);
    const int behind = tile.count - 1 - (min(rows, tile.row0 + 128) - 1) / a.group, first_behind = tile.count - 1 - tile.row0 / a.group;
    const int64_t slot = (int64_t)head * wa.padded + padded_row((int64_t)tile.first * a.group, tile.s) + tile.row0 + wave * 32;      // of the wavefront's first row
    const bool any = tile.row0 + wave * 32 < rows;              // (a wavefront without rows has no operands either)
    // The rows as operands: lane n + 32 half holds components D / 2 half .. of row n.  The blocks of the first keys leave them for k_weights_keys.
    f16x8 q[N];
    float back;
    {
        const int tok = live ? row / a.group : 0, qh = head * a.group + (live ? row - tok * a.group : 0);
        const int64_t at = (int64_t)(tile.first + tok) * a.q_token + (int64_t)qh * a.q_head + D / 2 * half;
        i32x4 raw[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            raw[i] = load8_raw(a.q, at + 8 * i, a.q_wide);
            if (!live) raw[i] = i32x4{0, 0, 0, 0};
        }
        float top = largest_finite<T>(raw);
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        float up;
        row_power(top, up, back);
        back *= wa.back_c;                                      // (a normal float: keys that are not there are -inf, which 0 would make NaN)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float f[8];
            widen8<T>(raw[i], f);
#pragma unroll
            for (int j = 0; j < 8; ++j) q[i][j] = (_Float16)(f[j] * up);
            if (any && split == 0) wa.q16[(slot / 32 * N + i) * 64 + lane] = q[i];
        }
        if (any && split == 0 && half == 0) wa.back[slot + n] = back;
    }
    const uint32_t page_bytes = (uint32_t)ROW << a.st.shift;
    int pg[PER], pg_step = 0;
    auto page_at = [&](const KeyTile& kt, int key) { return kt.pages[min(kt.k + key, kt.length - 1) >> a.st.shift]; };
    auto find_pages = [&](const KeyTile& kt) {
        if (!kt.have) return;
#pragma unroll
        for (int i = 0; i < PER; ++i) pg[i] = page_at(kt, (tid + i * 256) / (D / 16) % kTileKeys);
        pg_step = page_at(kt, lane);
    };
    auto row_of = [&](int page) { return (uint64_t)(uint32_t)(((uint32_t)page < (uint64_t)a.st.pages ? page : 0) * a.st.heads + head); };
    Piece ck[PER];
    uint32_t fk[PER];
    float rks = 0.0f;
    bool rhave = false;
    auto fetch = [&](const KeyTile& kt) {
        if (!kt.have) return;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int p = tid + i * 256, key = p / (D / 16), part = p % (D / 16);
            if (PIECES % 256 && p >= PIECES) break;
            const uint64_t r = row_of(pg[i]);
            const uint32_t at = (uint32_t)((kt.k + key) & (P - 1));
            ck[i] = *(const Piece*)(a.st.kc + r * page_bytes + at * ROW + part * (int)sizeof(Piece));
            if constexpr (BITS == 4) fk[i] = a.st.kf[(r << a.st.shift) + at];
        }
        if (wave == 0) {
            rhave = kt.k + lane < kt.length && (uint32_t)pg_step < (uint64_t)a.st.pages;
            rks = a.st.ks[(row_of(pg_step) << a.st.shift) + (uint32_t)((kt.k + lane) & (P - 1))];
        }
    };
    float largest = 0.0f;                                       // (first wavefront) of the lane's steps
    auto stage = [&](int kb) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int p = tid + i * 256, key = p / (D / 16), part = p % (D / 16);
            if (PIECES % 256 && p >= PIECES) break;
            f16x8 lo, hi;
            if constexpr (BITS == 8) codes_to_half(ck[i], lo, hi);
            else {
                const f16x8 r = spread(factor_pair(fk[i], (uint32_t)part / 2));
                lo = codes4_to_half((uint32_t)ck[i][0]) * r;
                hi = codes4_to_half((uint32_t)ck[i][1]) * r;
            }
            // key 32 h + 16 b + 4 g + r is row 32 b + 8 g + 4 h + r of the product, whose 32 results of a lane are then consecutive keys
            const int krow = (key & 16) * 2 + (key >> 2 & 3) * 8 + (key >> 5) * 4 + (key & 3);
            *(f16x8*)&lds_k[kb][krow * KS + 16 * part] = lo;
            *(f16x8*)&lds_k[kb][krow * KS + 16 * part + 8] = hi;
        }
        if (wave == 0) {
            const float step = rhave ? rks * wa.step_c : 0.0f;
            lds_step[kb][0][lane] = step;
            lds_step[kb][1][lane] = rhave ? 0.0f : -INFINITY;
            largest = fmaxf(largest, fabsf(step));
        }
    };
    float M = -INFINITY, L = 0.0f;
    auto pass = [&](auto first) {                               // first: steps take the row's factor first
        KeyTiles it;
        it.start(a, tile.s, split);
        it.next(a, tile.s, behind);
        KeyTile cur = it.t;
        find_pages(cur);
        fetch(cur);
        it.next(a, tile.s, behind);
        find_pages(it.t);
        if (cur.have) stage(0);
        KeyTile nxt = it.t;
        fetch(nxt);
        it.next(a, tile.s, behind);
        find_pages(it.t);
        int kb = 0;
        float left = decltype(first)::value ? 1.0f : back;      // what x is still to be multiplied by
        if constexpr (decltype(first)::value) asm("" : "+v"(left));       // (a product also where it is 1: x is rounded before m is taken off it)
        while (cur.have) {
            __syncthreads();                                    // tile `cur` is in buffer kb; the other has been read
            f32x16 s[2];
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int j = 0; j < 16; ++j) s[b][j] = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const f16x8 k = *(const f16x8*)&lds_k[kb][(32 * b + n) * KS + D / 2 * half + 8 * i];
                    s[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, q[i], s[b], 0, 0, 0);
                }
            if (nxt.have) stage(kb ^ 1);
            const KeyTile after = it.t;
            fetch(after);
            it.next(a, tile.s, behind);
            find_pages(it.t);
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    f32x4 sk = *(const f32x4*)&lds_step[kb][0][32 * half + 16 * b + 4 * g];
                    const f32x4 lv = *(const f32x4*)&lds_step[kb][1][32 * half + 16 * b + 4 * g];
                    if constexpr (decltype(first)::value) sk = sk * back;
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[b][4 * g + j] = fmaf(s[b][4 * g + j], sk[j], lv[j]);
                }
            if (cur.k + kTileKeys > cur.length - first_behind) {
                const int see = cur.length - see_after - cur.k - 32 * half;
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int j = 0; j < 16; ++j) s[b][j] = 16 * b + j < see ? s[b][j] : -INFINITY;
            }
            float top = M;                                      // (of x, as M until the end)
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int j = 0; j < 16; ++j) top = fmaxf(top, s[b][j]);
            const float m = top == -INFINITY ? 0.0f : top * left;
            float l[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int j = 0; j < 16; ++j) l[j & 3] += __builtin_amdgcn_exp2f(fmaf(s[b][j], left, -m));
            L = L * __builtin_amdgcn_exp2f(fmaf(M, left, -m)) + ((l[0] + l[1]) + (l[2] + l[3]));
            M = top;
            cur = nxt;
            nxt = after;
            kb ^= 1;
        }
        M *= left;                                              // (-inf: no key)
    };
    pass(std::false_type{});
    if (wave == 0) {
        const int met = __ballot(largest > kMostStep) != 0;
        if (lane == 0) lds_large = met;
    }
    __syncthreads();
    if (__builtin_amdgcn_readfirstlane(lds_large)) {
        M = -INFINITY;
        L = 0.0f;
        pass(std::true_type{});
    }
    join_sums(M, L, __shfl_xor(M, 32, 64), __shfl_xor(L, 32, 64));
    if (!any || half) return;
    if (a.splits == 1) {
        wa.row_m[slot + n] = M == -INFINITY ? 0.0f : M;
        wa.row_inv[slot + n] = live && L != 0.0f ? 1.0f / L : 0.0f;
    } else {
        const int64_t at = (int64_t)split * a.st.heads * wa.padded + slot + n;
        a.part_m[at] = M;
        a.part_l[at] = live ? L : 0.0f;
    }
}

// Joins the splits of each row, eight threads a row (rows of no sequence hold anything).
__global__ void __launch_bounds__(256) k_weights_join(WeightArgs wa) {
    const AttendArgs& a = wa.a;
    const int64_t all = a.st.heads * wa.padded, i = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 32 + (threadIdx.x >> 3);
    const int part = threadIdx.x & 7;
    float m = -INFINITY, l = 0.0f;
    if (i < all)
        for (int p = part; p < a.splits; p += 8) join_sums(m, l, a.part_m[p * all + i], a.part_l[p * all + i]);
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) join_sums(m, l, __shfl_xor(m, o, 64), __shfl_xor(l, o, 64));
    if (i >= all || part) return;
    wa.row_m[i] = m == -INFINITY ? 0.0f : m;
    wa.row_inv[i] = l == 0.0f ? 0.0f : 1.0f / l;
}

// v of the lane W away (W < 16), in the registers' own crossings: through LDS (a permute), the 31 exchanges below make up a tenth of a wavefront's instructions and wait for each round.
template <int W>
__device__ __forceinline__ float lane_across(float v) {
    const int x = __float_as_int(v);
    if constexpr (W == 8) return __int_as_float(__builtin_amdgcn_update_dpp(0, x, 0x128, 0xf, 0xf, true));            // row_ror:8
    else if constexpr (W == 4)                                                                                     // row_half_mirror, then quad_perm 3 2 1 0
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __builtin_amdgcn_update_dpp(0, x, 0x141, 0xf, 0xf, true), 0x1b, 0xf, 0xf, true));
    else if constexpr (W == 2) return __int_as_float(__builtin_amdgcn_update_dpp(0, x, 0x4e, 0xf, 0xf, true));        // quad_perm 2 3 0 1
    else return __int_as_float(__builtin_amdgcn_update_dpp(0, x, 0xb1, 0xf, 0xf, true));                              // quad_perm 1 0 3 2
}
// 2 W values of a lane are W of its pair's (lanes W apart) added up, and so on: after all rounds lane n has value n of the 32 that each of 32 lanes had, added up.
template <int W>
__device__ __forceinline__ void add_over_lanes(float (&v)[32]) {
    if constexpr (W == 16) {
#pragma unroll
        for (int j = 0; j < W; ++j) {                           // rows of 16 lanes: the odd ones of the first change places with the even ones of the second
            const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[j]), __float_as_uint(v[j + W]), false, false);
            v[j] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
        }
    } else {
        const bool upper = threadIdx.x & W;
#pragma unroll
        for (int j = 0; j < W; ++j) {
            const float give = upper ? v[j] : v[j + W], keep = upper ? v[j + W] : v[j];
            v[j] = keep + lane_across<W>(give);
        }
    }
    if constexpr (W > 1) add_over_lanes<W / 2>(v);
}

// Many rows: the sums.  A wavefront holds 64 keys as operands, rows pass by, 32 at a time.  SHARE: the block's four wavefronts have the same keys and take the rows in turn; else each
// has keys of its own.  Blocks: (chunk of keys, head, sequence).  The case of k_weights_rows: 40 us, bound in the same way.
template <int D, int BITS, bool SHARE>
__global__ void __launch_bounds__(256, 2) k_weights_keys(WeightArgs wa) {
    const AttendArgs& a = wa.a;
    constexpr int N = D / 16, ROW = D * BITS / 8;
    __shared__ float lds_sum[4][64];
    __shared__ __align__(16) float lds_step[4][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 31, half = lane >> 5;
    const int head = blockIdx.y, s = blockIdx.z, P = 1 << a.st.shift;
    const int64_t k0 = ((int64_t)blockIdx.x * (SHARE ? 1 : 4) + (SHARE ? 0 : wave)) * 64;
    int first, count;
    tokens_of(a, s, first, count);
    const int length = a.found ? min(max(a.lengths[s], 0), a.width << a.st.shift) : 0;
    const int rows = k0 < length ? count * a.group : 0;
    const int32_t* pages = a.tables + (int64_t)s * a.width;
    auto row_at = [&](int key, uint64_t& r, uint32_t& at) -> bool {
        const int64_t j = k0 + key;
        const int page = j < length ? pages[j >> a.st.shift] : -1;
        const bool ok = (uint32_t)page < (uint64_t)a.st.pages;
        r = (uint64_t)(uint32_t)((ok ? page : 0) * a.st.heads + head);
        at = (uint32_t)(j & (P - 1));
        return ok;
    };
    // the lane's two keys as operands; of its 32 results the keys are 32 half + 16 b + j, as in k_weights_rows: row 32 b + n of the product is the key below
    f16x8 k[2][N];
    f32x4 step[2][4];
    bool ok = false, large = false;                             // the lane's own key is there; a key of the wavefront is above kMostStep
    if (rows > 0) {
        uint64_t r;
        uint32_t at;
        ok = row_at(lane, r, at);
        const float own = ok ? a.st.ks[(r << a.st.shift) + at] * wa.step_c : 0.0f;           // (of a key that is not there: any)
        lds_step[wave][lane] = own;
        large = __ballot(fabsf(own) > kMostStep) != 0;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int key = 32 * (n >> 2 & 1) + 16 * b + 4 * (n >> 3) + (n & 3);
            row_at(key, r, at);
            const int8_t* from = a.st.kc + ((r << a.st.shift) + at) * ROW;
            uint32_t factors = 0;
            if constexpr (BITS == 4) factors = a.st.kf[(r << a.st.shift) + at];
#pragma unroll
            for (int i = 0; i < N; ++i) k[b][i] = key_operand<D, BITS>(from, D / 2 * half + 8 * i, factors);
        }
        wave_lds_order();
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int g = 0; g < 4; ++g) step[b][g] = *(const f32x4*)&lds_step[wave][32 * half + 16 * b + 4 * g];
    }
    float sum[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) sum[j] = 0.0f;
    // the first row that sees key k0, or behind the last one (the product passes 32 bits where a long table meets a large group)
    const int from_row = (int)min(max((int64_t)0, k0 - (length - count)) * a.group / 32 * 32, (int64_t)rows);
    const int64_t base = (int64_t)head * wa.padded + padded_row((int64_t)first * a.group, s);
    const f16x8* q16 = wa.q16 + base / 32 * N * 64 + lane;
    // the next 32 rows are requested before these are used
    f16x8 q[N];
    float back = 0.0f, m = 0.0f, inv = 0.0f;
    auto fetch = [&](int r0) {
        if (r0 >= rows) return;
#pragma unroll
        for (int i = 0; i < N; ++i) q[i] = q16[((int64_t)(r0 / 32) * N + i) * 64];
        back = wa.back[base + r0 + n];
        m = wa.row_m[base + r0 + n];
        inv = wa.row_inv[base + r0 + n];
    };
    constexpr int STRIDE = SHARE ? 128 : 32;
    int r0 = from_row + (SHARE ? wave * 32 : 0);
    if (large) {                                                // (as in k_weights_rows; nothing in flight, so that the registers hold it)
        float one = 1.0f;
        asm("" : "+v"(one));                                    // (a product also where it is 1: x is rounded before m is taken off it)
#pragma unroll 1
        for (; r0 < rows; r0 += STRIDE) {
            fetch(r0);
            const int row = r0 + n, see = row < rows ? (int)(length - count + row / a.group + 1 - k0) - 32 * half : 0;
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                f32x16 y;
#pragma unroll
                for (int j = 0; j < 16; ++j) y[j] = 0.0f;
#pragma unroll
                for (int i = 0; i < N; ++i) y = __builtin_amdgcn_mfma_f32_32x32x16_f16(k[b][i], q[i], y, 0, 0, 0);
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const float e = __builtin_amdgcn_exp2f(fmaf(y[j] * (step[b][j >> 2][j & 3] * back), one, -m)) * inv;
                    sum[16 * b + j] += 16 * b + j < see ? e : 0.0f;
                }
            }
        }
    }
    fetch(r0);
    for (; r0 < rows; r0 += STRIDE) {
        f32x16 y[2];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int j = 0; j < 16; ++j) y[b][j] = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int b = 0; b < 2; ++b) y[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k[b][i], q[i], y[b], 0, 0, 0);
        const int row = r0 + n;
        const float back_now = back, m_now = m, inv_now = inv;
        __builtin_amdgcn_sched_barrier(0);
        fetch(r0 + STRIDE);
        __builtin_amdgcn_sched_barrier(0);
        const int see = row < rows ? (int)(length - count + row / a.group + 1 - k0) - 32 * half : 0;
        if (__ballot(see < 32) == 0) {                          // every row sees all of the lane's keys
#pragma unroll
            for (int j = 0; j < 32; ++j) sum[j] = fmaf(__builtin_amdgcn_exp2f(fmaf(y[j >> 4][j & 15] * step[j >> 4][j >> 2 & 3][j & 3], back_now, -m_now)), inv_now, sum[j]);
        } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                const float e = __builtin_amdgcn_exp2f(fmaf(y[j >> 4][j & 15] * step[j >> 4][j >> 2 & 3][j & 3], back_now, -m_now)) * inv_now;
                sum[j] += j < see ? e : 0.0f;
            }
        }
    }
    add_over_lanes<16>(sum);                                    // (over the rows; lane n then has key n of its half)
    float mine = ok ? sum[0] : 0.0f;
    const int64_t key = k0 + lane;
    if constexpr (SHARE) {
        lds_sum[wave][lane] = mine;
        __syncthreads();
        if (wave) return;
        mine = ((lds_sum[0][lane] + lds_sum[1][lane]) + lds_sum[2][lane]) + lds_sum[3][lane];
    }
    if (key >= wa.keys) return;
    const int64_t at = ((int64_t)s * a.st.heads + head) * wa.keys + key;
    wa.sums[at] = (wa.before ? wa.before[at] : 0.0f) + mine;
}

}  // namespace lorann
