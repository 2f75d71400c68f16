// Softmax attention over the paged 8-bit state store (states_store.hpp).
//
// For query q and key j with codes K_j, V_j and steps sk_j, sv_j, in units of log2:
//   x_j = <q, K_j> (scale sk_j log2 e) + bias;   y_j = x_j + log2 sv_j;   M = max_j y_j (running);
//   w_j = 2^(y_j - M);   out = (sum_j w_j V_j) / (sum_j w_j / sv_j).
// The steps of the values are folded into the exponent, so the operand w of the second product lies in [0, 2^kSlack] whatever the steps are and the codes
// stay integers: both products are binary16 matrix products whose codes are exact (products of binary16 numbers added in float), and the only rounding before
// the answer's is w's to 11 bits (at most 2^-11 relative per weight; the answer's own rounding to bfloat16 is at most 2^-8).  The operand is 2^kLift w, which fills
// binary16's range to its top: weights keep their 11 bits down to 2^-23 of 2^M, and below that are off by at most 2^-34 of 2^M.  Queries become binary16
// with a power of two per row (k_attend_tile: per block while its rows lie within 2^12 of each other), which loses nothing of their 8 or 11 bits down to 2^-28 (2^-16) of
// the row's largest and 2^-39 (2^-27) of that below.  Scores, M, the sum and the answer are floats throughout.  (bfloat16 products instead would round the
// weights to 8 bits, at the same rate.)
#pragma once
#include "codes4.hpp"

namespace lorann {

constexpr int kTileKeys = 64;          // keys a wavefront takes at a time
constexpr int kRows = 16;              // query rows (token, head of the group) of a block of k_attend_rows
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
    float *part_acc, *part_m, *part_l; // [splits][tokens * query heads][dim] (2^kLift sum w V; not written where part_l is 0), and [splits][tokens * query heads] (splits > 1)
    bool q_wide, out_wide;             // rows are aligned to 16 / 8 bytes
};

// Which head, split and row tile a block has.  Consecutive blocks, which go to different dies (each with an L2 and a share of the memory bandwidth of its own), are the heads
// and then the splits of one row tile: one long sequence among short ones is read by all of them.  (With the row tiles consecutive, a token after 131072 keys
// beside 63 after 1000, 64 heads on 8 of 128, takes 1028 us, all of it on one die; 200 us so.)
struct BlockWork { int head, split, tile; };
__device__ __forceinline__ BlockWork block_work(const AttendArgs& a) {
    const int rest = blockIdx.x / a.st.heads, tile = rest / a.splits;
    return BlockWork{(int)blockIdx.x - rest * a.st.heads, rest - tile * a.splits, tile};
}

// Which tile of query rows a block has.
struct RowTile {
    int32_t s;             // sequence
    int32_t first, count;  // its tokens
    int32_t row0;          // first row of the tile: row = token * group + head of the group
};

// Tile `x` of the sequences' row tiles.  With q_start the tiles are counted by every wavefront, 64 sequences at a time.  false: none left.
// LONGEST: up to 64 sequences that read their own tables come in the order of their lengths instead of their own, so that what runs last is short
// (12 sequences of 128 to 500 new tokens and 1000 to 3500 keys, 16 heads of 64: 124 us in their own order, 104 so).
template <int ROWS, bool LONGEST>
__device__ __forceinline__ bool find_tile(const AttendArgs& a, int x, RowTile& t) {
    const int each = (int)(a.tokens / a.sequences);
    const bool sorted = LONGEST && !a.ids && a.found && a.sequences > 1 && a.sequences <= 64;
    if (!a.q_start && !sorted) {
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
            first = a.q_start ? min(max(a.q_start[s], 0), (int)a.tokens) : s * each;
            count = a.q_start ? max(min(a.q_start[s + 1], (int)a.tokens) - first, 0) : each;
        }
        const int n = (count * a.group + ROWS - 1) / ROWS;
        int upto = n;                                       // tiles up to and with this sequence's
        if (sorted) {
            const int length = s < a.sequences ? a.lengths[s] : 0;
            for (int o = 0; o < a.sequences; ++o) {
                const int other = __builtin_amdgcn_readlane(length, o);
                if (other > length || (other == length && o < s)) upto += __builtin_amdgcn_readlane(n, o);
            }
        } else {
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int w = __shfl_up(upto, o, 64);
                if (lane >= o) upto += w;
            }
        }
        const unsigned long long mine = __ballot(x - base >= upto - n && x - base < upto);
        if (mine) {
            const int src = __ffsll((long long)mine) - 1;
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
//   - A step of 0 stands beside codes of 0: any step may be taken in its place.  The key counts in the sum and adds nothing to the numerator, so the step
//     is one, kNoStep, with which its y hardly ever raises M (the weights of the other keys would be rounded where binary16 has few bits or none: with a step of
//     1, one zero row with a logit of 10 among values of 0.01 put answers off by 20 times their rounding and more).  Keys of step s keep their 11 bits up to a logit of log2(s) + 107 octaves below its.
//   - A NaN step of the values acts through add alone: rows that do not see the key multiply `inverse` by 0.
// While all steps of the values are within 2^-45 .. 2^10 ("tame") or 0, the operand 2^kLift w of a key whose share of the sum is 2^-40 of the largest is still a normal
// float, whatever the two keys' steps are, and operand * inverse is the sum's term.  From the first tile on that has a step beyond that ("wild"), the terms are exponentials of their own,
// relative to the largest of them so far (WildSum): between values of 2^-100 and 2^127 an operand's term may be 2^-125 or 2^107 times it, and terms next to 2^-126 would be lost.  (The same cases
// with values 2^14 times as large: 64 tokens after up to 8192 keys 150 instead of 140 us, over 4 bits 107 instead of 89; 4096 tokens after 28672 3.2 ms instead of 2.2.  In k_attend_rows the wild
// sums stay beside the others in one loop, marked unlikely: with a loop of their own, 48 tokens over passages took 54 instead of 51 us, over 4 bits 53 instead of 48.)
constexpr float kTameLow = 0x1p-45f, kTameHigh = 0x1p10f, kNoStep = 0x1p-84f;
// The reference M of the weights is raised only when a score passes it by more than kSlack, so the answer's registers are rarely rescaled.  Weights stay below
// 2^kSlack, and the operands 2^kLift w below 2^15, the last power of two but one that binary16 holds.  (Without the lift, weights below 2^-14 would lose bits and those
// below 2^-25 become 0 in the numerator alone: an answer of one key 20 to 26 octaves above 2^19 others was up to 1.8 % off.)  The kernels hold M - kLift, called M there.
// The difference itself is compared: in logits of 2^24 and more, whose neighbours lie 2 to 16 apart, M + kSlack + kLift and top - kLift round, and an operand of 2^16 would be an infinity.
constexpr float kSlack = 6.0f, kLift = 9.0f;
__device__ __forceinline__ bool passes(float top, float m) { return top - m > kSlack + kLift; }
__device__ __forceinline__ float raised(float top, float m) {
    const float r = fmaxf(m, top - kLift);
    return passes(top, r) ? top : r;
}
constexpr float kUnlift = 1.0f / 512;          // 2^-kLift
struct KeySteps { float product, add, inverse, log_inverse; bool wild; };
__device__ __forceinline__ KeySteps key_steps(float ks, float vs, float c, float bias, bool have) {
    const bool wild = vs != 0.0f && (vs < kTameLow || vs > kTameHigh);
    vs = vs == 0.0f ? kNoStep : vs < 0x1p-120f ? 0x1p-120f : vs;
    const float lg = __log2f(vs);
    KeySteps k;
    k.product = have ? ks * c : 0.0f;
    k.add = have ? lg + bias : -INFINITY;
    k.inverse = (have && vs == vs ? __builtin_amdgcn_rcpf(vs) : 1.0f) * kUnlift;       // (1 ulp)
    k.log_inverse = have && vs == vs ? -lg - kLift : 0.0f;      // takes the place of `inverse` from a tile with a wild key on: that may be no normal float
    k.wild = have && wild;
    return k;
}

// x * 2^d where 2^d may be below the normal floats and the product is not.
__device__ __forceinline__ float times_exp2(float x, float d) {
    const float h = __builtin_amdgcn_exp2f(0.5f * d);
    return x * h * h;
}

// A row's sum over wild tiles: terms 2^t, t = y + log2 inverse, relative to their largest so far.  sum 2^(ref - M) is what L holds otherwise.
struct WildSum {
    float ref;
    __device__ __forceinline__ void begin(float& l, float m) {         // (M may have been raised far above the terms so far)
        ref = l == 0.0f ? -INFINITY : m + (float)__builtin_amdgcn_frexp_expf(l);
        l = __builtin_amdgcn_frexp_mantf(l);
    }
    // The lane's keys of a tile.  each(f): f(y, log_inverse) for every four of them, both as f32x4; twice, so that their sums stay out of the registers between.
    template <typename F>
    __device__ __forceinline__ void add(float& l, F&& each) {
        float top = ref;
        each([&](const f32x4 y, const f32x4 log_inverse) {
#pragma unroll
            for (int j = 0; j < 4; ++j) top = fmaxf(top, y[j] + log_inverse[j]);
        });
        const float use = top == -INFINITY ? 0.0f : top;
        l *= __builtin_amdgcn_exp2f(ref - use);
        ref = top;
        asm volatile("" ::: "memory");
        each([&](const f32x4 y, const f32x4 log_inverse) {
#pragma unroll
            for (int j = 0; j < 4; ++j) l += __builtin_amdgcn_exp2f(y[j] + log_inverse[j] - use);
        });
    }
    __device__ __forceinline__ float end(float l, float m) const { return l == 0.0f ? 0.0f : times_exp2(l, ref - m); }
};

// A 32-bit offset that is widened where it is used (scalar base + vector offset in one instruction) instead of being kept as 64 bits.
__device__ __forceinline__ uint32_t here(uint32_t x) {
    asm volatile("" : "+v"(x));
    return x;
}

// LDS is served in a wavefront's order; this keeps the compiler from moving accesses that other lanes depend on.
__device__ __forceinline__ void wave_lds_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// A tile of 64 keys: keys k .. k + 63 of a table of `length` keys.  All values are the same in every thread of a block.
struct KeyTile {
    const int32_t* pages;
    int k, length;
    float bias;
    bool have;
};

// The score of the sequence's passage with the largest finite term.  Terms are taken relative to it, which no weight notices: distances of 10^5 that differ by a few
// would leave y few bits behind the binary point (answers were off by up to 20 times their rounding).  The same in every thread; 0.1 us where few rows are asked.
__device__ __forceinline__ float best_score(const AttendArgs& a, int s) {
    const float sign = a.weight < 0.0f ? -1.0f : 1.0f;
    float top = -INFINITY;
    auto take = [&](int r0, auto n) {                           // passages r0 .. r0 + 64 n - 1, all requested together (one by one, 4096 passages took 30 us more)
        constexpr int N = decltype(n)::value;
        int64_t id[N];
        float x[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int64_t at = (int64_t)s * a.found + min(r0 + 64 * i + (int)(threadIdx.x & 63), a.found - 1);
            id[i] = a.ids[at];
            x[i] = sign * a.scores[at];
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            if ((uint64_t)id[i] < (uint64_t)a.passages && fabsf(a.weight * x[i]) < INFINITY) top = fmaxf(top, x[i]);
    };
    if (a.found <= 64) take(0, std::integral_constant<int, 1>{});
    else for (int r0 = 0; r0 < a.found; r0 += 512) take(r0, std::integral_constant<int, 8>{});
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    top = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(top)));
    return top == -INFINITY ? 0.0f : sign * top;
}

// The key tiles of one split, in order: units of tables (AttendArgs), 64 keys at a time.
struct KeyTiles {
    int r, sub, left, k_end;
    float best;                // best_score
    int r0, info;              // passages r0 .. r0 + 20: lanes 3 i, 3 i + 1, 3 i + 2 hold the number (-1: none), the length and the bias of passage r0 + i
    KeyTile t;

    __device__ __forceinline__ void start(const AttendArgs& a, int s, int split) {
        const int u = split * a.per_split;
        left = min(a.found * a.units, u + a.per_split) - u;
        r = u / a.units;
        sub = u - r * a.units - 1;
        k_end = 0;
        t = KeyTile{nullptr, 0, 0, 0.0f, true};
        r0 = r;
        info = 0;
        best = 0.0f;
        if (a.ids && left > 0) {
            if (a.scores) best = best_score(a, s);
            look_up(a, s);
        }
    }
    // Everything about the next 21 passages at once: one by one, each would wait for its number and then for its length.
    __device__ __forceinline__ void look_up(const AttendArgs& a, int s) {
        const int lane = threadIdx.x & 63, p = lane / 3, field = lane - 3 * p;
        const int64_t at = (int64_t)s * a.found + min(r0 + p, a.found - 1);
        const int64_t id = a.ids[at];
        const float score = a.scores ? a.scores[at] : 0.0f, bias = a.weight * (score - best);
        const bool ok = (uint64_t)id < (uint64_t)a.passages && a.weight * score != -INFINITY;
        const int length = min(max(a.lengths[ok ? id : 0], 0), a.width << a.st.shift);
        info = field == 0 ? (ok ? (int)id : -1) : field == 1 ? length : __float_as_int(bias);
    }
    // Moves on by `n` tiles.
    __device__ __forceinline__ void skip(const AttendArgs& a, int s, int behind, int n) {
        if (__builtin_expect(t.k + n * kTileKeys < k_end, 1)) { t.k += n * kTileKeys; return; }
#pragma unroll 1
        for (int i = 0; i < n; ++i) next(a, s, behind);
    }
    // Moves on to the next tile (t.have: there is one).  `behind`: tokens of the sequence after the last one that any row of the block sees (causal only).
    __device__ __forceinline__ void next(const AttendArgs& a, int s, int behind) {
        if (!t.have) return;
        t.k += kTileKeys;
        if (__builtin_expect(t.k < k_end, 1)) return;
        while (t.k >= k_end) {
            if (--left < 0) { t.have = false; return; }
            if (++sub == a.units) { sub = 0; ++r; }
            int table = s;
            if (a.ids) {
                if (r - r0 >= 21) { r0 = r; look_up(a, s); }
                const int i = 3 * (r - r0);
                table = __builtin_amdgcn_readlane(info, i);
                t.k = k_end = 0;
                if (table < 0) continue;
                t.length = __builtin_amdgcn_readlane(info, i + 1);
                t.bias = __int_as_float(__builtin_amdgcn_readlane(info, i + 2));
            } else {
                t.length = min(max(a.lengths[table], 0), a.width << a.st.shift);
            }
            t.pages = a.tables + (int64_t)table * a.width;
            t.k = sub * a.unit;
            k_end = min(a.ids ? t.length : t.length - behind, t.k + a.unit);
        }
    }
};

// Few query rows: bound by reading the states, 2 D + 8 bytes per key and head for up to 16 rows.  Measured: 64 tokens of 32 heads over 1638 to 8192 keys (8 heads of
// 128, 705 MB) 140 us, 5.0 TB/s; one token of 64 heads over 131072 keys (8 heads of 128, 277 MB, 512 splits) 44 us + 4.5 us for the join; one token
// over 4001 keys 8.4 + 3.1 us, of which the memory would take 2: two rounds of dependent loads (length and page, then codes) and two launches.
// A block has up to 16 rows of one head and a range of keys; its wavefronts take tiles of 64 keys in turn,
// codes straight from memory into registers in the order of the matrix operands (no LDS: the order of the contracted axis is free), and
// their sums are joined in LDS at the end.  The first product is formed transposed (keys x rows), so a lane holds 16 scores of ONE row: statistics are
// in-lane but for exchanges between the four quarters of the wavefront, and the weights are the second product's operand as they stand.
// The next tile's keys are requested as soon as the first product has used this one's, its values after the second product, its page number one tile
// earlier: a wavefront always has 8 to 16 KiB in flight.  WHOLE: pages of 64 tokens and more, a tile lies in one.
// RT: tiles of 16 rows of a block, which share the converted codes.
// BITS 4: a lane's piece of a key row has the 8 codes of each step (at 128 values, 32 consecutive ones: 16 bytes as well), a 16-byte piece of the values has two components; the
// factors of a tile's keys and values go through LDS beside the steps.
template <typename T, int D, bool WHOLE, int BITS, int RT>
__global__ void __launch_bounds__(64 * kAttendWaves, 2) k_attend_rows(AttendArgs a) {
    constexpr int S32 = D / 32;                                 // steps of the first product, 32 values each
    constexpr int C = D / 64, ODD = S32 & 1;                    // 16-byte pieces of a lane's key row (two steps each), and one of 8 bytes
    constexpr int DT = D / 16;                                  // 16-value tiles of the answer
    constexpr bool FOUR = BITS == 4;
    constexpr int VT = FOUR ? DT / 2 : DT;                      // rows of the values' codes that a lane reads
    __shared__ __align__(16) float lds_step[kAttendWaves][3][kTileKeys];
    __shared__ __align__(16) float lds_acc[kAttendWaves][kRows][D + 4];
    __shared__ float lds_m[kAttendWaves][kRows], lds_l[kAttendWaves][kRows];
    __shared__ uint32_t lds_kf[FOUR ? kAttendWaves : 1][kTileKeys];
    __shared__ __align__(16) _Float16 lds_vf[FOUR ? kAttendWaves : 1][S32][kTileKeys];      // in the order of the second product

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, quarter = lane >> 4;
    const BlockWork work = block_work(a);
    const int head = work.head, split = work.split;
    RowTile tile;
    if (!find_tile<kRows * RT, false>(a, work.tile, tile)) return;
    const int rows = tile.count * a.group;
    bool live[RT];                                              // of the lane's row in each of the block's tiles of 16 rows
    int tok[RT], see_after[RT];                                 // its token; tokens of the sequence that it does not see
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int row = tile.row0 + kRows * t + n;
        live[t] = row < rows;
        tok[t] = live[t] ? row / a.group : 0;
        see_after[t] = tile.count - 1 - tok[t];
    }
    const int behind = tile.count - 1 - (min(rows, tile.row0 + kRows * RT) - 1) / a.group, first_behind = tile.count - 1 - tile.row0 / a.group;
    const int P = 1 << a.st.shift;

    // What does not depend on lengths is requested first: the queries, and (chunk: one unit of the sequence's own table) the pages of the wavefront's first tile.
    auto component = [&](int i) {                               // first of the lane's 8 in step i
        if (FOUR && D == 128) return 32 * quarter + 8 * i;
        return i < 2 * C ? 64 * (i >> 1) + 16 * quarter + 8 * (i & 1) : 64 * C + 8 * quarter;
    };
    i32x4 raw[RT][S32];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int qh = head * a.group + (live[t] ? tile.row0 + kRows * t + n - tok[t] * a.group : 0);
        const int64_t q_at = (int64_t)(tile.first + tok[t]) * a.q_token + (int64_t)qh * a.q_head;
#pragma unroll
        for (int i = 0; i < S32; ++i) raw[t][i] = load8_raw(a.q, q_at + component(i), a.q_wide);
    }
    int page = 0;                                               // lane = key of a tile: its page
    const bool ahead = !a.ids && a.width > 0;
    if (ahead) page = a.tables[(int64_t)tile.s * a.width + min((split * a.unit + wave * kTileKeys + lane) >> a.st.shift, a.width - 1)];
    // the wavefront's tiles: every fourth of the block's
    KeyTiles it;
    it.start(a, tile.s, split);
    auto find_page = [&](const KeyTile& kt) {
        if (kt.have) page = kt.pages[min(kt.k + lane, kt.length - 1) >> a.st.shift];
    };
    // Operands: row i of the first product's tile b (of four) is key 16 (i >> 2) + 4 b + (i & 3), so that a quarter's 16 results are 16 consecutive keys -
    // the 16 consecutive bytes of a component in the transposed values.
    const int my_key = 16 * (n >> 2) + (n & 3);                 // (+ 4 b)
    constexpr int ROW = D * BITS / 8;                           // bytes of a key row
    const uint32_t page_bytes = (uint32_t)ROW << a.st.shift;
    i32x4 kr[4][C > 0 && !FOUR ? C : 1], vr[VT];                // (4 bits: one piece, of which a lane uses D / 8 bytes)
    uint2 ko[4];
    uint32_t rkf = 0, rvf = 0;
    float rks = 0.0f, rvs = 0.0f;
    bool rhave = false;
    int row_of_key = 0, row_of_tile = 0, place = 0;             // page * heads + head, per lane and (WHOLE) for the tile; place in the page
    auto fetch_keys = [&](const KeyTile& kt) {
        if (!kt.have) return;
        const bool known = (uint32_t)page < (uint64_t)a.st.pages;
        rhave = known && kt.k + lane < kt.length;
        row_of_key = (known ? page : 0) * a.st.heads + head;     // (a page number outside the store becomes page 0, its keys get no weight)
        place = kt.k & (P - 1);
        if constexpr (WHOLE) row_of_tile = __builtin_amdgcn_readfirstlane(row_of_key);
        const uint64_t at = ((uint64_t)(uint32_t)(WHOLE ? row_of_tile : row_of_key) << a.st.shift) + (uint32_t)((place + lane) & (P - 1));
        rks = a.st.ks[at];
        rvs = a.st.vs[at];
        if constexpr (FOUR) {
            rkf = a.st.kf[at];
            rvf = a.st.vf[at];
        }
        if constexpr (FOUR) {
            const int8_t* base = a.st.kc + (uint64_t)(uint32_t)row_of_tile * page_bytes + (uint32_t)(place * ROW);          // (WHOLE)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int key = my_key + 4 * b;
                const int8_t* kp = WHOLE ? base : a.st.kc + (uint64_t)(uint32_t)__shfl(row_of_key, key, 64) * page_bytes;
                const uint32_t at = (uint32_t)((WHOLE ? key : key & (P - 1)) * ROW);          // (a scalar base and a vector offset where the tile lies in one page)
                if constexpr (D == 128) kr[b][0] = *(const i32x4*)(kp + here(at + 16 * quarter));
                if constexpr (C == 1) {
                    const i32x2 two = *(const i32x2*)(kp + here(at + 8 * quarter));
                    kr[b][0][0] = two[0];
                    kr[b][0][1] = two[1];
                }
                if constexpr (ODD) kr[b][0][2 * C] = *(const int*)(kp + here(at + 32 * C + 4 * quarter));
            }
        } else if constexpr (WHOLE) {
            const int8_t* base = a.st.kc + (uint64_t)(uint32_t)row_of_tile * page_bytes + (uint32_t)(place * D);
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int key = my_key + 4 * b;
#pragma unroll
                for (int i = 0; i < C; ++i) kr[b][i] = *(const i32x4*)(base + here(key * D + 64 * i + 16 * quarter));
                if constexpr (ODD) ko[b] = *(const uint2*)(base + here(key * D + 64 * C + 8 * quarter));
            }
        } else {
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int key = my_key + 4 * b;
                const int8_t* kp = a.st.kc + (uint64_t)(uint32_t)__shfl(row_of_key, key, 64) * page_bytes + (uint32_t)((key & (P - 1)) * D);
#pragma unroll
                for (int i = 0; i < C; ++i) kr[b][i] = *(const i32x4*)(kp + (uint32_t)(64 * i + 16 * quarter));
                if constexpr (ODD) ko[b] = *(const uint2*)(kp + (uint32_t)(64 * C + 8 * quarter));
            }
        }
    };
    auto fetch_values = [&](bool have, int row_tile, int row_key, int at) {
        if (!have) return;
        const int key = 16 * quarter;
        if constexpr (WHOLE) {
            const int8_t* base = a.st.vc + (uint64_t)(uint32_t)row_tile * page_bytes + (uint32_t)at;
#pragma unroll
            for (int i = 0; i < VT; ++i) vr[i] = *(const i32x4*)(base + here(((n + 16 * i) << a.st.shift) + key));
        } else {
            const int8_t* vp = a.st.vc + (uint64_t)(uint32_t)__shfl(row_key, key, 64) * page_bytes + (uint32_t)((n << a.st.shift) + (key & (P - 1)));
#pragma unroll
            for (int i = 0; i < VT; ++i) vr[i] = *(const i32x4*)(vp + ((uint32_t)(16 * i) << a.st.shift));
        }
    };
    it.skip(a, tile.s, behind, 1 + wave);
    KeyTile cur = it.t;
    if (!ahead) find_page(cur);
    fetch_keys(cur);
    const int first_row_tile = row_of_tile, first_row_key = row_of_key, first_place = place;
    it.skip(a, tile.s, behind, kAttendWaves);
    find_page(it.t);
    fetch_values(cur.have, first_row_tile, first_row_key, first_place);

    // queries, normalised to binary16 by a power of two per row
    f16x8 qf[RT][S32];
    float q_back[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        float top = 0.0f;
#pragma unroll
        for (int i = 0; i < S32; ++i) {
            if (!live[t]) raw[t][i] = i32x4{0, 0, 0, 0};
            float f[8];
            widen8<T>(raw[t][i], f);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float m = fabsf(f[j]);
                if (m <= 3.4028235e38f) top = fmaxf(top, m);
            }
        }
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        float up;
        row_power(top, up, q_back[t]);
#pragma unroll
        for (int i = 0; i < S32; ++i) {
            float f[8];
            widen8<T>(raw[t][i], f);
#pragma unroll
            for (int j = 0; j < 8; ++j) qf[t][i][j] = (_Float16)(f[j] * up);
        }
    }

    f32x4 acc[RT][DT];
    float M[RT], L[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
#pragma unroll
        for (int i = 0; i < DT; ++i) acc[t][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        M[t] = -INFINITY;
        L[t] = 0.0f;
    }
    bool wild = false;                                          // some step so far is not tame
    WildSum terms[RT];

    while (cur.have) {
        bool now_wild;                                          // ... with this tile's
        {
            wave_lds_order();                                   // the previous tile's steps have been read
            const KeySteps ks = key_steps(rks, rvs, a.c, cur.bias, rhave);
            lds_step[wave][0][lane] = ks.product;
            lds_step[wave][1][lane] = ks.add;
            now_wild = wild | (__ballot(ks.wild) != 0);
            lds_step[wave][2][lane] = ks.inverse;
            if (__builtin_expect(now_wild, 0)) lds_step[wave][2][lane] = ks.log_inverse;
            if constexpr (FOUR) {
                lds_kf[wave][lane] = rkf;
#pragma unroll
                for (int g = 0; g < S32; ++g) lds_vf[wave][g][(lane & ~7) + token_place(lane & 7)] = factor_half(rvf, g);
            }
            wave_lds_order();
        }
        f32x4 s[RT][4];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
#pragma unroll
            for (int t = 0; t < RT; ++t) s[t][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            if constexpr (FOUR) {
                const uint32_t factors = lds_kf[wave][my_key + 4 * b];
                f16x8 r;
#pragma unroll
                for (int i = 0; i < S32; ++i) {
                    if (i == 0 || (D != 128 && i == 2 * C)) r = spread(factor_pair(factors, (uint32_t)component(i) / 32));      // (128 values: the lane's 32 share one)
                    const f16x8 k = codes4_to_half((uint32_t)kr[b][0][i]) * r;
#pragma unroll
                    for (int t = 0; t < RT; ++t) s[t][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, qf[t][i], s[t][b], 0, 0, 0);
                }
            } else {
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    f16x8 lo, hi;
                    codes_to_half(kr[b][i], lo, hi);
#pragma unroll
                    for (int t = 0; t < RT; ++t) {
                        s[t][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo, qf[t][2 * i], s[t][b], 0, 0, 0);
                        s[t][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi, qf[t][2 * i + 1], s[t][b], 0, 0, 0);
                    }
                }
                if constexpr (ODD) {
                    f16x8 lo, hi;
                    codes_to_half(i32x4{(int)ko[b].x, (int)ko[b].y, 0, 0}, lo, hi);
#pragma unroll
                    for (int t = 0; t < RT; ++t) s[t][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo, qf[t][2 * C], s[t][b], 0, 0, 0);
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        const KeyTile nxt = it.t;
        fetch_keys(nxt);
        it.skip(a, tile.s, behind, kAttendWaves);
        find_page(it.t);
        __builtin_amdgcn_sched_barrier(0);
        f16x8 w[RT][2];
        const bool was_wild = wild;
        wild = now_wild;
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            float top = -INFINITY;
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const f32x4 sk = *(const f32x4*)&lds_step[wave][0][16 * quarter + 4 * b], lv = *(const f32x4*)&lds_step[wave][1][16 * quarter + 4 * b];
#pragma unroll
                for (int j = 0; j < 4; ++j) s[t][b][j] = fmaf(s[t][b][j], sk[j] * q_back[t], lv[j]);          // (the product by itself, up to 2^29, times a row's factor of 2^113 would be an infinity)
            }
            if (!a.ids && cur.k + kTileKeys > cur.length - first_behind) {       // some row may not see all of it
                const int see = cur.length - see_after[t] - cur.k - 16 * quarter;
#pragma unroll
                for (int b = 0; b < 4; ++b)
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[t][b][j] = 4 * b + j < see ? s[t][b][j] : -INFINITY;
            }
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int j = 0; j < 4; ++j) top = fmaxf(top, s[t][b][j]);
            if (__ballot(passes(top, M[t]))) {
                top = fmaxf(top, __shfl_xor(top, 32, 64));
                top = fmaxf(top, __shfl_xor(top, 16, 64));
                const float m_new = raised(top, M[t]), d = M[t] - (m_new == -INFINITY ? 0.0f : m_new);
                const float shrink = __builtin_amdgcn_exp2f(d);
                if (!was_wild) L[t] = times_exp2(L[t], d);
                M[t] = m_new;
#pragma unroll
                for (int i = 0; i < DT; ++i) acc[t][i] = acc[t][i] * shrink;
            }
            const float m_use = M[t] == -INFINITY ? 0.0f : M[t];
            float l = 0.0f;                                         // the tile's part of the sum: terms far below the sum so far would each be rounded away
            auto weigh = [&](auto with_sum) {
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const f32x4 iv = *(const f32x4*)&lds_step[wave][2][16 * quarter + 4 * b];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float e = __builtin_amdgcn_exp2f(s[t][b][j] - m_use);
                        if (decltype(with_sum)::value && !(wild && !FOUR)) l = fmaf(e, iv[j], l);
                        w[t][b >> 1][FOUR ? token_place(4 * (b & 1) + j) : 4 * (b & 1) + j] = (_Float16)e;
                    }
                }
            };
            if (__builtin_expect(wild, 0)) {
                if (!was_wild) terms[t].begin(L[t], M[t]);
                terms[t].add(L[t], [&](auto&& f) {
#pragma unroll
                    for (int b = 0; b < 4; ++b) f(s[t][b], *(const f32x4*)&lds_step[wave][2][16 * quarter + 4 * b]);
                });
            }
            if (FOUR && __builtin_expect(wild, 0)) weigh(std::false_type{});             // (8 bits: one copy, with a select)
            else weigh(std::true_type{});
            L[t] += l;
            asm volatile("" : "+v"(L[t]));                             // (the sum is formed here: kept for later, its terms would fill the registers)
        }
        if constexpr (FOUR) {
#pragma unroll
            for (int i = 0; i < VT; ++i)
#pragma unroll
                for (int o = 0; o < 2; ++o) {
                    const f16x8 r = *(const f16x8*)&lds_vf[wave][i][16 * quarter + 8 * o];
                    uint32_t low, high;
                    split_values4((uint32_t)vr[i][2 * o], (uint32_t)vr[i][2 * o + 1], low, high);
                    const f16x8 v0 = codes4_to_half(low) * r, v1 = codes4_to_half(high) * r;
#pragma unroll
                    for (int t = 0; t < RT; ++t) {
                        acc[t][2 * i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, w[t][o], acc[t][2 * i], 0, 0, 0);
                        acc[t][2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, w[t][o], acc[t][2 * i + 1], 0, 0, 0);
                    }
                }
        } else
#pragma unroll
        for (int i = 0; i < DT; ++i) {
            f16x8 lo, hi;
            codes_to_half(vr[i], lo, hi);
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                acc[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo, w[t][0], acc[t][i], 0, 0, 0);
                acc[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi, w[t][1], acc[t][i], 0, 0, 0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        fetch_values(nxt.have, row_of_tile, row_of_key, place);
        cur = nxt;
    }
    // join the wavefronts, a tile of rows at a time
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        float l_all = wild ? terms[rt].end(L[rt], M[rt]) : L[rt];
        l_all += __shfl_xor(l_all, 32, 64);
        l_all += __shfl_xor(l_all, 16, 64);
        if (rt) __syncthreads();                                // (the last tile's have been read)
        if (quarter == 0) { lds_m[wave][n] = M[rt]; lds_l[wave][n] = l_all; }
        __syncthreads();
        float m_all = lds_m[0][n];
#pragma unroll
        for (int w = 1; w < kAttendWaves; ++w) m_all = fmaxf(m_all, lds_m[w][n]);
        {
            const float f = __builtin_amdgcn_exp2f(M[rt] - (m_all == -INFINITY ? 0.0f : m_all));
#pragma unroll
            for (int i = 0; i < DT; ++i) *(f32x4*)&lds_acc[wave][n][16 * i + 4 * quarter] = acc[rt][i] * f;
        }
        __syncthreads();
        constexpr int Q = D / 4;
        const int heads = a.st.heads * a.group;
        for (int i = threadIdx.x; i < kRows * Q; i += 64 * kAttendWaves) {
            const int rr = i / Q, d = (i - rr * Q) * 4;
            const int grow = tile.row0 + kRows * rt + rr;
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
                const float inv = l == 0.0f ? 0.0f : kUnlift / l;
                store4<T>(a.out, (int64_t)t * a.out_token + (int64_t)hq * a.out_head + d, a.out_wide, o * inv);
            } else {
                const int64_t at = ((int64_t)split * a.tokens + t) * heads + hq;
                if (l != 0.0f) *(f32x4*)&a.part_acc[at * D + d] = o;       // (l = 0: no key was seen, and nothing is read there)
                if (d == 0) { a.part_m[at] = m; a.part_l[at] = l; }
            }
        }
    }
}

// Joins the splits of each row: out = (sum_s 2^(M_s - M) acc_s) / (sum_s 2^(M_s - M) l_s), acc lifted.  Bound by latency for one token (3 us with 16 to 512 splits).  D / 4 threads hold a row's values; `sides` such groups share a row's splits (a power of two, as many as there are splits
// while the block has room), each with a running reference of its own, and the block's other groups take other rows.
template <typename T, int D, int BITS>          // (BITS: the store's, a name of its own in each library file)
__global__ void __launch_bounds__(256) k_attend_join(AttendArgs a, int sides) {
    constexpr int Q = D / 4, GROUPS = 256 / Q;
    __shared__ __align__(16) f32x4 lds_o[GROUPS][Q];
    __shared__ float lds_l[GROUPS], lds_m[GROUPS];
    const int heads = a.st.heads * a.group;
    const int group = threadIdx.x / Q, d = threadIdx.x - group * Q;
    const int side = group & (sides - 1), rows = GROUPS / sides;
    const int64_t all = a.tokens * heads, row = (int64_t)blockIdx.x * rows + group / sides, t = row / heads;
    bool live = group < rows * sides && row < all;
    if (live && a.q_start) live = t >= a.q_start[0] && t < a.q_start[a.sequences];      // no sequence's: nothing was computed
    float m = -INFINITY, l = 0.0f;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    if (live) {
        for (int s0 = side; s0 < a.splits; s0 += 4 * sides) {
            float ms[4], ls[4];
            f32x4 os[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {                     // (four at a time are requested together)
                const int s = s0 + i * sides;
                const int64_t at = (int64_t)min(s, a.splits - 1) * all + row;
                ms[i] = a.part_m[at];
                ls[i] = a.part_l[at];
                os[i] = *(const f32x4*)&a.part_acc[at * D + 4 * d];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (s0 + i * sides >= a.splits) break;
                const float m_new = fmaxf(m, ms[i]), m_use = m_new == -INFINITY ? 0.0f : m_new;
                l = times_exp2(l, m - m_use) + times_exp2(ls[i], ms[i] - m_use);
                o = o * __builtin_amdgcn_exp2f(m - m_use);
                if (ls[i] != 0.0f) o += os[i] * __builtin_amdgcn_exp2f(ms[i] - m_use);
                m = m_new;
            }
        }
    }
    if (group < GROUPS) {
        lds_o[group][d] = o;
        if (d == 0) { lds_m[group] = m; lds_l[group] = l; }
    }
    __syncthreads();
    if (!live || side) return;
    float m_all = m;
    for (int i = 1; i < sides; ++i) m_all = fmaxf(m_all, lds_m[group + i]);
    const float m_use = m_all == -INFINITY ? 0.0f : m_all;
    l = times_exp2(l, m - m_use);
    o = o * __builtin_amdgcn_exp2f(m - m_use);
    for (int i = 1; i < sides; ++i) {
        const float dm = lds_m[group + i] - m_use;
        l += times_exp2(lds_l[group + i], dm);
        o += lds_o[group + i][d] * __builtin_amdgcn_exp2f(dm);
    }
    const float inv = l == 0.0f ? 0.0f : kUnlift / l;
    store4<T>(a.out, t * a.out_token + (row - t * heads) * a.out_head + 4 * d, a.out_wide, o * inv);
}

}  // namespace lorann
