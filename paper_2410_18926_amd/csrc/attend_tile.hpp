// Attention of many query rows (a chunk of new tokens, questions over passages).  Mathematics in attend.hpp.
//
// What bounds it: per 64 keys and 32 rows a wavefront issues D / 4 matrix instructions of 32 cycles (D = 128: 1024 cycles) and 240 to 310 vector instructions
// of 4, its 32 exponentials of 8 (per score: y, half a maximum, y - M, the exponential, the sum, half a conversion; then the codes' conversion).  Counted at D = 128: 1224 cycles of
// vector instructions with 8 wavefronts, 1505 with 4; at D = 64 with pages of 16: 1394.  The two overlap little: where blocks are many and alike, a wavefront's tile
// takes 2471 cycles of its SIMD at D = 128, half of them with a vector instruction, 41 % with a matrix instruction.  The clock falls to 2.0 - 2.2 GHz meanwhile.
// Measured: 4096 tokens of 32 heads after 28672 (8 heads of 128) 2.2 ms, 0.93 PFLOP/s; 12 sequences of up to 500 tokens after up to 3000 (16 heads of 64)
// 90 - 102 us, a tile's SIMD time 3009 cycles (blocks of unequal length: some SIMDs have nothing left); 24 questions of up to 96 tokens over 10 passages of up to 512 keys 142 - 166 us,
// 3958 cycles (448 blocks that have rows for 256 CUs, a fifth of their rows empty).
#pragma once
#include "attend.hpp"

namespace lorann {

__device__ __forceinline__ int pick4(const i32x4 v, int i) { return i & 2 ? (i & 1 ? v[3] : v[2]) : (i & 1 ? v[1] : v[0]); }

// f(0) .. f(N - 1) with the number as a constant of its type (array elements picked by it stay in registers).
template <int I, int N, typename F>
__device__ __forceinline__ void unrolled(F&& f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        unrolled<I + 1, N>(f);
    }
}

// A block has NW * 32 query rows of one head; a wavefront 32 of them.  The block's threads convert each tile of 64 keys and values once to
// binary16 in LDS, in the order of the matrix operands (next tile's codes are in flight and are converted into the other buffer while this one
// is used; one barrier per tile).  As in k_attend_rows the scores come out transposed, a lane holds scores of one row, and the weights
// are the second product's operand as they stand.  Conversion once per block is why a block has 128 or 256 rows and why LDS is used at all: straight to
// registers, as k_attend_rows does, each wavefront would convert all codes itself (320 instructions per tile at D = 128 instead of 80 or 40).
// BITS 4: a piece has 16 codes all the same, in 8 bytes: of a key, or of two components and 8 tokens, which come to lie in the order of token_place (the weights likewise).  A piece's codes
// are multiplied by their factors as they are converted; the values' factors are in LDS one tile ahead, written with the steps.
template <typename T, int D, int NW, bool WHOLE, int BITS>
__global__ void __launch_bounds__(64 * NW, 2) k_attend_tile(AttendArgs a) {
    constexpr int C = D / 32, ROWS = NW * 32, THREADS = 64 * NW;
    constexpr int KS = D + 8, VS = kTileKeys + 8;               // row strides in LDS (16 bytes of padding: rows start in other banks)
    constexpr int PIECES = kTileKeys * D / 16;                  // 16-code pieces of the keys, and of the values
    constexpr int PER = (PIECES + THREADS - 1) / THREADS;
    constexpr bool FOUR = BITS == 4;
    constexpr int ROW = D * BITS / 8;                           // bytes of a key row
    typedef std::conditional_t<FOUR, i32x2, i32x4> Piece;
    __shared__ __align__(16) _Float16 lds_k[2][kTileKeys * KS];
    __shared__ __align__(16) _Float16 lds_v[2][D * VS];
    __shared__ __align__(16) float lds_step[3][3][kTileKeys];
    __shared__ int lds_flag[NW], lds_wild[3];
    __shared__ __align__(16) _Float16 lds_vf[FOUR ? 3 : 1][C][kTileKeys];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, half = lane >> 5;
    const BlockWork work = block_work(a);
    const int head = work.head, split = work.split;
    RowTile tile;
    if (!find_tile<ROWS, true>(a, work.tile, tile)) return;
    const int rows = tile.count * a.group;
    const int P = 1 << a.st.shift;

    // queries
    int tok, see_after;
    f16x8 qf[2 * C];
    float row_up;                                               // of rows whose power of two is not the block's
    int e_block;
    bool mixed;
    {
        i32x4 raw[2 * C];
        int e_row;
        int e_max = -1000, e_min = 1000;
        const int row = tile.row0 + wave * 32 + n;
        const bool live = row < rows;
        tok = live ? row / a.group : 0;
        see_after = tile.count - 1 - tok;
        const int qh = head * a.group + (live ? row - tok * a.group : 0);
        const int64_t at = (int64_t)(tile.first + tok) * a.q_token + (int64_t)qh * a.q_head;
        float top = 0.0f;
#pragma unroll
        for (int i = 0; i < 2 * C; ++i) {
            float f[8];
            raw[i] = load8_raw(a.q, at + 16 * i + 8 * half, a.q_wide);
            if (!live) raw[i] = i32x4{0, 0, 0, 0};
            widen8<T>(raw[i], f);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float m = fabsf(f[j]);
                if (m <= 3.4028235e38f) top = fmaxf(top, m);
            }
        }
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        e_row = top < kTinyRow ? -1000 : (int)((__float_as_uint(top) >> 23) & 255) - 127;
        if (e_row > -1000) { e_max = max(e_max, e_row); e_min = min(e_min, e_row); }
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { e_max = max(e_max, __shfl_xor(e_max, o, 64)); e_min = min(e_min, __shfl_xor(e_min, o, 64)); }
        if (lane == 0) lds_flag[wave] = (e_max + 1000) << 12 | (e_min + 1000);
        __syncthreads();
        e_max = -1000; e_min = 1000;
#pragma unroll
        for (int w = 0; w < NW; ++w) { e_max = max(e_max, (lds_flag[w] >> 12) - 1000); e_min = min(e_min, (lds_flag[w] & 4095) - 1000); }
        e_max = __builtin_amdgcn_readfirstlane(e_max);
        e_min = __builtin_amdgcn_readfirstlane(e_min);
        e_block = e_max > -1000 ? e_max : 14;
        mixed = e_max - e_min > 12 && e_max > -1000;
        const int e = mixed && e_row > -1000 ? e_row : e_block;
        const float up = ldexpf(1.0f, 14 - e);
        row_up = ldexpf(1.0f, e - e_block);
#pragma unroll
        for (int i = 0; i < 2 * C; ++i) {
            float f[8];
            widen8<T>(raw[i], f);
#pragma unroll
            for (int j = 0; j < 8; ++j) qf[i][j] = (_Float16)(f[j] * up);
        }
    }
    const float c = ldexpf(a.c, e_block - 14);

    f32x16 acc[C];
    float M = -INFINITY, L = 0.0f;
#pragma unroll
    for (int i = 0; i < C; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) acc[i][j] = 0.0f;

    // Loading: the thread's pieces of the keys (a key, 16 of its values) and of the values (a component, 16 keys), and in one of three wavefronts in turn
    // the steps of a key per lane.  Page numbers are requested one tile before they are used: pages of 64 tokens and more (WHOLE) hold a tile in one
    // piece, smaller ones are looked up for each piece.  A page number outside the store becomes page 0, its keys get no weight.
    // (Vector loads, all lanes the same where the page is: scalar loads would have to return before the next wait for LDS does.)
    int pg[WHOLE ? 1 : PER], pg_step = 0;                       // WHOLE: the tile's page; else the pages of the thread's keys and of the lane's key
    int pv[WHOLE ? 1 : PER];                                    // ... and of the thread's values, of the tile before (WHOLE: as page * heads + head)
    auto page_at = [&](const KeyTile& kt, int key) { return kt.pages[min(kt.k + key, kt.length - 1) >> a.st.shift]; };
    auto find_pages = [&](const KeyTile& kt) {
        if (!kt.have) return;
        if constexpr (WHOLE) pg[0] = *(const int32_t*)((const char*)(kt.pages + (kt.k >> a.st.shift)) + here(0));
        else {
#pragma unroll
            for (int i = 0; i < PER; ++i) pg[i] = page_at(kt, (tid + i * THREADS) / (D / 16) % kTileKeys);
            pg_step = page_at(kt, lane);
        }
    };
    auto row_of = [&](int page) { return ((uint32_t)page < (uint64_t)a.st.pages ? page : 0) * a.st.heads + head; };
    Piece ck[PER], cv[PER];
    uint32_t fk[PER], rvf = 0;                                  // 4 bits: factors of the pieces' keys, and of the values of the lane's key
    float rks = 0.0f, rvs = 0.0f;
    bool rhave = false;
    const uint32_t page_bytes = (uint32_t)ROW << a.st.shift;
    int off_v = 0;                                              // place in the page of the tile whose values are requested next
    bool have_v = false;
    // requests the keys of a tile, its steps in wavefront `by`, and notes where its values are
    auto fetch_keys = [&](const KeyTile& kt, int by) {
        have_v = kt.have;
        if (!kt.have) return;
        const int off = kt.k & (P - 1);                         // (a tile starts at a multiple of 64: within a page, or at a page's start)
        off_v = off;
        if constexpr (WHOLE) {
            const int page = __builtin_amdgcn_readfirstlane(pg[0]);
            pv[0] = row_of(page);
            const int8_t* base = a.st.kc + (uint64_t)(uint32_t)pv[0] * page_bytes + (uint32_t)(off * ROW);
            const uint64_t at = ((uint64_t)(uint32_t)pv[0] << a.st.shift) + (uint32_t)off;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int p = tid + i * THREADS;
                if (PIECES % THREADS && p >= PIECES) break;
                ck[i] = *(const Piece*)(base + here((int)sizeof(Piece) * p));
                if constexpr (FOUR) fk[i] = *(const uint32_t*)((const char*)(a.st.kf + at) + here(4 * (p / (D / 16))));
            }
            if (wave == by) {
                rhave = kt.k + lane < kt.length && (uint32_t)page < (uint64_t)a.st.pages;
                rks = *(const float*)((const char*)(a.st.ks + at) + here(4 * lane));
                rvs = *(const float*)((const char*)(a.st.vs + at) + here(4 * lane));
                if constexpr (FOUR) rvf = *(const uint32_t*)((const char*)(a.st.vf + at) + here(4 * lane));
            }
        } else {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int p = tid + i * THREADS;
                if (PIECES % THREADS && p >= PIECES) break;
                const int key = p / (D / 16), part = p % (D / 16);
                ck[i] = *(const Piece*)(a.st.kc + (uint64_t)(uint32_t)row_of(pg[i]) * page_bytes + (uint32_t)((key & (P - 1)) * ROW + (int)sizeof(Piece) * part));
                if constexpr (FOUR) fk[i] = a.st.kf[((uint64_t)(uint32_t)row_of(pg[i]) << a.st.shift) + (uint32_t)(key & (P - 1))];
                pv[i] = page_at(kt, FOUR ? 8 * (p % 8) : 16 * (p % 4));
            }
            if (wave == by) {
                rhave = kt.k + lane < kt.length && (uint32_t)pg_step < (uint64_t)a.st.pages;
                const uint64_t at = ((uint64_t)(uint32_t)row_of(pg_step) << a.st.shift) + (uint32_t)(lane & (P - 1));
                rks = a.st.ks[at];
                rvs = a.st.vs[at];
                if constexpr (FOUR) rvf = a.st.vf[at];
            }
        }
    };
    auto fetch_values = [&]() {
        if (!have_v) return;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int p = tid + i * THREADS;
            if (PIECES % THREADS && p >= PIECES) break;
            if constexpr (FOUR) {
                const int row = p / 8, key = 8 * (p % 8);
                if constexpr (WHOLE) cv[i] = *(const Piece*)(a.st.vc + (uint64_t)(uint32_t)pv[0] * page_bytes + (uint32_t)off_v + here((row << a.st.shift) + key));
                else cv[i] = *(const Piece*)(a.st.vc + (uint64_t)(uint32_t)row_of(pv[i]) * page_bytes + (uint32_t)((row << a.st.shift) + (key & (P - 1))));
            } else {
                const int comp = p / 4, grp = p % 4;
                if constexpr (WHOLE) cv[i] = *(const Piece*)(a.st.vc + (uint64_t)(uint32_t)pv[0] * page_bytes + (uint32_t)off_v + here((comp << a.st.shift) + 16 * grp));
                else cv[i] = *(const Piece*)(a.st.vc + (uint64_t)(uint32_t)row_of(pv[i]) * page_bytes + (uint32_t)((comp << a.st.shift) + ((16 * grp) & (P - 1))));
            }
        }
    };
    auto put = [&](_Float16* to, const i32x4 codes) {
        f16x8 lo, hi;
        codes_to_half(codes, lo, hi);
        *(f16x8*)to = lo;
        *(f16x8*)(to + 8) = hi;
    };
    auto stage_keys = [&](int kb, int i) {
        const int p = tid + i * THREADS;
        if (PIECES % THREADS && p >= PIECES) return;
        const int key = p / (D / 16), part = p % (D / 16);
        // key 32 h + 16 b + 4 g + q is row 32 b + 8 g + 4 h + q of the first product
        const int krow = (key & 16) * 2 + (key >> 2 & 3) * 8 + (key >> 5) * 4 + (key & 3);
        if constexpr (FOUR) {
            const f16x8 r = spread(factor_pair(fk[i], (uint32_t)part / 2));
            *(f16x8*)&lds_k[kb][krow * KS + 16 * part] = codes4_to_half((uint32_t)ck[i][0]) * r;
            *(f16x8*)&lds_k[kb][krow * KS + 16 * part + 8] = codes4_to_half((uint32_t)ck[i][1]) * r;
        } else put(&lds_k[kb][krow * KS + 16 * part], ck[i]);
    };
    auto stage_values = [&](int kb, int i, int sb) {            // sb: the steps' buffer of the same tile
        const int p = tid + i * THREADS;
        if (PIECES % THREADS && p >= PIECES) return;
        if constexpr (FOUR) {
            const int row = p / 8, g = row / 16, comp = 16 * g + row, at = 8 * (p % 8);
            const f16x8 r = *(const f16x8*)&lds_vf[sb][g][at];
            uint32_t low, high;
            split_values4((uint32_t)cv[i][0], (uint32_t)cv[i][1], low, high);
            *(f16x8*)&lds_v[kb][comp * VS + at] = codes4_to_half(low) * r;
            *(f16x8*)&lds_v[kb][(comp + 16) * VS + at] = codes4_to_half(high) * r;
        } else put(&lds_v[kb][p / 4 * VS + 16 * (p % 4)], cv[i]);
    };
    // where the weight of key j of eight stands
    auto place_of = [](int j) { return FOUR ? token_place(j) : j; };
    auto stage_steps = [&](int vb, const KeyTile& kt, bool wild_now) {          // (by the wavefront that requested them: tiles go round)
        if (wave != vb) return;
        const KeySteps ks = key_steps(rks, rvs, c, kt.bias, rhave);
        lds_step[vb][0][lane] = ks.product;
        lds_step[vb][1][lane] = ks.add;
        const int w = wild_now || __ballot(ks.wild) != 0;
        lds_step[vb][2][lane] = w ? ks.log_inverse : ks.inverse;
        if constexpr (FOUR) {
#pragma unroll
            for (int g = 0; g < C; ++g) lds_vf[vb][g][(lane & ~7) + token_place(lane & 7)] = factor_half(rvf, g);
        }
        if (lane == 0) lds_wild[vb] = w;
    };

    const int last_row = min(rows, tile.row0 + ROWS) - 1;
    const int behind = tile.count - 1 - last_row / a.group;
    const int first_behind = tile.count - 1 - tile.row0 / a.group;

    // first product of a tile
    auto scores = [&](int kb, f32x16 (&s)[2]) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int j = 0; j < 16; ++j) s[b][j] = 0.0f;
#pragma unroll
        for (int i = 0; i < 2 * C; ++i)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const f16x8 k = *(const f16x8*)&lds_k[kb][(32 * b + n) * KS + 16 * i + 8 * half];
                s[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, qf[i], s[b], 0, 0, 0);
            }
    };
    // what a row does not see becomes -inf
    auto hide = [&](const KeyTile& kt, f32x16 (&s)[2]) -> bool {
        if (a.ids || kt.k + kTileKeys <= kt.length - first_behind) return false;
        const int see = kt.length - see_after - kt.k - 32 * half;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int j = 0; j < 16; ++j) s[b][j] = 16 * b + j < see ? s[b][j] : -INFINITY;
        return true;
    };
    // y of a tile from its products; what a row does not see is -inf
    auto logits = [&](int vb, const KeyTile& kt, f32x16 (&s)[2], bool mixed_now) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int at = 32 * half + 16 * b + 4 * g;
                const f32x4 sk = *(const f32x4*)&lds_step[vb][0][at], lv = *(const f32x4*)&lds_step[vb][1][at];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float x = mixed_now ? s[b][4 * g + j] * row_up : s[b][4 * g + j];
                    s[b][4 * g + j] = fmaf(x, sk[j], lv[j]);
                }
            }
        hide(kt, s);
    };
    auto top_of = [&](const f32x16 (&s)[2]) {
        float top = s[0][0];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int j = 0; j < 16; ++j) top = fmaxf(top, s[b][j]);
        return top;
    };
    // raises the reference where a row's largest score passes it by more than kSlack (M is kLift below it)
    auto raise = [&](float top, bool wild_now) {
        if (__ballot(passes(top, M))) {
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float m_new = raised(top, M), d = M - (m_new == -INFINITY ? 0.0f : m_new);
            const float shrink = __builtin_amdgcn_exp2f(d);
            if (!wild_now) L = times_exp2(L, d);
            M = m_new;
#pragma unroll
            for (int i = 0; i < C; ++i)
#pragma unroll
                for (int j = 0; j < 16; ++j) acc[i][j] *= shrink;
        }
    };
    // the weights of a tile and their sum (wild: WildSum's)
    auto weights = [&](int vb, const f32x16 (&y)[2], f16x8 (&w)[2][2], bool wild_now) {
        const float m_use = M == -INFINITY ? 0.0f : M;
        float l = 0.0f;                  // the tile's part of the sum: terms far below the sum so far would each be rounded away
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 iv = *(const f32x4*)&lds_step[vb][2][32 * half + 16 * b + 4 * g];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float e = __builtin_amdgcn_exp2f(y[b][4 * g + j] - m_use);
                    if (!wild_now) l = fmaf(e, iv[j], l);
                    w[b][g >> 1][place_of(4 * (g & 1) + j)] = (_Float16)e;
                }
            }
        L += l;
    };
    // second product
    auto gather = [&](int kb, const f16x8 (&w)[2][2]) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    const f16x8 v = *(const f16x8*)&lds_v[kb][(32 * i + n) * VS + 32 * half + 16 * b + 8 * j];
                    acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, w[b][j], acc[i], 0, 0, 0);
                }
    };

    // Pipeline, for tile t in turn: the first product of t + 1 runs beside the exponentials of t; the second product of t beside the conversion of the keys
    // of t + 2 and the values of t + 1 into LDS and the scores of t + 1; then the codes of the tiles after those are requested.
    static_assert(NW >= 3, "three wavefronts form the steps in turn");
    KeyTiles it;
    KeyTile d0, d1, d2;
    it.start(a, tile.s, split);
    it.next(a, tile.s, behind);
    d0 = it.t;
    find_pages(d0);
    fetch_keys(d0, 0);
    fetch_values();
#pragma unroll
    for (int i = 0; i < PER; ++i) stage_keys(0, i);
    stage_steps(0, d0, false);
    if constexpr (FOUR) __syncthreads();                        // (the values' factors)
#pragma unroll
    for (int i = 0; i < PER; ++i) stage_values(0, i, 0);
    it.next(a, tile.s, behind);
    d1 = it.t;
    find_pages(d1);
    fetch_keys(d1, 1);
    fetch_values();
#pragma unroll
    for (int i = 0; i < PER; ++i) stage_keys(1, i);
    stage_steps(1, d1, false);
    it.next(a, tile.s, behind);
    d2 = it.t;
    find_pages(d2);
    fetch_keys(d2, 2);
    it.next(a, tile.s, behind);
    find_pages(it.t);
    __syncthreads();
    int kb = 0, vb = 0;                  // buffers of tile t: keys and values, steps
    // requests the keys of t + 3 and the values of t + 2 and moves on
    auto advance = [&]() {
        fetch_values();
        fetch_keys(it.t, vb);
        d0 = d1;
        d1 = d2;
        d2 = it.t;
        it.next(a, tile.s, behind);
        find_pages(it.t);
        kb ^= 1;
        vb = vb == 2 ? 0 : vb + 1;
    };
    if (!mixed && d0.have) {
        f32x16 y[2];
        scores(0, y);
        logits(0, d0, y, false);
        float top = top_of(y);
        raise(top, false);
        int wild_now = lds_wild[0];
        __syncthreads();
        while (d0.have && !__builtin_amdgcn_readfirstlane(wild_now)) {
            const int v1 = vb == 2 ? 0 : vb + 1, v2 = v1 == 2 ? 0 : v1 + 1;
            f32x16 s[2];
            f16x8 w[2][2];
            {
                const float m_use = M == -INFINITY ? 0.0f : M;
                float l = 0.0f;          // (as in weights; the first term needs no addition)
                __builtin_amdgcn_sched_barrier(0);
                // operands are read from LDS two steps ahead of the products that use them
                constexpr int STEPS = 4 * C;
                f16x8 k[3];
                f32x4 iv[2];
                auto read_k = [&](auto xc) {
                    constexpr int x = decltype(xc)::value, b = x / (2 * C), i = x % (2 * C);
                    if constexpr (x < STEPS) k[x % 3] = *(const f16x8*)&lds_k[kb ^ 1][(32 * b + n) * KS + 16 * i + 8 * half];
                };
                auto read_iv = [&](auto xc) {
                    constexpr int x = decltype(xc)::value;
                    if constexpr (x < 8) iv[x % 2] = *(const f32x4*)&lds_step[vb][2][32 * half + 16 * (x >> 2) + 4 * (x & 3)];
                };
                read_k(std::integral_constant<int, 0>{});
                read_iv(std::integral_constant<int, 0>{});
                read_k(std::integral_constant<int, 1>{});
                unrolled<0, STEPS>([&](auto xc) {
                    constexpr int x = decltype(xc)::value, b = x / (2 * C), i = x % (2 * C);
                    read_k(std::integral_constant<int, x + 2>{});
                    if constexpr (i == 0) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) s[b][j] = 0.0f;
                    }
                    s[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k[x % 3], qf[i], s[b], 0, 0, 0);
                    unrolled<8 * i / (2 * C), 8 * (i + 1) / (2 * C)>([&](auto pc) {      // pairs of scores
                        constexpr int pr = decltype(pc)::value, g = 4 * b + pr / 2;
                        if constexpr (pr % 2 == 0) read_iv(std::integral_constant<int, g + 1>{});
#pragma unroll
                        for (int j = 2 * pr; j < 2 * pr + 2; ++j) {
                            const float e = __builtin_amdgcn_exp2f(y[b][j] - m_use);
                            l = b == 0 && j == 0 ? e * iv[g % 2][j % 4] : fmaf(e, iv[g % 2][j % 4], l);
                            w[b][j / 8][place_of(j % 8)] = (_Float16)e;
                        }
                    });
                    asm volatile("" : "+v"(l));       // (the sum is formed here, not where it is next used)
                    __builtin_amdgcn_sched_barrier(0);
                });
                L += l;
            }
            wild_now = lds_wild[v1];
            {
                // (pieces and steps of a tile that is not there are converted all the same, into a buffer that nothing reads)
                constexpr int STEPS = 4 * C, AHEAD = 2, FIRST = STEPS / 2;
                top = -INFINITY;
                f16x8 v[AHEAD + 1];
                f32x4 sk[2], lv[2];
                auto read_v = [&](auto xc) {
                    constexpr int x = decltype(xc)::value;
                    if constexpr (x < STEPS) v[x % (AHEAD + 1)] = *(const f16x8*)&lds_v[kb][(32 * (x % C) + n) * VS + 32 * half + 8 * (x / C)];
                };
                auto read_step = [&](auto bg) {
                    constexpr int x = decltype(bg)::value;
                    if constexpr (x < 8) {
                        sk[x % 2] = *(const f32x4*)&lds_step[v1][0][32 * half + 16 * (x >> 2) + 4 * (x & 3)];
                        lv[x % 2] = *(const f32x4*)&lds_step[v1][1][32 * half + 16 * (x >> 2) + 4 * (x & 3)];
                    }
                };
                unrolled<0, AHEAD>(read_v);
                unrolled<0, STEPS>([&](auto xc) {
                    constexpr int x = decltype(xc)::value, bj = x / C, i = x % C;
                    read_v(std::integral_constant<int, x + AHEAD>{});
                    if constexpr (x == FIRST - 1) read_step(std::integral_constant<int, 0>{});
                    acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v[x % (AHEAD + 1)], w[bj >> 1][bj & 1], acc[i], 0, 0, 0);
                    // beside the products: first the conversions, then the scores of the next tile
                    if constexpr (x < FIRST) {
                        unrolled<2 * PER * x / FIRST, 2 * PER * (x + 1) / FIRST>([&](auto uc) {
                            constexpr int u = decltype(uc)::value;
                            if constexpr (u & 1) stage_values(kb ^ 1, u >> 1, v1); else stage_keys(kb, u >> 1);
                        });
                    } else {
                        unrolled<8 * (x - FIRST) / (STEPS - FIRST), 8 * (x - FIRST + 1) / (STEPS - FIRST)>([&](auto bg) {
                            constexpr int z = decltype(bg)::value, b = z >> 2, g = z & 3;
                            read_step(std::integral_constant<int, z + 1>{});
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                s[b][4 * g + j] = fmaf(s[b][4 * g + j], sk[z % 2][j], lv[z % 2][j]);
                                top = fmaxf(top, s[b][4 * g + j]);
                            }
                            asm volatile("" : "+v"(top));
                        });
                    }
                    __builtin_amdgcn_sched_barrier(0);
                });
            }
            stage_steps(v2, d2, false);
            if (hide(d1, s)) {
                top = top_of(s);
            }
            advance();
            if (d0.have) raise(top, false);
#pragma unroll
            for (int b = 0; b < 2; ++b) y[b] = s[b];
            __syncthreads();
        }
    }
    // Queries of very different sizes in one block, or steps of the values that are not tame (key_steps): the same step by step, for the tiles that are left.
    bool wild = false;
    WildSum terms;
    while (d0.have) {
        const int v1 = vb == 2 ? 0 : vb + 1, v2 = v1 == 2 ? 0 : v1 + 1;
        const bool logs = __builtin_amdgcn_readfirstlane(lds_wild[vb]);
        if (logs && !wild) terms.begin(L, M);
        wild = wild || logs;
        f32x16 s[2];
        f16x8 w[2][2];
        scores(kb, s);
        logits(vb, d0, s, true);
        float top = top_of(s);
        raise(top, wild);
        weights(vb, s, w, wild);
        if (wild) {
            if (!logs) {                                        // (staged before the first wild tile was met)
                __syncthreads();
                if (tid < kTileKeys) lds_step[vb][2][tid] = __log2f(lds_step[vb][2][tid]);
                __syncthreads();
            }
            terms.add(L, [&](auto&& f) {
#pragma unroll
                for (int g = 0; g < 8; ++g) {
                    const f32x16& y = s[g >> 2];
                    f(f32x4{y[4 * (g & 3)], y[4 * (g & 3) + 1], y[4 * (g & 3) + 2], y[4 * (g & 3) + 3]}, *(const f32x4*)&lds_step[vb][2][32 * half + 16 * (g >> 2) + 4 * (g & 3)]);
                }
            });
        }
        gather(kb, w);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PER; ++i) { stage_keys(kb, i); stage_values(kb ^ 1, i, v1); }
        stage_steps(v2, d2, wild);
        advance();
        __syncthreads();
    }

    const int heads = a.st.heads * a.group;
    if (wild) L = terms.end(L, M);
    const float l = L + __shfl_xor(L, 32, 64);
    const int row = tile.row0 + wave * 32 + n;
    if (row >= rows) return;
    const int64_t at_tok = tile.first + tok;
    const int qh = head * a.group + row - tok * a.group;
    if (a.splits == 1) {
        const float inv = l == 0.0f ? 0.0f : kUnlift / l;
#pragma unroll
        for (int i = 0; i < C; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 o = {acc[i][4 * g] * inv, acc[i][4 * g + 1] * inv, acc[i][4 * g + 2] * inv, acc[i][4 * g + 3] * inv};
                store4<T>(a.out, at_tok * a.out_token + (int64_t)qh * a.out_head + 32 * i + 8 * g + 4 * half, a.out_wide, o);
            }
    } else {
        const int64_t at = ((int64_t)split * a.tokens + at_tok) * heads + qh;
        if (l != 0.0f) {
#pragma unroll
            for (int i = 0; i < C; ++i)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *(f32x4*)&a.part_acc[at * D + 32 * i + 8 * g + 4 * half] = f32x4{acc[i][4 * g], acc[i][4 * g + 1], acc[i][4 * g + 2], acc[i][4 * g + 3]};
        }
        if (half == 0) { a.part_m[at] = M; a.part_l[at] = l; }
    }
}

}  // namespace lorann
