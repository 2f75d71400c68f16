// Host side that the state stores' entry points share: argument checks, the plan of an attention and its launches.  No call allocates, waits or keeps anything.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/lorann_states.h"
#include "../../include/lorann_states4.h"
#include "attend.hpp"
#include "attend_tile.hpp"
#include "error.hpp"

namespace lorann {
namespace {

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool aligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
int log2_of(int v) { int s = 0; while ((1 << s) < v) ++s; return s; }

// St: lorann_states or lorann_states4.
template <typename St>
int check_sizes(const St* st) {
    if (!st) return fail(LORANN_E_INVAL, "the store is NULL");
    if (st->pages < 1 || st->heads < 1) return fail(LORANN_E_INVAL, "a store needs at least one page and one head (pages %lld, heads %d)", (long long)st->pages, st->heads);
    if (st->page_size < 1 || (st->page_size & (st->page_size - 1))) return fail(LORANN_E_INVAL, "page_size %d is not a power of two", st->page_size);
    if (st->dim < 1) return fail(LORANN_E_INVAL, "dim %d is not positive", st->dim);
    if (st->page_size < LORANN_MIN_PAGE || st->page_size > LORANN_MAX_PAGE)
        return fail(LORANN_E_UNSUPPORTED, "page_size %d is outside %d .. %d", st->page_size, LORANN_MIN_PAGE, LORANN_MAX_PAGE);
    if (st->dim % 32 || st->dim > LORANN_MAX_DIM) return fail(LORANN_E_UNSUPPORTED, "dim %d is not a multiple of 32 up to %d", st->dim, LORANN_MAX_DIM);
    if (st->heads > LORANN_MAX_HEADS) return fail(LORANN_E_UNSUPPORTED, "%d heads are more than %d", st->heads, LORANN_MAX_HEADS);
    if (st->pages > 0x7fffffff / st->heads) return fail(LORANN_E_UNSUPPORTED, "%lld pages of %d heads are more than 32 bits count", (long long)st->pages, st->heads);
    return LORANN_OK;
}

// `current`: the current device, -1 until the first pointer asks for it (a call checks up to twelve).
int check_device(const void* p, const char* name, int& current) {
    if (!p) return fail(LORANN_E_INVAL, "%s is NULL", name);
    int gpu = -1;
    if (!is_device_ptr(p, &gpu)) return fail(LORANN_E_INVAL, "%s is not a device pointer", name);
    if (current < 0) HIP_TRY(hipGetDevice(&current));
    if (gpu >= 0 && gpu != current) return fail(LORANN_E_INVAL, "%s is memory of GPU %d, the current device is %d", name, gpu, current);
    return LORANN_OK;
}

template <typename St>
int check_store(const St* st, int& gpu) {
    constexpr bool four = std::is_same_v<St, lorann_states4>;
    int rc;
    if ((rc = check_sizes(st))) return rc;
    if (!st->k_codes || !st->v_codes || !st->k_scales || !st->v_scales) return fail(LORANN_E_INVAL, "an array of the store is NULL");
    if constexpr (four) {
        if (!st->k_factors || !st->v_factors) return fail(LORANN_E_INVAL, "an array of the store is NULL");
        if (!aligned(st->k_factors, 4) || !aligned(st->v_factors, 4)) return fail(LORANN_E_INVAL, "the store's factors are not 4-byte aligned");
    }
    if (!aligned(st->k_codes, 16) || !aligned(st->v_codes, 16)) return fail(LORANN_E_INVAL, "the store's codes are not 16-byte aligned");
    if (!aligned(st->k_scales, 4) || !aligned(st->v_scales, 4)) return fail(LORANN_E_INVAL, "the store's steps are not 4-byte aligned");
    if ((rc = check_device(st->k_codes, "k_codes", gpu)) || (rc = check_device(st->v_codes, "v_codes", gpu))) return rc;
    if ((rc = check_device(st->k_scales, "k_scales", gpu)) || (rc = check_device(st->v_scales, "v_scales", gpu))) return rc;
    if constexpr (four) {
        if ((rc = check_device(st->k_factors, "k_factors", gpu)) || (rc = check_device(st->v_factors, "v_factors", gpu))) return rc;
    }
    return LORANN_OK;
}

template <typename St>
Store view(const St* st) {
    Store s{};
    s.kc = (int8_t*)st->k_codes; s.vc = (int8_t*)st->v_codes; s.ks = st->k_scales; s.vs = st->v_scales;
    if constexpr (std::is_same_v<St, lorann_states4>) { s.kf = (uint32_t*)st->k_factors; s.vf = (uint32_t*)st->v_factors; }
    s.pages = st->pages; s.heads = st->heads; s.shift = log2_of(st->page_size);
    return s;
}

int element_size(int32_t type) { return type == LORANN_F32 ? 4 : type == LORANN_F16 || type == LORANN_BF16 ? 2 : 0; }

TokenRows rows_of(void* p, int64_t token, int64_t head, int32_t type) {
    const int per = 16 / element_size(type);
    return TokenRows{p, token, head, aligned(p, 16) && token % per == 0 && head % per == 0};
}

template <typename St>
int check_tokens(const St* st, int32_t type, int64_t tokens) {
    if (!element_size(type)) return fail(LORANN_E_INVAL, "unknown element type %d", type);
    if (tokens < 0) return fail(LORANN_E_INVAL, "%lld tokens", (long long)tokens);
    if (tokens > 0x7fffffffLL / st->heads || tokens >= 1 << 30) return fail(LORANN_E_UNSUPPORTED, "%lld tokens of %d heads in one call", (long long)tokens, st->heads);
    return LORANN_OK;
}

// ---- attention ----

struct Plan {
    int32_t waves;                   // wavefronts of a block of k_attend_tile (32 rows each); 0: k_attend_rows
    int32_t row_tiles;               // tiles of 16 rows of a block of k_attend_rows
    int64_t tiles;                   // row tiles over all sequences, at most
    int32_t unit, units, splits, per_split;
    int64_t workspace;
};

// Splitting.  Two blocks of either kernel fit a CU: 512 fill the GPU, more only add to what is joined (a token of 64 heads after 131071 keys: 50 us with 256 or 512, 54
// with 1024, 62 with 1536).  The host does not know the lengths, only the tables' width: where that is long, a block still gets at most so many keys, so that one long sequence
// among short ones does not run on a few CUs alone.  One token each of 64 sequences, one of 131072 keys, the others of 1000: 169 / 178 / 289 us with at most 8192 / 16384 / 32768
// keys a block, 1012 uncut; 300 tokens each of 4 sequences, one of 131072 keys: 1116 / 1114 / 1633 with 16384 / 32768 / 65536, 3205 uncut.
constexpr int64_t kBlocksWanted = 512;
constexpr int64_t kMostKeys = 16384, kMostTileKeys = 32768, kMostPartRows = 1 << 17;      // (and no more than that many rows of partial answers)
// Rows per sequence and head (tokens x group) up to which k_attend_rows is taken, which reads the states once for every 16 rows.  32 sequences of 4096 keys, 8 heads
// of 128, us of k_attend_rows / k_attend_tile: 16 rows 50 / 97, 32 rows 58 / 94, 48 rows 83 / 99, 64 rows 105 / 100, 128 rows 198 / 118.
// The rows are the call's mean, one kernel takes all its sequences, and the figures are of sequences alike.  Pieces of prompts beside single tokens may do better in calls of
// their own: 200 single tokens and a piece of 512, each over 2000 keys, 227 us together, 157 + 60 apart; 63 and 1024: 174, 44 + 83; 255 and 2048: 497, 189 + 153.
constexpr int64_t kMostFewRows = 48;
// 4 bits: a block of k_attend_rows may have two tiles of 16 rows, for which the codes are converted once, and is taken up to more rows.  us of k_attend_tile / one tile / two, over 32 sequences of
// 4096 keys and over ten passages of 512 for each of 24:
//   values, heads, page    32 rows                       48 rows                        64 rows                          96 rows
//   64, 16, 16             140 72 60   156 71 71         144 99 110   160 110 114       143 126 109   159 130 114        150 185 160   160 187 170
//   96, 8, 32              158 51 49   123 66 62         164 75 68    183 100 85        165 97 69     184 103 84         169 137 105   184 160 130
//   128, 8, 64             133 59 59   115 72 71         136 86 79    154 108 95        134 110 81    152 111 96         140 156 119   154 169 146
//   128, 8, 16             159 59 73   123 72 84         159 89 90    168 111 106       161 109 92    170 114 107        167 158 146   170 172 172
// (Four tiles of 64 values: 125 at 64 rows, the registers spill.)
constexpr int64_t kMostFewRows4 = 64, kMostWideRows4 = 96;      // up to 64 values, and above
template <typename St>
int32_t row_tiles4(const St* st, int64_t mean_rows) {
    const int64_t tiles = ceil_div(mean_rows, kRows);
    if (tiles <= 1) return 1;
    if (st->dim <= 64) return tiles % 2 ? 1 : 2;
    return tiles == 2 && st->dim == 128 && st->page_size < 64 ? 1 : 2;
}
// Blocks of k_attend_tile have 4 wavefronts, or 8 where they still fill the GPU and little of them is empty: then the codes are converted for 256 rows at once.
// us of 4 / 8 wavefronts: 4096 tokens of 32 heads over 32768 keys 2336 / 2161, 16 x 256 tokens over 4352 keys 344 / 324; 8 heads of 96, 4096 tokens over 12288
// keys 724 / 679; with 256 blocks only, 2048 tokens over 16384 keys, 610 / 595; at a dimension of 64, 4096 tokens over 16384 keys 769 / 729, but 16 x 512 over 2048
// 234 / 236 and 12 x 512 over 3500 with pages of 16 171 / 194.
constexpr int64_t kManyBlocks = 512, kManyRows = 1024;
constexpr int kDimForFour = 64;
constexpr int64_t kKeysPerBlock = 64 * kAttendWaves;

template <typename St>
int check_questions(const St* st, const lorann_questions* qs, int32_t found, int32_t width) {
    if (!qs) return fail(LORANN_E_INVAL, "the questions are NULL");
    if (qs->type != LORANN_F16 && qs->type != LORANN_BF16) return fail(qs->type == LORANN_F32 ? LORANN_E_UNSUPPORTED : LORANN_E_INVAL, "queries are LORANN_F16 or LORANN_BF16 (type %d)", qs->type);
    if (qs->tokens < 0 || qs->sequences < 0) return fail(LORANN_E_INVAL, "%lld tokens of %lld sequences", (long long)qs->tokens, (long long)qs->sequences);
    if (qs->heads < 1 || qs->heads % st->heads) return fail(LORANN_E_INVAL, "%d query heads are not a multiple of the store's %d", qs->heads, st->heads);
    if (qs->heads > LORANN_MAX_HEADS) return fail(LORANN_E_UNSUPPORTED, "%d query heads are more than %d", qs->heads, LORANN_MAX_HEADS);
    if (!(std::fabs(qs->scale) <= 1.0e38f)) return fail(LORANN_E_INVAL, "the scale is not finite");
    if (width < 0 || found < 0) return fail(LORANN_E_INVAL, "table width %d, %d passages per sequence", width, found);
    if (found > LORANN_MAX_FOUND) return fail(LORANN_E_UNSUPPORTED, "%d passages per sequence are more than %d", found, LORANN_MAX_FOUND);
    if ((int64_t)width * st->page_size > (1 << 30)) return fail(LORANN_E_UNSUPPORTED, "tables of %d pages of %d tokens are longer than 2^30 tokens", width, st->page_size);
    if (qs->sequences > 0x3fffffff || qs->tokens > 0x3fffffffLL / qs->heads) return fail(LORANN_E_UNSUPPORTED, "%lld tokens of %d heads, %lld sequences in one call", (long long)qs->tokens, qs->heads, (long long)qs->sequences);
    return LORANN_OK;
}

template <typename St>
Plan plan_of(const St* st, const lorann_questions* qs, int32_t found, int32_t width) {
    Plan p{};
    const int64_t group = qs->heads / st->heads;
    const int64_t sequences = std::max<int64_t>(qs->sequences, 1), mean_rows = qs->tokens * group / sequences;
    auto tiles_of = [&](int64_t rows) { return qs->q_start ? qs->tokens * group / rows + sequences : sequences * ceil_div(mean_rows, rows); };
    constexpr bool four = std::is_same_v<St, lorann_states4>;
    p.row_tiles = four ? row_tiles4(st, mean_rows) : 1;
    p.waves = mean_rows <= (!four ? kMostFewRows : st->dim > kDimForFour ? kMostWideRows4 : kMostFewRows4) ? 0 : tiles_of(256) * st->heads >= kManyBlocks && mean_rows >= kManyRows && st->dim > kDimForFour ? 8 : 4;
    p.tiles = tiles_of(p.waves ? 32 * p.waves : kRows * p.row_tiles);
    const int64_t table_keys = std::max<int64_t>((int64_t)width * st->page_size, 1), tables = std::max(found, 1), keys = tables * table_keys;
    const int64_t blocks = std::max<int64_t>(p.tiles * st->heads, 1), rows = std::max<int64_t>(qs->tokens * qs->heads, 1);
    const int64_t want = std::max(std::max<int64_t>(1, std::min(kBlocksWanted / blocks, ceil_div(keys, kKeysPerBlock))), std::min(ceil_div(keys, p.waves ? kMostTileKeys : kMostKeys), kMostPartRows / rows));
    if (want <= tables) {              // whole tables per split
        p.unit = (int32_t)(ceil_div(table_keys, kTileKeys) * kTileKeys);
        p.units = 1;
        p.per_split = (int32_t)ceil_div(tables, want);
        p.splits = (int32_t)ceil_div(tables, p.per_split);
    } else {                           // tables cut
        p.unit = (int32_t)(ceil_div(ceil_div(table_keys, ceil_div(want, tables)), kKeysPerBlock) * kKeysPerBlock);
        p.units = (int32_t)ceil_div(table_keys, p.unit);
        p.per_split = 1;               // (k_attend_rows counts on one unit per split where a sequence has one table)
        p.splits = (int32_t)(tables * p.units);
    }
    p.workspace = p.splits > 1 ? (int64_t)p.splits * rows * (st->dim + 2) * 4 : 0;
    return p;
}

// `grid`, `block`: of the first kernel.
template <typename T, int D, int BITS>
void launch_attend(const Plan& p, const AttendArgs& a, dim3 grid, dim3 block, hipStream_t stream) {
    const bool whole = a.st.shift >= 6;          // pages of 64 tokens and more: a tile of keys lies in one
    if (p.waves == 8) {
        if constexpr (D > kDimForFour) {
            if (whole) hipLaunchKernelGGL((k_attend_tile<T, D, 8, true, BITS>), grid, block, 0, stream, a);
            else hipLaunchKernelGGL((k_attend_tile<T, D, 8, false, BITS>), grid, block, 0, stream, a);
        }
    } else if (p.waves) {
        if (whole) hipLaunchKernelGGL((k_attend_tile<T, D, 4, true, BITS>), grid, block, 0, stream, a);
        else hipLaunchKernelGGL((k_attend_tile<T, D, 4, false, BITS>), grid, block, 0, stream, a);
    } else if (p.row_tiles == 1) {
        if (whole) hipLaunchKernelGGL((k_attend_rows<T, D, true, BITS, 1>), grid, block, 0, stream, a);
        else hipLaunchKernelGGL((k_attend_rows<T, D, false, BITS, 1>), grid, block, 0, stream, a);
    } else if constexpr (BITS == 4) {
        if (whole) hipLaunchKernelGGL((k_attend_rows<T, D, true, BITS, 2>), grid, block, 0, stream, a);
        else hipLaunchKernelGGL((k_attend_rows<T, D, false, BITS, 2>), grid, block, 0, stream, a);
    }
    if (p.splits > 1) {
        constexpr int groups = 256 / (D / 4);
        int sides = 1;
        while (sides < p.splits && 2 * sides <= groups) sides *= 2;
        const int64_t rows = a.tokens * a.st.heads * a.group;
        hipLaunchKernelGGL((k_attend_join<T, D, BITS>), dim3((unsigned)ceil_div(rows, groups / sides)), dim3(256), 0, stream, a, sides);
    }
}

template <typename St>
int attend(const St* st, const lorann_questions* qs, const int64_t* ids, int32_t found, const float* scores, float score_weight,
           const int32_t* tables, int32_t width, const int32_t* lengths, int64_t passages, void* workspace, int64_t workspace_bytes, hipStream_t stream, int& gpu) {
    constexpr int bits = std::is_same_v<St, lorann_states4> ? 4 : 8;
    int rc;
    if (qs->tokens == 0 || qs->sequences == 0) return LORANN_OK;
    if ((rc = check_store(st, gpu))) return rc;
    if (!qs->q_start && qs->tokens % qs->sequences) return fail(LORANN_E_INVAL, "%lld tokens do not divide over %lld sequences", (long long)qs->tokens, (long long)qs->sequences);
    if ((rc = check_device(qs->q, "q", gpu)) || (rc = check_device(qs->out, "out", gpu))) return rc;
    if (!aligned(qs->q, 2) || !aligned(qs->out, 2)) return fail(LORANN_E_INVAL, "q or out is not aligned to its type");
    if (qs->q_start && (rc = check_device(qs->q_start, "q_start", gpu))) return rc;
    if (width > 0 && (!ids || passages > 0) && (!ids || found > 0) && ((rc = check_device(tables, "tables", gpu)) || (rc = check_device(lengths, "lengths", gpu)))) return rc;
    const Plan p = plan_of(st, qs, found, width);
    const int64_t blocks = p.tiles * st->heads * p.splits;
    if (p.tiles > 0x7fffffff || blocks > 0xffffffffLL / (64 * std::max(p.waves, kAttendWaves)))       // (threads of a grid)
        return fail(LORANN_E_UNSUPPORTED, "%lld tokens of %lld sequences are more than one launch holds", (long long)qs->tokens, (long long)qs->sequences);
    if (p.workspace) {
        if (!workspace || workspace_bytes < p.workspace) return fail(LORANN_E_INVAL, "the workspace holds %lld bytes, %lld are needed", (long long)(workspace ? workspace_bytes : 0), (long long)p.workspace);
        if (!aligned(workspace, 16)) return fail(LORANN_E_INVAL, "the workspace is not 16-byte aligned");
        if ((rc = check_device(workspace, "workspace", gpu))) return rc;
    }
    AttendArgs a{};
    a.st = view(st);
    a.q = qs->q; a.out = qs->out;
    a.q_token = qs->q_token; a.q_head = qs->q_head; a.out_token = qs->out_token; a.out_head = qs->out_head;
    a.tokens = qs->tokens; a.sequences = (int32_t)qs->sequences; a.group = qs->heads / st->heads;
    a.q_start = qs->q_start;
    a.c = qs->scale * 1.44269504088896341f;
    a.tables = tables; a.width = width; a.lengths = lengths;
    a.ids = ids; a.found = ids ? found : 1; a.passages = passages; a.scores = scores; a.weight = score_weight * 1.44269504088896341f;
    if (width == 0 || (ids && passages == 0)) a.found = 0;       // nothing to see: zeros
    a.unit = p.unit; a.units = p.units; a.splits = p.splits; a.per_split = p.per_split;
    const int64_t rows = qs->tokens * qs->heads;
    a.part_acc = (float*)workspace;
    a.part_m = a.part_acc + (int64_t)p.splits * rows * st->dim;
    a.part_l = a.part_m + (int64_t)p.splits * rows;
    a.q_wide = aligned(qs->q, 16) && qs->q_token % 8 == 0 && qs->q_head % 8 == 0;
    a.out_wide = aligned(qs->out, 8) && qs->out_token % 4 == 0 && qs->out_head % 4 == 0;
    const dim3 grid((unsigned)blocks), block(64 * (p.waves ? p.waves : kAttendWaves));
#define LAUNCH_DIM(D_) do { if (qs->type == LORANN_F16) launch_attend<_Float16, D_, bits>(p, a, grid, block, stream); else launch_attend<__bf16, D_, bits>(p, a, grid, block, stream); } while (0)
    switch (st->dim) {
        case 32: LAUNCH_DIM(32); break;
        case 64: LAUNCH_DIM(64); break;
        case 96: LAUNCH_DIM(96); break;
        default: LAUNCH_DIM(128); break;
    }
#undef LAUNCH_DIM
    HIP_TRY(hipGetLastError());
    return LORANN_OK;
}

template <typename St>
int attend_chunk(const St* st, const lorann_questions* qs, const int32_t* tables, int32_t width, const int32_t* lengths, void* workspace, int64_t workspace_bytes, void* hip_stream) {
    int rc, gpu = -1;
    if ((rc = check_sizes(st)) || (rc = check_questions(st, qs, 0, width))) return rc;
    return attend(st, qs, nullptr, 0, nullptr, 0.0f, tables, width, lengths, 0, workspace, workspace_bytes, (hipStream_t)hip_stream, gpu);
}

template <typename St>
int attend_passages(const St* st, const lorann_questions* qs, const int64_t* ids, int32_t found, const float* scores, float score_weight, const int32_t* tables, int32_t width,
                    const int32_t* lengths, int64_t passages, void* workspace, int64_t workspace_bytes, void* hip_stream) {
    int rc, gpu = -1;
    if ((rc = check_sizes(st)) || (rc = check_questions(st, qs, found, width))) return rc;
    if (passages < 0) return fail(LORANN_E_INVAL, "%lld passages", (long long)passages);
    if (passages > 0x7fffffff) return fail(LORANN_E_UNSUPPORTED, "%lld passages are more than 32 bits count", (long long)passages);
    if (!(std::fabs(score_weight) <= 1.0e38f)) return fail(LORANN_E_INVAL, "the weight of the scores is not finite");
    if (found < 1) return fail(LORANN_E_INVAL, "%d passages per sequence", found);
    if (qs->tokens > 0 && qs->sequences > 0) {
        if ((rc = check_device(ids, "ids", gpu)) || (scores && (rc = check_device(scores, "scores", gpu)))) return rc;
    }
    return attend(st, qs, ids, found, scores, score_weight, tables, width, lengths, passages, workspace, workspace_bytes, (hipStream_t)hip_stream, gpu);
}

template <typename St>
int64_t attend_workspace(const St* st, const lorann_questions* qs, int32_t found, int32_t width) {
    int rc;
    if ((rc = check_sizes(st)) || (rc = check_questions(st, qs, found, width))) return rc;
    if (qs->tokens == 0 || qs->sequences == 0) return 0;
    return plan_of(st, qs, found, width).workspace;
}

// Checks of a call that writes or reads tokens; the grid of its kernel.
template <typename St>
int check_rows(const St* st, const int64_t* slots, const void* k, const void* v, int32_t type, bool both, int& gpu) {
    int rc;
    if ((rc = check_store(st, gpu))) return rc;
    if (!both && (rc = check_device(slots, "slots", gpu))) return rc;
    if (((k || both) && (rc = check_device(k, "k", gpu))) || ((v || both) && (rc = check_device(v, "v", gpu)))) return rc;
    if (both && (rc = check_device(slots, "slots", gpu))) return rc;
    if (!aligned(k, element_size(type)) || !aligned(v, element_size(type))) return fail(LORANN_E_INVAL, "k or v is not aligned to its type");
    return LORANN_OK;
}
template <typename St>
dim3 rows_grid(const St* st, int64_t tokens) { return dim3((unsigned)ceil_div(tokens, kBlockTokens), (unsigned)st->heads, 2); }
// Heads first, keys and values of the same tokens side by side (k_states4_write).
template <typename St>
dim3 heads_grid(const St* st, int64_t tokens) {
    const int64_t blocks = ceil_div(tokens, kBlockTokens), y = std::min<int64_t>(blocks, 32768);
    return dim3((unsigned)(2 * st->heads), (unsigned)y, (unsigned)ceil_div(blocks, y));
}

}  // namespace
}  // namespace lorann
