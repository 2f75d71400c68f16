// C ABI (include/lorann_states.h) of the state store and its attention: argument checks, plans and launches.  No call allocates, waits or keeps anything.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/lorann_states.h"
#include "attend.hpp"
#include "attend_tile.hpp"
#include "error.hpp"
#include "states_store.hpp"

using namespace lorann;

namespace {

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool aligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
int log2_of(int v) { int s = 0; while ((1 << s) < v) ++s; return s; }

int check_sizes(const lorann_states* st) {
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

int check_store(const lorann_states* st, int& gpu) {
    int rc;
    if ((rc = check_sizes(st))) return rc;
    if (!st->k_codes || !st->v_codes || !st->k_scales || !st->v_scales) return fail(LORANN_E_INVAL, "an array of the store is NULL");
    if (!aligned(st->k_codes, 16) || !aligned(st->v_codes, 16)) return fail(LORANN_E_INVAL, "the store's codes are not 16-byte aligned");
    if (!aligned(st->k_scales, 4) || !aligned(st->v_scales, 4)) return fail(LORANN_E_INVAL, "the store's steps are not 4-byte aligned");
    if ((rc = check_device(st->k_codes, "k_codes", gpu)) || (rc = check_device(st->v_codes, "v_codes", gpu))) return rc;
    if ((rc = check_device(st->k_scales, "k_scales", gpu)) || (rc = check_device(st->v_scales, "v_scales", gpu))) return rc;
    return LORANN_OK;
}

Store view(const lorann_states* st) {
    Store s;
    s.kc = st->k_codes; s.vc = st->v_codes; s.ks = st->k_scales; s.vs = st->v_scales;
    s.pages = st->pages; s.heads = st->heads; s.shift = log2_of(st->page_size);
    return s;
}

int element_size(int32_t type) { return type == LORANN_F32 ? 4 : type == LORANN_F16 || type == LORANN_BF16 ? 2 : 0; }

TokenRows rows_of(void* p, int64_t token, int64_t head, int32_t type) {
    const int per = 16 / element_size(type);
    return TokenRows{p, token, head, aligned(p, 16) && token % per == 0 && head % per == 0};
}

int check_tokens(const lorann_states* st, int32_t type, int64_t tokens) {
    if (!element_size(type)) return fail(LORANN_E_INVAL, "unknown element type %d", type);
    if (tokens < 0) return fail(LORANN_E_INVAL, "%lld tokens", (long long)tokens);
    if (tokens > 0x7fffffffLL / st->heads || tokens >= 1 << 30) return fail(LORANN_E_UNSUPPORTED, "%lld tokens of %d heads in one call", (long long)tokens, st->heads);
    return LORANN_OK;
}

// ---- attention ----

struct Plan {
    int32_t waves;                   // wavefronts of a block of k_attend_tile (32 rows each); 0: k_attend_rows
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
// Blocks of k_attend_tile have 4 wavefronts, or 8 where they still fill the GPU and little of them is empty: then the codes are converted for 256 rows at once.
// us of 4 / 8 wavefronts: 4096 tokens of 32 heads over 32768 keys 2336 / 2161, 16 x 256 tokens over 4352 keys 344 / 324; 8 heads of 96, 4096 tokens over 12288
// keys 724 / 679; with 256 blocks only, 2048 tokens over 16384 keys, 610 / 595; at a dimension of 64, 4096 tokens over 16384 keys 769 / 729, but 16 x 512 over 2048
// 234 / 236 and 12 x 512 over 3500 with pages of 16 171 / 194.
constexpr int64_t kManyBlocks = 512, kManyRows = 1024;
constexpr int kDimForFour = 64;
constexpr int64_t kKeysPerBlock = 64 * kAttendWaves;

int check_questions(const lorann_states* st, const lorann_questions* qs, int32_t found, int32_t width) {
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

Plan plan_of(const lorann_states* st, const lorann_questions* qs, int32_t found, int32_t width) {
    Plan p{};
    const int64_t group = qs->heads / st->heads;
    const int64_t sequences = std::max<int64_t>(qs->sequences, 1), mean_rows = qs->tokens * group / sequences;
    auto tiles_of = [&](int64_t rows) { return qs->q_start ? qs->tokens * group / rows + sequences : sequences * ceil_div(mean_rows, rows); };
    p.waves = mean_rows <= kMostFewRows ? 0 : tiles_of(256) * st->heads >= kManyBlocks && mean_rows >= kManyRows && st->dim > kDimForFour ? 8 : 4;
    p.tiles = tiles_of(p.waves ? 32 * p.waves : kRows);
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
template <typename T, int D>
void launch_attend(const Plan& p, const AttendArgs& a, dim3 grid, dim3 block, hipStream_t stream) {
    const bool whole = a.st.shift >= 6;          // pages of 64 tokens and more: a tile of keys lies in one
    if (p.waves == 8) {
        if constexpr (D > kDimForFour) {
            if (whole) hipLaunchKernelGGL((k_attend_tile<T, D, 8, true>), grid, block, 0, stream, a);
            else hipLaunchKernelGGL((k_attend_tile<T, D, 8, false>), grid, block, 0, stream, a);
        }
    } else if (p.waves) {
        if (whole) hipLaunchKernelGGL((k_attend_tile<T, D, 4, true>), grid, block, 0, stream, a);
        else hipLaunchKernelGGL((k_attend_tile<T, D, 4, false>), grid, block, 0, stream, a);
    } else {
        if (whole) hipLaunchKernelGGL((k_attend_rows<T, D, true>), grid, block, 0, stream, a);
        else hipLaunchKernelGGL((k_attend_rows<T, D, false>), grid, block, 0, stream, a);
    }
    if (p.splits > 1) {
        constexpr int groups = 256 / (D / 4);
        int sides = 1;
        while (sides < p.splits && 2 * sides <= groups) sides *= 2;
        const int64_t rows = a.tokens * a.st.heads * a.group;
        hipLaunchKernelGGL((k_attend_join<T, D>), dim3((unsigned)ceil_div(rows, groups / sides)), dim3(256), 0, stream, a, sides);
    }
}

int attend(const lorann_states* st, const lorann_questions* qs, const int64_t* ids, int32_t found, const float* scores, float score_weight,
           const int32_t* tables, int32_t width, const int32_t* lengths, int64_t passages, void* workspace, int64_t workspace_bytes, hipStream_t stream, int& gpu) {
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
#define LAUNCH_DIM(D_) do { if (qs->type == LORANN_F16) launch_attend<_Float16, D_>(p, a, grid, block, stream); else launch_attend<__bf16, D_>(p, a, grid, block, stream); } while (0)
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

}  // namespace

extern "C" {

int lorann_states_write(const lorann_states* st, const void* k, const void* v, int32_t type, int64_t tokens,
                        int64_t k_token, int64_t k_head, int64_t v_token, int64_t v_head, const int64_t* slots, void* hip_stream) {
    int rc, gpu = -1;
    if ((rc = check_sizes(st)) || (rc = check_tokens(st, type, tokens))) return rc;
    if (tokens == 0) return LORANN_OK;
    if ((rc = check_store(st, gpu))) return rc;
    if ((rc = check_device(k, "k", gpu)) || (rc = check_device(v, "v", gpu)) || (rc = check_device(slots, "slots", gpu))) return rc;
    if (!aligned(k, element_size(type)) || !aligned(v, element_size(type))) return fail(LORANN_E_INVAL, "k or v is not aligned to its type");
    const dim3 grid((unsigned)ceil_div(tokens, kBlockTokens), (unsigned)st->heads, 2);
    const TokenRows kr = rows_of(const_cast<void*>(k), k_token, k_head, type), vr = rows_of(const_cast<void*>(v), v_token, v_head, type);
    hipStream_t s = (hipStream_t)hip_stream;
    if (type == LORANN_F32) hipLaunchKernelGGL((k_states_write<float>), grid, dim3(256), 0, s, view(st), kr, vr, slots, tokens, st->dim);
    else if (type == LORANN_F16) hipLaunchKernelGGL((k_states_write<_Float16>), grid, dim3(256), 0, s, view(st), kr, vr, slots, tokens, st->dim);
    else hipLaunchKernelGGL((k_states_write<__bf16>), grid, dim3(256), 0, s, view(st), kr, vr, slots, tokens, st->dim);
    HIP_TRY(hipGetLastError());
    return LORANN_OK;
}

int lorann_states_read(const lorann_states* st, const int64_t* slots, int64_t tokens, void* k, void* v, int32_t type,
                       int64_t k_token, int64_t k_head, int64_t v_token, int64_t v_head, void* hip_stream) {
    int rc, gpu = -1;
    if ((rc = check_sizes(st)) || (rc = check_tokens(st, type, tokens))) return rc;
    if (tokens == 0 || (!k && !v)) return LORANN_OK;
    if ((rc = check_store(st, gpu))) return rc;
    if ((rc = check_device(slots, "slots", gpu))) return rc;
    if ((k && (rc = check_device(k, "k", gpu))) || (v && (rc = check_device(v, "v", gpu)))) return rc;
    if (!aligned(k, element_size(type)) || !aligned(v, element_size(type))) return fail(LORANN_E_INVAL, "k or v is not aligned to its type");
    const dim3 grid((unsigned)ceil_div(tokens, kBlockTokens), (unsigned)st->heads, 2);
    const TokenRows kr = rows_of(k, k_token, k_head, type), vr = rows_of(v, v_token, v_head, type);
    hipStream_t s = (hipStream_t)hip_stream;
    if (type == LORANN_F32) hipLaunchKernelGGL((k_states_read<float>), grid, dim3(256), 0, s, view(st), slots, tokens, kr, vr, st->dim);
    else if (type == LORANN_F16) hipLaunchKernelGGL((k_states_read<_Float16>), grid, dim3(256), 0, s, view(st), slots, tokens, kr, vr, st->dim);
    else hipLaunchKernelGGL((k_states_read<__bf16>), grid, dim3(256), 0, s, view(st), slots, tokens, kr, vr, st->dim);
    HIP_TRY(hipGetLastError());
    return LORANN_OK;
}

int64_t lorann_attend_workspace(const lorann_states* st, const lorann_questions* qs, int32_t found, int32_t width) {
    int rc;
    if ((rc = check_sizes(st)) || (rc = check_questions(st, qs, found, width))) return rc;
    if (qs->tokens == 0 || qs->sequences == 0) return 0;
    return plan_of(st, qs, found, width).workspace;
}

int lorann_attend_chunk(const lorann_states* st, const lorann_questions* qs, const int32_t* tables, int32_t width, const int32_t* lengths,
                        void* workspace, int64_t workspace_bytes, void* hip_stream) {
    int rc, gpu = -1;
    if ((rc = check_sizes(st)) || (rc = check_questions(st, qs, 0, width))) return rc;
    return attend(st, qs, nullptr, 0, nullptr, 0.0f, tables, width, lengths, 0, workspace, workspace_bytes, (hipStream_t)hip_stream, gpu);
}

int lorann_attend_passages(const lorann_states* st, const lorann_questions* qs, const int64_t* ids, int32_t found, const float* scores,
                           float score_weight, const int32_t* tables, int32_t width, const int32_t* lengths, int64_t passages,
                           void* workspace, int64_t workspace_bytes, void* hip_stream) {
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

}  // extern "C"
