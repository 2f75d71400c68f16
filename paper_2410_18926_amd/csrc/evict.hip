// C ABI (include/lorann_evict.h): weights that attention gives each key, and eviction by them.  No call allocates, waits or keeps anything.
#include "../../include/lorann_evict.h"
#include "attend_weights.hpp"
#include "evict.hpp"
#include "states_host.hpp"

using namespace lorann;

namespace {

struct WeightPlan {
    bool many;
    int64_t tiles, padded, row_keys;
    int32_t unit, splits;
    int64_t y, parts, q16, rows, workspace;      // bytes: scores; m and l of the splits; operands; back, m, 1 / l of a row
};

// Rows per sequence and head (their mean over the call) up to which the scores are kept, and how much memory they may take: otherwise they are formed twice.  us kept / formed twice:
//   rows                                                     4          16         32         48         64         128
//   32 sequences, 4096 keys, 8 heads of 128, 8 bits     45 / 117   52 / 114   96 / 114  144 / 127  200 / 125  400 / 149
//   the same, 4 bits                                    43 / 114   44 / 113   65 / 110  117 / 126  171 / 124  360 / 152
//   16 sequences, 4000 keys, 16 heads of 64, 8 bits                           59 / 88   114 / 99   162 / 98
//   one sequence, 16000 keys, 8 heads of 128, 8 bits    20 / 42    26 / 44    39 / 43               64 / 44
//   two sequences, 9000 keys, 4 heads of 64, 4 bits                           32 / 28    43 / 29    54 / 29
// The memory follows from the tables' width, whatever the lengths are: very wide tables of many sequences lose the better way.  64 single tokens of 32 heads after 4096 keys, 8 heads of 128,
// 8 / 4 bits, in tables of 4096 keys 78 / 54, of 65536 235 / 175, of 131072 (1 GiB of scores) 288 / 229 (more sums are read and written), of 131136, formed twice, 1129 / 1109.
// Blocks wanted: of k_weights_scores many more than the GPU holds, since sequences differ in length and a split costs two numbers a row (64 tokens after up to 8192 keys, 8 heads, us with
// 512 / 1024 / 2048 / 4096 / 8192: 102 / 101 / 104 / 89 / 96); of k_weights_rows 4 a CU (4 x 32 tokens after 16000 keys, 512 / 768 / 1024 / 1536 / 2048: 53 / 52 / 40 / 41 / 49; with 1536 calls of
// 16 x 64 tokens after 4000 and of 300 after 60000 were 5 to 7 % faster, of 12 x 200 after 6000 2 % slower).
constexpr int64_t kScoreBlocks = 4096, kRowBlocks = 1024, kFewWeightRows = 32, kMostScores = (int64_t)1 << 30;

// Keys of a block of k_weights_keys: 256, each wavefront with 64 of its own and all rows, or 64 that its wavefronts share with a quarter of the rows each (four times the blocks).  512 blocks are on
// the GPU at a time, and what a wavefront does before its first rows takes as long as 11 steps of 32 rows.  us of a call, 64 shared / 256 apart, one sequence, 8 heads of 128, 8 bits:
//   rows    1000 keys    4000       8000       16000      60000
//   64      23 / 23      23 / 24    29 / 24
//   400     26 / 32      37 / 38    52 / 48
//   1200    36 / 55      60 / 69    95 / 107   161 / 152  497 / 477
bool share_keys(int64_t blocks_apart, int64_t mean_rows) {
    const double fill = 512, before = 11, steps = (double)mean_rows / 32;
    return std::max(1.0, 4 * blocks_apart / fill) * (before + steps / 4) < std::max(1.0, blocks_apart / fill) * (before + steps);
}

template <typename St>
WeightPlan weight_plan(const St* st, const lorann_questions* qs, int32_t width) {
    WeightPlan p{};
    const int64_t group = qs->heads / st->heads, rows = qs->tokens * group, mean_rows = rows / qs->sequences;
    const int64_t keys = (int64_t)width * st->page_size;
    auto tiles_of = [&](int64_t n) { return qs->q_start ? rows / n + qs->sequences : qs->sequences * ceil_div(mean_rows, n); };
    p.row_keys = ceil_div(std::max<int64_t>(keys, 1), kTileKeys) * kTileKeys;
    p.y = rows * st->heads * p.row_keys * 4;
    p.many = mean_rows > kFewWeightRows || p.y > kMostScores;
    p.tiles = tiles_of(p.many ? 128 : kRows);
    const int64_t blocks = std::max<int64_t>(p.tiles * st->heads, 1);
    const int64_t want = std::max<int64_t>(1, std::min((p.many ? kRowBlocks : kScoreBlocks) / blocks, ceil_div(keys, kKeysPerBlock)));
    const int64_t most = std::max(want, ceil_div(keys, p.many ? kMostTileKeys : kMostKeys));
    p.unit = (int32_t)(ceil_div(ceil_div(std::max<int64_t>(keys, 1), most), kKeysPerBlock) * kKeysPerBlock);
    p.splits = (int32_t)ceil_div(std::max<int64_t>(keys, 1), p.unit);
    if (p.many) {
        p.padded = ceil_div(rows, 32) * 32 + 32 * qs->sequences;
        p.y = 0;
        p.q16 = p.padded * st->heads * st->dim * 2;
        p.rows = 3 * p.padded * st->heads * 4;
        p.parts = p.splits > 1 ? 2 * (int64_t)p.splits * p.padded * st->heads * 4 : 0;
    } else p.parts = 2 * (int64_t)p.splits * rows * st->heads * 4;
    p.workspace = ceil_div(p.y + p.parts + p.q16 + p.rows, 16) * 16;
    return p;
}

template <typename St>
int check_weights(const St* st, const lorann_questions* qs, int32_t width) {
    int rc;
    if ((rc = check_sizes(st)) || (rc = check_questions(st, qs, 0, width))) return rc;
    if (qs->sequences > 65535) return fail(LORANN_E_UNSUPPORTED, "%lld sequences are more than 65535", (long long)qs->sequences);          // (a dimension of a grid)
    return LORANN_OK;
}

template <int D, int BITS>
void launch_weights(const WeightPlan& p, const WeightArgs& w, int32_t type, hipStream_t stream) {
    const AttendArgs& a = w.a;
    const dim3 grid((unsigned)(p.tiles * a.st.heads * a.splits));
    if (!p.many) {
        if (type == LORANN_F16) hipLaunchKernelGGL((k_weights_scores<_Float16, D, BITS>), grid, dim3(64 * kAttendWaves), 0, stream, w);
        else hipLaunchKernelGGL((k_weights_scores<__bf16, D, BITS>), grid, dim3(64 * kAttendWaves), 0, stream, w);
        return;
    }
    if (type == LORANN_F16) hipLaunchKernelGGL((k_weights_rows<_Float16, D, BITS>), grid, dim3(256), 0, stream, w);
    else hipLaunchKernelGGL((k_weights_rows<__bf16, D, BITS>), grid, dim3(256), 0, stream, w);
    if (a.splits > 1) {
        const int64_t blocks = ceil_div(a.st.heads * w.padded, 32), x = std::min<int64_t>(blocks, 4096);          // (one dimension would pass 2^32 threads from 2^29 rows and heads on)
        hipLaunchKernelGGL(k_weights_join, dim3((unsigned)x, (unsigned)ceil_div(blocks, x)), dim3(256), 0, stream, w);
    }
    const bool share = share_keys(ceil_div(w.keys, 256) * a.st.heads * a.sequences, a.tokens * a.group / a.sequences);
    const dim3 chunks((unsigned)ceil_div(w.keys, share ? 64 : 256), (unsigned)a.st.heads, (unsigned)a.sequences);
    if (share) hipLaunchKernelGGL((k_weights_keys<D, BITS, true>), chunks, dim3(256), 0, stream, w);
    else hipLaunchKernelGGL((k_weights_keys<D, BITS, false>), chunks, dim3(256), 0, stream, w);
}

template <typename St>
int attend_weights(const St* st, const lorann_questions* qs, const int32_t* tables, int32_t width, const int32_t* lengths, const float* before, float* sums,
                   void* workspace, int64_t workspace_bytes, hipStream_t stream) {
    constexpr int bits = std::is_same_v<St, lorann_states4> ? 4 : 8;
    int rc, gpu = -1;
    if ((rc = check_weights(st, qs, width))) return rc;
    if (qs->sequences == 0 || width == 0) return LORANN_OK;
    if (!qs->q_start && qs->tokens % qs->sequences) return fail(LORANN_E_INVAL, "%lld tokens do not divide over %lld sequences", (long long)qs->tokens, (long long)qs->sequences);
    if ((rc = check_store(st, gpu))) return rc;
    if (qs->tokens > 0) {
        if ((rc = check_device(qs->q, "q", gpu))) return rc;
        if (!aligned(qs->q, 2)) return fail(LORANN_E_INVAL, "q is not aligned to its type");
        if (qs->q_start && (rc = check_device(qs->q_start, "q_start", gpu))) return rc;
    }
    if ((rc = check_device(tables, "tables", gpu)) || (rc = check_device(lengths, "lengths", gpu))) return rc;
    if ((before && (rc = check_device(before, "before", gpu))) || (rc = check_device(sums, "sums", gpu))) return rc;
    if (!aligned(before, 4) || !aligned(sums, 4)) return fail(LORANN_E_INVAL, "before or sums is not 4-byte aligned");
    WeightPlan p = weight_plan(st, qs, width);
    const int64_t blocks = p.tiles * st->heads * p.splits;
    if (p.tiles > 0x7fffffff || blocks > 0xffffffffLL / 256) return fail(LORANN_E_UNSUPPORTED, "%lld tokens of %lld sequences are more than one launch holds", (long long)qs->tokens, (long long)qs->sequences);
    if (p.workspace) {
        if (!workspace || workspace_bytes < p.workspace) return fail(LORANN_E_INVAL, "the workspace holds %lld bytes, %lld are needed", (long long)(workspace ? workspace_bytes : 0), (long long)p.workspace);
        if (!aligned(workspace, 16)) return fail(LORANN_E_INVAL, "the workspace is not 16-byte aligned");
        if ((rc = check_device(workspace, "workspace", gpu))) return rc;
    }
    WeightArgs w{};
    AttendArgs& a = w.a;
    a.st = view(st);
    a.q = qs->q;
    a.q_token = qs->q_token; a.q_head = qs->q_head;
    a.tokens = qs->tokens; a.sequences = (int32_t)qs->sequences; a.group = qs->heads / st->heads;
    a.q_start = qs->tokens > 0 ? qs->q_start : nullptr;
    a.c = qs->scale * 1.44269504088896341f;
    a.tables = tables; a.width = width; a.lengths = lengths;
    a.found = 1;
    a.unit = p.unit; a.units = a.splits = p.splits; a.per_split = 1;
    a.q_wide = aligned(qs->q, 16) && qs->q_token % 8 == 0 && qs->q_head % 8 == 0;
    // as much of the scale's power of two goes with the rows as leaves their factors (2^-114 .. 2^113: row_power) normal floats, the rest with the keys' steps
    int power = 0;
    const float part = std::frexp(a.c, &power);
    const int with_rows = std::min(std::max(power, -12), 14);
    w.step_c = std::ldexp(part, power - with_rows);
    w.back_c = std::ldexp(1.0f, with_rows);
    w.before = before; w.sums = sums; w.keys = (int64_t)width * st->page_size; w.row_keys = p.row_keys; w.padded = p.padded;
    char* at = (char*)workspace;
    if (p.many) {
        w.q16 = (f16x8*)at;
        at += p.q16;
        w.back = (float*)at;
        w.row_m = w.back + p.padded * st->heads;
        w.row_inv = w.row_m + p.padded * st->heads;
        at += p.rows;
    } else {
        w.y = (float*)at;
        at += p.y;
    }
    a.part_m = (float*)at;
    a.part_l = a.part_m + p.parts / 8;
    if (qs->tokens > 0) {
        switch (st->dim) {
            case 32: launch_weights<32, bits>(p, w, qs->type, stream); break;
            case 64: launch_weights<64, bits>(p, w, qs->type, stream); break;
            case 96: launch_weights<96, bits>(p, w, qs->type, stream); break;
            default: launch_weights<128, bits>(p, w, qs->type, stream); break;
        }
    }
    if (qs->tokens == 0 || !p.many) hipLaunchKernelGGL(k_weights_add, dim3((unsigned)ceil_div(w.keys, kAddKeys), (unsigned)st->heads, (unsigned)qs->sequences), dim3(256), 0, stream, w);
    HIP_TRY(hipGetLastError());
    return LORANN_OK;
}

template <typename St>
int64_t attend_weights_workspace(const St* st, const lorann_questions* qs, int32_t width) {
    int rc;
    if ((rc = check_weights(st, qs, width))) return rc;
    if (qs->sequences == 0 || width == 0 || qs->tokens == 0) return 0;
    return weight_plan(st, qs, width).workspace;
}

// Tables whose keys fit a block's registers (16 a thread) are chosen from in one launch, longer ones in chunks.
constexpr int64_t kChooseKeys = 16 * kChooseThreads;
int64_t evict_chunks(int64_t keys) { return ceil_div(keys, kChunk); }
int64_t evict_room(int64_t seats, int64_t keys) {
    if (keys <= kChooseKeys) return 0;
    return ceil_div(seats * evict_chunks(keys) * (2 * kBins + 3) * 4 + seats * 16, 16) * 16;
}

template <typename St>
int evict(const St* st, const int32_t* tables, int32_t width, const int32_t* lengths, int64_t sequences, const float* sums, int32_t budget, int32_t recent, const int32_t* to_tables,
          int32_t to_width, int32_t* kept, int32_t* kept_lengths, float* kept_sums, void* workspace, int64_t workspace_bytes, hipStream_t stream) {
    constexpr int bits = std::is_same_v<St, lorann_states4> ? 4 : 8;
    int rc, gpu = -1;
    if ((rc = check_sizes(st))) return rc;
    if (sequences < 0 || width < 0 || to_width < 0) return fail(LORANN_E_INVAL, "%lld sequences, tables of width %d and %d", (long long)sequences, width, to_width);
    if (sequences > 65535) return fail(LORANN_E_UNSUPPORTED, "%lld sequences are more than 65535", (long long)sequences);
    if (budget < 0 || recent < 0 || recent > budget) return fail(LORANN_E_INVAL, "a budget of %d tokens, %d of them the newest", budget, recent);
    if ((int64_t)width * st->page_size > (1 << 30) || (int64_t)to_width * st->page_size > (1 << 30))
        return fail(LORANN_E_UNSUPPORTED, "tables of %d and %d pages of %d tokens are longer than 2^30 tokens", width, to_width, st->page_size);
    if ((int64_t)to_width * st->page_size < budget) return fail(LORANN_E_INVAL, "destinations of %d pages hold no %d tokens", to_width, budget);
    if (sequences == 0) return LORANN_OK;
    if ((rc = check_store(st, gpu))) return rc;
    if (width > 0 && ((rc = check_device(tables, "tables", gpu)) || (rc = check_device(sums, "sums", gpu)))) return rc;
    if ((rc = check_device(lengths, "lengths", gpu)) || (rc = check_device(kept_lengths, "kept_lengths", gpu))) return rc;
    if (budget > 0 && (rc = check_device(kept, "kept", gpu))) return rc;
    if (to_width > 0 && (budget > 0 || kept_sums) && (rc = check_device(to_tables, "to_tables", gpu))) return rc;          // (where the move runs, it reads them)
    if (kept_sums && to_width > 0 && (rc = check_device(kept_sums, "kept_sums", gpu))) return rc;
    if (!aligned(sums, 4) || !aligned(kept, 4) || !aligned(kept_lengths, 4) || !aligned(kept_sums, 4)) return fail(LORANN_E_INVAL, "an array is not 4-byte aligned");
    const int64_t seats = sequences * st->heads, keys = (int64_t)width * st->page_size, room = evict_room(seats, keys), chunks = evict_chunks(keys);
    const int64_t tokens = kept_sums ? (int64_t)to_width * st->page_size : budget;
    if (seats * (room ? chunks : 1) > 0xffffffffLL / kChooseThreads || ceil_div(tokens, 64) > 0xffffffffLL / 256)       // (threads of a grid)
        return fail(LORANN_E_UNSUPPORTED, "%lld sequences of %d heads, tables of %lld tokens are more than one launch holds", (long long)sequences, st->heads, (long long)keys);
    if (room) {
        if (!workspace || workspace_bytes < room) return fail(LORANN_E_INVAL, "the workspace holds %lld bytes, %lld are needed", (long long)(workspace ? workspace_bytes : 0), (long long)room);
        if (!aligned(workspace, 16)) return fail(LORANN_E_INVAL, "the workspace is not 16-byte aligned");
        if ((rc = check_device(workspace, "workspace", gpu))) return rc;
    }
    EvictArgs a{};
    a.st = view(st);
    a.tables = tables; a.width = width; a.lengths = lengths; a.sums = sums; a.keys = keys;
    a.budget = budget; a.recent = recent; a.to_tables = to_tables; a.to_width = to_width;
    a.kept = kept; a.kept_lengths = kept_lengths; a.kept_sums = to_width > 0 ? kept_sums : nullptr;
    const bool wide = aligned(sums, 16);
    if (!room) {
        const dim3 grid((unsigned)seats), block(kChooseThreads);
        if (keys <= 4 * kChooseThreads) hipLaunchKernelGGL(k_evict_choose<4>, grid, block, 0, stream, a, wide);
        else if (keys <= 8 * kChooseThreads) hipLaunchKernelGGL(k_evict_choose<8>, grid, block, 0, stream, a, wide);
        else hipLaunchKernelGGL(k_evict_choose<16>, grid, block, 0, stream, a, wide);
    } else {
        ChunkArgs c{};
        c.a = a;
        c.chunks = (int32_t)chunks;
        c.hist[0] = (uint32_t*)workspace;
        c.hist[1] = c.hist[0] + seats * chunks * kBins;
        c.there = (uint2*)(c.hist[1] + seats * chunks * kBins);
        c.place = (uint32_t*)(c.there + seats * chunks);
        c.state = c.place + seats * chunks;
        const dim3 grid((unsigned)(seats * chunks)), block(kChooseThreads);
        hipLaunchKernelGGL(k_evict_chunks<0>, grid, block, 0, stream, c, wide);
        hipLaunchKernelGGL(k_evict_chunks<1>, grid, block, 0, stream, c, wide);
        hipLaunchKernelGGL(k_evict_chunks<2>, grid, block, 0, stream, c, wide);
        hipLaunchKernelGGL(k_evict_chunks<3>, grid, block, 0, stream, c, wide);
    }
    if (tokens > 0) hipLaunchKernelGGL((k_evict_move<bits>), dim3((unsigned)ceil_div(tokens, 64), (unsigned)st->heads, (unsigned)sequences), dim3(256), 0, stream, a, st->dim);
    HIP_TRY(hipGetLastError());
    return LORANN_OK;
}

}  // namespace

extern "C" {

int lorann_attend_weights(const lorann_states* st, const lorann_questions* qs, const int32_t* tables, int32_t width, const int32_t* lengths,
                          const float* before, float* sums, void* workspace, int64_t workspace_bytes, void* hip_stream) {
    return attend_weights(st, qs, tables, width, lengths, before, sums, workspace, workspace_bytes, (hipStream_t)hip_stream);
}

int lorann_attend4_weights(const lorann_states4* st, const lorann_questions* qs, const int32_t* tables, int32_t width, const int32_t* lengths,
                           const float* before, float* sums, void* workspace, int64_t workspace_bytes, void* hip_stream) {
    return attend_weights(st, qs, tables, width, lengths, before, sums, workspace, workspace_bytes, (hipStream_t)hip_stream);
}

int64_t lorann_attend_weights_workspace(const lorann_states* st, const lorann_questions* qs, int32_t width) { return attend_weights_workspace(st, qs, width); }

int64_t lorann_attend4_weights_workspace(const lorann_states4* st, const lorann_questions* qs, int32_t width) { return attend_weights_workspace(st, qs, width); }

int lorann_states_evict(const lorann_states* st, const int32_t* tables, int32_t width, const int32_t* lengths, int64_t sequences, const float* sums, int32_t budget, int32_t recent,
                        const int32_t* to_tables, int32_t to_width, int32_t* kept, int32_t* kept_lengths, float* kept_sums, void* workspace, int64_t workspace_bytes, void* hip_stream) {
    return evict(st, tables, width, lengths, sequences, sums, budget, recent, to_tables, to_width, kept, kept_lengths, kept_sums, workspace, workspace_bytes, (hipStream_t)hip_stream);
}

int lorann_states4_evict(const lorann_states4* st, const int32_t* tables, int32_t width, const int32_t* lengths, int64_t sequences, const float* sums, int32_t budget, int32_t recent,
                         const int32_t* to_tables, int32_t to_width, int32_t* kept, int32_t* kept_lengths, float* kept_sums, void* workspace, int64_t workspace_bytes, void* hip_stream) {
    return evict(st, tables, width, lengths, sequences, sums, budget, recent, to_tables, to_width, kept, kept_lengths, kept_sums, workspace, workspace_bytes, (hipStream_t)hip_stream);
}

int64_t lorann_evict_workspace(int32_t heads, int64_t table_tokens, int64_t sequences) {
    if (heads < 1 || table_tokens < 0 || sequences < 0) return fail(LORANN_E_INVAL, "%d heads, tables of %lld tokens, %lld sequences", heads, (long long)table_tokens, (long long)sequences);
    if (table_tokens > 1 << 30 || sequences > 65535) return fail(LORANN_E_UNSUPPORTED, "tables of %lld tokens, %lld sequences", (long long)table_tokens, (long long)sequences);
    return evict_room(heads * sequences, table_tokens);
}

}  // extern "C"
