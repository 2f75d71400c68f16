// C ABI (include/lorann_states4.h) of the 4-bit state store and its attention: argument checks, plans and launches.  No call allocates, waits or keeps anything.
#include "states_host.hpp"
#include "states4_store.hpp"

using namespace lorann;

extern "C" {

int lorann_states4_write(const lorann_states4* st, const void* k, const void* v, int32_t type, int64_t tokens,
                        int64_t k_token, int64_t k_head, int64_t v_token, int64_t v_head, const int64_t* slots, void* hip_stream) {
    int rc, gpu = -1;
    if ((rc = check_sizes(st)) || (rc = check_tokens(st, type, tokens))) return rc;
    if (tokens == 0) return LORANN_OK;
    if ((rc = check_rows(st, slots, k, v, type, true, gpu))) return rc;
    const dim3 grid = heads_grid(st, tokens);
    const TokenRows kr = rows_of(const_cast<void*>(k), k_token, k_head, type), vr = rows_of(const_cast<void*>(v), v_token, v_head, type);
    hipStream_t s = (hipStream_t)hip_stream;
    if (type == LORANN_F32) hipLaunchKernelGGL((k_states4_write<float>), grid, dim3(256), 0, s, view(st), kr, vr, slots, tokens, st->dim);
    else if (type == LORANN_F16) hipLaunchKernelGGL((k_states4_write<_Float16>), grid, dim3(256), 0, s, view(st), kr, vr, slots, tokens, st->dim);
    else hipLaunchKernelGGL((k_states4_write<__bf16>), grid, dim3(256), 0, s, view(st), kr, vr, slots, tokens, st->dim);
    HIP_TRY(hipGetLastError());
    return LORANN_OK;
}

int lorann_states4_read(const lorann_states4* st, const int64_t* slots, int64_t tokens, void* k, void* v, int32_t type,
                       int64_t k_token, int64_t k_head, int64_t v_token, int64_t v_head, void* hip_stream) {
    int rc, gpu = -1;
    if ((rc = check_sizes(st)) || (rc = check_tokens(st, type, tokens))) return rc;
    if (tokens == 0 || (!k && !v)) return LORANN_OK;
    if ((rc = check_rows(st, slots, k, v, type, false, gpu))) return rc;
    const dim3 grid = rows_grid(st, tokens);
    const TokenRows kr = rows_of(k, k_token, k_head, type), vr = rows_of(v, v_token, v_head, type);
    hipStream_t s = (hipStream_t)hip_stream;
    if (type == LORANN_F32) hipLaunchKernelGGL((k_states4_read<float>), grid, dim3(256), 0, s, view(st), slots, tokens, kr, vr, st->dim);
    else if (type == LORANN_F16) hipLaunchKernelGGL((k_states4_read<_Float16>), grid, dim3(256), 0, s, view(st), slots, tokens, kr, vr, st->dim);
    else hipLaunchKernelGGL((k_states4_read<__bf16>), grid, dim3(256), 0, s, view(st), slots, tokens, kr, vr, st->dim);
    HIP_TRY(hipGetLastError());
    return LORANN_OK;
}

int64_t lorann_attend4_workspace(const lorann_states4* st, const lorann_questions* qs, int32_t found, int32_t width) {
    return attend_workspace(st, qs, found, width);
}

int lorann_attend4_chunk(const lorann_states4* st, const lorann_questions* qs, const int32_t* tables, int32_t width, const int32_t* lengths,
                        void* workspace, int64_t workspace_bytes, void* hip_stream) {
    return attend_chunk(st, qs, tables, width, lengths, workspace, workspace_bytes, hip_stream);
}

int lorann_attend4_passages(const lorann_states4* st, const lorann_questions* qs, const int64_t* ids, int32_t found, const float* scores,
                           float score_weight, const int32_t* tables, int32_t width, const int32_t* lengths, int64_t passages,
                           void* workspace, int64_t workspace_bytes, void* hip_stream) {
    return attend_passages(st, qs, ids, found, scores, score_weight, tables, width, lengths, passages, workspace, workspace_bytes, hip_stream);
}

}  // extern "C"
