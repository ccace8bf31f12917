// Argument checks that the C entry points of the paged caches share.
#pragma once

#include "paged.cuh"

namespace tkv {

template <typename... A>
inline trimkv_status refuse(trimkv_status s, const char* fmt, A... args) {
    set_last_error(fmt, args...);
    return s;
}
inline bool ok16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool ok4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

inline trimkv_status done(cudaError_t e, const char* what) {
    if (e == cudaSuccess) return TRIMKV_OK;
    cudaGetLastError();
    return refuse(TRIMKV_E_CUDA, "%s launch failed: %s", what, cudaGetErrorString(e));
}

// What the attention calls share: requests, tokens, q, out, tables, scale, workspace.
trimkv_status paged_check_batch(const PagedView& pv, int is_bf16, size_t workspace_needed, int32_t n_req, int64_t n_tokens, int32_t q_heads, const void* q,
                                int64_t q_stride, const int32_t* cu_new, const int32_t* lens, const int32_t* block_table, int32_t table_width, float scale,
                                const void* out, const void* workspace, size_t workspace_bytes, int32_t* status, PagedBatch* pb);

}  // namespace tkv
