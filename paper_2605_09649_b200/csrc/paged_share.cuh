// Sharing, compacting and moving pages: arguments and launchers.  Not part of the public ABI.
#pragma once

#include "paged.cuh"

namespace tkv {

struct ShareArgs {
    int R, W;
    const int32_t* source;                    // share only, as the next three but old_lens
    const int32_t* old_lens;
    const int32_t* keep_lens;
    const int32_t* new_lens;
    const int32_t* table;                     // [R][W]
    int32_t* table_out;
    const int32_t* refs;                      // [n_pages]; compact: may be null, with refs_out
    int32_t* refs_out;
    const int32_t* free_pages;                // [n_pages], a stack of *free_count
    int32_t* free_out;
    int n_pages;
    const int32_t* free_count;
    int32_t* free_count_out;
    int max_tokens;
    int32_t* lens_out;
    int32_t* cu_new;
    int32_t* slot_map;
    int32_t* positions;                       // may be null
    int max_moves;
    int32_t* move_src;
    int32_t* move_dst;
    int32_t* move_count;
    int32_t* status;
};
cudaError_t launch_paged_share(const ShareArgs& a, cudaStream_t st);
cudaError_t launch_paged_compact(const ShareArgs& a, const unsigned long long* keep_bits, cudaStream_t st);

// Arrays of pages [n_pages][heads][64][row_bytes] whose rows are moved, a launch's worth of them.
constexpr int MOVE_ARRAYS = 128;
struct MoveArray { char* pages; int heads, row_bytes; };
struct MoveArrays { MoveArray a[MOVE_ARRAYS]; int n; };
struct MoveBound { const char* pages; char* bounds; int heads, row_bytes; };
struct MoveBounds { MoveBound a[MOVE_ARRAYS]; int n; };
struct MoveList { const int32_t* src; const int32_t* dst; const int32_t* count; int max_moves, n_pages; int32_t* status; };
cudaError_t launch_paged_move(const MoveArrays& arrays, const MoveList& list, cudaStream_t st);
cudaError_t launch_paged_bounds(const MoveBounds& arrays, int is_bf16, const MoveList& list, cudaStream_t st);

}  // namespace tkv
