// C entry points that share, compact and move pages: argument checks.
#include <limits.h>

#include <algorithm>

#include "paged_check.cuh"
#include "paged_share.cuh"

using namespace tkv;

namespace {

trimkv_status check_rows(const ShareArgs& a, int64_t max_tokens, int64_t max_moves) {
    if (a.R < 1 || a.R > PAGED_MAX_REQ) return refuse(TRIMKV_E_ARG, "n_req must be in [1, %d]", PAGED_MAX_REQ);
    if (a.W < 1 || a.W > TRIMKV_PAGED_MAX_WIDTH) return refuse(TRIMKV_E_ARG, "table_width must be in [1, %d]", TRIMKV_PAGED_MAX_WIDTH);
    if (a.n_pages < 1 || a.n_pages > TRIMKV_PAGED_MAX_PAGES) return refuse(TRIMKV_E_ARG, "n_pages must be in [1, %d]", TRIMKV_PAGED_MAX_PAGES);
    if (max_tokens < 0 || max_tokens > (1LL << 30)) return refuse(TRIMKV_E_ARG, "max_tokens must be in [0, 2^30]");
    if (max_moves < 0 || max_moves > (1LL << 30)) return refuse(TRIMKV_E_ARG, "max_moves must be in [0, 2^30]");
    if (!a.old_lens || !a.table || !a.table_out || !a.free_pages || !a.free_out || !a.free_count || !a.free_count_out || !a.lens_out || !a.move_count ||
        (max_moves > 0 && (!a.move_src || !a.move_dst)))
        return refuse(TRIMKV_E_ARG, "NULL buffer");
    if (a.table_out == a.table) return refuse(TRIMKV_E_ARG, "table_out must not be the table");
    if (a.lens_out == a.old_lens || a.lens_out == a.keep_lens || a.lens_out == a.new_lens || a.lens_out == a.source) return refuse(TRIMKV_E_ARG, "lens_out must not be an input");
    const void* all[] = {a.source, a.old_lens, a.keep_lens, a.new_lens, a.table, a.table_out, a.refs, a.refs_out, a.free_pages, a.free_out, a.free_count,
                         a.free_count_out, a.lens_out, a.cu_new, a.slot_map, a.positions, a.move_src, a.move_dst, a.move_count, a.status};
    for (const void* p : all)
        if (!ok4(p)) return refuse(TRIMKV_E_ARG, "int32 buffers must be 4-byte aligned");
    return TRIMKV_OK;
}

}  // namespace

extern "C" {

trimkv_status trimkv_paged_share(int32_t n_req, const int32_t* source, const int32_t* old_lens, const int32_t* keep_lens, const int32_t* new_lens,
                                 const int32_t* block_table, int32_t* table_out, int32_t table_width, const int32_t* page_refs, int32_t* refs_out,
                                 const int32_t* free_pages, int32_t* free_out, int32_t n_pages, const int32_t* free_count, int32_t* free_count_out,
                                 int64_t max_tokens, int32_t* lens_out, int32_t* cu_new, int32_t* slot_map, int32_t* positions, int64_t max_moves,
                                 int32_t* move_src, int32_t* move_dst, int32_t* move_count, int32_t* status, void* stream) {
    ShareArgs a = {n_req, table_width, source, old_lens, keep_lens, new_lens, block_table, table_out, page_refs, refs_out, free_pages, free_out, n_pages,
                   free_count, free_count_out, (int)max_tokens, lens_out, cu_new, slot_map, positions, (int)max_moves, move_src, move_dst, move_count, status};
    const trimkv_status s = check_rows(a, max_tokens, max_moves);
    if (s != TRIMKV_OK) return s;
    if (!source || !keep_lens || !new_lens || !page_refs || !refs_out || !cu_new || (max_tokens > 0 && !slot_map)) return refuse(TRIMKV_E_ARG, "NULL buffer");
    return done(launch_paged_share(a, (cudaStream_t)stream), "share");
}

trimkv_status trimkv_paged_compact(int32_t n_req, const int32_t* lens, const uint64_t* keep_bits, const int32_t* block_table, int32_t* table_out,
                                   int32_t table_width, const int32_t* page_refs, int32_t* refs_out, const int32_t* free_pages, int32_t* free_out,
                                   int32_t n_pages, const int32_t* free_count, int32_t* free_count_out, int32_t* lens_out, int64_t max_moves,
                                   int32_t* move_src, int32_t* move_dst, int32_t* move_count, int32_t* status, void* stream) {
    ShareArgs a = {n_req, table_width, nullptr, lens, nullptr, nullptr, block_table, table_out, page_refs, refs_out, free_pages, free_out, n_pages,
                   free_count, free_count_out, 0, lens_out, nullptr, nullptr, nullptr, (int)max_moves, move_src, move_dst, move_count, status};
    const trimkv_status s = check_rows(a, 0, max_moves);
    if (s != TRIMKV_OK) return s;
    if (!keep_bits || (reinterpret_cast<uintptr_t>(keep_bits) & 7u)) return refuse(TRIMKV_E_ARG, "keep_bits must be non-NULL and 8-byte aligned");
    if (!page_refs != !refs_out) return refuse(TRIMKV_E_ARG, "page_refs and refs_out go together");
    return done(launch_paged_compact(a, (const unsigned long long*)keep_bits, (cudaStream_t)stream), "compact");
}

trimkv_status trimkv_paged_move(int32_t n_arrays, const trimkv_paged_rows* arrays, int32_t n_pages, int64_t max_moves, const int32_t* move_src,
                                const int32_t* move_dst, const int32_t* move_count, int32_t* status, void* stream) {
    if (n_arrays < 0 || n_arrays > TRIMKV_PAGED_MAX_ARRAYS || (n_arrays > 0 && !arrays)) return refuse(TRIMKV_E_ARG, "n_arrays must be in [0, %d], arrays non-NULL", TRIMKV_PAGED_MAX_ARRAYS);
    if (n_pages < 1 || n_pages > TRIMKV_PAGED_MAX_PAGES) return refuse(TRIMKV_E_ARG, "n_pages must be in [1, %d]", TRIMKV_PAGED_MAX_PAGES);
    if (max_moves < 0 || max_moves > (1LL << 30)) return refuse(TRIMKV_E_ARG, "max_moves must be in [0, 2^30]");
    if (max_moves > 0 && (!move_src || !move_dst || !move_count || !ok4(move_src) || !ok4(move_dst) || !ok4(move_count)))
        return refuse(TRIMKV_E_ARG, "move_src, move_dst and move_count must be non-NULL and aligned");
    if (!ok4(status)) return refuse(TRIMKV_E_ARG, "status must be aligned");
    for (int i = 0; i < n_arrays; ++i) {
        const trimkv_paged_rows& r = arrays[i];
        if (!r.pages || !ok16(r.pages) || !ok16(r.key_bounds)) return refuse(TRIMKV_E_ARG, "array %d: pages must be non-NULL, pages and key_bounds 16-byte aligned", i);
        if (r.heads < 1 || r.heads > 1024) return refuse(TRIMKV_E_ARG, "array %d: heads must be in [1, 1024]", i);
        if (r.row_bytes < 1 || r.row_bytes > 4096) return refuse(TRIMKV_E_ARG, "array %d: row_bytes must be in [1, 4096]", i);
        if (r.reserved != 0) return refuse(TRIMKV_E_ARG, "array %d: reserved must be 0", i);
        if (r.key_bounds && ((r.dtype != TRIMKV_DTYPE_BF16 && r.dtype != TRIMKV_DTYPE_F32) || r.row_bytes % 16))
            return refuse(TRIMKV_E_ARG, "array %d: key_bounds want bf16 or fp32 rows of a multiple of 16 bytes", i);
    }
    if (n_arrays == 0 || max_moves == 0) return TRIMKV_OK;
    const cudaStream_t st = (cudaStream_t)stream;
    const MoveList list = {move_src, move_dst, move_count, (int)max_moves, n_pages, status};
    cudaError_t e = cudaSuccess;
    for (int i0 = 0; i0 < n_arrays && e == cudaSuccess; i0 += MOVE_ARRAYS) {
        MoveArrays m;
        m.n = std::min(n_arrays - i0, MOVE_ARRAYS);
        for (int i = 0; i < m.n; ++i) m.a[i] = {(char*)arrays[i0 + i].pages, arrays[i0 + i].heads, arrays[i0 + i].row_bytes};
        e = launch_paged_move(m, list, st);
    }
    for (int bf16 = 0; bf16 < 2; ++bf16) {
        MoveBounds b;
        b.n = 0;
        for (int i = 0; i <= n_arrays && e == cudaSuccess; ++i) {
            if (b.n == MOVE_ARRAYS || (i == n_arrays && b.n > 0)) {
                e = launch_paged_bounds(b, bf16, list, st);
                b.n = 0;
            }
            if (i < n_arrays && arrays[i].key_bounds && (arrays[i].dtype == TRIMKV_DTYPE_BF16) == (bf16 == 1))
                b.a[b.n++] = {(const char*)arrays[i].pages, (char*)arrays[i].key_bounds, arrays[i].heads, arrays[i].row_bytes};
        }
    }
    return done(e, "move");
}

}  // extern "C"
