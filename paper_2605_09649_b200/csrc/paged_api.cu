// C entry points of the caller-owned paged cache: argument checks, workspace layout, choice of kernels.
#include <limits.h>
#include <math.h>

#include <algorithm>

#include "paged.cuh"

using namespace tkv;

namespace {

template <typename... A>
trimkv_status refuse(trimkv_status s, const char* fmt, A... args) {
    set_last_error(fmt, args...);
    return s;
}
bool ok16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool ok4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

trimkv_status done(cudaError_t e, const char* what) {
    if (e == cudaSuccess) return TRIMKV_OK;
    cudaGetLastError();
    return refuse(TRIMKV_E_CUDA, "%s launch failed: %s", what, cudaGetErrorString(e));
}

trimkv_status check_cache(const trimkv_paged_cache* c, PagedView* pv) {
    if (!c || !c->k_pages || !c->v_pages) return refuse(TRIMKV_E_ARG, "cache, k_pages and v_pages must not be NULL");
    if (c->reserved != 0) return refuse(TRIMKV_E_ARG, "reserved must be 0");
    if (c->kv_dtype != TRIMKV_DTYPE_BF16 && c->kv_dtype != TRIMKV_DTYPE_F32) return refuse(TRIMKV_E_ARG, "unknown kv_dtype %d", c->kv_dtype);
    if (c->page_size != PAGE) return refuse(TRIMKV_E_UNSUPPORTED, "page_size must be %d", PAGE);
    if (c->n_pages < 1 || c->n_pages > TRIMKV_PAGED_MAX_PAGES) return refuse(TRIMKV_E_ARG, "n_pages must be in [1, %d]", TRIMKV_PAGED_MAX_PAGES);
    if (c->kv_heads < 1 || c->kv_heads > 1024) return refuse(TRIMKV_E_ARG, "kv_heads must be in [1, 1024]");
    if (c->head_dim < 8 || c->head_dim % 8 || c->head_dim > 256) return refuse(TRIMKV_E_UNSUPPORTED, "head_dim must be a multiple of 8 up to 256");
    // rows of the tensor maps and slots are 32-bit numbers
    if ((long long)c->n_pages * c->kv_heads * PAGE > INT_MAX) return refuse(TRIMKV_E_UNSUPPORTED, "n_pages x kv_heads x %d must be below 2^31", PAGE);
    if (!ok16(c->k_pages) || !ok16(c->v_pages) || !ok16(c->key_bounds)) return refuse(TRIMKV_E_ARG, "k_pages, v_pages and key_bounds must be 16-byte aligned");
    pv->k = (const char*)c->k_pages;
    pv->v = (const char*)c->v_pages;
    pv->bounds = (const char*)c->key_bounds;
    pv->n_pages = c->n_pages;
    pv->H = c->kv_heads;
    pv->d = c->head_dim;
    return TRIMKV_OK;
}

// Workspace: two areas {shared units, partial results}.  The first serves the kernel that a call always has or the
// only one, the second the tensor-core kernel, where the head size has one.  Sizes depend on the head size alone.
size_t area_bytes(int rows, int d) { return PAGED_SHARED_BYTES + paged_partial_bytes(rows, d); }
// The most (workers x rows of a unit) of the first kernels: the fp32 kernel's units are 16 rows; the warp kernel's 8 or 16 with
// four workers per SM, 32 or 64 with two.
constexpr int FIRST_ROWS = PAGED_SMS * 2 * PAGED_WARP_ROWS;
static_assert(PAGED_F32_CTAS * PAGED_F32_ROWS <= 2 * PAGED_WARP_ROWS && PAGED_WARPS * 16 <= 2 * PAGED_WARP_ROWS, "every kernel fits");
size_t first_area(int d) { return area_bytes(FIRST_ROWS, d); }
size_t work_bytes(int d) { return first_area(d) + (d <= PAGED_TC_HEAD ? area_bytes(PAGED_SMS * PAGED_TC_ROWS, d) : 0); }
PagedWork carve(void* area, int rows, int d) {
    char* p = (char*)area;
    PagedWork w;
    w.shared = (int4*)p;
    w.part_o = (float*)(p + PAGED_SHARED_BYTES);
    w.part_ml = w.part_o + (size_t)2 * rows * d;
    return w;
}

trimkv_status check_batch(const PagedView& pv, int is_bf16, int32_t n_req, int64_t n_tokens, int32_t q_heads, const void* q, int64_t q_stride,
                          const int32_t* cu_new, const int32_t* lens, const int32_t* block_table, int32_t table_width, float scale,
                          const void* out, const void* workspace, size_t workspace_bytes, int32_t* status, PagedBatch* pb) {
    if (n_req < 1 || n_req > PAGED_MAX_REQ) return refuse(TRIMKV_E_ARG, "n_req must be in [1, %d]", PAGED_MAX_REQ);
    if (table_width < 1 || table_width > TRIMKV_PAGED_MAX_WIDTH) return refuse(TRIMKV_E_ARG, "table_width must be in [1, %d]", TRIMKV_PAGED_MAX_WIDTH);
    if (q_heads < pv.H || q_heads % pv.H || q_heads / pv.H > 128) return refuse(TRIMKV_E_ARG, "q_heads must be kv_heads times 1 to 128");
    if (n_tokens < 0 || n_tokens * q_heads > (1LL << 30)) return refuse(TRIMKV_E_ARG, "n_tokens x q_heads must be in [0, 2^30]");
    if (n_tokens > 0) {
        if (!q || !out || !ok16(q) || !ok16(out)) return refuse(TRIMKV_E_ARG, "q and out must be non-NULL and 16-byte aligned");
        if (q_stride < (int64_t)q_heads * pv.d || q_stride > (1LL << 31) || (q_stride * (is_bf16 ? 2 : 4)) % 16)
            return refuse(TRIMKV_E_ARG, "q_stride must cover a token's q and be a multiple of 16 bytes");
        // several workers read a row of q, and any of them may be the first to write its part of out
        const size_t elt = is_bf16 ? 2 : 4, row = (size_t)q_heads * pv.d * elt;
        const uintptr_t q0 = reinterpret_cast<uintptr_t>(q), o0 = reinterpret_cast<uintptr_t>(out);
        if (q0 < o0 + n_tokens * row && o0 < q0 + (n_tokens - 1) * (size_t)q_stride * elt + row) return refuse(TRIMKV_E_ARG, "out must not overlap q");
    }
    if (!cu_new || !lens || !block_table || !ok4(cu_new) || !ok4(lens) || !ok4(block_table) || !ok4(status))
        return refuse(TRIMKV_E_ARG, "cu_new, lens and block_table must be non-NULL and aligned");
    if (!(scale > 0.f) || isinf(scale)) return refuse(TRIMKV_E_ARG, "scale must be positive and finite");
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return refuse(TRIMKV_E_ARG, "workspace must be non-NULL and 256-byte aligned");
    const size_t need = work_bytes(pv.d);
    if (workspace_bytes < need) return refuse(TRIMKV_E_ARG, "workspace too small: %zu bytes, %zu needed", workspace_bytes, need);
    *pb = PagedBatch{};
    pb->cu_new = cu_new;
    pb->lens = lens;
    pb->table = block_table;
    pb->R = n_req;
    pb->W = table_width;
    pb->T = (int)n_tokens;
    pb->Hq = q_heads;
    pb->g = q_heads / pv.H;
    pb->by_g = FastDiv::by(pb->g);
    pb->by_h = FastDiv::by(pv.H);
    pb->q_stride = q_stride;
    pb->status = status;
    return TRIMKV_OK;
}

}  // namespace

extern "C" {

trimkv_status trimkv_paged_plan(int32_t n_req, const int32_t* old_lens, const int32_t* keep_lens, const int32_t* new_lens,
                                int32_t* block_table, int32_t table_width, int32_t* free_pages, int32_t n_pages,
                                const int32_t* free_count, int32_t* free_count_out, int64_t max_tokens, int32_t* lens_out,
                                int32_t* cu_new, int32_t* slot_map, int32_t* positions, int32_t* status, void* stream) {
    if (n_req < 1 || n_req > PAGED_MAX_REQ) return refuse(TRIMKV_E_ARG, "n_req must be in [1, %d]", PAGED_MAX_REQ);
    if (table_width < 1 || table_width > TRIMKV_PAGED_MAX_WIDTH) return refuse(TRIMKV_E_ARG, "table_width must be in [1, %d]", TRIMKV_PAGED_MAX_WIDTH);
    if (n_pages < 1 || n_pages > TRIMKV_PAGED_MAX_PAGES) return refuse(TRIMKV_E_ARG, "n_pages must be in [1, %d]", TRIMKV_PAGED_MAX_PAGES);
    if (max_tokens < 0 || max_tokens > (1LL << 30)) return refuse(TRIMKV_E_ARG, "max_tokens must be in [0, 2^30]");
    if (!old_lens || !new_lens || !block_table || !free_pages || !free_count || !free_count_out || !lens_out || !cu_new || (max_tokens > 0 && !slot_map))
        return refuse(TRIMKV_E_ARG, "NULL buffer");
    if (!ok4(old_lens) || !ok4(keep_lens) || !ok4(new_lens) || !ok4(block_table) || !ok4(free_pages) || !ok4(free_count) || !ok4(free_count_out) ||
        !ok4(lens_out) || !ok4(cu_new) || !ok4(status) || !ok16(slot_map) || !ok16(positions))
        return refuse(TRIMKV_E_ARG, "misaligned buffer (slot_map and positions 16 B, the others 4 B)");
    return done(launch_paged_plan(n_req, old_lens, keep_lens, new_lens, block_table, table_width, free_pages, n_pages, free_count, free_count_out,
                                  (int)max_tokens, lens_out, cu_new, slot_map, positions, status, (cudaStream_t)stream),
                "plan");
}

trimkv_status trimkv_paged_append(const trimkv_paged_cache* cache, int64_t n_tokens, const void* k, int64_t k_stride, const void* v,
                                  int64_t v_stride, const int32_t* slot_map, int32_t* status, void* stream) {
    PagedView pv;
    const trimkv_status s = check_cache(cache, &pv);
    if (s != TRIMKV_OK) return s;
    if (n_tokens < 0 || n_tokens * pv.H > (1LL << 30)) return refuse(TRIMKV_E_ARG, "n_tokens x kv_heads must be in [0, 2^30]");
    if (n_tokens == 0) return TRIMKV_OK;
    const int is_bf16 = cache->kv_dtype == TRIMKV_DTYPE_BF16, elt = is_bf16 ? 2 : 4;
    if (!k || !v || !slot_map || !ok16(k) || !ok16(v) || !ok4(slot_map) || !ok4(status)) return refuse(TRIMKV_E_ARG, "k, v and slot_map must be non-NULL; k and v 16-byte aligned");
    const int64_t row = (int64_t)pv.H * pv.d;
    if (k_stride < row || v_stride < row || k_stride > (1LL << 31) || v_stride > (1LL << 31) || (k_stride * elt) % 16 || (v_stride * elt) % 16)
        return refuse(TRIMKV_E_ARG, "k_stride and v_stride must cover a token's row and be multiples of 16 bytes");
    return done(launch_paged_append(pv, (char*)cache->k_pages, (char*)cache->v_pages, (char*)cache->key_bounds, is_bf16, (int)n_tokens, k, k_stride, v,
                                    v_stride, slot_map, status, (cudaStream_t)stream),
                "append");
}

size_t trimkv_paged_workspace_bytes(int32_t q_heads, int32_t kv_heads, int32_t head_dim) {
    if (kv_heads < 1 || q_heads < kv_heads || q_heads % kv_heads || head_dim < 8 || head_dim > 256 || head_dim % 8 || q_heads / kv_heads > 128) return 0;
    return work_bytes(head_dim);
}

trimkv_status trimkv_paged_attention(const trimkv_paged_cache* cache, int32_t n_req, int64_t n_tokens, int32_t max_new, int32_t q_heads,
                                     const void* q, int64_t q_stride, const int32_t* cu_new, const int32_t* lens,
                                     const int32_t* block_table, int32_t table_width, float scale, int32_t window, void* out,
                                     void* workspace, size_t workspace_bytes, int32_t* status, void* stream) {
    PagedView pv;
    PagedBatch pb;
    trimkv_status s = check_cache(cache, &pv);
    if (s != TRIMKV_OK) return s;
    const int is_bf16 = cache->kv_dtype == TRIMKV_DTYPE_BF16;
    s = check_batch(pv, is_bf16, n_req, n_tokens, q_heads, q, q_stride, cu_new, lens, block_table, table_width, scale, out, workspace, workspace_bytes, status, &pb);
    if (s != TRIMKV_OK) return s;
    if (window < 0 || window > (1 << 30)) return refuse(TRIMKV_E_ARG, "window must be in [0, 2^30]");
    if (max_new < 0) return refuse(TRIMKV_E_ARG, "max_new must not be negative");
    if (n_tokens == 0) return TRIMKV_OK;
    pb.window = window;
    const cudaStream_t st = (cudaStream_t)stream;
    const PagedWork w = carve(workspace, FIRST_ROWS, pv.d);
    if (!is_bf16) return done(launch_paged_attention_f32(pv, pb, q, out, scale, w, st), "attention");
    // Requests of up to 64 rows (tokens x query heads of a KV head) stream through the warp kernel, larger ones go to the
    // tcgen05 kernel; of a batch with both, those of up to 32.  max_new may be wrong: every kernel takes any request, and where
    // both run the device sorts them.
    const long long most = (long long)(max_new > 0 ? max_new : n_tokens) * pb.g;
    const bool tc = pv.d <= PAGED_TC_HEAD;
    cudaError_t e = cudaSuccess;
    if (most <= PAGED_WARP_ROWS || !tc) {
        e = launch_paged_attention_warp(pv, pb, q, out, scale, w, most <= 8 ? 8 : most <= 16 ? 16 : most <= 32 ? 32 : 64, INT_MAX, st);
    } else {
        const bool equal = max_new > 0 && n_tokens == (int64_t)n_req * max_new;    // every request has max_new tokens: one kernel
        const PagedWork w2 = carve((char*)workspace + first_area(pv.d), PAGED_SMS * PAGED_TC_ROWS, pv.d);
        e = launch_paged_attention_tc(pv, pb, q, out, scale, w2, equal ? 1 : 33, st);
        if (e == cudaSuccess && !equal) e = launch_paged_attention_warp(pv, pb, q, out, scale, w, 32, 32, st);
    }
    return done(e, "attention");
}

trimkv_status trimkv_paged_sparse_attention(const trimkv_paged_cache* cache, int32_t n_req, int64_t n_tokens, int32_t q_heads, const void* q,
                                            int64_t q_stride, const int32_t* cu_new, const int32_t* lens, const int32_t* block_table,
                                            int32_t table_width, float scale, int32_t top_pages, int32_t sink_pages, int32_t recent_pages,
                                            int32_t* selected, void* out, void* workspace, size_t workspace_bytes, int32_t* status,
                                            void* stream) {
    PagedView pv;
    PagedBatch pb;
    trimkv_status s = check_cache(cache, &pv);
    if (s != TRIMKV_OK) return s;
    const int is_bf16 = cache->kv_dtype == TRIMKV_DTYPE_BF16;
    s = check_batch(pv, is_bf16, n_req, n_tokens, q_heads, q, q_stride, cu_new, lens, block_table, table_width, scale, out, workspace, workspace_bytes, status, &pb);
    if (s != TRIMKV_OK) return s;
    if (!pv.bounds) return refuse(TRIMKV_E_ARG, "the cache has no key_bounds");
    if (sink_pages < 0 || recent_pages < 1 || top_pages > TRIMKV_PAGED_MAX_WIDTH || sink_pages > top_pages || recent_pages > top_pages - sink_pages)
        return refuse(TRIMKV_E_ARG, "sink_pages >= 0, recent_pages >= 1 and sink_pages + recent_pages <= top_pages <= %d are wanted", TRIMKV_PAGED_MAX_WIDTH);
    if (n_tokens == 0) return TRIMKV_OK;
    if (!selected || !ok4(selected)) return refuse(TRIMKV_E_ARG, "selected must be non-NULL and aligned");
    if (paged_select_smem(table_width, pb.g, pv.d, is_bf16) > (size_t)PAGED_SELECT_SMEM)
        return refuse(TRIMKV_E_UNSUPPORTED, "%d query heads per KV head of %d and a table of %d pages do not fit the selection's shared memory", pb.g, pv.d, table_width);
    pb.top = top_pages;
    pb.sink = sink_pages;
    pb.recent = recent_pages;
    pb.selected = selected;
    s = done(launch_paged_select(pv, pb, is_bf16, q, selected, (cudaStream_t)stream), "page selection");
    if (s != TRIMKV_OK) return s;
    const cudaStream_t st = (cudaStream_t)stream;
    const PagedWork w = carve(workspace, FIRST_ROWS, pv.d);
    cudaError_t e = cudaSuccess;
    // a token's g rows are one unit, or several of the most rows that the kernel holds
    const int most = is_bf16 ? (pv.d > 128 ? 32 : PAGED_WARP_ROWS) : PAGED_F32_ROWS;
    pb.sub_rows = pb.g < most ? pb.g : most;
    pb.sub = (pb.g + pb.sub_rows - 1) / pb.sub_rows;
    pb.by_sub = FastDiv::by(pb.sub);
    if (is_bf16) {
        // A token that reads its own pages costs 2.7 ns a page and KV head (out of L2; up to 4.5 from HBM), a unit that walks the union of its
        // tokens' pages 4 ns for each page up to the request's last, and 30 us a call to begin with, of which every token bears its part:
        // a request walks the union while its pages are at most pick_pages.  (Fitted to 172 calls: one or two requests of 16 to 512
        // tokens over 32 to 1024 pages, 1 to 16 query heads per KV head, 8 to 48 pages each, queries independent or alike.  It takes the
        // faster way or one at most 15 % slower, 1 % on average.  2 x 512 tokens, 8 x 4 heads, top 32, over 256 pages: 411 us, token by token 827;
        // 2 x 128 tokens, 2 x 8 heads, over 1024 pages: 173, token by token 111.)
        const long long OWN = 27, UNION = 40, START = 300000;            // tenths of a nanosecond
        const long long heads = n_tokens * pv.H, gain = heads * std::min(top_pages, table_width) * OWN - START;
        const bool forced = (global_test_hooks() & TRIMKV_TEST_UNION_OF_PAGES) != 0;
        // The union needs a bit per token of the unit and page, and room for its list.
        const int unit_tokens = PAGED_TC_ROWS / pb.g + 2 + 1;            // and the union's own row of bits
        const long long fit = std::min<long long>(PAGED_PICK_PAGES, 32LL * (PAGED_PICK_WORDS / unit_tokens - 1));
        pb.pick_pages = (int)(forced ? fit : std::min(fit, gain > 0 ? gain * PAGED_TC_ROWS / (heads * UNION * pb.g) : 0LL));
        // The host sees no lengths.  Some request surely may have PAGED_PICK_ROWS rows if the tokens leave it that many beside one for each
        // other request.  Fewer tokens may be a decode step, where the union's kernel finds nothing to do (7 us), or a chunk among requests
        // without new tokens: it is launched where that is two hundredths of the call (256 single tokens over 2048 entries each 345 to 352 us,
        // over 8192 408 to 417; 200 tokens of one of 256 requests 152 to 63, 197 to 124), not where it is ten (64 single tokens 92 to
        // 100; 64 tokens of one of 64 requests would go from 60 to 39 us, over 8192 entries from 76 to 77).
        const long long DOUBT = 1300000;
        const bool likely = (n_tokens - n_req + 1) * pb.g >= PAGED_PICK_ROWS || (gain >= DOUBT - START && n_tokens * pb.g >= PAGED_PICK_ROWS);
        const bool walk = pv.d <= PAGED_TC_HEAD && pb.pick_pages > 0 && likely;
        if (walk) {
            PagedBatch pu = pb;
            pu.top = 0;
            pu.pick = 1;
            pu.pick_top = top_pages;
            const PagedWork w2 = carve((char*)workspace + first_area(pv.d), PAGED_SMS * PAGED_TC_ROWS, pv.d);
            e = launch_paged_attention_tc(pv, pu, q, out, scale, w2, 1, st);
            pb.pick = -1;
        }
        if (e == cudaSuccess)
            e = launch_paged_attention_warp(pv, pb, q, out, scale, w, pb.g <= 8 ? 8 : pb.g <= 16 ? 16 : pb.g <= 32 ? 32 : 64, INT_MAX, st);
    } else
        e = launch_paged_attention_f32(pv, pb, q, out, scale, w, st);
    return done(e, "attention");
}

}  // extern "C"
