// C entry points of the paged cache held in 4 bits: argument checks, workspace layout, choice of kernels.
#include <limits.h>

#include "paged4.cuh"
#include "paged_check.cuh"

using namespace tkv;

namespace {

trimkv_status check_cache4(const trimkv_paged4_cache* c, int32_t dtype, Paged4View* v) {
    if (!c || !c->k_codes || !c->k_scales || !c->v_codes || !c->v_scales) return refuse(TRIMKV_E_ARG, "cache, codes and scales must not be NULL");
    if (c->reserved != 0) return refuse(TRIMKV_E_ARG, "reserved must be 0");
    if (dtype != TRIMKV_DTYPE_BF16 && dtype != TRIMKV_DTYPE_F32) return refuse(TRIMKV_E_ARG, "unknown dtype %d", dtype);
    if (c->page_size != PAGE) return refuse(TRIMKV_E_UNSUPPORTED, "page_size must be %d", PAGE);
    if (c->n_pages < 1 || c->n_pages > TRIMKV_PAGED_MAX_PAGES) return refuse(TRIMKV_E_ARG, "n_pages must be in [1, %d]", TRIMKV_PAGED_MAX_PAGES);
    if (c->kv_heads < 1 || c->kv_heads > 1024) return refuse(TRIMKV_E_ARG, "kv_heads must be in [1, 1024]");
    if (c->head_dim < 32 || c->head_dim % 32 || c->head_dim > 256) return refuse(TRIMKV_E_UNSUPPORTED, "head_dim must be a multiple of 32 up to 256");
    if ((long long)c->n_pages * c->kv_heads * PAGE > INT_MAX) return refuse(TRIMKV_E_UNSUPPORTED, "n_pages x kv_heads x %d must be below 2^31", PAGE);
    if (!ok16(c->k_codes) || !ok16(c->k_scales) || !ok16(c->v_codes) || !ok16(c->v_scales)) return refuse(TRIMKV_E_ARG, "codes and scales must be 16-byte aligned");
    if (!ok4(c->k_shift) || !ok4(c->v_shift)) return refuse(TRIMKV_E_ARG, "shifts must be 4-byte aligned");
    *v = Paged4View{};
    v->pv.n_pages = c->n_pages;
    v->pv.H = c->kv_heads;
    v->pv.d = c->head_dim;
    v->codes[0] = (const uint8_t*)c->k_codes;
    v->codes[1] = (const uint8_t*)c->v_codes;
    v->scales[0] = (const uint8_t*)c->k_scales;
    v->scales[1] = (const uint8_t*)c->v_scales;
    v->shift[0] = c->k_shift;
    v->shift[1] = c->v_shift;
    return TRIMKV_OK;
}

// Workspace: {shared units, partial results} of the warp kernel, then of the tensor-core kernel, where the head size has one.
size_t first_bytes4(int d) { return P4_SHARED_BYTES + paged_partial_bytes(P4_WORKER_ROWS, d); }
size_t work_bytes4(int d) { return first_bytes4(d) + (d <= PAGED_TC_HEAD ? PAGED_SHARED_BYTES + paged_partial_bytes(PAGED_SMS * PAGED_TC_ROWS, d) : 0); }
PagedWork carve4(void* area, size_t shared_bytes, int rows, int d) {
    PagedWork w;
    w.shared = (int4*)area;
    w.part_o = (float*)((char*)area + shared_bytes);
    w.part_ml = w.part_o + (size_t)2 * rows * d;
    return w;
}

}  // namespace

extern "C" {

trimkv_status trimkv_paged4_append(const trimkv_paged4_cache* cache, int32_t dtype, int64_t n_tokens, const void* k, int64_t k_stride, const void* v,
                                   int64_t v_stride, const int32_t* slot_map, int32_t* status, void* stream) {
    Paged4View c;
    const trimkv_status s = check_cache4(cache, dtype, &c);
    if (s != TRIMKV_OK) return s;
    if (n_tokens < 0 || n_tokens > (1LL << 30) / c.pv.H) return refuse(TRIMKV_E_ARG, "n_tokens x kv_heads must be in [0, 2^30]");
    if (n_tokens == 0) return TRIMKV_OK;
    const int elt = dtype == TRIMKV_DTYPE_BF16 ? 2 : 4;
    if (!k || !v || !slot_map || !ok16(k) || !ok16(v) || !ok4(slot_map) || !ok4(status)) return refuse(TRIMKV_E_ARG, "k, v and slot_map must be non-NULL; k and v 16-byte aligned");
    const int64_t row = (int64_t)c.pv.H * c.pv.d;
    if (k_stride < row || v_stride < row || k_stride > (1LL << 31) || v_stride > (1LL << 31) || (k_stride * elt) % 16 || (v_stride * elt) % 16)
        return refuse(TRIMKV_E_ARG, "k_stride and v_stride must cover a token's row and be multiples of 16 bytes");
    return done(launch_paged4_append(c, elt == 2, (int)n_tokens, k, k_stride, v, v_stride, slot_map, status, (cudaStream_t)stream), "append");
}

trimkv_status trimkv_paged4_read(const trimkv_paged4_cache* cache, int32_t dtype, int64_t n_slots, const int32_t* slot_map, void* k, void* v, int32_t* status,
                                 void* stream) {
    Paged4View c;
    const trimkv_status s = check_cache4(cache, dtype, &c);
    if (s != TRIMKV_OK) return s;
    if (n_slots < 0 || n_slots > (1LL << 30) / c.pv.H) return refuse(TRIMKV_E_ARG, "n_slots x kv_heads must be in [0, 2^30]");
    if (n_slots == 0) return TRIMKV_OK;
    if (!k || !v || !slot_map || !ok16(k) || !ok16(v) || !ok4(slot_map) || !ok4(status)) return refuse(TRIMKV_E_ARG, "k, v and slot_map must be non-NULL; k and v 16-byte aligned");
    return done(launch_paged4_read(c, dtype == TRIMKV_DTYPE_BF16, (int)n_slots, slot_map, k, v, status, (cudaStream_t)stream), "read");
}

size_t trimkv_paged4_workspace_bytes(int32_t q_heads, int32_t kv_heads, int32_t head_dim) {
    if (kv_heads < 1 || q_heads < kv_heads || q_heads % kv_heads || head_dim < 32 || head_dim > 256 || head_dim % 32 || q_heads / kv_heads > 128) return 0;
    return work_bytes4(head_dim);
}

trimkv_status trimkv_paged4_attention(const trimkv_paged4_cache* cache, int32_t dtype, int32_t n_req, int64_t n_tokens, int32_t max_new, int32_t q_heads,
                                      const void* q, int64_t q_stride, const int32_t* cu_new, const int32_t* lens, const int32_t* block_table,
                                      int32_t table_width, float scale, int32_t window, void* out, void* workspace, size_t workspace_bytes,
                                      int32_t* status, void* stream) {
    Paged4View c;
    PagedBatch pb;
    trimkv_status s = check_cache4(cache, dtype, &c);
    if (s != TRIMKV_OK) return s;
    const int is_bf16 = dtype == TRIMKV_DTYPE_BF16;
    s = paged_check_batch(c.pv, is_bf16, work_bytes4(c.pv.d), n_req, n_tokens, q_heads, q, q_stride, cu_new, lens, block_table, table_width, scale, out, workspace,
                          workspace_bytes, status, &pb);
    if (s != TRIMKV_OK) return s;
    if (window < 0 || window > (1 << 30)) return refuse(TRIMKV_E_ARG, "window must be in [0, 2^30]");
    if (max_new < 0) return refuse(TRIMKV_E_ARG, "max_new must not be negative");
    if (n_tokens == 0) return TRIMKV_OK;
    pb.window = window;
    const cudaStream_t st = (cudaStream_t)stream;
    const PagedWork w = carve4(workspace, P4_SHARED_BYTES, P4_WORKER_ROWS, c.pv.d);
    // Requests of up to 32 rows (tokens x query heads of a KV head) go to the warp kernel, larger ones to the tcgen05 kernel, where there is
    // one.  The warp kernel's time grows with every 16 rows, the other's stays to 128; where they cross depends on the lengths, which the host does
    // not see.  Warp kernel against tcgen05 at 32, 48 and 64 rows, us:
    //   32 requests over 2.3 K entries, 8 KV heads of 128    68, 90, 128    110, 111, 113
    //   8 over 16 K, 8 of 128                               103, 142, 181    153, 154, 155
    //   1 over 32 K, 8 of 128                                54, 61, 69       60, 61, 61
    //   4 over 16 K, 8 of 64                                 44, 54, 66       77, 78, 78
    //   16 over 1 K, 2 of 128 (a unit's pages to one warp)   42, 42, 42       22, 23, 23
    // So 33 to 48 rows lose up to 24 us (a quarter, with heads of 64 a third) over many long requests, and 9 to 32 rows 20 us over few short ones.
    // max_new may be wrong: every kernel takes any request, and where both run the device sorts them.
    const long long most = (long long)(max_new > 0 ? max_new : n_tokens) * pb.g;
    const int tile = most <= 8 || (c.pv.d > PAGED_TC_HEAD && most <= PAGED_WARP_ROWS) ? 8 : 16;
    cudaError_t e = cudaSuccess;
    if (most <= 32 || !is_bf16 || c.pv.d > PAGED_TC_HEAD) {
        e = launch_paged4_attention_warp(c, pb, is_bf16, q, out, scale, w, tile, INT_MAX, st);
    } else {
        const bool equal = max_new > 0 && n_tokens == (int64_t)n_req * max_new;    // every request has max_new tokens: one kernel
        const PagedWork w2 = carve4((char*)workspace + first_bytes4(c.pv.d), PAGED_SHARED_BYTES, PAGED_SMS * PAGED_TC_ROWS, c.pv.d);
        e = launch_paged4_attention_tc(c, pb, q, out, scale, w2, equal ? 1 : 33, st);
        if (e == cudaSuccess && !equal) e = launch_paged4_attention_warp(c, pb, is_bf16, q, out, scale, w, tile, 32, st);
    }
    return done(e, "attention");
}

}  // extern "C"
