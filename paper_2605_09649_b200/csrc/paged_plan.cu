// Block tables and slot maps of the caller-owned paged cache, from request lengths, and the append that follows a slot map.
//
// Plan.  Request r goes from ceil(old / 64) to ceil(new / 64) pages; tokens keep .. new - 1 are the call's new ones.  Pages
// given back are pushed on the free stack in (request, page) order, then the missing ones are popped in (request, page)
// order, so the result is a pure function of the inputs: three prefix sums over the requests (tokens, pages taken, pages
// given back) place everything.  One cluster of 16 CTAs does it in one launch: every CTA computes the sums for itself from
// shared memory (3 x R words), the cluster barrier separates the last read of an input from the first write (inputs and
// outputs may be the same arrays), and the output is dealt out over all 16384 threads.  Bound by latency: 7.3 us for 64
// requests with one token each (22 KB), whatever the cluster's size; 11.3 us for 256 requests of up to 1024 new tokens (1.6 MB),
// where clusters of 1, 2, 4 and 8 CTAs take 96, 50, 28 and 17 us: each token costs its search in shared memory.
//
// Append.  A copy of k and v rows to their slots, 16 bytes per thread and step; the grid's second half looks
// for tokens that complete a page (slot % 64 = 63) and reduces the page's 64 keys to its channelwise bounds.  Rows of
// the page that this same call writes are read from the call's input, so the halves need not wait for one another.  One
// token for each of 32 requests (8 heads of 128, bf16) takes 2.2 us, the latency of a launch and two dependent reads; 32
// chunks of up to 512 move 106 MB in 23.8 us, 0.69 of the measured copy rate: the copy is short, its first and last loads stand
// alone (two or eight rows in flight per thread: 27 and 31 us; 888 to 9472 blocks: 23.4 to 30 us).
#include <cooperative_groups.h>

#include <algorithm>

#include "mma_sync.cuh"
#include "paged.cuh"
#include "paged_bounds.cuh"

namespace tkv {

namespace {

namespace cg = cooperative_groups;

constexpr int PLAN_CTAS = 16, PLAN_THREADS = 1024;

// Last r with at[r] <= x (at ascending, at[0] = 0, x < at[n]).  Empty requests are passed over: their successor has the
// same offset.
__device__ __forceinline__ int plan_find(const int* at, int n, int x) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (at[mid] <= x) lo = mid; else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ int plan_pages(int n) { return (int)(((unsigned)n + PAGE - 1u) / PAGE); }

__global__ void __launch_bounds__(PLAN_THREADS, 1)
paged_plan_kernel(int R, const int32_t* old_lens, const int32_t* keep_lens, const int32_t* new_lens, int32_t* table, int W,
                  int32_t* free_pages, int n_pages, const int32_t* free_count, int32_t* free_count_out, int max_tokens,
                  int32_t* lens_out, int32_t* cu_new, int32_t* slot_map, int32_t* positions, int32_t* status) {
    extern __shared__ int s_plan[];
    int* s_old = s_plan;                      // [R] each
    int* s_keep = s_old + R;
    int* s_new = s_keep + R;
    int* s_tok = s_new + R;                   // [R + 1] each: sums before request r
    int* s_take = s_tok + R + 1;
    int* s_back = s_take + R + 1;
    __shared__ long long w_sum[3][32];
    __shared__ int s_bad;
    cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) s_bad = 0;
    grid_dependency_wait();
    grid_dependents_may_launch();
    __syncthreads();

    // ---- lengths, and their sums: thread i takes the requests [i per, (i + 1) per)
    const int per = (R + PLAN_THREADS - 1) / PLAN_THREADS;
    const int r0 = min(R, tid * per), r1 = min(R, r0 + per);
    long long mine[3] = {0, 0, 0};
    for (int r = r0; r < r1; ++r) {
        const int o = old_lens[r], n = new_lens[r], k = keep_lens ? keep_lens[r] : min(o, n);
        s_old[r] = o; s_new[r] = n; s_keep[r] = k;
        const long long cap = (long long)W * PAGE;
        if (o < 0 || n < 0 || k < 0 || k > o || k > n || o > cap || n > cap) { s_bad = TRIMKV_E_ARG; continue; }
        const int diff = plan_pages(n) - plan_pages(o);
        mine[0] += n - k;
        mine[1] += max(diff, 0);
        mine[2] += max(-diff, 0);
    }
    long long incl[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        incl[i] = mine[i];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(0xffffffffu, incl[i], o);
            if (lane >= o) incl[i] += v;
        }
        if (lane == 31) w_sum[i][warp] = incl[i];
    }
    __syncthreads();
    if (warp < 3) {
        long long v = w_sum[warp][lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long u = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v += u;
        }
        w_sum[warp][lane] = v;
    }
    __syncthreads();
    const long long tokens = w_sum[0][31], taken = w_sum[1][31], back = w_sum[2][31];
    const int fc = *free_count;
    int bad = s_bad;
    if (!bad && (fc < 0 || fc + back > n_pages || tokens > max_tokens)) bad = TRIMKV_E_ARG;
    if (!bad && fc + back < taken) bad = TRIMKV_E_NOMEM;
    if (!bad) {
        long long at[3];
#pragma unroll
        for (int i = 0; i < 3; ++i) at[i] = (warp ? w_sum[i][warp - 1] : 0) + incl[i] - mine[i];
        for (int r = r0; r < r1; ++r) {
            s_tok[r] = (int)at[0]; s_take[r] = (int)at[1]; s_back[r] = (int)at[2];
            const int diff = plan_pages(s_new[r]) - plan_pages(s_old[r]);
            at[0] += s_new[r] - s_keep[r];
            at[1] += max(diff, 0);
            at[2] += max(-diff, 0);
        }
        if (tid == 0) { s_tok[R] = (int)tokens; s_take[R] = (int)taken; s_back[R] = (int)back; }
    }
    __syncthreads();
    cluster.sync();                           // every input length and the free count have been read

    const int gt = (int)cluster.block_rank() * PLAN_THREADS + tid, GT = PLAN_CTAS * PLAN_THREADS;
    if (bad) {                                // nothing changes hands; the call's tokens are none
        for (int r = gt; r <= R; r += GT) {
            cu_new[r] = 0;
            if (r < R) lens_out[r] = s_old[r];
        }
        for (int i = gt; i < max_tokens; i += GT) { slot_map[i] = -1; if (positions) positions[i] = -1; }
        if (gt == 0) { *free_count_out = fc; latch_error(status, bad); }
        return;
    }
    for (int r = gt; r <= R; r += GT) {
        cu_new[r] = s_tok[r];
        if (r < R) lens_out[r] = s_new[r];
    }
    if (gt == 0) *free_count_out = fc + (int)back - (int)taken;
    auto given_back = [&](int i) {            // i-th page given back
        const int r = plan_find(s_back, R, i);
        return table[(size_t)r * W + plan_pages(s_new[r]) + (i - s_back[r])];
    };
    auto taken_page = [&](int i) {            // i-th page taken; -1 where the free list or the table holds no page
        const int s = fc + (int)back - 1 - i;
        const int p = s >= fc ? given_back(s - fc) : free_pages[s];
        return (p >= 0 && p < n_pages) ? p : -1;
    };
    bool wrong = false;
    for (int i = gt; i < (int)back; i += GT) {    // (a table entry that is no page keeps its place on the stack, as -1)
        const int p = given_back(i);
        free_pages[fc + i] = p >= 0 && p < n_pages ? p : -1;
        wrong |= p < 0 || p >= n_pages;
    }
    for (int i = gt; i < (int)taken; i += GT) {
        const int r = plan_find(s_take, R, i), p = taken_page(i);
        table[(size_t)r * W + plan_pages(s_old[r]) + (i - s_take[r])] = p;
        wrong |= p < 0;
    }
    // four consecutive tokens per thread: one search, one 16-byte store each
    for (long long i0 = 4LL * gt; i0 < max_tokens; i0 += 4LL * GT) {
        int slot[4], pos[4];
        int r = i0 < tokens ? plan_find(s_tok, R, (int)i0) : R;
        int page_of = -1, page = -1;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = (int)i0 + e;
            slot[e] = pos[e] = -1;
            if (i0 + e >= tokens) continue;
            if (i >= s_tok[r + 1]) { r = plan_find(s_tok, R, i); page_of = -1; }
            const int p = s_keep[r] + (i - s_tok[r]), lp = p / PAGE;
            if (page_of != lp) {
                const int had = plan_pages(s_old[r]);
                page_of = lp;
                page = lp < had ? table[(size_t)r * W + lp] : taken_page(s_take[r] + lp - had);
                if (page < 0 || page >= n_pages) { page = -1; wrong = true; }
            }
            pos[e] = p;
            slot[e] = page < 0 ? -1 : page * PAGE + p % PAGE;
        }
        if (i0 + 4 <= max_tokens) {           // the arrays are 16-byte aligned
            *reinterpret_cast<int4*>(slot_map + i0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
            if (positions) *reinterpret_cast<int4*>(positions + i0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
        } else {
            for (int e = 0; e < 4 && i0 + e < max_tokens; ++e) {
                slot_map[i0 + e] = slot[e];
                if (positions) positions[i0 + e] = pos[e];
            }
        }
    }
    if (wrong) latch_error(status, TRIMKV_E_ARG);
}

// ---------------------------------------------------------------- append
constexpr int APP_THREADS = 256, APP_UNROLL = 4;

// Blocks [0, copy_blocks) copy rows: 16-byte chunk c of the T x H x (d * elt / 16) chunks of k, and the same of v.  The
// others take `group` tokens of one head each and reduce the pages that these tokens complete, eight rows per warp.
template <typename T>
__global__ void __launch_bounds__(APP_THREADS)
paged_append_kernel(char* k_pages, char* v_pages, char* bounds, int n_pages, int H, int d, int T_rows, const char* k, long long k_stride,
                    const char* v, long long v_stride, const int32_t* slot_map, int32_t* status, int copy_blocks, int group) {
    constexpr int WARPS = APP_THREADS / 32;
    __shared__ uint4 s_part[2][WARPS][16];
    const int rb = d * (int)sizeof(T), cpr = rb / 16;         // bytes, 16-byte chunks per row
    const int slots = n_pages * PAGE;
    grid_dependency_wait();
    grid_dependents_may_launch();
    if ((int)blockIdx.x < copy_blocks) {
        const unsigned per_tok = (unsigned)(H * cpr);
        const long long n = (long long)T_rows * per_tok;
        const long long step = (long long)copy_blocks * APP_THREADS;
        for (long long c0 = (long long)blockIdx.x * APP_THREADS + threadIdx.x; c0 < n; c0 += APP_UNROLL * step) {
            int s[APP_UNROLL];
            unsigned tok[APP_UNROLL], rest[APP_UNROLL];
#pragma unroll
            for (int u = 0; u < APP_UNROLL; ++u) {
                const long long c = c0 + u * step;
                tok[u] = n < (1LL << 32) ? (unsigned)c / per_tok : (unsigned)(c / per_tok);
                rest[u] = (unsigned)(c - (long long)tok[u] * per_tok);
                s[u] = c < n ? slot_map[tok[u]] : -1;
            }
            uint4 kv[APP_UNROLL], vv[APP_UNROLL];
#pragma unroll
            for (int u = 0; u < APP_UNROLL; ++u) {            // all loads in flight before the first store
                if (s[u] < 0 || s[u] >= slots) {
                    if (s[u] != -1 && rest[u] == 0) latch_error(status, TRIMKV_E_ARG);
                    s[u] = -1;
                    continue;
                }
                kv[u] = *reinterpret_cast<const uint4*>(k + ((size_t)tok[u] * k_stride) * sizeof(T) + (size_t)rest[u] * 16);
                vv[u] = *reinterpret_cast<const uint4*>(v + ((size_t)tok[u] * v_stride) * sizeof(T) + (size_t)rest[u] * 16);
            }
#pragma unroll
            for (int u = 0; u < APP_UNROLL; ++u)
                if (s[u] >= 0) {
                    const unsigned h = rest[u] / (unsigned)cpr, ch = rest[u] - h * cpr;
                    const size_t dst = (((size_t)(s[u] / PAGE) * H + h) * PAGE + s[u] % PAGE) * rb + (size_t)ch * 16;
                    *reinterpret_cast<uint4*>(k_pages + dst) = kv[u];
                    *reinterpret_cast<uint4*>(v_pages + dst) = vv[u];
                }
        }
        return;
    }
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int item = (int)blockIdx.x - copy_blocks, h = item % H;
    const long long t_first = (long long)(item / H) * group;
    for (int g0 = 0; g0 < group && t_first + g0 < T_rows; g0 += 32) {
        const int t0 = (int)t_first + g0;
        const int my_slot = g0 + lane < group && t0 + lane < T_rows ? slot_map[t0 + lane] : -1;
        unsigned full = __ballot_sync(0xffffffffu, my_slot >= 0 && my_slot < slots && my_slot % PAGE == PAGE - 1);
        while (full) {                                        // the same for every warp of the block
            const int b = __ffs(full) - 1, t = t0 + b;
            full &= full - 1;
            const int s = __shfl_sync(0xffffffffu, my_slot, b), page = s / PAGE;
            // row i of the page is this call's token t - 63 + i if that token was given the row's slot
            const int my_row = warp * 8 + (lane & 7), my_tok = t - (PAGE - 1) + my_row;
            const unsigned here = __ballot_sync(0xffffffffu, my_tok >= 0 && slot_map[max(my_tok, 0)] == page * PAGE + my_row);
            const char* page_rows = k_pages + ((size_t)page * H + h) * PAGE * (size_t)rb;
            char* out = bounds + ((size_t)page * H + h) * 2 * rb;
            for (int c0 = 0; c0 < cpr; c0 += 16) {            // half a warp per row, four rows each
                const int ch = c0 + (lane & 15), half = lane >> 4;
                const bool on = ch < cpr;
                uint4 val[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int i = 2 * j + half, row = warp * 8 + i;
                    const char* src = (here >> i) & 1u ? k + ((size_t)(t - (PAGE - 1) + row) * k_stride) * sizeof(T) + (size_t)h * rb
                                                       : page_rows + (size_t)row * rb;
                    val[j] = on ? *reinterpret_cast<const uint4*>(src + (size_t)ch * 16) : make_uint4(0u, 0u, 0u, 0u);
                }
                MinMax16<T> mm;
                mm.start(val[0]);
#pragma unroll
                for (int j = 1; j < 4; ++j) mm.add(val[j]);
                uint4 lo = *reinterpret_cast<uint4*>(mm.lo), hi = *reinterpret_cast<uint4*>(mm.hi), olo, ohi;
                olo.x = __shfl_xor_sync(0xffffffffu, lo.x, 16); olo.y = __shfl_xor_sync(0xffffffffu, lo.y, 16);
                olo.z = __shfl_xor_sync(0xffffffffu, lo.z, 16); olo.w = __shfl_xor_sync(0xffffffffu, lo.w, 16);
                ohi.x = __shfl_xor_sync(0xffffffffu, hi.x, 16); ohi.y = __shfl_xor_sync(0xffffffffu, hi.y, 16);
                ohi.z = __shfl_xor_sync(0xffffffffu, hi.z, 16); ohi.w = __shfl_xor_sync(0xffffffffu, hi.w, 16);
                mm.join(olo, ohi);
                if (half == 0) {
                    s_part[0][warp][lane] = *reinterpret_cast<uint4*>(mm.lo);
                    s_part[1][warp][lane] = *reinterpret_cast<uint4*>(mm.hi);
                }
                __syncthreads();
                if (warp == 0 && half == 0 && on) {
                    for (int x = 1; x < WARPS; ++x) mm.join(s_part[0][x][lane], s_part[1][x][lane]);
                    *reinterpret_cast<uint4*>(out + (size_t)ch * 16) = *reinterpret_cast<uint4*>(mm.lo);
                    *reinterpret_cast<uint4*>(out + rb + (size_t)ch * 16) = *reinterpret_cast<uint4*>(mm.hi);
                }
                __syncthreads();
            }
        }
    }
}

}  // namespace

cudaError_t launch_paged_plan(int R, const int32_t* old_lens, const int32_t* keep_lens, const int32_t* new_lens, int32_t* table,
                              int W, int32_t* free_pages, int n_pages, const int32_t* free_count, int32_t* free_count_out,
                              int max_tokens, int32_t* lens_out, int32_t* cu_new, int32_t* slot_map, int32_t* positions,
                              int32_t* status, cudaStream_t st) {
    const size_t smem = ((size_t)6 * R + 3) * sizeof(int);
    static std::atomic<unsigned long long> done{0};
    const cudaError_t e = paged_allow_smem(reinterpret_cast<const void*>(paged_plan_kernel),
                                           (int)(((size_t)6 * PAGED_MAX_REQ + 3) * sizeof(int)), done, true);
    if (e != cudaSuccess) return e;
    return paged_launch(paged_plan_kernel, dim3(PLAN_CTAS), dim3(PLAN_THREADS), smem, PLAN_CTAS, true, st, R, old_lens, keep_lens, new_lens,
                        table, W, free_pages, n_pages, free_count, free_count_out, max_tokens, lens_out, cu_new, slot_map, positions, status);
}

cudaError_t launch_paged_append(const PagedView& pv, char* k_pages, char* v_pages, char* bounds, int is_bf16, int T, const void* k,
                                long long k_stride, const void* v, long long v_stride, const int32_t* slot_map, int32_t* status,
                                cudaStream_t st) {
    const long long chunks = (long long)T * pv.H * (pv.d * (is_bf16 ? 2 : 4) / 16);
    // one chunk per thread while that leaves the GPU unfilled, then up to APP_UNROLL per thread
    long long copy_blocks = (chunks + APP_THREADS - 1) / APP_THREADS;
    if (copy_blocks > PAGED_SMS * 8) copy_blocks = std::max<long long>(PAGED_SMS * 8, std::min<long long>(PAGED_SMS * 64, (copy_blocks + APP_UNROLL - 1) / APP_UNROLL));
    // tokens per reducing block: few, so that the pages of a decode step (each token may complete one) are reduced side by
    // side; a prompt completes one page in 64 tokens
    int group = 1;
    while (group < 64 && (long long)((T + group - 1) / group) * pv.H > PAGED_SMS * 8) group *= 2;
    const long long items = bounds ? (long long)((T + group - 1) / group) * pv.H : 0;
    const unsigned blocks = (unsigned)(copy_blocks + items);
    auto go = [&](auto kernel) {
        return paged_launch(kernel, dim3(blocks), dim3(APP_THREADS), 0, 1, true, st, k_pages, v_pages, bounds, pv.n_pages, pv.H, pv.d, T, (const char*)k, k_stride,
                            (const char*)v, v_stride, slot_map, status, (int)copy_blocks, group);
    };
    return is_bf16 ? go(paged_append_kernel<__nv_bfloat16>) : go(paged_append_kernel<float>);
}

}  // namespace tkv
