// The caller-owned paged cache: views, work split and launchers shared by the paged kernels.  Not part of the public ABI.
//
// Pages hold 64 entries of every KV head: k_pages, v_pages [n_pages][H][64][d].  A request's entries 0 .. len-1 lie in the
// pages of its block-table row, in order.  The n new tokens of request r are rows cu_new[r] .. cu_new[r+1]-1 of q and out;
// new token j stands at position len - n + j and sees the entries up to it.
#pragma once

#include <limits.h>

#include <cuda.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "trimkv_internal.cuh"

namespace tkv {

// Opts the kernel in to `bytes` of dynamic shared memory on the current device, once per device.  The bit is set after the
// call has succeeded, so a thread that finds it set may launch; two threads that race both make the call.
inline cudaError_t paged_allow_smem(const void* kernel, int bytes, std::atomic<unsigned long long>& done, bool wide_cluster = false) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const unsigned long long bit = dev < 64 ? 1ull << dev : 0;
    if (bit & done.load(std::memory_order_acquire)) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && wide_cluster) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_release);
    return e;
}

// Division by a number that the host knows, in three instructions (a division by a variable is thirty, and these kernels'
// short runs are paced by fetching their code): q = (mulhi(n, m) + n) >> s with s = ceil(log2 d), m = floor(2^32 (2^s - d) / d) + 1,
// for 0 <= n < 2^31 (Granlund and Montgomery, Division by Invariant Integers using Multiplication).
struct FastDiv {
    uint32_t m, s, d;
    static FastDiv by(int d) {
        FastDiv f = {1u, 0u, (uint32_t)d};
        while ((1ull << f.s) < (unsigned long long)d) ++f.s;
        f.m = (uint32_t)((((1ull << f.s) - (unsigned long long)d) << 32) / (unsigned long long)d) + 1u;
        return f;
    }
    __device__ __forceinline__ int div(int n) const { return (int)((__umulhi((uint32_t)n, m) + (uint32_t)n) >> s); }
    __device__ __forceinline__ int mod(int n) const { return n - div(n) * (int)d; }
};

struct PagedView {
    const char* k;
    const char* v;
    const char* bounds;       // [n_pages][H][2][d]: channelwise smallest and largest key of a full page; may be null
    int n_pages, H, d;
};

struct PagedBatch {
    const int32_t* cu_new;    // [R + 1]
    const int32_t* lens;      // [R]
    const int32_t* table;     // [R][W]
    int R, W, T;              // requests, table width, rows of q
    int Hq, g;                // query heads, query heads per KV head
    long long q_stride;       // elements from one token's q to the next
    int window;               // > 0: a token sees the last `window` entries up to its own; 0: all of them
    int top, sink, recent;    // page selection (top = 0: every page is read)
    int sub;                  // ... units per token: its g rows in blocks of sub_rows
    int sub_rows;
    const int32_t* selected;  // [T][H][top] pages to read, ascending, -1 behind the last
    // Page selection may run two kernels: pick < 0 marks the one that reads each token's pages for itself (top > 0), pick > 0 the
    // one that walks the union of a unit's tokens' pages (top = 0, the selection's width in pick_top).  A request goes to the
    // second if it has at least PAGED_PICK_ROWS rows and at most pick_pages pages.  0: one kernel takes all requests.
    int pick, pick_top, pick_pages;
    int32_t* status;          // latched status, may be null
    FastDiv by_g, by_h, by_sub;
};

constexpr int PAGED_MAX_REQ = 8192;
constexpr int PAGED_PICK_ROWS = 64;           // see PagedBatch::pick
constexpr int PAGED_PICK_WORDS = 3456;        // shared memory of the union: bits (tokens of a unit x pages / 32)
constexpr int PAGED_PICK_PAGES = 1024;        // ... and its list of pages

// Rows and length of request r; a request whose offsets or length are out of range counts as having no rows.
struct PagedReq { int row0, n, len; };
__device__ __forceinline__ PagedReq paged_checked(const PagedBatch& pb, int row0, int end, int len) {
    PagedReq q;
    q.row0 = row0;
    q.len = len;
    q.n = end - row0;
    if (row0 < 0 || end < row0 || end > pb.T || len < 0 || len > pb.W * (long long)PAGE) {
        latch_error(pb.status, TRIMKV_E_ARG);
        q.row0 = q.n = q.len = 0;
    }
    return q;
}
__device__ __forceinline__ PagedReq paged_request(const PagedBatch& pb, int r) { return paged_checked(pb, pb.cu_new[r], pb.cu_new[r + 1], pb.lens[r]); }

// ---------------------------------------------------------------- work split
// A request has U units per KV head -- blocks of `tile_rows` of its n * g (token, query head) rows, or single tokens when
// pages are selected -- and each unit counts C steps of one page (the most pages any of its units reads; at least 1, so
// that a unit with nothing to read still writes its zeros).  All units of all requests, laid end to end, form one line of
// `total` steps, and worker w of N takes the steps [total w / N, total (w + 1) / N): equal shares whatever the lengths, no
// counters.  A worker's first and last unit may be shared with its neighbours; then it stores a partial result
// (m, l, O) -- slot 2 w for a unit that it did not begin, slot 2 w + 1 for one that it began and did not end -- and a
// second kernel joins the partials.  Where whole units balance about as well (many short ones, or few that are short), a
// worker takes whole units instead and nothing is joined.
struct PagedCost { int U, C; };
// SEL: whether pages are selected, where a kernel knows it (0, 1); -1: the batch says (top > 0).
template <int SEL>
__device__ __forceinline__ bool paged_selects(const PagedBatch& pb) { return SEL < 0 ? pb.top > 0 : SEL != 0; }

template <int SEL>
__device__ __forceinline__ PagedCost paged_cost(const PagedBatch& pb, const PagedReq& q, int tile_rows, int min_rows, int max_rows) {
    PagedCost c;
    const int rows = q.n * pb.g;
    int pages = (q.len + PAGE - 1) / PAGE;
    const bool walks = rows >= PAGED_PICK_ROWS && pages <= pb.pick_pages;
    if (q.n == 0 || rows < min_rows || rows > max_rows || (pb.pick != 0 && walks != (pb.pick > 0))) { c.U = 0; c.C = 1; return c; }
    if (paged_selects<SEL>(pb)) {
        c.U = q.n * pb.sub;
        pages = min(pages, pb.top);
    } else {
        c.U = (rows + tile_rows - 1) / tile_rows;
        if (pb.window > 0) {                              // entries that the tokens of one unit see, spread over pages
            const long long span = (long long)pb.window + min(q.n, pb.by_g.div(tile_rows) + 2);
            pages = (int)min((long long)pages, span / PAGE + 2);
        }
    }
    c.C = max(pages, 1);
    return c;
}

// 64-bit quotients are a long routine; nearly all of them have operands of 32 bits.
__device__ __forceinline__ long long paged_div(long long a, int b) {
    return (unsigned long long)a >> 32 ? a / b : (long long)((unsigned)a / (unsigned)b);
}

// Where the host can tell that every batch of these sizes is dealt out in whole units (paged_choose_whole): a unit for each worker, none
// longer than a join is worth.  Then no join is launched (2.5 us of a short call's host time).
constexpr int PAGED_GROUPS = 480;
inline bool paged_always_whole(const PagedBatch& pb, int H, int tile_rows, int workers, int join_steps) {
    // units of one KV head: whole ones per token, or those that the tokens fill and a last one of each request
    const long long units = pb.top > 0 ? (long long)pb.T * pb.sub
                                       : std::min((long long)pb.T * ((pb.g + tile_rows - 1) / tile_rows), (long long)pb.T * pb.g / tile_rows + pb.R);
    long long longest = pb.top > 0 && pb.top < pb.W ? pb.top : pb.W;
    if (pb.window > 0) longest = std::min(longest, ((long long)pb.window + tile_rows / pb.g + 2) / PAGE + 2);      // as paged_cost
    return pb.R <= PAGED_GROUPS && units * H <= workers && longest <= join_steps;
}

// Shared memory of the table: PAGED_GROUPS groups of consecutive requests, and what each of the block's warps sums up over them.  (A kernel
// has room for its own warps, no more: with 200 bytes too many the fp32 kernel takes 23.8 us instead of 23.3 for a prompt of 512.)
struct PagedTableLine {
    long long grp[PAGED_GROUPS + 1];          // steps before a group
    int4 req[PAGED_GROUPS];                   // {row0, n, len, units} of each request where a group is one request
};
template <int WARPS>
struct PagedTableMemOf : PagedTableLine {
    long long steps[WARPS], units[WARPS];     // of the requests of each warp
    int longest[WARPS], whole;
};
using PagedTableMem = PagedTableMemOf<18>;    // (the tensor-core kernel has 18)
struct PagedTable {
    PagedTableLine* mem;
    int gsz, ngrp, heads;
    int tile_rows, min_rows, max_rows;
    long long total;
    int workers;                              // workers that take part: no share is under min_share steps
    bool whole;                               // the line counts whole units, not steps
    long long quot;                           // total = quot * workers + rem
    int rem;
    // First step of worker w: floor(total w / workers).
    __device__ __forceinline__ long long share(int w) const { return quot * w + (long long)((unsigned)(rem * w) / (unsigned)workers); }
};

__device__ __forceinline__ void paged_finish_table(PagedTable& t, int max_workers, int min_share) {
    t.total = t.mem->grp[t.ngrp];
    t.workers = (int)min((long long)max_workers, t.whole ? t.total : paged_div(t.total + min_share - 1, min_share));
    t.quot = t.workers ? paged_div(t.total, t.workers) : 0;
    t.rem = (int)(t.total - t.quot * t.workers);
}
// steps, units and the longest unit of all requests: do whole units do?
// join_steps: what joining parts costs, in steps of the kernel.
__device__ __forceinline__ bool paged_choose_whole(long long steps, long long units, int longest, int max_workers, int join_steps) {
    return paged_div(units + max_workers - 1, max_workers) * longest <= paged_div(steps, max_workers) + join_steps;
}

// Every thread of the block calls it.
template <int SEL, int WARPS>
__device__ __forceinline__ void paged_build_table(PagedTable& t, const PagedBatch& pb, int heads, int tile_rows, int min_rows,
                                                  int max_rows, int max_workers, int min_share, int join_steps, PagedTableMemOf<WARPS>* mem) {
    t.mem = mem;
    t.heads = heads;
    t.tile_rows = tile_rows; t.min_rows = min_rows; t.max_rows = max_rows;
    if (pb.R <= 32) {                         // by one warp
        t.gsz = 1;
        t.ngrp = pb.R;
        if (threadIdx.x < 32) {
            const int r = threadIdx.x;
            PagedReq q = {0, 0, 0};
            PagedCost c = {0, 1};
            if (r < pb.R) {
                q = paged_request(pb, r);
                c = paged_cost<SEL>(pb, q, tile_rows, min_rows, max_rows);
            }
            const int units = c.U * heads;
            long long all_steps = (long long)units * c.C, all_units = units;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                all_steps += __shfl_xor_sync(0xffffffffu, all_steps, o);
                all_units += __shfl_xor_sync(0xffffffffu, all_units, o);
            }
            const int longest = __reduce_max_sync(0xffffffffu, c.U ? c.C : 0);
            t.whole = paged_choose_whole(all_steps, all_units, longest, max_workers, join_steps);
            const long long mine = t.whole ? units : (long long)units * c.C;
            long long sum = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long v = __shfl_up_sync(0xffffffffu, sum, o);
                if (r >= o) sum += v;
            }
            mem->req[r] = make_int4(q.row0, q.n, q.len, 0);
            mem->grp[r + 1] = sum;
            if (r == 0) { mem->grp[0] = 0; mem->whole = t.whole; }
        }
        __syncthreads();
        t.whole = mem->whole;
        paged_finish_table(t, max_workers, min_share);
        return;
    }
    // a thread takes neighbouring groups; sums over the threads by shuffles and one sum per warp in shared memory
    t.gsz = (pb.R + PAGED_GROUPS - 1) / PAGED_GROUPS;
    t.ngrp = (pb.R + t.gsz - 1) / t.gsz;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    if (t.gsz == 1) {                         // every load in flight at once
        for (int r = threadIdx.x; r < pb.R; r += blockDim.x) mem->req[r] = make_int4(pb.cu_new[r], pb.cu_new[r + 1], pb.lens[r], 0);
        __syncthreads();
    }
    const int per = (t.ngrp + (int)blockDim.x - 1) / (int)blockDim.x;
    const int g0 = min(t.ngrp, (int)threadIdx.x * per), g1 = min(t.ngrp, g0 + per);
    long long my_steps = 0, my_units = 0;
    int my_longest = 0;
    for (int gi = g0; gi < g1; ++gi) {
        long long steps = 0, units = 0;
        for (int r = gi * t.gsz; r < min(pb.R, (gi + 1) * t.gsz); ++r) {
            PagedReq q;
            if (t.gsz == 1) { const int4 v = mem->req[r]; q = paged_checked(pb, v.x, v.y, v.z); } else q = paged_request(pb, r);
            const PagedCost c = paged_cost<SEL>(pb, q, tile_rows, min_rows, max_rows);
            units += c.U * heads;
            steps += (long long)(c.U * heads) * c.C;
            if (c.U) my_longest = max(my_longest, c.C);
            if (t.gsz == 1) mem->req[gi] = make_int4(q.row0, q.n, q.len, (int)units);
        }
        mem->grp[gi + 1] = steps;
        my_steps += steps;
        my_units += units;
    }
    long long steps_to = my_steps, units_to = my_units;           // of the warp's threads up to this one
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long a = __shfl_up_sync(0xffffffffu, steps_to, o), b = __shfl_up_sync(0xffffffffu, units_to, o);
        if (lane >= o) { steps_to += a; units_to += b; }
    }
    my_longest = __reduce_max_sync(0xffffffffu, my_longest);
    if (lane == 31) { mem->steps[warp] = steps_to; mem->units[warp] = units_to; mem->longest[warp] = my_longest; }
    __syncthreads();
    long long steps = 0, units = 0;
    for (int x = 0; x < warps; ++x) {
        if (x == warp) { steps_to += steps; units_to += units; }
        steps += mem->steps[x];
        units += mem->units[x];
        my_longest = max(my_longest, mem->longest[x]);
    }
    // (groups of several requests keep to steps: their units are not kept apart)
    t.whole = t.gsz == 1 && paged_choose_whole(steps, units, my_longest, max_workers, join_steps);
    long long run = t.whole ? units_to - my_units : steps_to - my_steps;
    for (int gi = g0; gi < g1; ++gi) {
        run += t.whole ? (long long)mem->req[gi].w : mem->grp[gi + 1];
        mem->grp[gi + 1] = run;
    }
    if (threadIdx.x == 0) mem->grp[0] = 0;
    __syncthreads();
    paged_finish_table(t, max_workers, min_share);
}

// The worker whose share holds step x, from the line's total and the number of workers.
__device__ __forceinline__ int paged_owner(long long total, int workers, long long x) {
    const long long quot = paged_div(total, workers);
    const int rem = (int)(total - quot * workers);
    auto share = [&](int w) { return quot * w + (long long)((unsigned)(rem * w) / (unsigned)workers); };
    int w = min(workers - 1, (int)((float)x / (float)total * (float)workers));       // near; then exact
    while (w > 0 && share(w) > x) --w;
    while (w + 1 < workers && share(w + 1) <= x) ++w;
    return w;
}

// Order of a request's units on the line: last, first, last but one, second, ...  Later units see more entries, so pairs of
// neighbours cost about the same and equal shares of the line stay equal shares of the work.
__device__ __forceinline__ int paged_fold(int v, int U) { return (v & 1) ? v / 2 : U - 1 - v / 2; }

// First of the request's n * g (token, query head) rows that belong to unit u, and how many do.
template <int SEL>
__device__ __forceinline__ int paged_unit_first(const PagedBatch& pb, int u, int tile_rows) {
    if (!paged_selects<SEL>(pb)) return u * tile_rows;
    const int t = pb.by_sub.div(u);
    return t * pb.g + (u - t * pb.sub) * pb.sub_rows;
}
template <int SEL>
__device__ __forceinline__ int paged_unit_rows(const PagedBatch& pb, int u, int n, int tile_rows) {
    return paged_selects<SEL>(pb) ? min(pb.sub_rows, pb.g - pb.by_sub.mod(u) * pb.sub_rows) : min(tile_rows, n * pb.g - u * tile_rows);
}

// One stretch of a unit, as a worker meets it.
struct PagedItem {
    int r, h, u;            // request, KV head, unit of the request
    PagedReq q;
    int p0, p1;             // first page and one past the last (of the unit's pages, or places in its list of selected pages)
    long long steps;        // steps of the line that it covers
    int slot;               // -1: the whole unit (the result is final); else 2 w or 2 w + 1, see above
    int cost;               // steps of the unit
    int tok0, tok1;         // tokens (of the request) that the unit's rows belong to, tok1 inclusive
};

template <int SEL>
__device__ __forceinline__ PagedItem paged_item(const PagedTable& t, const PagedBatch& pb, long long x, long long end, int w) {
    PagedItem it;
    int lo = 0, hi = t.ngrp - 1;
    while (lo < hi) {                                     // last group that begins at or before x
        const int mid = (lo + hi + 1) >> 1;
        if (t.mem->grp[mid] <= x) lo = mid; else hi = mid - 1;
    }
    long long base = t.mem->grp[lo];
    int r = lo * t.gsz;
    PagedReq q;
    PagedCost c;
    if (t.gsz == 1) {
        const int4 v = t.mem->req[lo];
        q.row0 = v.x; q.n = v.y; q.len = v.z;
        c = paged_cost<SEL>(pb, q, t.tile_rows, t.min_rows, t.max_rows);
    } else {
        for (;; ++r) {
            q = paged_request(pb, r);
            c = paged_cost<SEL>(pb, q, t.tile_rows, t.min_rows, t.max_rows);
            const long long s = (long long)(c.U * t.heads) * c.C;
            if (x < base + s || r + 1 >= pb.R) break;
            base += s;
        }
    }
    const long long off = x - base;
    const int unit = t.whole ? (int)off : (int)paged_div(off, c.C), v0 = t.whole ? 0 : (int)(off - (long long)unit * c.C);
    it.steps = t.whole ? 1 : min((long long)(c.C - v0), end - x);
    const int v1 = t.whole ? c.C : v0 + (int)it.steps;
    it.r = r;
    it.q = q;
    it.cost = c.C;
    it.h = unit / c.U;
    it.u = paged_fold(unit - it.h * c.U, c.U);
    int first, count;                                     // the unit's pages
    if (paged_selects<SEL>(pb)) {
        it.tok0 = it.tok1 = pb.by_sub.div(it.u);
        const int pos = q.len - q.n + it.tok0;
        first = 0;
        count = pos < 0 ? 0 : min(pb.top, pos / PAGE + 1);
    } else {
        it.tok0 = pb.by_g.div(it.u * t.tile_rows);
        it.tok1 = min(q.n - 1, pb.by_g.div((it.u + 1) * t.tile_rows - 1));
        const int plo = q.len - q.n + it.tok0, phi = q.len - q.n + it.tok1;
        first = pb.window > 0 ? max(0, plo - pb.window + 1) / PAGE : 0;
        count = phi < 0 ? 0 : phi / PAGE + 1 - first;
    }
    it.p0 = first + (count == c.C ? v0 : (int)paged_div((long long)count * v0, c.C));
    it.p1 = first + (count == c.C ? v1 : (int)paged_div((long long)count * v1, c.C));
    it.slot = (v0 == 0 && v1 == c.C) ? -1 : (v0 == 0 ? 2 * w + 1 : 2 * w);
    return it;
}

// The request of token t and what it holds, by the whole warp: the last r with cu_new[r] <= t.  In a decode step token t is
// request t's, so that is looked at first, its length with it; otherwise 32 offsets per step.
__device__ __forceinline__ int paged_find_request(const PagedBatch& pb, int t, PagedReq& rq) {
    const int lane = threadIdx.x & 31, guess = min(t, pb.R - 1);
    rq = paged_request(pb, guess);
    if (rq.row0 <= t && t < rq.row0 + rq.n) return guess;
    int lo = 0, n = pb.R;
    while (n > 1) {
        const int step = (n + 31) / 32, i = lane * step;
        const int v = i < n ? pb.cu_new[lo + i] : INT_MAX;
        const int k = max(__popc(__ballot_sync(0xffffffffu, i < n && v <= t)), 1) - 1;
        lo += k * step;
        n = min(step, n - k * step);
    }
    rq = paged_request(pb, lo);
    return lo;
}

// Physical page of a logical one, or -1 (latched) where the table's entry is out of range: its entries count as masked.
__device__ __forceinline__ int paged_physical(const PagedBatch& pb, const PagedView& pv, int r, int page) {
    const int p = (page >= 0 && page < pb.W) ? pb.table[(size_t)r * pb.W + page] : -1;
    if (p < 0 || p >= pv.n_pages) {
        latch_error(pb.status, TRIMKV_E_ARG);
        return -1;
    }
    return p;
}

// ---------------------------------------------------------------- workspace
// Of each kernel: [shared units, one per worker: int4][partial results, two slots per worker].
constexpr int PAGED_SMS = 148;
constexpr int PAGED_WARP_ROWS = 64, PAGED_WARPS = 4;              // warp kernel: rows per unit at most, workers per SM (2 above 16 rows)
constexpr int PAGED_F32_ROWS = 16, PAGED_F32_CTAS = 2;        // fp32 kernel: rows per unit, CTAs per SM at most
constexpr int PAGED_TC_ROWS = 256, PAGED_TC_HEAD = 128;           // tensor-core kernel: rows per unit, one CTA per SM; largest head size
constexpr size_t PAGED_SHARED_BYTES = (size_t)PAGED_SMS * PAGED_WARPS * 16;      // the warp kernel has the most workers
static_assert(PAGED_SHARED_BYTES % 256 == 0, "partial results are aligned");
// partial results of `rows` rows (workers x rows per unit), two slots each
constexpr size_t paged_partial_bytes(int rows, int d) { return ((size_t)2 * rows * (d + 2) * 4 + 255) & ~(size_t)255; }

struct PagedWork {
    int4* shared;             // [workers]: see paged_note_shared
    float* part_o;            // [slots][rows][d]
    float* part_ml;           // [slots][rows][2]: running maximum (log2 units) and sum
};

// The unit that worker w began, at step x of the line, and did not end: {row0 of its request, its first row, rows | parts << 12,
// KV head}; worker w's own part is in slot 2 w + 1, the next workers' in slots 2 (w + 1), 2 (w + 2), ...  Workers without
// such a unit leave zeros (paged_note_none).
__device__ __forceinline__ void paged_note_none(const PagedWork& wk, int w) { wk.shared[w] = make_int4(0, 0, 0, 0); }
__device__ __forceinline__ void paged_note_shared(const PagedWork& wk, const PagedTable& t, const PagedItem& it, long long x, int w, int first, int rows) {
    const int parts = paged_owner(t.total, t.workers, x + it.cost - 1) - w + 1;
    wk.shared[w] = make_int4(it.q.row0, first, rows | parts << 12, it.h);
}

// ---------------------------------------------------------------- launchers (host)
// Every kernel of this family is launched as a programmatic dependent of whatever precedes it in the stream: it may be placed
// (barriers, descriptors) while its predecessor finishes, every one of its threads calls grid_dependency_wait() before it
// touches memory or returns, and it lets its own successor be placed early.  Their parameters carry no __restrict__: it would
// promise that the memory does not change from the kernel's start on, so a load could be moved before that wait.  Behind a kernel
// that does not take part this is an ordinary launch.  cluster: CTAs per cluster, or 1.  early = false: an ordinary launch.
template <typename... KArgs, typename... Args>
inline cudaError_t paged_launch(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem_bytes, int cluster, bool early, cudaStream_t stream, Args&&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem_bytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = early ? 1 : 0;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    count_launch();
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

cudaError_t launch_paged_plan(int R, const int32_t* old_lens, const int32_t* keep_lens, const int32_t* new_lens, int32_t* table,
                              int W, int32_t* free_pages, int n_pages, const int32_t* free_count, int32_t* free_count_out,
                              int max_tokens, int32_t* lens_out, int32_t* cu_new, int32_t* slot_map, int32_t* positions,
                              int32_t* status, cudaStream_t st);
cudaError_t launch_paged_append(const PagedView& pv, char* k_pages, char* v_pages, char* bounds, int is_bf16, int T, const void* k,
                                long long k_stride, const void* v, long long v_stride, const int32_t* slot_map, int32_t* status,
                                cudaStream_t st);
constexpr int PAGED_SELECT_SMEM = 196 * 1024;
size_t paged_select_smem(int W, int g, int d, int is_bf16);        // must not exceed PAGED_SELECT_SMEM
cudaError_t launch_paged_select(const PagedView& pv, const PagedBatch& pb, int is_bf16, const void* q, int32_t* selected,
                                cudaStream_t st);
// Joins the partial results of a kernel of `workers` workers whose units have up to unit_rows rows; blocks: 0 or, for very many workers, how
// many blocks look through their notes (at least a sixteenth of them).
cudaError_t launch_paged_join(const PagedView& pv, const PagedBatch& pb, int is_bf16, void* out, const PagedWork& w, int unit_rows,
                              int workers, cudaStream_t st, int blocks = 0);
// fp32 caches.
cudaError_t launch_paged_attention_f32(const PagedView& pv, const PagedBatch& pb, const void* q, void* out, float scale, const PagedWork& w,
                                       cudaStream_t st);
cudaError_t paged_tensor_map(CUtensorMap* map, const char* base, const PagedView& pv, int box_rows, int box_planes);      // see its definition
// The bf16 forms: head sizes up to 256 (warp kernel) and 128 (tensor-core kernel).  Warp kernel: requests of min_rows = 1 to max_rows rows in units of tile_rows = 8,
// 16, 32 or 64.  Tensor-core kernel: the requests of more than min_rows - 1 rows.
cudaError_t launch_paged_attention_warp(const PagedView& pv, const PagedBatch& pb, const void* q, void* out, float scale, const PagedWork& w,
                                        int tile_rows, int max_rows, cudaStream_t st);
cudaError_t launch_paged_attention_tc(const PagedView& pv, const PagedBatch& pb, const void* q, void* out, float scale, const PagedWork& w,
                                      int min_rows, cudaStream_t st);

}  // namespace tkv
