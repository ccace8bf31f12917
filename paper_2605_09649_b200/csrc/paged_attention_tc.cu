// Attention over the caller-owned paged cache for many query rows, on tcgen05: bf16, head sizes up to 128 (padded to 64 or 128 in
// shared memory, the missing columns zero).
//
// A unit is 256 (token, query head) rows of one KV head in two groups of 128 that share every K/V tile; a tile is two pages
// (128 entries; the last of a stretch may be one).  One persistent CTA per SM takes an equal share of the line of page steps
// (paged.cuh) and meets a stretch of a unit at a time.  TMA copies K and V as 64-column planes with the 128-byte swizzle:
// K planes (both pages' rows) are K-major operands of S = Q K^T, V planes MN-major operands of O += P V.  Warps 0-7 / 8-15 are
// the softmax warps of group 0 / 1, two threads per row with a page of the tile each (S from tensor memory, masked,
// exponentiated, P back over it as the A operand of P V), warp 16 issues the copies, warp 17 the products, group 0's and group
// 1's in turn: the pipe runs P V and the next S of one group while the other group's softmax works on its S.  (With an issuer
// per group the pipe served both at once, and the groups fell into step: products, then softmax, 5800 cycles a tile.)
//
// The reference m of a row's weights lags: a tile is weighed against the maximum known from the tiles before it, which the two
// threads of a row exchange through shared memory without a barrier of their own (the hand-over of the tile orders it), and
// m is raised, and O rescaled, when that maximum exceeds it by more than 2^8.  Only the first tile that a row sees finds its
// maximum beforehand.  Weights above 2^64, a row whose logits leap by that much within one stretch, send the whole stretch
// round again with the maximum found first in every tile.  A third of the
// exponentials are evaluated on the FMA pipe (7.5e-5 relative).  P is rounded to V's type, which both operands of a product share: off
// by 2^-8 at most, as the output's own rounding; the sum takes the unrounded weights, which are at hand.  A unit of 128 rows or fewer leaves group 1 idle.  V rows behind a request's last
// entry are zeroed in shared memory before the product reads them (they may hold NaN).  Every wait is bounded; one that runs
// out latches TRIMKV_E_TIMEOUT.
//
// Why 128 entries: an S of 64 columns reads 6 KB of operands from shared memory for 32 cycles of products, more than the
// 128 bytes a cycle it delivers, and doubles the hand-overs between the pipes per entry (measured with 64: 610 us for 4 x 512
// tokens over 16K, the pipe 45 % busy).
//
// Order: a worker's share of the line is the rest of a unit that another one began, whole units, and the beginning of one.  It puts
// the rest off to the end, so that every CTA begins a unit at its first page at the same time and those of one KV head read each
// page together, once from HBM and then from L2 (4 x 512 tokens over 16K, 8 KV heads: 0.70 GB from HBM instead of 2.09 GB for
// 0.27 GB of pages; the power saved keeps the clock up: 515-605 us instead of 600-670, 0.9 to 1.05 PFLOP/s of useful products,
// the tensor pipe 54 % busy).  What bounds it is the chain S - softmax - P V of a group, of which the other group
// hides most but not all.
//
// PICK: attention over selected pages for requests with many tokens.  A unit walks the union of its tokens' pages once and masks, row
// by row, the pages that a token did not select (a bit per token and page in shared memory), instead of fetching every token's
// pages for itself.  (128 tokens with 32 of 256 pages each: the union is 166 pages where their queries are alike, 254 where
// they are independent.  The walk of 3744 such steps takes 67 us, half of it for its 13 tiles a CTA, half for what a stretch
// begins and ends with.)
#include "paged.cuh"
#include "paged_tc.cuh"

namespace tkv {

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr int T_ROWS = 128, T_UNIT = PAGED_TC_ROWS;
constexpr int T_PLANE = PAGE * 128;                                   // 64 entries x 64 columns
constexpr int T_QPLANE = T_ROWS * 128;
constexpr int T_SOFT = 16;                                            // softmax warps
constexpr int T_THREADS = (T_SOFT + 2) * 32;
constexpr int T_TMEM_COLS = 512;      // group g: S of page h at columns 128 g + 64 h (P over its first 32); O at 256 + 128 g
constexpr int T_POLY_EVERY = 3;
constexpr int T_JOIN_STEPS = 4;       // what a join costs, in pages
constexpr float T_RESCALE_STEP = 8.0f, T_LEAP = 64.0f;
constexpr int T_STAGES = 2;           // tiles of K, and of V, in shared memory
constexpr int T_E0 = 8;               // ring of the tiles' first entries (two pages each): more than the tiles in flight
constexpr int T_NO_PAGE = INT_MAX / 2;

template <int D, bool PICK>
struct TcShape {
    static constexpr int PLANES = D / 64;
    static constexpr int KPLANE = 2 * T_PLANE;                        // 128 entries x 64 columns
    static constexpr int TILE = PLANES * KPLANE;                      // K of a tile; V of a tile
    static constexpr int OFF_V = T_STAGES * TILE;
    static constexpr int OFF_Q = 2 * T_STAGES * TILE;
    static constexpr int OFF_BAR = OFF_Q + 2 * PLANES * T_QPLANE;
    static constexpr int OFF_E0 = OFF_BAR + 256;
    static constexpr int OFF_MX = OFF_E0 + T_E0 * 8;                  // [tile parity; 2: sums][group][page of the tile][row]: maxima so far
    static constexpr int OFF_TAB = OFF_MX + 3 * 2 * 2 * T_ROWS * 4;
    static constexpr int OFF_BITS = (OFF_TAB + (int)sizeof(PagedTableMem) + 15) & ~15;
    static constexpr int OFF_LIST = OFF_BITS + (PICK ? PAGED_PICK_WORDS * 4 : 0);
    static constexpr int SMEM = OFF_LIST + (PICK ? PAGED_PICK_PAGES * 2 : 0) + 1024;      // 1024: alignment slack
    // D fp32, A and B bf16, M = 128.  S: both K-major, N = 64 per page.  P V: B (V) MN-major, N = D.
    static constexpr uint32_t IDESC_S1 = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(64 >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
    static constexpr uint32_t IDESC_S2 = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(128 >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
    static constexpr uint32_t IDESC_PV = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
};

// EXACT: the head size is D; otherwise smaller, and the columns from pv.d on are zeros in shared memory.
template <int D, bool PICK, bool EXACT>
__global__ void __launch_bounds__(T_THREADS, 1)
paged_attn_tc_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, PagedView pv, PagedBatch pb,
                     const __nv_bfloat16* q, __nv_bfloat16* out, float scale_log2, PagedWork wk, int min_rows) {
    using S = TcShape<D, PICK>;
    extern __shared__ unsigned char t_smem_raw[];
    const uint32_t raw = a_smem(t_smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    unsigned char* gen = t_smem_raw + (base - raw);
    const uint32_t bars = base + S::OFF_BAR;
    const uint32_t k_full = bars, k_empty = bars + 16, v_full = bars + 32, v_empty = bars + 48 /* [stage] each */, s_ready0 = bars + 64,
                   p_ready0 = bars + 80, done0 = bars + 96 /* [group] each */, pair0 = bars + 112 /* [group][32 rows] */;
    volatile uint32_t* s_tmem = reinterpret_cast<volatile uint32_t*>(gen + S::OFF_BAR + 240);
    volatile int* s_fail = reinterpret_cast<volatile int*>(gen + S::OFF_BAR + 244);
    volatile int* s_redo = reinterpret_cast<volatile int*>(gen + S::OFF_BAR + 252);
    volatile int* s_nlist = reinterpret_cast<volatile int*>(gen + S::OFF_BAR + 248);
    volatile int* s_e0 = reinterpret_cast<volatile int*>(gen + S::OFF_E0);
    float* s_mx = reinterpret_cast<float*>(gen + S::OFF_MX);
    PagedTableMem* table_mem = reinterpret_cast<PagedTableMem*>(gen + S::OFF_TAB);
    uint32_t* s_bits = reinterpret_cast<uint32_t*>(gen + S::OFF_BITS);
    uint16_t* s_list = reinterpret_cast<uint16_t*>(gen + S::OFF_LIST);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = pb.g, d = EXACT ? D : pv.d;

    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            a_bar_init(k_full + 8 * i, 1);
            a_bar_init(k_empty + 8 * i, 1);
            a_bar_init(v_full + 8 * i, 1);
            a_bar_init(v_empty + 8 * i, 1);
            a_bar_init(s_ready0 + 8 * i, 1);
            a_bar_init(p_ready0 + 8 * i, T_SOFT / 2);
            a_bar_init(done0 + 8 * i, 1);
        }
        for (int i = 0; i < 8; ++i) a_bar_init(pair0 + 8 * i, 2);
        *s_fail = 0;
        *s_redo = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        a_prefetch_map(&map_k);
        a_prefetch_map(&map_v);
    }
    grid_dependency_wait();
    PagedTable tab;
    paged_build_table<0>(tab, pb, pv.H, T_UNIT, min_rows, INT_MAX, (int)gridDim.x, 4, T_JOIN_STEPS, table_mem);
    grid_dependents_may_launch();
    const int w = blockIdx.x;
    if (threadIdx.x == 0) paged_note_none(wk, w);
    if (w >= tab.workers) return;                                     // the whole block, before it holds tensor memory
    if (warp == T_SOFT + 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(a_smem((const void*)s_tmem)), "r"(T_TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    a_fence_before();
    __syncthreads();
    a_fence_after();
    const uint32_t tmem = *s_tmem;
    // softmax warps: group, page of the tile, 32 rows of the group (a warp reaches the tensor-memory lanes of its number mod 4)
    const int grp = (warp >> 3) & 1, half = (warp >> 2) & 1, wl = warp & 3;
    const int r = wl * 32 + lane, R = grp * T_ROWS + r;               // row: lane of tensor memory, row of the unit

    const long long begin = tab.share(w);
    long long end = tab.share(w + 1);
    // tiles of the stretches before this one: of the rings, and of group 1, whose barriers rest while it has no rows; and the
    // stretches with tiles, of group 0 and 1
    unsigned ct = 0, ct1 = 0, st0 = 0, st1 = 0;
    unsigned ex = 0;                                                  // barriers of the two warps of a row so far
    bool careful = false;                                             // this stretch again, every tile's maximum first
    // The rest of a unit that another worker began comes last: the workers then begin units at their first page at the same time, and
    // those of one KV head read the same pages from L2.
    long long last = 0;                                               // end of that rest, if it was put off
    for (long long x = begin; x < end || last;) {
        if (x >= end) { x = begin; end = last; }
        const PagedItem it = paged_item<0>(tab, pb, x, end, w);
        if (x == begin && !last && it.slot == 2 * w && x + it.steps < end) { last = x += it.steps; continue; }
        if (end == last) last = 0;
        int npage = it.p1 - it.p0;
        const int row_first = it.u * T_UNIT, rows = min(T_UNIT, it.q.n * g - row_first);
        const bool both = rows > T_ROWS;
        const bool soft = warp < T_SOFT && (grp == 0 || both);
        const bool valid = soft && R < rows;
        const int tok = valid ? pb.by_g.div(row_first + R) : it.tok0, head = valid ? row_first + R - tok * g : 0;
        const int pos = it.q.len - it.q.n + tok;
        const int see_hi = valid ? max(pos + 1, 0) : 0;               // entries the row sees: see_lo .. see_hi - 1
        const int see_lo = valid && pb.window > 0 ? max(pos + 1 - pb.window, 0) : 0;
        const int w0 = it.p0 >> 5, nw = npage > 0 ? ((it.p1 - 1) >> 5) - w0 + 1 : 0;      // words of the stretch's pages
        if (PICK && npage > 0) {
            // ---- which token selected which page of the stretch; the union, ascending
            const int ntok = it.tok1 - it.tok0 + 1;
            for (int i = threadIdx.x; i < (ntok + 1) * nw; i += T_THREADS) s_bits[i] = 0u;      // a row of bits per token, the union last
            __syncthreads();
            for (int i = threadIdx.x; i < ntok * pb.pick_top; i += T_THREADS) {
                const int tk = i / pb.pick_top, e = i - tk * pb.pick_top;
                const int page = pb.selected[((size_t)(it.q.row0 + it.tok0 + tk) * pv.H + it.h) * pb.pick_top + e];
                if (page >= it.p0 && page < it.p1) {
                    const int word = (page >> 5) - w0;
                    const uint32_t bit = 1u << (page & 31);
                    atomicOr(&s_bits[tk * nw + word], bit);
                    if (!(reinterpret_cast<volatile uint32_t*>(s_bits)[ntok * nw + word] & bit)) atomicOr(&s_bits[ntok * nw + word], bit);
                }
            }
            __syncthreads();
            if (warp == 0) {
                int at = 0;
                for (int i0 = 0; i0 < nw; i0 += 32) {
                    uint32_t any = i0 + lane < nw ? s_bits[ntok * nw + i0 + lane] : 0u;
                    int before = __popc(any);
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) {
                        const int v = __shfl_up_sync(0xffffffffu, before, o);
                        if (lane >= o) before += v;
                    }
                    const int all = __shfl_sync(0xffffffffu, before, 31);
                    int put = at + before - __popc(any);
                    while (any) {
                        const int b = __ffs(any) - 1;
                        any &= any - 1;
                        s_list[put++] = (uint16_t)((w0 + i0 + lane) * 32 + b);
                    }
                    at += all;
                }
                if (lane == 0) *s_nlist = at;
            }
            __syncthreads();
            npage = *s_nlist;
        }
        const int ntile = (npage + 1) / 2;
        if (ntile > 0) {
            if (soft) {
                // neighbouring lanes have neighbouring 16 bytes of a row (a row per lane: 32 cache lines per load, 4100 cycles in all)
                constexpr int CPR = D / 16;                           // 16-byte chunks of half a row
                const int c = half * CPR + lane % CPR;
#pragma unroll
                for (int k = 0; k < CPR; ++k) {
                    const int rq = wl * 32 + k * (32 / CPR) + lane / CPR, row = row_first + grp * T_ROWS + rq, qt = pb.by_g.div(row);
                    const __nv_bfloat16* src = q + (size_t)(it.q.row0 + qt) * pb.q_stride + (size_t)(it.h * g + row - qt * g) * d + c * 8;
                    const uint4 v = grp * T_ROWS + rq < rows && c * 8 < d ? *reinterpret_cast<const uint4*>(src) : make_uint4(0u, 0u, 0u, 0u);
                    *reinterpret_cast<uint4*>(gen + S::OFF_Q + (grp * S::PLANES + (c >> 3)) * T_QPLANE + rq * 128 + (((c & 7) ^ (rq & 7)) << 4)) = v;
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // Q and the barriers, before the async proxy uses them
            a_fence_before();
            // everyone but the warp that copies K and V: its rings are free since the end of the stretch before
            if (warp != T_SOFT) asm volatile("bar.sync 1, %0;" ::"n"(T_THREADS - 32) : "memory");
            a_fence_after();

            if (warp == T_SOFT) {
                // ---- TMA producer: lane l holds page l of the current run of 32
                int page = 0, phys = 0;
                auto copy = [&](uint32_t dst, const CUtensorMap* map, int plane, int row, uint32_t bar) {    // a page's plane
                    if (EXACT || d % 64 == 0) a_tma_3d(dst, map, 0, row, plane, bar);
                    else a_tma_2d(dst, map, plane * 64, row, bar);    // the last plane's missing columns arrive as zeros
                };
                for (int i = 0; i < ntile; ++i) {
                    if ((i & 15) == 0) {
                        const int e = 2 * i + lane;
                        page = e < npage ? (PICK ? (int)s_list[e] : it.p0 + e) : -1;
                        phys = e < npage ? paged_physical(pb, pv, it.r, page) : -1;
                    }
                    const int src = (2 * i) & 31;
                    const int pg0 = __shfl_sync(0xffffffffu, page, src), pg1 = __shfl_sync(0xffffffffu, page, src + 1);
                    const int ph0 = __shfl_sync(0xffffffffu, phys, src), ph1 = __shfl_sync(0xffffffffu, phys, src + 1);
                    const unsigned c = ct + i, s = c % T_STAGES;
                    int ok = 1;
                    if (lane == 0) {
                        const bool two = 2 * i + 1 < npage;
                        if (c >= T_STAGES) ok = a_bar_wait(k_empty + 8 * s, ((c / T_STAGES) - 1) & 1) ? 1 : 0;
                        if (ok) {
                            // a page that does not exist: the copy reads page 0 and every row masks the page
                            s_e0[c % T_E0 * 2] = ph0 < 0 ? T_NO_PAGE : pg0 * PAGE;
                            s_e0[c % T_E0 * 2 + 1] = !two ? -1 : ph1 < 0 ? T_NO_PAGE : pg1 * PAGE;
                            const int row0 = (max(ph0, 0) * pv.H + it.h) * PAGE, row1 = (max(ph1, 0) * pv.H + it.h) * PAGE;
                            const uint32_t kd = base + s * S::TILE, vd = base + S::OFF_V + s * S::TILE;
                            a_bar_expect_tx(k_full + 8 * s, two ? S::TILE : S::TILE / 2);
#pragma unroll
                            for (int p = 0; p < S::PLANES; ++p) {
                                copy(kd + p * S::KPLANE, &map_k, p, row0, k_full + 8 * s);
                                if (two) copy(kd + p * S::KPLANE + T_PLANE, &map_k, p, row1, k_full + 8 * s);
                            }
                            if (c >= T_STAGES) ok = a_bar_wait(v_empty + 8 * s, ((c / T_STAGES) - 1) & 1) ? 1 : 0;
                            if (ok) {
                                a_bar_expect_tx(v_full + 8 * s, two ? S::TILE : S::TILE / 2);
#pragma unroll
                                for (int p = 0; p < S::PLANES; ++p) {
                                    copy(vd + p * T_PLANE, &map_v, p, row0, v_full + 8 * s);
                                    if (two) copy(vd + (S::PLANES + p) * T_PLANE, &map_v, p, row1, v_full + 8 * s);
                                }
                            }
                        }
                    }
                    if (__shfl_sync(0xffffffffu, ok, 0) == 0) {
                        if (lane == 0) *s_fail = 1;
                        // the copies already issued land before the block leaves (bounded); K of this tile may be among them
                        for (unsigned k = c >= T_STAGES ? c - T_STAGES : 0; k <= c; ++k) {
                            a_bar_wait(k_full + 8 * (k % T_STAGES), (k / T_STAGES) & 1);
                            if (k < c) a_bar_wait(v_full + 8 * (k % T_STAGES), (k / T_STAGES) & 1);
                        }
                        break;
                    }
                }
            } else if (warp > T_SOFT) {
                // ---- MMA issuer: P V of a tile, then S of the next, which overwrites that tile's P (the pipe runs in issue
                // order), for one group after the other
                bool ok = true;
                const uint32_t leader = t_elect();
                const uint32_t ub = t_uniform(base), ut = t_uniform(tmem), uct = t_uniform(ct), uct1 = t_uniform(ct1);
                const int un = (int)t_uniform((uint32_t)ntile), upages = (int)t_uniform((uint32_t)npage), uboth = (int)t_uniform(both ? 1u : 0u);
                auto issue_s = [&](int i, int gq) {
                    const uint32_t c = uct + i, s = c % T_STAGES;
                    ok = __all_sync(0xffffffffu, a_bar_wait(k_full + 8 * s, (c / T_STAGES) & 1));
                    if (!ok) return;
                    a_fence_after();
                    const uint32_t k_lo = t_desc_lo(ub, 16) + s * (S::TILE >> 4), q_lo = t_desc_lo(ub + S::OFF_Q, 16) + gq * (S::PLANES * T_QPLANE >> 4);
                    const uint32_t idesc = 2 * i + 1 < upages ? S::IDESC_S2 : S::IDESC_S1;
#pragma unroll
                    for (int p = 0; p < S::PLANES; ++p)
#pragma unroll
                        for (int j = 0; j < 4; ++j)                   // 16 channels per instruction, 32 bytes along the row
                            t_umma(leader, ut + 128 * gq, q_lo + (p * T_QPLANE + j * 32) / 16, k_lo + (p * S::KPLANE + j * 32) / 16, idesc, (p | j) != 0);
                    t_commit(leader, bars + 64 + 8 * gq);             // S ready (and everything issued before: O up to the last tile)
                    if (gq == 1 || !uboth) t_commit(leader, k_empty + 8 * s);
                };
                auto wait_v = [&](int i) {                            // V of the tile; what lies behind the last entry becomes zero
                    const uint32_t c = uct + i, s = c % T_STAGES;
                    ok = __all_sync(0xffffffffu, a_bar_wait(v_full + 8 * s, (c / T_STAGES) & 1));
                    if (!ok) return;
                    for (int h = 0; h < 2 && 2 * i + h < upages; ++h) {      // (held <= 0 for a page that does not exist: all of its V)
                        const int held = it.q.len - s_e0[c % T_E0 * 2 + h];
                        if (held >= PAGE) continue;
                        unsigned char* vg = gen + S::OFF_V + s * S::TILE + h * S::PLANES * T_PLANE;
                        for (int e = max(held, 0) * 8 + lane; e < PAGE * 8; e += 32)
#pragma unroll
                            for (int p = 0; p < S::PLANES; ++p) *reinterpret_cast<uint4*>(vg + p * T_PLANE + e * 16) = make_uint4(0u, 0u, 0u, 0u);
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                    }
                };
                auto issue_pv = [&](int i, int gq) {
                    const uint32_t c = uct + i, s = c % T_STAGES;
                    const uint32_t v_lo = t_desc_lo(ub + S::OFF_V, T_PLANE) + s * (S::TILE >> 4);     // the next 64 channels: one plane further
                    const uint32_t d_o = ut + 256 + 128 * gq, a_p = ut + 128 * gq;
                    ok = __all_sync(0xffffffffu, a_bar_wait(p_ready0 + 8 * gq, ((gq ? uct1 : uct) + i) & 1));
                    if (!ok) return;
                    a_fence_after();
#pragma unroll
                    for (int j = 0; j < PAGE / 16; ++j)               // 16 entries per instruction: P +8 columns, V +2 row groups
                        t_umma_ts(leader, d_o, a_p + j * 8, v_lo + j * 128, S::IDESC_PV, i != 0 || j != 0);
                    if (2 * i + 1 < upages) {
#pragma unroll
                        for (int j = 0; j < PAGE / 16; ++j)
                            t_umma_ts(leader, d_o, a_p + 64 + j * 8, v_lo + S::PLANES * T_PLANE / 16 + j * 128, S::IDESC_PV, 1u);
                    }
                    if (gq == 1 || !uboth) t_commit(leader, v_empty + 8 * s);
                    if (i + 1 == un) t_commit(leader, done0 + 8 * gq);
                };
                issue_s(0, 0);
                if (ok && uboth) issue_s(0, 1);
                for (int i = 0; i < un && ok; ++i) {
                    wait_v(i);
                    if (ok) issue_pv(i, 0);
                    if (ok && i + 1 < un) issue_s(i + 1, 0);
                    if (ok && uboth) issue_pv(i, 1);
                    if (ok && uboth && i + 1 < un) issue_s(i + 1, 1);
                }
                if (!ok && lane == 0) *s_fail = 1;
            }
        }
        if (soft) {
            // ---- softmax warps: page `half` of every tile
            const uint32_t lane_addr = tmem + ((uint32_t)(wl * 32) << 16);
            const uint32_t s_addr = lane_addr + (uint32_t)(128 * grp + 64 * half), o_addr = lane_addr + (uint32_t)(256 + 128 * grp + half * (D / 2));
            const uint32_t pair = pair0 + 8 * (grp * 4 + wl);
            float* mx_mine = s_mx + (grp * 2 + half) * T_ROWS + r;
            const float* mx_other = s_mx + (grp * 2 + (half ^ 1)) * T_ROWS + r;
            constexpr int MX = 4 * T_ROWS;                            // from one buffer of maxima to the next
            const unsigned gt = grp ? ct1 : ct;
            const uint64_t sc2 = a_pack2(scale_log2, scale_log2);
            float m_used = -INFINITY, m_mine = -INFINITY, l = 0.f;    // the reference (the same in both threads), this thread's maximum, its sum
            bool ok = true;
            // entries that every row of the warp sees (rows without a query see whatever the others do); once every row has a
            // maximum, a tile of two pages in this span needs no look at the rows
            const int all_hi = PICK ? 0 : __reduce_min_sync(0xffffffffu, valid ? see_hi : INT_MAX), all_lo = __reduce_max_sync(0xffffffffu, see_lo);
            bool primed = false;
            for (int i = 0; i < ntile; ++i) {
                ok = __all_sync(0xffffffffu, a_bar_wait(s_ready0 + 8 * grp, (gt + i) & 1));
                if (!ok) break;
                a_fence_after();
                // first entries of both pages (-1: the tile is one page); what the row sees of them
                const int e0 = s_e0[(ct + i) % T_E0 * 2 + half], e1 = s_e0[(ct + i) % T_E0 * 2 + (half ^ 1)];
                auto sees = [&](int e) {
                    if (!(valid && e >= 0 && e < see_hi && e + PAGE > see_lo)) return false;
                    return !PICK || ((s_bits[(tok - it.tok0) * nw + (e / PAGE >> 5) - w0] >> (e / PAGE & 31)) & 1u) != 0u;
                };
                const bool inside = primed && !careful && min(e0, e1) >= all_lo && max(e0, e1) + PAGE <= all_hi;      // (e1 < 0: not inside)
                bool mine = true, some = true, edge = false, first = false;
                if (!inside) {
                    mine = sees(e0);
                    some = __any_sync(0xffffffffu, mine);             // of the warp's rows
                    // a row that sees nothing of the page is weighed to nothing below (mref); only what lies behind the last
                    // entry has to go, it may be NaN
                    edge = mine ? e0 + PAGE > see_hi || e0 < see_lo : e0 + PAGE > it.q.len;
                    // the same for both warps of the rows: a row that has seen nothing yet finds its maximum first
                    first = careful || i == 0 || __any_sync(0xffffffffu, m_used == -INFINITY && (mine || sees(e1)));
                }
                uint32_t sv[32];
                auto load = [&](int k) {                              // entries 32 k .. of the page, masked
                    a_tmem_ld32(s_addr + 32 * k, sv);
                    t_tmem_wait_ld();
                    if (edge) {
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (e0 + 32 * k + e >= see_hi || e0 + 32 * k + e < see_lo) sv[e] = 0xff800000u;        // -inf
                    }
                };
                float m_all;
                if (first) {
                    if (some) {
#pragma unroll 1
                        for (int k = 0; k < 2; ++k) {
                            load(k);
                            float mq[2] = {-INFINITY, -INFINITY};
#pragma unroll
                            for (int e = 0; e < 32; e += 4) {
                                mq[0] = a_max3(mq[0], __uint_as_float(sv[e]), __uint_as_float(sv[e + 1]));
                                mq[1] = a_max3(mq[1], __uint_as_float(sv[e + 2]), __uint_as_float(sv[e + 3]));
                            }
                            if (mine) m_mine = fmaxf(m_mine, fmaxf(mq[0], mq[1]) * scale_log2);  // scale_log2 > 0
                        }
                    }
                    mx_mine[(i & 1) * MX] = m_mine;
                    ok = t_pair_sync(pair, ex);
                    if (!ok) break;
                    ++ex;
                    m_all = fmaxf(m_mine, mx_other[(i & 1) * MX]);
                } else
                    m_all = fmaxf(m_mine, mx_other[((i - 1) & 1) * MX]);
                if (__any_sync(0xffffffffu, m_all > m_used + T_RESCALE_STEP)) {
                    const float mn = fmaxf(m_used, m_all);
                    const float alpha = (m_used == -INFINITY) ? 0.0f : exp2f(m_used - mn);
                    m_used = mn;
                    l *= alpha;
                    if (i > 0) {                                      // (O is complete up to the previous tile: see the commit of S)
#pragma unroll 1
                        for (int k = 0; k < D / 32; ++k) {
                            uint32_t ov[16];
                            t_tmem_ld16(o_addr + k * 16, ov);
                            t_tmem_wait_ld();
#pragma unroll
                            for (int e = 0; e < 16; ++e) ov[e] = __float_as_uint(__uint_as_float(ov[e]) * alpha);
                            t_tmem_st16(o_addr + k * 16, ov);
                        }
                    }
                }
                if (!primed) primed = __all_sync(0xffffffffu, m_used > -INFINITY || !valid);
                if (some) {
                    // a row that sees nothing of the page weighs it against +inf: every weight is 0
                    const float mref = !mine ? INFINITY : (m_used == -INFINITY) ? 0.0f : m_used;
                    const uint64_t nm2 = a_pack2(-mref, -mref);
                    uint64_t sq[2] = {0ull, 0ull};
                    float mq[2] = {-INFINITY, -INFINITY};
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        load(k);
                        uint32_t pk[16];
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            const uint64_t x2 = a_fma2(a_pack2(__uint_as_float(sv[e]), __uint_as_float(sv[e + 1])), sc2, nm2);
                            float x0, x1, p0, p1;
                            a_unpack2(x2, x0, x1);
                            mq[(e >> 1) & 1] = a_max3(mq[(e >> 1) & 1], x0, x1);
                            if ((e >> 1) % T_POLY_EVERY == T_POLY_EVERY - 1) {
                                a_exp2_fma2(x2, p0, p1);
                            } else {
                                p0 = a_ex2(x0);
                                p1 = a_ex2(x1);
                            }
                            sq[(e >> 1) & 1] = a_add2(sq[(e >> 1) & 1], a_pack2(p0, p1));
                            pk[e >> 1] = a_bf16x2(p0, p1);
                        }
                        t_tmem_st16(s_addr + 16 * k, pk);             // P: two entries per column, over the page's first 32 columns of S
                    }
                    float a0, a1;
                    a_unpack2(a_add2(sq[0], sq[1]), a0, a1);
                    l += a0 + a1;
                    const float mx = fmaxf(mq[0], mq[1]);
                    if (mine) {
                        m_mine = fmaxf(m_mine, mref + mx);
                        if (!first && mx > T_LEAP) *s_redo = 1;
                    }
                } else if (e0 >= 0) {
                    uint32_t pk[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) pk[e] = 0u;
                    t_tmem_st16(s_addr, pk);
                    t_tmem_st16(s_addr + 16, pk);
                }
                if (!first) mx_mine[(i & 1) * MX] = m_mine;           // read by the other thread at the next tile
                t_tmem_wait_st();
                a_fence_before();
                __syncwarp();
                if (lane == 0) a_bar_arrive(p_ready0 + 8 * grp);
            }
            if (ok && ntile > 0) ok = __all_sync(0xffffffffu, a_bar_wait(done0 + 8 * grp, (grp ? st1 : st0) & 1));
            mx_mine[2 * MX] = l;                                      // the two threads' sums
            if (ok) ok = t_pair_sync(pair, ex);
            if (!ok) {
                if (lane == 0) *s_fail = 1;
            } else {
                ++ex;
                a_fence_after();
                l += mx_other[2 * MX];
                if (m_used == -INFINITY && !(l != l)) l = 0.f;        // a row that sees nothing (the polynomial gives masked entries 2^-125)
                const float inv = l > 0.f ? 1.0f / l : (l == 0.f ? 0.f : l);
                uint4* op = reinterpret_cast<uint4*>(out + ((size_t)(it.q.row0 + tok) * pb.Hq + (size_t)(it.h * g + head)) * d + half * (D / 2));
                const size_t pr = (size_t)(it.slot < 0 ? 0 : it.slot) * T_UNIT + R;
                float* po = wk.part_o + pr * d + half * (D / 2);
                const bool zero = l == 0.f;                           // (also a stretch without tiles, whose O was never written)
#pragma unroll 1
                for (int k = 0; k < D / 32; ++k) {
                    uint32_t ov[16];
                    if (ntile > 0) {
                        t_tmem_ld16(o_addr + k * 16, ov);
                        t_tmem_wait_ld();
                    }
#pragma unroll
                    for (int e = 0; e < 16; ++e) ov[e] = zero ? 0u : ov[e];
                    if (!valid) continue;
                    if (it.slot < 0) {
#pragma unroll
                        for (int e = 0; e < 16; e += 8) {
                            uint32_t v[4];
#pragma unroll
                            for (int k2 = 0; k2 < 4; ++k2)
                                v[k2] = a_bf16x2(__uint_as_float(ov[e + 2 * k2]) * inv, __uint_as_float(ov[e + 2 * k2 + 1]) * inv);
                            if (half * (D / 2) + k * 16 + e < d) op[k * 2 + (e >> 3)] = make_uint4(v[0], v[1], v[2], v[3]);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 16; e += 8)
                            if (half * (D / 2) + k * 16 + e < d) t_store32(po + k * 16 + e, ov + e);
                    }
                }
                if (valid && it.slot >= 0 && half == 0) {
                    wk.part_ml[pr * 2] = m_used;
                    wk.part_ml[pr * 2 + 1] = l;
                }
            }
        }
        ct += (unsigned)ntile;
        st0 += ntile > 0;
        if (both) { ct1 += (unsigned)ntile; st1 += ntile > 0; }
        a_fence_before();
        __syncthreads();                                              // Q, the lists and tensor memory are free for the next stretch
        a_fence_after();
        if (*s_fail) break;
        careful = !careful && *s_redo;                                // (a careful stretch sets no flag)
        if (!careful) {
            if (it.slot >= 0 && (it.slot & 1) && threadIdx.x == 0) paged_note_shared(wk, tab, it, x, w, row_first, rows);
            x += it.steps;
        }
        else {
            __syncthreads();                                          // everyone has read the flag
            if (threadIdx.x == 0) *s_redo = 0;
        }
    }
    __syncthreads();
    if (warp == T_SOFT + 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(T_TMEM_COLS) : "memory");
    if (threadIdx.x == 0 && *s_fail) latch_error(pb.status, TRIMKV_E_TIMEOUT);
}

template <int D, bool PICK, bool EXACT>
cudaError_t run_tc(const PagedView& pv, const PagedBatch& pb, const void* q, void* out, float scale, const PagedWork& w, int min_rows, cudaStream_t st) {
    using S = TcShape<D, PICK>;
    static_assert(S::SMEM <= 227 * 1024, "shared memory of one SM");
    static std::atomic<unsigned long long> done{0};
    cudaError_t e = paged_allow_smem(reinterpret_cast<const void*>(paged_attn_tc_kernel<D, PICK, EXACT>), S::SMEM, done);
    if (e != cudaSuccess) return e;
    CUtensorMap mk, mv;
    e = paged_tensor_map(&mk, pv.k, pv, PAGE, 1);                     // plane by plane: a tile's plane of K holds the rows of two pages
    if (e == cudaSuccess) e = paged_tensor_map(&mv, pv.v, pv, PAGE, 1);
    if (e != cudaSuccess) return e;
    e = paged_launch(paged_attn_tc_kernel<D, PICK, EXACT>, dim3(PAGED_SMS), dim3(T_THREADS), S::SMEM, 1, true, st, mk, mv, pv, pb, (const __nv_bfloat16*)q,
                     (__nv_bfloat16*)out, scale * LOG2E, w, min_rows);
    if (e != cudaSuccess || paged_always_whole(pb, pv.H, T_UNIT, PAGED_SMS, T_JOIN_STEPS)) return e;
    return launch_paged_join(pv, pb, 1, out, w, T_UNIT, PAGED_SMS, st);
}

}  // namespace

cudaError_t launch_paged_attention_tc(const PagedView& pv, const PagedBatch& pb, const void* q, void* out, float scale, const PagedWork& w,
                                      int min_rows, cudaStream_t st) {
    auto go = [&](auto d, auto pick) {
        constexpr int D = decltype(d)::value;
        constexpr bool PICK = decltype(pick)::value;
        return pv.d == D ? run_tc<D, PICK, true>(pv, pb, q, out, scale, w, min_rows, st) : run_tc<D, PICK, false>(pv, pb, q, out, scale, w, min_rows, st);
    };
    using D64 = std::integral_constant<int, 64>;
    using D128 = std::integral_constant<int, 128>;
    if (pb.pick > 0) return pv.d <= 64 ? go(D64{}, std::true_type{}) : go(D128{}, std::true_type{});
    return pv.d <= 64 ? go(D64{}, std::false_type{}) : go(D128{}, std::false_type{});
}

}  // namespace tkv
