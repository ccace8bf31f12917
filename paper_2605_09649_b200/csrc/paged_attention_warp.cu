// Attention over the caller-owned paged cache for few query rows: bf16, head sizes up to 256 (padded to 64, 128 or 256 in shared
// memory, the missing columns zero).
//
// A decode step does 2 g flops per byte of K and V, far below the machine's balance, so the kernel is a stream from HBM:
// one CTA per SM, four independent warps, each with a ring of its own (48 KB) that TMA fills 32 entries at a time, one
// or two 64-column boxes of K and of V (a team: 64 entries), 128-byte swizzled so that ldmatrix meets no bank conflict.  A warp takes an equal
// share of the line of page steps (paged.cuh), computes S^T = K Q^T and O^T += V^T P^T with mma.sync m16n8k16 -- the
// (token, head) rows are the N dimension, 8 or 16 columns, so little is wasted on padding -- and keeps the
// softmax in registers.  Units of up to 32 or 64 rows (drafted tokens): teams of four warps share a ring of 96 KB and every
// tile, each warp with 8 or 16 of the rows.  (One warp with 32 columns took 80 us for 32 requests x 5 tokens x 4 heads over
// 0.6 to 2.3 K entries: a warp alone on its scheduler waits for each of its own products.)
// Measured: 1.07 GB of K and V of a decode step (8 requests of up to 32 K) in 170 us, 0.98 of the measured copy rate; 81 MB (4
// of up to 16 K) in 26 us and the 184 MB of those drafts in 42 us, of which about 10 are the launch, the table of requests,
// the first pages' way here and the join.
// P is rounded to bf16 for the second product, and the sum takes the rounded values, so the weights
// still add up to one.  Rows behind a request's last entry are zeroed in shared memory (they may hold NaN, and 0 x NaN is
// NaN).  Every wait is bounded: on expiry the warp latches TRIMKV_E_TIMEOUT, drains its copies and returns.
#include "async_copy.cuh"
#include "mma_sync.cuh"
#include "paged.cuh"
#include "tcgen05_attn.cuh"

namespace tkv {

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr int W_JOIN_STEPS = 8;                                       // what a join costs, in pages
constexpr float W_RESCALE_STEP = 8.0f;                                // log2 units the reference of the weights may lag behind the maximum

// NT: column tiles of 8 rows per warp.  TW: warps of a team, which share a ring and a unit, each with rows of its own.
template <int D, int NT, int TW>
struct WarpShape {
    static constexpr int TEAMS = TW == 1 ? PAGED_WARPS : 2;
    static constexpr int ROWS = NT * 8 * TW;                          // rows of a unit
    static constexpr int TILE = (TW == 1 ? 32 : 64) / (D == 256 ? 2 : 1);       // entries per stage
    static constexpr int PER_PAGE = PAGE / TILE;
    static constexpr int PLANE = TILE * 128;                          // entries x 64 columns
    static constexpr int PLANES = D / 64;
    static constexpr int STAGE = 2 * PLANES * PLANE;                  // K planes, V planes
    static constexpr int STAGES = 192 * 1024 / TEAMS / STAGE;         // 3; d = 64: 6
    static constexpr int LAG = TW == 1 ? 0 : 1;                       // tiles that the rest of a team may be behind a refill
    static constexpr int RING = STAGES * STAGE;
    static constexpr int OFF_BAR = TEAMS * RING;                      // full and empty barrier of each stage
    static constexpr int OFF_META = OFF_BAR + TEAMS * STAGES * 16;
    static constexpr int OFF_TAB = (OFF_META + TEAMS * STAGES * 4 + 15) & ~15;
    static constexpr int SMEM = OFF_TAB + (int)sizeof(PagedTableMem) + 1024;      // 1024: alignment slack
};

// A place on the line and the stretch of a unit that begins there.
struct WarpCursor {
    long long x;
    PagedItem it;
    int ntile;          // tiles to read
    bool on;
};

// EXACT: the head size is D; otherwise smaller, and the columns from pv.d on are zeros in shared memory.
template <int D, int NT, int TW, bool SELECT, bool EXACT>
__global__ void __launch_bounds__(WarpShape<D, NT, TW>::TEAMS * TW * 32, 1)
paged_attn_warp_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, PagedView pv, PagedBatch pb,
                       const __nv_bfloat16* q, __nv_bfloat16* out, float scale_log2, PagedWork wk, int max_rows) {
    using S = WarpShape<D, NT, TW>;
    constexpr int KS = D / 16, MT = S::TILE / 16;
    extern __shared__ unsigned char w_smem_raw[];
    unsigned char* smem = w_smem_raw + ((1024u - (smem_u32(w_smem_raw) & 1023u)) & 1023u);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = pb.g;
    const int team = warp / TW, tw = warp % TW;
    unsigned char* ring = smem + (size_t)team * S::RING;
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + S::OFF_BAR) + team * S::STAGES * 2;
    uint64_t* empty = bars + S::STAGES;
    volatile int* meta = reinterpret_cast<volatile int*>(smem + S::OFF_META) + team * S::STAGES;      // first entry of the stage's tile; -1: skip
    PagedTableMem* table_mem = reinterpret_cast<PagedTableMem*>(smem + S::OFF_TAB);
    const int unit_rows = SELECT ? pb.sub_rows : S::ROWS, d = EXACT ? D : pv.d;

    if (lane == 0 && tw == 0)
        for (int s = 0; s < S::STAGES; ++s) { mbar_init(bars + s, 1); mbar_init(empty + s, TW); }
    if (threadIdx.x == 0) { a_prefetch_map(&map_k); a_prefetch_map(&map_v); }
    fence_proxy_async_smem();
    grid_dependency_wait();
    PagedTable tab;
    paged_build_table<SELECT>(tab, pb, pv.H, S::ROWS, 1, max_rows, (int)gridDim.x * S::TEAMS, 4, W_JOIN_STEPS, table_mem);      // (synchronises the block)
    grid_dependents_may_launch();
    // workers are spread over the SMs first, so that a short line uses many of them
    const int w = team * (int)gridDim.x + (int)blockIdx.x;
    if (lane == 0 && tw == 0) paged_note_none(wk, w);
    if (w >= tab.workers) return;
    const long long end = tab.share(w + 1);

    auto at = [&](long long x) {
        WarpCursor c;
        c.x = x;
        c.ntile = 0;
        c.on = x < end;
        if (!c.on) return c;
        c.it = paged_item<SELECT>(tab, pb, x, end, w);
        c.ntile = S::PER_PAGE * (c.it.p1 - c.it.p0);
        // the page of the unit's last token: its last tiles may lie behind what is seen
        if (S::PER_PAGE > 1 && c.ntile) {
            const int phi = c.it.q.len - c.it.q.n + c.it.tok1, np = phi / PAGE + 1;
            const bool last = SELECT ? c.it.p1 == min(pb.top, np) : c.it.p1 == np;
            if (last) c.ntile -= S::PER_PAGE - 1 - phi % PAGE / S::TILE;
        }
        return c;
    };
    WarpCursor cons = at(tab.share(w)), prod = cons;
    int prod_tile = 0, log_page = 0, phys_page = 0;                   // lane l: page l of the current run of 32
    unsigned issued = 0, consumed = 0;
    bool failed = false;

    auto issue_one = [&]() {                                          // the team's first warp
        while (prod.on && prod_tile == prod.ntile) { prod = at(prod.x + prod.it.steps); prod_tile = 0; }
        if (!prod.on) return;
        if (prod_tile % (32 * S::PER_PAGE) == 0) {                    // the next 32 pages
            const int p = prod.it.p0 + prod_tile / S::PER_PAGE + lane;
            log_page = -1;
            if (p < prod.it.p1) log_page = SELECT ? pb.selected[((size_t)(prod.it.q.row0 + prod.it.tok0) * pv.H + prod.it.h) * pb.top + p] : p;
            phys_page = p < prod.it.p1 ? paged_physical(pb, pv, prod.it.r, log_page) : -1;
        }
        const int src = (prod_tile / S::PER_PAGE) & 31, half = prod_tile % S::PER_PAGE;
        const int lp = __shfl_sync(0xffffffffu, log_page, src), pp = __shfl_sync(0xffffffffu, phys_page, src);
        const unsigned s = issued % S::STAGES;
        if (TW > 1 && issued >= S::STAGES && !mbar_wait_bounded(empty + s, (issued / S::STAGES - 1) & 1u)) { failed = true; return; }
        if (lane == 0) {
            meta[s] = pp < 0 ? -1 : lp * PAGE + half * S::TILE;
            if (pp < 0) {
                mbar_arrive(bars + s);
            } else {
                const uint32_t dst = smem_u32(ring + s * S::STAGE), bar = smem_u32(bars + s);
                const int row = (pp * pv.H + prod.it.h) * PAGE + half * S::TILE;
                mbar_expect_tx(bars + s, S::STAGE);                   // (the zeroing of rows below carries its own proxy fence)
                if (EXACT || d % 64 == 0) {
                    a_tma_3d(dst, &map_k, 0, row, 0, bar);
                    a_tma_3d(dst + S::PLANES * S::PLANE, &map_v, 0, row, 0, bar);
                } else {                                              // the last plane's missing columns arrive as zeros
#pragma unroll
                    for (int p = 0; p < S::PLANES; ++p) {
                        a_tma_2d(dst + p * S::PLANE, &map_k, p * 64, row, bar);
                        a_tma_2d(dst + (S::PLANES + p) * S::PLANE, &map_v, p * 64, row, bar);
                    }
                }
            }
        }
        ++issued;
        ++prod_tile;
    };
    if (tw == 0)
        for (int s = 0; s < S::STAGES - 1 - S::LAG; ++s) issue_one();

    uint32_t bq[NT][KS][2];
    float o[NT][KS][4];
    float m_run[NT][2], l_run[NT][2];

    while (cons.on && !failed) {
        const PagedItem& it = cons.it;
        const int unit_first = paged_unit_first<SELECT>(pb, it.u, S::ROWS), unit_n = paged_unit_rows<SELECT>(pb, it.u, it.q.n, S::ROWS);
        const int row_first = unit_first + tw * NT * 8;               // this warp's rows
        const int rows = max(0, min(NT * 8, unit_n - tw * NT * 8));
        // ---- Q fragments (B operand: k = channel, n = row)
        int all_lo, all_hi;                                           // entries that every row of the unit sees
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int row = nt * 8 + (lane >> 2);
            const int qr = row_first + row;
            const int qt = row < rows ? pb.by_g.div(qr) : 0, qj = row < rows ? qr - qt * g : 0;
            const __nv_bfloat16* p = q + (size_t)(it.q.row0 + qt) * pb.q_stride + (size_t)(it.h * g + qj) * d + 2 * (lane & 3);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                bq[nt][ks][0] = row < rows && ks * 16 < d ? *reinterpret_cast<const uint32_t*>(p + ks * 16) : 0u;
                bq[nt][ks][1] = row < rows && ks * 16 + 8 < d ? *reinterpret_cast<const uint32_t*>(p + ks * 16 + 8) : 0u;
                o[nt][ks][0] = o[nt][ks][1] = o[nt][ks][2] = o[nt][ks][3] = 0.f;
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                m_run[nt][c] = -INFINITY;
                l_run[nt][c] = 0.f;
            }
        }
        {                                                             // from the warp's first and last row
            const int p0 = it.q.len - it.q.n + pb.by_g.div(row_first), p1 = it.q.len - it.q.n + pb.by_g.div(max(row_first + rows - 1, 0));
            all_hi = max(p0 + 1, 0);
            all_lo = pb.window > 0 ? max(p1 + 1 - pb.window, 0) : 0;
        }

        for (int tt = 0; tt < cons.ntile; ++tt) {
            if (tw == 0) issue_one();                                 // refill the stage freed by the previous tile (a team: the one before)
            const unsigned s = consumed % S::STAGES;
            if (failed || !mbar_wait_bounded(bars + s, (consumed / S::STAGES) & 1u)) { failed = true; break; }
            ++consumed;
            const int e0 = meta[s];
            if (e0 < 0 || rows == 0) {                                // a page that does not exist; no rows for this warp
                __syncwarp();
                if (TW > 1 && lane == 0) mbar_arrive(empty + s);
                continue;
            }
            const uint32_t kbase = smem_u32(ring + s * S::STAGE), vbase = kbase + S::PLANES * S::PLANE;
            const int held = it.q.len - e0;                           // entries of the tile, if it is not full
            if (held < S::TILE) {
                for (int i = max(held, 0) * 8 + lane; i < S::TILE * 8; i += 32)
#pragma unroll
                    for (int p = 0; p < S::PLANES; ++p)
                        *reinterpret_cast<uint4*>(ring + s * S::STAGE + (S::PLANES + p) * S::PLANE + i * 16) = make_uint4(0u, 0u, 0u, 0u);
                fence_proxy_async_smem();                             // before a later copy into this stage
                __syncwarp();
            }
            // ---- S^T[entry][row] = K Q^T
            float sacc[MT][NT][4];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) sacc[mt][nt][0] = sacc[mt][nt][1] = sacc[mt][nt][2] = sacc[mt][nt][3] = 0.f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    const int row = mt * 16 + (lane & 7) + ((lane >> 3) & 1) * 8;
                    const int c = 2 * ks + (lane >> 4);
                    uint32_t a[4];
                    ldsm_x4(a, kbase + (c >> 3) * S::PLANE + row * 128 + (((c & 7) ^ (row & 7)) << 4));
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma_bf16(sacc[mt][nt], a, bq[nt][ks][0], bq[nt][ks][1]);
                }
            }
            // ---- softmax over the entries; this thread owns rows 2 (lane & 3), + 1 of each column tile.  m_ref, the
            // reference of a row's weights, is raised only when some logit exceeds it by 2^8: until then a tile needs one vote
            // and no exchange between lanes, and the weights stay below 2^8.
            const bool edge = e0 + S::TILE > all_hi || e0 < all_lo;
            float mx[NT][2];
            bool raise = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                if (edge) {                                           // rows of the column's token see entries lo .. pos
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int col = nt * 8 + 2 * (lane & 3) + c;
                        const int pos = col < rows ? it.q.len - it.q.n + pb.by_g.div(row_first + col) : -1;
                        const int lo = pb.window > 0 ? pos + 1 - pb.window : 0;
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                            for (int i = c; i < 4; i += 2) {
                                const int e = e0 + mt * 16 + (lane >> 2) + (i >> 1) * 8;
                                if (e > pos || e < lo) sacc[mt][nt][i] = -INFINITY;
                            }
                    }
                }
                mx[nt][0] = mx[nt][1] = -INFINITY;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    mx[nt][0] = fmaxf(mx[nt][0], fmaxf(sacc[mt][nt][0], sacc[mt][nt][2]));
                    mx[nt][1] = fmaxf(mx[nt][1], fmaxf(sacc[mt][nt][1], sacc[mt][nt][3]));
                }
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    mx[nt][c] *= scale_log2;                          // > 0
                    raise |= mx[nt][c] > m_run[nt][c] + W_RESCALE_STEP;
                }
            }
            if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float m = mx[nt][c];
#pragma unroll
                        for (int off = 4; off < 32; off <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
                        m = fmaxf(m, m_run[nt][c]);
                        const float f = m == -INFINITY ? 1.f : a_ex2(m_run[nt][c] - m);      // (0 the first time)
                        m_run[nt][c] = m;
                        l_run[nt][c] *= f;
#pragma unroll
                        for (int dt = 0; dt < KS; ++dt) { o[nt][dt][c] *= f; o[nt][dt][c + 2] *= f; }
                    }
            }
            uint32_t pbf[MT][NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float ref0 = m_run[nt][0] == -INFINITY ? 0.f : m_run[nt][0], ref1 = m_run[nt][1] == -INFINITY ? 0.f : m_run[nt][1];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    const float* sc = sacc[mt][nt];                   // (a row that has seen nothing: every weight is 2^-inf = 0)
                    const __nv_bfloat162 plo = __floats2bfloat162_rn(a_ex2(fmaf(sc[0], scale_log2, -ref0)), a_ex2(fmaf(sc[1], scale_log2, -ref1)));
                    const __nv_bfloat162 phi = __floats2bfloat162_rn(a_ex2(fmaf(sc[2], scale_log2, -ref0)), a_ex2(fmaf(sc[3], scale_log2, -ref1)));
                    l_run[nt][0] += __low2float(plo) + __low2float(phi);     // the sum of what the tensor cores will see
                    l_run[nt][1] += __high2float(plo) + __high2float(phi);
                    pbf[mt][nt][0] = movmatrix_trans(*reinterpret_cast<const uint32_t*>(&plo));
                    pbf[mt][nt][1] = movmatrix_trans(*reinterpret_cast<const uint32_t*>(&phi));
                }
            }
            // ---- O^T[channel][row] += V^T P^T
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
                for (int dt = 0; dt < KS; ++dt) {
                    const int row = mt * 16 + (lane & 7) + (lane >> 4) * 8;
                    const int c = 2 * dt + ((lane >> 3) & 1);
                    uint32_t a[4];
                    ldsm_x4_trans(a, vbase + (c >> 3) * S::PLANE + row * 128 + (((c & 7) ^ (row & 7)) << 4));
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma_bf16(o[nt][dt], a, pbf[mt][nt][0], pbf[mt][nt][1]);
                }
            }
            __syncwarp();                                             // all lanes are done with the stage before it is refilled
            if (TW > 1 && lane == 0) mbar_arrive(empty + s);
        }
        if (failed) break;

        // ---- the unit's result, or this worker's part of it
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float l = l_run[nt][c];
#pragma unroll
                for (int off = 4; off < 32; off <<= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
                const int col = nt * 8 + 2 * (lane & 3) + c;
                if (col >= rows) continue;
                const int dr = lane >> 2;
                if (it.slot < 0) {
                    const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
                    const int qt = pb.by_g.div(row_first + col), qj = row_first + col - qt * g;
                    __nv_bfloat16* op = out + ((size_t)(it.q.row0 + qt) * pb.Hq + (size_t)(it.h * g + qj)) * d + dr;
#pragma unroll
                    for (int dt = 0; dt < KS; ++dt) {
                        if (dt * 16 < d) op[dt * 16] = __float2bfloat16_rn(o[nt][dt][c] * inv);
                        if (dt * 16 + 8 < d) op[dt * 16 + 8] = __float2bfloat16_rn(o[nt][dt][c + 2] * inv);
                    }
                } else {
                    const size_t pr = (size_t)it.slot * unit_rows + tw * NT * 8 + col;
                    float* op = wk.part_o + pr * d + dr;
#pragma unroll
                    for (int dt = 0; dt < KS; ++dt) {
                        if (dt * 16 < d) op[dt * 16] = o[nt][dt][c];
                        if (dt * 16 + 8 < d) op[dt * 16 + 8] = o[nt][dt][c + 2];
                    }
                    if (dr == 0) { wk.part_ml[pr * 2] = m_run[nt][c]; wk.part_ml[pr * 2 + 1] = l; }
                }
            }
        if (it.slot >= 0 && (it.slot & 1) && lane == 0 && tw == 0) paged_note_shared(wk, tab, it, cons.x, w, unit_first, unit_n);
        const long long next = cons.x + it.steps;
        if (tw == 0 && prod.on && prod.x == next) cons = prod; else cons = at(next);
    }
    if (failed) {
        if (lane == 0) latch_error(pb.status, TRIMKV_E_TIMEOUT);
        while (consumed < issued) {                                   // wait (bounded) for the copies still in flight
            mbar_wait_bounded(bars + consumed % S::STAGES, (consumed / S::STAGES) & 1u);
            ++consumed;
        }
    }
}

template <int D, int NT, int TW, bool SELECT, bool EXACT>
cudaError_t run_warp(const PagedView& pv, const PagedBatch& pb, const void* q, void* out, float scale, const PagedWork& w, int max_rows,
                     cudaStream_t st) {
    using S = WarpShape<D, NT, TW>;
    static std::atomic<unsigned long long> done{0};
    cudaError_t e = paged_allow_smem(reinterpret_cast<const void*>(paged_attn_warp_kernel<D, NT, TW, SELECT, EXACT>), S::SMEM, done);
    if (e != cudaSuccess) return e;
    CUtensorMap mk, mv;
    e = paged_tensor_map(&mk, pv.k, pv, S::TILE, S::PLANES);
    if (e == cudaSuccess) e = paged_tensor_map(&mv, pv.v, pv, S::TILE, S::PLANES);
    if (e != cudaSuccess) return e;
    e = paged_launch(paged_attn_warp_kernel<D, NT, TW, SELECT, EXACT>, dim3(PAGED_SMS), dim3(S::TEAMS * TW * 32), S::SMEM, 1, true, st, mk, mv, pv, pb,
                     (const __nv_bfloat16*)q, (__nv_bfloat16*)out, scale * LOG2E, w, max_rows);
    if (e != cudaSuccess || paged_always_whole(pb, pv.H, S::ROWS, PAGED_SMS * S::TEAMS, W_JOIN_STEPS)) return e;
    return launch_paged_join(pv, pb, 1, out, w, SELECT ? pb.sub_rows : S::ROWS, PAGED_SMS * S::TEAMS, st);
}

}  // namespace

// The pages as n_pages x H x 64 rows of d bf16.  d a multiple of 64: columns cut into planes of 64, dimensions {64, rows, d / 64}; a
// box is box_rows rows of box_planes planes, each plane 128-byte swizzled, plane after plane.  Otherwise: dimensions {d, rows}, a
// box is 64 columns (those behind d are filled with zeros) of box_rows rows.
cudaError_t paged_tensor_map(CUtensorMap* map, const char* base, const PagedView& pv, int box_rows, int box_planes) {
    EncodeTiledFnA fn = a_encode_fn();
    if (!fn) return cudaErrorNotSupported;
    const cuuint64_t rows = (cuuint64_t)pv.n_pages * pv.H * PAGE, row_bytes = (cuuint64_t)pv.d * 2;
    const bool planes = pv.d % 64 == 0;
    const cuuint64_t dims[3] = {planes ? 64 : (cuuint64_t)pv.d, rows, (cuuint64_t)pv.d / 64};
    const cuuint64_t strides[2] = {row_bytes, 128};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, (cuuint32_t)box_planes};
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, planes ? 3 : 2, const_cast<char*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
               ? cudaSuccess : cudaErrorInvalidValue;
}

cudaError_t launch_paged_attention_warp(const PagedView& pv, const PagedBatch& pb, const void* q, void* out, float scale, const PagedWork& w,
                                        int tile_rows, int max_rows, cudaStream_t st) {
    auto go = [&](auto d, auto nt, auto tw) {
        constexpr int D = decltype(d)::value, NT = decltype(nt)::value, TW = decltype(tw)::value;
        if (pv.d == D)
            return pb.top > 0 ? run_warp<D, NT, TW, true, true>(pv, pb, q, out, scale, w, max_rows, st)
                              : run_warp<D, NT, TW, false, true>(pv, pb, q, out, scale, w, max_rows, st);
        return pb.top > 0 ? run_warp<D, NT, TW, true, false>(pv, pb, q, out, scale, w, max_rows, st)
                          : run_warp<D, NT, TW, false, false>(pv, pb, q, out, scale, w, max_rows, st);
    };
    auto rows = [&](auto d) {
        using One = std::integral_constant<int, 1>;
        using Two = std::integral_constant<int, 2>;
        using Four = std::integral_constant<int, 4>;
        return tile_rows <= 8 ? go(d, One{}, One{}) : tile_rows <= 16 ? go(d, Two{}, One{}) : tile_rows <= 32 ? go(d, One{}, Four{}) : go(d, Two{}, Four{});
    };
    if (pv.d <= 64) return rows(std::integral_constant<int, 64>{});
    if (pv.d <= 128) return rows(std::integral_constant<int, 128>{});
    // the accumulators of 16 rows of 256 do not fit the registers of a warp: 8 rows, or a team's 32
    using D256 = std::integral_constant<int, 256>;
    return tile_rows <= 8 ? go(D256{}, std::integral_constant<int, 1>{}, std::integral_constant<int, 1>{})
                          : go(D256{}, std::integral_constant<int, 1>{}, std::integral_constant<int, 4>{});
}

}  // namespace tkv
