// Attention over the paged cache held in 4 bits for many query rows, on tcgen05: bf16, head sizes up to 128 (padded to 64 or 128 in
// shared memory, the missing columns zero).
//
// The chunk kernel of the bf16 cache (paged_attention_tc.cu: units of 256 rows in two groups, tiles of two pages, 16 softmax warps, one issuing
// warp, the order of a worker's stretches) with another producer: one warp has the copy engine bring codes and scales of a page into a
// ring of three, eight warps turn them into fp16 (exact, see paged4.cuh) and store them where TMA would have put a bf16 tile:
// rows of 128 bytes, 128-byte swizzled, 64-column planes.  Eight neighbouring lanes take four rows and two parts, so the stores meet
// no bank conflict.  Each kind of warp has its loop in code of its own, and they divide the block's registers; the place on the line is
// kept in shared memory, since local memory has almost no cache beside it.
// Both products are fp16: Q's rows are scaled by powers of two (largest value in 2^10 .. 2^11) and P by 2^4: weights may exceed their
// reference by 2^11 before a stretch goes round again (fp16 ends at 2^16), and what is lost of a small one is 2^-29 of the reference.
// V behind a request's last entry, and pages that do not exist, are stored as zeros.
//
// What bounds it: the feed.  Beside the products' own reads a way to shared memory and back takes some 200 cycles, and a page of K or V costs a
// feeding warp several of them in turn.  4 x 512 tokens over 16K, 8 x 4 heads of 128: 622 to 660 us, 0.82 to 0.87 PFLOP/s of useful products (the bf16 cache's
// kernel, fed by TMA alone: 521).  Steps: three warps with loads of their own 1683 us, the loads of four steps in flight 1180, seven
// warps 1062, copies by the copy engine 864, the place on the line in shared memory 703, a page ahead in registers 635, barriers asked ahead 627.
#include "paged4.cuh"
#include "paged_tc.cuh"

namespace tkv {

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr int T_ROWS = 128, T_UNIT = PAGED_TC_ROWS;
constexpr int T_PLANE = PAGE * 128;                                   // 64 entries x 64 columns
constexpr int T_QPLANE = T_ROWS * 128;
constexpr int T_SOFT = 16, T_FEED = 8;                                // softmax warps; warps that make K and V; then one that copies, one that issues, two to fill the group
constexpr int T_THREADS = (T_SOFT + T_FEED + 4) * 32;
constexpr int T_REGS = 72, T_SOFT_REGS = 96, T_REST_REGS = 40;        // a thread's registers at the launch, and as the warps divide them
static_assert(T_SOFT * T_SOFT_REGS + (T_THREADS / 32 - T_SOFT) * T_REST_REGS <= T_THREADS / 32 * T_REGS, "no more than the block was launched with");
using TableMem = PagedTableMemOf<T_THREADS / 32>;
static_assert(T_SOFT % 4 == 0 && T_THREADS / 32 % 4 == 0, "registers are divided by groups of four warps");
constexpr int T_TMEM_COLS = 512;      // group g: S of page h at columns 128 g + 64 h (P over its first 32); O at 256 + 128 g
constexpr int T_POLY_EVERY = 3;
constexpr int T_JOIN_STEPS = 4;       // what a join costs, in pages
constexpr float T_RESCALE_STEP = 4.0f, T_OFFSET = 4.0f, T_LEAP = 15.0f;      // log2; weights are 2^T_OFFSET times their value, at most 2^T_LEAP
constexpr int T_STAGES = 2;           // tiles of K, and of V, in shared memory
constexpr int T_E0 = 8;               // ring of the tiles' first entries (two pages each): more than the tiles in flight
constexpr int T_NO_PAGE = INT_MAX / 2;

// The feed.  TMA brings codes and scales of a page's K or V, page after page, into a ring of T_RAW places; a step turns ROWS of its rows into fp16, 32
// channels a lane.
constexpr int T_RAW = 3;
template <int D>
struct Feed {
    static constexpr int PARTS = D / 32, ROWS = 32 / PARTS, STEPS = PAGE / ROWS, RAW = PAGE * (D / 2 + D / 16);
    static_assert(T_FEED % STEPS == 0 && T_FEED <= 2 * STEPS, "a warp has one step of a page, or of one of a tile's two");
};
// Whether the phase is over, without waiting: asked well before the answer is used, it hides the way to shared memory and back, which
// takes some 200 cycles beside the tensor cores' own reads.
__device__ __forceinline__ uint32_t t_test(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok;
}
__device__ __forceinline__ void t_bulk(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

// A worker's share of the line and the stretch of it that the block is at, in shared memory: one warp moves it on between two barriers of the block,
// the others keep none of it in registers.  The rest of a unit that another worker began comes last: the workers then begin units
// at their first page at the same time, and those of one KV head read the same pages from L2.
struct Walk {
    PagedTable tab;
    long long begin, x, end, last;            // last: end of that rest, if it was put off
    PagedItem it;
    int more;                                 // whether there is a stretch
    int careful;                              // this stretch again, every tile's maximum first
};

template <int D>
struct Tc4Shape {
    static constexpr int PLANES = D / 64;
    static constexpr int KPLANE = 2 * T_PLANE;                        // 128 entries x 64 columns
    static constexpr int TILE = PLANES * KPLANE;                      // K of a tile; V of a tile
    static constexpr int OFF_V = T_STAGES * TILE;
    static constexpr int OFF_Q = 2 * T_STAGES * TILE;
    static constexpr int OFF_BAR = OFF_Q + 2 * PLANES * T_QPLANE;
    static constexpr int OFF_E0 = OFF_BAR + 256;
    static constexpr int OFF_MX = OFF_E0 + T_E0 * 8;                  // [tile parity; 2: sums][group][page of the tile][row]: maxima so far
    static constexpr int OFF_TAB = OFF_MX + 3 * 2 * 2 * T_ROWS * 4;
    static constexpr int OFF_UP = (OFF_TAB + (int)sizeof(TableMem) + 15) & ~15;      // from a row's S to log2 units
    static constexpr int OFF_WALK = OFF_UP + T_UNIT * 4;
    static constexpr int OFF_RAW = (OFF_WALK + (int)sizeof(Walk) + 15) & ~15;
    static constexpr int SMEM = OFF_RAW + T_RAW * Feed<D>::RAW + 1024;      // 1024: alignment slack
    // D fp32, A and B fp16, M = 128.  S: both K-major, N = 64 per page.  P V: B (V) MN-major, N = D.
    static constexpr uint32_t IDESC_S1 = (1u << 4) | ((uint32_t)(64 >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
    static constexpr uint32_t IDESC_S2 = (1u << 4) | ((uint32_t)(128 >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
    static constexpr uint32_t IDESC_PV = (1u << 4) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
};

// By one warp: the first stretch, or the one behind that which is done (or the same again).
__device__ __forceinline__ void walk_on(Walk* k, bool begun, const PagedBatch& pb, const PagedWork& wk, int w, int unit_rows, volatile int* s_redo) {
    const PagedTable tab = k->tab;
    const long long begin = k->begin;
    long long x = k->x, end = k->end, last = k->last;
    PagedItem it = k->it;
    const bool again = begun && !k->careful && *s_redo;       // (a careful stretch sets no flag)
    bool more = again;
    if (begun && !again) {
        if (it.slot >= 0 && (it.slot & 1) && (threadIdx.x & 31) == 0)
            paged_note_shared(wk, tab, it, x, w, it.u * unit_rows, min(unit_rows, it.q.n * pb.g - it.u * unit_rows));
        x += it.steps;
    }
    while (!again && (x < end || last)) {
        if (x >= end) { x = begin; end = last; }
        it = paged_item<0>(tab, pb, x, end, w);
        if (x == begin && !last && it.slot == 2 * w && x + it.steps < end) { last = x += it.steps; continue; }
        if (end == last) last = 0;
        more = true;
        break;
    }
    __syncwarp();
    if ((threadIdx.x & 31) == 0) {
        k->x = x;
        k->end = end;
        k->last = last;
        k->it = it;
        k->more = more;
        k->careful = again;
        *s_redo = 0;
    }
}

template <int D>
__global__ void __launch_bounds__(T_THREADS, 1) /* T_REGS registers */
paged4_attn_tc_kernel(Paged4View cache, PagedBatch pb, const __nv_bfloat16* q, __nv_bfloat16* out, float scale_log2, PagedWork wk, int min_rows) {
    using S = Tc4Shape<D>;
    const PagedView& pv = cache.pv;
    extern __shared__ unsigned char t_smem_raw[];
    const uint32_t raw = a_smem(t_smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    unsigned char* gen = t_smem_raw + (base - raw);
    const uint32_t bars = base + S::OFF_BAR;
    const uint32_t k_full = bars, k_empty = bars + 16, v_full = bars + 32, v_empty = bars + 48 /* [stage] each */, s_ready0 = bars + 64,
                   p_ready0 = bars + 80, done0 = bars + 96 /* [group] each */, pair0 = bars + 112 /* [group][32 rows] */,
                   raw_full = bars + 176, raw_empty = bars + 200 /* [place] each */;
    volatile uint32_t* s_tmem = reinterpret_cast<volatile uint32_t*>(gen + S::OFF_BAR + 240);
    volatile int* s_fail = reinterpret_cast<volatile int*>(gen + S::OFF_BAR + 244);
    volatile int* s_real = reinterpret_cast<volatile int*>(gen + S::OFF_BAR + 224);      // [place]: rows of the page that count
    volatile int* s_redo = reinterpret_cast<volatile int*>(gen + S::OFF_BAR + 252);
    volatile int* s_e0 = reinterpret_cast<volatile int*>(gen + S::OFF_E0);
    float* s_mx = reinterpret_cast<float*>(gen + S::OFF_MX);
    TableMem* table_mem = reinterpret_cast<TableMem*>(gen + S::OFF_TAB);
    float* s_up = reinterpret_cast<float*>(gen + S::OFF_UP);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = pb.g, d = pv.d;

    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            a_bar_init(k_full + 8 * i, T_FEED);
            a_bar_init(k_empty + 8 * i, 1);
            a_bar_init(v_full + 8 * i, T_FEED);
            a_bar_init(v_empty + 8 * i, 1);
            a_bar_init(s_ready0 + 8 * i, 1);
            a_bar_init(p_ready0 + 8 * i, T_SOFT / 2);
            a_bar_init(done0 + 8 * i, 1);
        }
        for (int i = 0; i < 8; ++i) a_bar_init(pair0 + 8 * i, 2);
        for (int i = 0; i < T_RAW; ++i) { a_bar_init(raw_full + 8 * i, 1); a_bar_init(raw_empty + 8 * i, T_FEED); }
        *s_fail = 0;
        *s_redo = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    grid_dependency_wait();
    PagedTable tab;
    paged_build_table<0>(tab, pb, pv.H, T_UNIT, min_rows, INT_MAX, (int)gridDim.x, 4, T_JOIN_STEPS, table_mem);
    grid_dependents_may_launch();
    const int w = blockIdx.x;
    if (threadIdx.x == 0) paged_note_none(wk, w);
    if (w >= tab.workers) return;                                     // the whole block, before it holds tensor memory
    if (warp == T_SOFT + T_FEED + 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(a_smem((const void*)s_tmem)), "r"(T_TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    a_fence_before();
    __syncthreads();
    a_fence_after();
    const uint32_t tmem = *s_tmem;
    Walk* walk = reinterpret_cast<Walk*>(gen + S::OFF_WALK);
    if (threadIdx.x == 0) {
        walk->tab = tab;
        walk->begin = walk->x = tab.share(w);
        walk->end = tab.share(w + 1);
        walk->last = 0;
        walk->careful = 0;
    }
    __syncwarp();
    if (warp == 0) walk_on(walk, false, pb, wk, w, T_UNIT, s_redo);
    __syncthreads();
    const PagedItem& it = walk->it;
    auto stretch_done = [&]() {                                       // false: a wait gave up
        a_fence_before();
        __syncthreads();                                              // Q and tensor memory are free for the next stretch
        a_fence_after();
        if (*s_fail) return false;
        if (warp == 0) walk_on(walk, true, pb, wk, w, T_UNIT, s_redo);
        __syncthreads();
        return true;
    };
    // Tiles of the stretches before this one: of the rings, and of group 1, whose barriers rest while it has no rows; and the
    // stretches with tiles, of group 0 and 1.
    unsigned ct = 0, ct1 = 0, st0 = 0, st1 = 0;

    if (warp < T_SOFT) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(T_SOFT_REGS));
        // group, page of the tile, 32 rows of the group (a warp reaches the tensor-memory lanes of its number mod 4)
        const int grp = (warp >> 3) & 1, half = (warp >> 2) & 1, wl = warp & 3;
        const int r = wl * 32 + lane, R = grp * T_ROWS + r;           // row: lane of tensor memory, row of the unit
        unsigned ex = 0;                                              // barriers of the two warps of a row so far
        while (walk->more) {
            const bool again = walk->careful != 0;
            const int npage = it.p1 - it.p0, ntile = (npage + 1) / 2;
            const int row_first = it.u * T_UNIT, rows = min(T_UNIT, it.q.n * g - row_first);
            const bool both = rows > T_ROWS, soft = grp == 0 || both;
            const bool valid = soft && R < rows;
            const int tok = valid ? pb.by_g.div(row_first + R) : it.tok0, head = valid ? row_first + R - tok * g : 0;
            const int pos = it.q.len - it.q.n + tok;
            const int see_hi = valid ? max(pos + 1, 0) : 0;           // entries the row sees: see_lo .. see_hi - 1
            const int see_lo = valid && pb.window > 0 ? max(pos + 1 - pb.window, 0) : 0;
            if (ntile > 0) {
                if (soft) {
                    // neighbouring lanes have neighbouring 16 bytes of a row; the two warps of 32 rows take 16 each
                    constexpr int CPR = D / 8;                            // 16-byte chunks of a row
                    const int c = lane % CPR, ksh = p4_shift(cache, 0, it.h);
#pragma unroll 2
                    for (int k = 0; k < CPR / 2; ++k) {
                        const int rq = wl * 32 + half * 16 + k * (32 / CPR) + lane / CPR, row = row_first + grp * T_ROWS + rq, qt = pb.by_g.div(row);
                        const __nv_bfloat16* src = q + (size_t)(it.q.row0 + qt) * pb.q_stride + (size_t)(it.h * g + row - qt * g) * d + c * 8;
                        const uint4 v = grp * T_ROWS + rq < rows && c * 8 < d ? *reinterpret_cast<const uint4*>(src) : make_uint4(0u, 0u, 0u, 0u);
                        const uint32_t vw[4] = {v.x, v.y, v.z, v.w};
                        float top = 0.f;
#pragma unroll
                        for (int e = 0; e < 4; ++e) top = fmaxf(top, fmaxf(fabsf(__uint_as_float(vw[e] << 16)), fabsf(__uint_as_float(vw[e] & 0xffff0000u))));
#pragma unroll
                        for (int o = 1; o < CPR; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                        const int up = top > 0.f ? max(-60, min(60, 137 - (int)(__float_as_uint(top) >> 23))) : 0;
                        const float f = p4_pow2(up);
                        uint32_t w4[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) w4[e] = p4_f16x2(__uint_as_float(vw[e] << 16) * f, __uint_as_float(vw[e] & 0xffff0000u) * f);
                        *reinterpret_cast<uint4*>(gen + S::OFF_Q + (grp * S::PLANES + (c >> 3)) * T_QPLANE + rq * 128 + (((c & 7) ^ (rq & 7)) << 4)) = make_uint4(w4[0], w4[1], w4[2], w4[3]);
                        if (c == 0) s_up[grp * T_ROWS + rq] = p4_to_log2(scale_log2, ksh - up);
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // Q, before the async proxy uses it
                a_fence_before();
                asm volatile("bar.sync 1, %0;" ::"n"((T_SOFT + 1) * 32) : "memory");      // with the issuing warp
                a_fence_after();
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
                const float to_log2 = ntile > 0 ? s_up[R] : 0.f;
                const uint64_t sc2 = a_pack2(to_log2, to_log2);
                float m_used = -INFINITY, m_mine = -INFINITY, l = 0.f;    // the reference (the same in both threads), this thread's maximum, its sum
                bool ok = true;
                // entries that every row of the warp sees (rows without a query see whatever the others do); once every row has a
                // maximum, a tile of two pages in this span needs no look at the rows
                const int all_hi = __reduce_min_sync(0xffffffffu, valid ? see_hi : INT_MAX), all_lo = __reduce_max_sync(0xffffffffu, see_lo);
                bool primed = false;
                for (int i = 0; i < ntile; ++i) {
                    ok = __all_sync(0xffffffffu, a_bar_wait(s_ready0 + 8 * grp, (gt + i) & 1));
                    if (!ok) break;
                    a_fence_after();
                    // first entries of both pages (-1: the tile is one page); what the row sees of them
                    const int e0 = s_e0[(ct + i) % T_E0 * 2 + half], e1 = s_e0[(ct + i) % T_E0 * 2 + (half ^ 1)];
                    auto sees = [&](int e) {
                        return valid && e >= 0 && e < see_hi && e + PAGE > see_lo;
                    };
                    const bool inside = primed && !again && min(e0, e1) >= all_lo && max(e0, e1) + PAGE <= all_hi;      // (e1 < 0: not inside)
                    bool mine = true, some = true, edge = false, first = false;
                    if (!inside) {
                        mine = sees(e0);
                        some = __any_sync(0xffffffffu, mine);             // of the warp's rows
                        // a row that sees nothing of the page is weighed to nothing below (mref); only what lies behind the last
                        // entry has to go, it may be NaN
                        edge = mine ? e0 + PAGE > see_hi || e0 < see_lo : e0 + PAGE > it.q.len;
                        // the same for both warps of the rows: a row that has seen nothing yet finds its maximum first
                        first = again || i == 0 || __any_sync(0xffffffffu, m_used == -INFINITY && (mine || sees(e1)));
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
                                if (mine) m_mine = fmaxf(m_mine, fmaxf(mq[0], mq[1]) * to_log2);     // to_log2 > 0
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
                        const uint64_t nm2 = a_pack2(T_OFFSET - mref, T_OFFSET - mref);
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
                                pk[e >> 1] = p4_f16x2(p0, p1);
                            }
                            t_tmem_st16(s_addr + 16 * k, pk);             // P: two entries per column, over the page's first 32 columns of S
                        }
                        float a0, a1;
                        a_unpack2(a_add2(sq[0], sq[1]), a0, a1);
                        l += a0 + a1;
                        const float mx = fmaxf(mq[0], mq[1]);
                        if (mine) {
                            m_mine = fmaxf(m_mine, mref - T_OFFSET + mx);
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
                    const float v_up = p4_pow2(p4_shift(cache, 1, it.h)), inv = l > 0.f ? v_up / l : (l == 0.f ? 0.f : l);
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
                        for (int e = 0; e < 16; ++e) ov[e] = zero ? 0u : it.slot < 0 ? ov[e] : __float_as_uint(__uint_as_float(ov[e]) * v_up);
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
            if (!stretch_done()) break;
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(T_REST_REGS));      // (one instruction for the four warps of a group)
        if (warp < T_SOFT + T_FEED) {
            // ---- K and V
            // Lanes: eight neighbours store four rows and two parts, all 32 banks.
            using F = Feed<D>;
            const int fw = warp - T_SOFT, part = (lane & 1) | (F::PARTS == 4 ? lane >> 4 << 1 : 0), lrow = (lane >> 1) % F::ROWS;
            const int code_row = d / 2, scale_row = d / 16;
            const bool on = part * 32 < d;                                // not a missing column
            const uint32_t out0 = base + (fw % F::STEPS * F::ROWS + lrow) * 128 + ((part % 2 * 4) ^ (lrow & 7)) * 16;
            const uint32_t code0 = base + S::OFF_RAW + (fw % F::STEPS * F::ROWS + lrow) * code_row + (on ? part * 16 : 0), scale0 = base + S::OFF_RAW + PAGE * code_row + (fw % F::STEPS * F::ROWS + lrow) * scale_row + (on ? part * 2 : 0);
            const int row0 = fw % F::STEPS * F::ROWS;                     // this warp's step of a page; (heads of 64: of every other page)
            unsigned slot = 0, phase = 0;                                 // place in the ring of the page that is read next
            bool ok = true;
            while (walk->more) {
                const int npage = it.p1 - it.p0, ntile = (npage + 1) / 2;
                uint32_t word[4], scale;
                int real;
                auto take = [&](uint32_t (&wd)[4], uint32_t& sc, int& n) {
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(wd[0]), "=r"(wd[1]), "=r"(wd[2]), "=r"(wd[3]) : "r"(code0 + slot * F::RAW));
                    asm volatile("{\n\t.reg .b16 t;\n\tld.shared.b16 t, [%1];\n\tcvt.u32.u16 %0, t;\n\t}" : "=r"(sc) : "r"(scale0 + slot * F::RAW));
                    n = s_real[slot];
                };
                if (npage > 0) {
                    ok = __all_sync(0xffffffffu, a_bar_wait(raw_full + 8 * slot, phase));
                    take(word, scale, real);
                }
                uint32_t raw_ready = 0u, stage_ready = 0u;                // of the page behind, of the part behind
                unsigned c = ct;
                int kv = 0, h = 0, left = npage;                          // page h of K or V of tile c; pages of the tile and those behind it
#pragma unroll 1
                for (int n = 0; n < 2 * npage && ok; ++n) {
                    __syncwarp();
                    if (lane == 0) a_bar_arrive(raw_empty + 8 * slot);    // in registers
                    if (++slot == T_RAW) { slot = 0; phase ^= 1; }
                    uint32_t next[4] = {0u, 0u, 0u, 0u}, next_scale = 0u;
                    int next_real = 0;
                    if (n + 1 < 2 * npage) {
                        if (!__all_sync(0xffffffffu, raw_ready != 0u)) ok = __all_sync(0xffffffffu, a_bar_wait(raw_full + 8 * slot, phase));
                        take(next, next_scale, next_real);
                    }
                    raw_ready = t_test(raw_full + (slot + 1 == T_RAW ? 0u : 8 * (slot + 1)), slot + 1 == T_RAW ? phase ^ 1u : phase);
                    const unsigned s = c % T_STAGES;
                    if (h == 0 && c >= T_STAGES && ok && !__all_sync(0xffffffffu, stage_ready != 0u))
                        ok = __all_sync(0xffffffffu, a_bar_wait((kv ? v_empty : k_empty) + 8 * s, ((c / T_STAGES) - 1) & 1));
                    if (!ok) break;
                    const bool last_page = h == 1 || left == 1;           // of the tile
                    if (last_page) {
                        const unsigned nc = c + kv;                       // the next part: V of this tile, or K of the next
                        stage_ready = t_test((kv ? k_empty : v_empty) + 8 * (nc % T_STAGES), ((nc / T_STAGES) - 1) & 1);
                    }
                    if (F::STEPS == T_FEED || fw / F::STEPS == h) {
                        // K: a plane holds the rows of both pages; V: planes of a page, then of the next
                        const uint32_t out = out0 + s * S::TILE + (kv ? S::OFF_V + (h * S::PLANES + part / 2) * T_PLANE : part / 2 * S::KPLANE + h * T_PLANE);
                        const uint32_t sc = p4_scales(on && row0 + lrow < real ? scale : 0u), lo = p4_both_low(sc), hi = p4_both_high(sc);
#pragma unroll
                        for (int x = 0; x < 4; ++x) {                     // (chunk x lies 16 x further, but for the swizzle)
                            uint32_t r4[4];
                            p4_codes(word[x], r4);
                            const uint32_t by = x < 2 ? lo : hi;
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(out ^ (x * 16)), "r"(p4_mul(r4[0], by)), "r"(p4_mul(r4[1], by)),
                                         "r"(p4_mul(r4[2], by)), "r"(p4_mul(r4[3], by)) : "memory");
                        }
                    }
                    if (last_page) {
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                        if (lane == 0) a_bar_arrive((kv ? v_full : k_full) + 8 * s);
                        h = 0;
                        if (kv) { ++c; left -= 2; }
                        kv ^= 1;
                    } else {
                        h = 1;
                    }
#pragma unroll
                    for (int x = 0; x < 4; ++x) word[x] = next[x];
                    scale = next_scale;
                    real = next_real;
                }
                if (!ok && lane == 0) *s_fail = 1;
                ct += (unsigned)ntile;
                if (!stretch_done()) break;
            }
        } else if (warp == T_SOFT + T_FEED) {
            // ---- copies: lane l holds page l of the current run of 32
            unsigned rc = 0;
            bool ok = true;
            while (walk->more) {
                const int npage = it.p1 - it.p0, ntile = (npage + 1) / 2;
                int phys = -1;
#pragma unroll 1
                for (int i = 0; i < ntile && ok; ++i) {
                    if ((i & 15) == 0) phys = 2 * i + lane < npage ? paged_physical(pb, pv, it.r, it.p0 + 2 * i + lane) : -1;
                    const int two = 2 * i + 1 < npage, page0 = __shfl_sync(0xffffffffu, phys, (2 * i) & 31), page1 = __shfl_sync(0xffffffffu, phys, (2 * i + 1) & 31);
                    if (lane == 0) {                                      // a page that does not exist: every row masks it
                        const unsigned c = ct + i;
                        s_e0[c % T_E0 * 2] = page0 < 0 ? T_NO_PAGE : (it.p0 + 2 * i) * PAGE;
                        s_e0[c % T_E0 * 2 + 1] = !two ? -1 : page1 < 0 ? T_NO_PAGE : (it.p0 + 2 * i + 1) * PAGE;
                    }
#pragma unroll 1
                    for (int n = 0; n < 2 * (1 + two) && ok; ++n, ++rc) {
                        const int kv = n > two, p = two && (n & 1) ? page1 : page0;
                        const unsigned slot = rc % T_RAW;
                        if (rc >= T_RAW) ok = __all_sync(0xffffffffu, a_bar_wait(raw_empty + 8 * slot, ((rc / T_RAW) - 1) & 1));
                        if (!ok) break;
                        if (lane == 0) {
                            // none of a page that does not exist; of V those up to the last entry (their weights are 0, but scales may be NaN)
                            s_real[slot] = p < 0 ? 0 : kv ? it.q.len - (it.p0 + 2 * i + (two ? n & 1 : 0)) * PAGE : PAGE;
                            if (p < 0) {
                                a_bar_arrive(raw_full + 8 * slot);
                            } else {
                                const size_t row = ((size_t)p * pv.H + it.h) * PAGE;
                                const uint32_t dst = base + S::OFF_RAW + slot * Feed<D>::RAW;
                                a_bar_expect_tx(raw_full + 8 * slot, PAGE * (d / 2 + d / 16));
                                t_bulk(dst, (kv ? cache.codes[1] : cache.codes[0]) + row * (d / 2), PAGE * (d / 2), raw_full + 8 * slot);
                                t_bulk(dst + PAGE * (d / 2), (kv ? cache.scales[1] : cache.scales[0]) + row * (d / 16), PAGE * (d / 16), raw_full + 8 * slot);
                            }
                        }
                        __syncwarp();
                    }
                }
                if (!ok && lane == 0) *s_fail = 1;
                ct += (unsigned)ntile;
                if (!stretch_done()) {                                     // copies in flight land before the block leaves (bounded)
                    for (unsigned k = rc > T_RAW ? rc - T_RAW : 0; k < rc; ++k) a_bar_wait(raw_full + 8 * (k % T_RAW), (k / T_RAW) & 1);
                    break;
                }
            }
        } else if (warp > T_SOFT + T_FEED + 1) {
            while (walk->more && stretch_done()) {}
        } else {
            // ---- MMA issuer: P V of a tile, then S of the next, which overwrites that tile's P (the pipe runs in issue order), for one group
            // after the other
            while (walk->more) {
                const int npage = it.p1 - it.p0, ntile = (npage + 1) / 2;
                const bool both = min(T_UNIT, it.q.n * g - it.u * T_UNIT) > T_ROWS;
                if (ntile > 0) {
                    a_fence_before();
                    asm volatile("bar.sync 1, %0;" ::"n"((T_SOFT + 1) * 32) : "memory");      // Q is there
                    a_fence_after();
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
                    auto wait_v = [&](int i) {
                        const uint32_t c = uct + i;
                        ok = __all_sync(0xffffffffu, a_bar_wait(v_full + 8 * (c % T_STAGES), (c / T_STAGES) & 1));
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
                ct += (unsigned)ntile;
                if (both) ct1 += (unsigned)ntile;
                if (!stretch_done()) break;
            }
        }
    }
    __syncthreads();
    if (warp == T_SOFT + T_FEED + 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(T_TMEM_COLS) : "memory");
    if (threadIdx.x == 0 && *s_fail) latch_error(pb.status, TRIMKV_E_TIMEOUT);
}

template <int D>
cudaError_t run_tc4(const Paged4View& c, const PagedBatch& pb, const void* q, void* out, float scale, const PagedWork& w, int min_rows, cudaStream_t st) {
    using S = Tc4Shape<D>;
    static_assert(S::SMEM <= 227 * 1024, "shared memory of one SM");
    static std::atomic<unsigned long long> done{0};
    cudaError_t e = paged_allow_smem(reinterpret_cast<const void*>(paged4_attn_tc_kernel<D>), S::SMEM, done);
    if (e != cudaSuccess) return e;
    e = paged_launch(paged4_attn_tc_kernel<D>, dim3(PAGED_SMS), dim3(T_THREADS), S::SMEM, 1, true, st, c, pb, (const __nv_bfloat16*)q, (__nv_bfloat16*)out, scale * LOG2E, w,
                     min_rows);
    if (e != cudaSuccess || paged_always_whole(pb, c.pv.H, T_UNIT, PAGED_SMS, T_JOIN_STEPS)) return e;
    return launch_paged_join(c.pv, pb, 1, out, w, T_UNIT, PAGED_SMS, st);
}

}  // namespace

cudaError_t launch_paged4_attention_tc(const Paged4View& c, const PagedBatch& pb, const void* q, void* out, float scale, const PagedWork& w, int min_rows,
                                       cudaStream_t st) {
    return c.pv.d <= 64 ? run_tc4<64>(c, pb, q, out, scale, w, min_rows, st) : run_tc4<128>(c, pb, q, out, scale, w, min_rows, st);
}

}  // namespace tkv
