// Attention over the paged cache held in 4 bits, for few query rows (and for fp32 and head sizes above 128, any number).
//
// One CTA per SM.  Its warps are independent, each with a ring of its own in shared memory and an equal share of the line of page steps
// (paged.cuh); one or two more walk those shares for them, a lane for each warp: they describe a page, then have the copy engine
// bring its codes and scales.  A computing warp forms S^T = K Q^T and O^T += V^T P^T with mma.sync m16n8k16 in fp16, 32 entries at a
// time, the (token, head) rows as the N dimension: fp16 holds every value of the cache exactly (paged4.cuh), and Q once each row
// is scaled by a power of two (its largest value in 2^10 .. 2^11; what is lost of the smallest ones is 2^-35 of the largest).  fp32:
// Q and P in two fp16 parts each, 2^-22 relative, and the sums of 32 entries apart.
//
// The operands are made in registers.  K (A operand, rows = entries): a thread takes d / 4 neighbouring channels of an entry, so the order of
// channels along k is a permutation, which Q follows; a word of codes is the A registers of two products.  V (A operand, rows =
// channels): a thread takes d / 8 neighbouring channels of entries in pairs, and three-input logic puts the codes of one channel
// of two entries into a byte, which one conversion makes the register.  Each register is then multiplied by its scale (of two entries for V).
// 16 entries of heads of 128 cost a warp 270 instructions, 122 of them on the ALU (64 conversions) and 95 on the FMA pipe (64 products
// with scales).
//
// What bounds it: 302 MB of a decode step (8 requests of 32 K, 8 x 4 heads of 128) take 73 us, 16 of which no length changes (launch, table of
// requests, first pages, join) and the rest 5.3 TB/s, 0.8 of the copy rate; without the conversions, or without the products with
// scales, it takes 9 us less.  Steps: 8 warps that fetch for themselves 121 us, 16 of them 100, head size known at compile time 82, 11 warps fed by
// another 77.6, 14 fed by two 77.1, descriptions ahead of the copies and a join of 296 blocks 74.5.
//
// The reference of a row's weights lags its maximum by up to 2^8, and weights are 2^7 times their value: at most 2^15, and what
// fp16 cannot hold is below 2^-32 of the row's largest weight.
// Entries behind the request's last one: any code is finite, so only their scales are put to zero (for V; K's products are masked).
// Every wait is bounded and, where a whole warp computes, voted on: on expiry the warp leaves as a whole, latches TRIMKV_E_TIMEOUT and returns;
// those that bring tiles once their copies have landed.
#include "async_copy.cuh"
#include "mma_sync.cuh"
#include "paged4.cuh"
#include "tcgen05_attn.cuh"

namespace tkv {

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr unsigned W4_IDLE_LIMIT = 1u << 22, W4_NAP = 20;             // rounds without progress, and ns between them
// Pages up to which units stay whole (paged_choose_whole), and up to which a table's width alone tells the host that no join is needed, whose launch is 3.5 us.
// A lone warp takes 1.75 us a page.  16 against 4, us: 9 pages 20.9, 19.5 (32 requests of 8 heads of 128), 19.7, 24.2 (64, heads of 64), 28.3, 29.7
// (32 x 5 tokens); 16 pages 33.2, 21.5; 30.6, 26.2; 44.9, 39.4; and 33.0, 16.6 for 8 requests.  So it is kind to many requests and dear to few.
constexpr int W4_JOIN_STEPS = 16;
constexpr float W4_RESCALE_STEP = 8.0f, W4_OFFSET = 7.0f;             // log2: how far the reference may lag; what the weights are scaled by

// A tile that a warp is to read, and the stretch of a unit that it belongs to.
constexpr int W4_AHEAD = 4, W4_MOST_STAGES = 4;                       // pages that are described to a warp at most; places of its ring
constexpr int TILE_FIRST = 1, TILE_LAST = 2, TILE_END = 4;            // of the stretch; nothing more to do
struct __align__(16) Tile4 {
    int e0, flags;                                                    // first entry
    int real;                                                         // whether there is something to read; written last, with the copy
    int row0, n, len, row_first, rows, h, slot;                       // see PagedItem, paged_unit_first, paged_unit_rows
    int pad[2];
};

template <int D, int NT, bool F32>
struct Warp4Shape {
    // Warps that bring tiles, and those that compute.  As the registers allow: 128 a thread with 16 in all, 168 with 12, 255 with 8.  One warp feeds
    // up to 11 in time (a page costs it some 500 cycles).
    static constexpr int FEED = D <= 128 && NT == 1 && !F32 ? 2 : 1;
    static constexpr int WARPS = (D > 128 || F32 ? 8 : NT == 2 ? 12 : 16) - FEED;
    static constexpr int EACH = (WARPS + FEED - 1) / FEED;            // warps that one feeds
    static constexpr int ROWS = NT * 8;                               // rows of a unit
    static constexpr int STEP = 32;                                   // entries that are worked on at a time
    // A place of a ring holds a page's codes and scales of K and of V, or, where that leaves too few places, of one of them.
    static constexpr bool WHOLE = D <= 128 && (NT > 1 || F32);
    static constexpr int HALF = PAGE * (D / 2 + D / 16), STAGE = WHOLE ? 2 * HALF : HALF;
    static constexpr int MOST = WHOLE ? W4_MOST_STAGES - 1 : W4_MOST_STAGES;
    static constexpr int STAGES = 208 * 1024 / WARPS / STAGE < MOST ? 208 * 1024 / WARPS / STAGE : MOST;
    static_assert(STAGES >= (WHOLE ? 2 : 3) && (WHOLE ? STAGES : (STAGES + 1) / 2) + 1 <= W4_AHEAD, "a description stays while its page is in the ring");
    static constexpr int OFF_BAR = WARPS * STAGES * STAGE;
    static constexpr int OFF_TOLD = OFF_BAR + WARPS * STAGES * 16;    // pages described to each warp
    static constexpr int OFF_DESC = (OFF_TOLD + WARPS * 4 + 15) & ~15;
    static constexpr int OFF_TAB = OFF_DESC + WARPS * W4_AHEAD * (int)sizeof(Tile4);
    static constexpr int SMEM = OFF_TAB + (int)sizeof(PagedTableMem) + 128;       // 128: alignment slack
    static_assert(SMEM <= 227 * 1024, "shared memory of one SM");
    static_assert(WARPS * ROWS * PAGED_SMS <= P4_WORKER_ROWS, "the workspace holds the workers' partial results");
};

__device__ __forceinline__ void w4_mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ bool w4_test(uint64_t* bar, uint32_t parity) {      // whether the phase is over, without waiting
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity) : "memory");
    return ok != 0;
}
// For the whole warp, whose lanes agree on the answer.  (The first try mostly does, and needs no loop with lanes that leave it apart.)
__device__ __forceinline__ bool w4_wait(uint64_t* bar, uint32_t parity) {
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    return __all_sync(0xffffffffu, mbar_wait_bounded(bar, parity));
}
// Entry that row r (0 .. 15) of a product's 16 stands for: neighbours and every second row fall on both halves of the 32 banks.
__device__ __forceinline__ int w4_entry(int r) { return r ^ ((r >> 1) & 1); }
template <int BYTES>
__device__ __forceinline__ void w4_load(uint32_t* w, const unsigned char* p) {
    if constexpr (BYTES == 4) w[0] = *reinterpret_cast<const uint32_t*>(p);
    if constexpr (BYTES == 8) { const uint2 v = *reinterpret_cast<const uint2*>(p); w[0] = v.x; w[1] = v.y; }
    if constexpr (BYTES == 16) { const uint4 v = *reinterpret_cast<const uint4*>(p); w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w; }
}
__device__ __forceinline__ float w4_exp2(float x, std::false_type) { return a_ex2(x); }
__device__ __forceinline__ float w4_exp2(float x, std::true_type) { return exp2f(x); }
__device__ __forceinline__ void w4_load8(float (&v)[8], const __nv_bfloat16* p) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t w = reinterpret_cast<const uint32_t*>(&u)[i >> 1];
        v[i] = __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
    }
}
__device__ __forceinline__ void w4_load8(float (&v)[8], const float* p) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void w4_store8(__nv_bfloat16* p, const float (&v)[8]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}
__device__ __forceinline__ void w4_store8(float* p, const float (&v)[8]) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}

// EXACT: the head size is D; otherwise smaller, a multiple of 32.  T: type of q and out.
template <int D, int NT, bool EXACT, typename T>
__global__ void __launch_bounds__((Warp4Shape<D, NT, sizeof(T) == 4>::WARPS + Warp4Shape<D, NT, sizeof(T) == 4>::FEED) * 32, 1)
paged4_attn_warp_kernel(Paged4View cache, PagedBatch pb, const T* q, T* out, float scale_log2, PagedWork wk, int max_rows) {
    using S = Warp4Shape<D, NT, sizeof(T) == 4>;
    constexpr bool F32 = sizeof(T) == 4;
    using Exact = std::integral_constant<bool, F32>;
    constexpr int KS = D / 16, MT = S::STEP / 16, PARTS = F32 ? 2 : 1;
    constexpr int KW = D / 32, VW = D / 64;                           // words of codes that a thread takes of an entry's K, and of its V
    extern __shared__ unsigned char w4_smem_raw[];
    unsigned char* smem = w4_smem_raw + ((128u - (smem_u32(w4_smem_raw) & 127u)) & 127u);
    const PagedView& pv = cache.pv;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = pb.g, d = EXACT ? D : pv.d, gq = lane >> 2, tq = lane & 3;
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + S::OFF_BAR);      // [warp][stage]
    uint64_t* empty = full + S::WARPS * S::STAGES;
    volatile unsigned* told = reinterpret_cast<volatile unsigned*>(smem + S::OFF_TOLD);
    Tile4* desc = reinterpret_cast<Tile4*>(smem + S::OFF_DESC);
    PagedTableMem* table_mem = reinterpret_cast<PagedTableMem*>(smem + S::OFF_TAB);
    const int code_row = d / 2, scale_row = d / 16;
    const int off_scale = PAGE * code_row;                            // within a stage

    if (threadIdx.x < S::WARPS * S::STAGES) { mbar_init(full + threadIdx.x, 1); mbar_init(empty + threadIdx.x, 1); }
    if (threadIdx.x < S::WARPS) told[threadIdx.x] = 0u;
    fence_proxy_async_smem();
    grid_dependency_wait();
    PagedTable tab;
    paged_build_table<0>(tab, pb, pv.H, S::ROWS, 1, max_rows, (int)gridDim.x * S::WARPS, 4, W4_JOIN_STEPS, table_mem);      // (synchronises the block)
    grid_dependents_may_launch();
    if (warp >= S::WARPS) {
        // ---- the warps that bring tiles: each lane those of one warp, at a place of its own on the line
        const int c = (warp - S::WARPS) * S::EACH + lane;
        bool done = lane >= S::EACH || c >= S::WARPS;
        const int w = c * (int)gridDim.x + (int)blockIdx.x;           // workers are spread over the SMs first
        if (!done) paged_note_none(wk, w);
        const long long end = !done && w < tab.workers ? tab.share(w + 1) : 0;
        long long x = !done && w < tab.workers ? tab.share(w) : 0;
        PagedItem it;
        int ntile = 0, tile = 0, entry = -1, phys = -1;               // entry: the table's, on its way
        auto table_entry = [&](int page) { return page < pb.W ? pb.table[(size_t)it.r * pb.W + page] : -1; };
        auto begin = [&]() {                                          // the stretch at x
            it = paged_item<0>(tab, pb, x, end, w);
            tile = 0;
            ntile = it.p1 - it.p0;
            entry = ntile ? table_entry(it.p0) : -1;
        };
        if (x < end) begin();
        // Part p is K (p even) or V of page p / 2, or page p where a place holds both, and lies in place p mod STAGES of the ring.
        unsigned n = 0, part = 0, place = 0, parity = 1, idle = 0;    // page; (the first round of a ring finds it empty)
        while (__any_sync(0xffffffffu, !done)) {
            const unsigned at = (done ? 0 : c) * S::STAGES + place;
            const bool go = !done && (part < (unsigned)S::STAGES || w4_test(empty + at, parity));
            if (go) {
                Tile4* t = desc + c * W4_AHEAD + n % W4_AHEAD;
                const int kv = S::WHOLE ? 0 : part & 1;
                const bool last = tile + 1 >= ntile;
                if (!kv) {
                    if (x >= end) {
                        t->flags = TILE_END;
                        done = true;
                    } else {
                        t->e0 = (it.p0 + tile) * PAGE;
                        t->flags = (tile == 0 ? TILE_FIRST : 0) | (last ? TILE_LAST : 0);
                        if (tile == 0 || last) {                      // (at the first page all of it is read, at the last where the result goes)
                            t->row0 = it.q.row0; t->n = it.q.n; t->len = it.q.len;
                            t->row_first = paged_unit_first<0>(pb, it.u, S::ROWS);
                            t->rows = paged_unit_rows<0>(pb, it.u, it.q.n, S::ROWS);
                            t->h = it.h; t->slot = it.slot;
                        }
                    }
                    __threadfence_block();
                    told[c] = n + 1;
                    if (!done) {
                        phys = entry >= 0 && entry < pv.n_pages ? entry : -1;
                        if (phys < 0 && ntile > 0) latch_error(pb.status, TRIMKV_E_ARG);
                        t->real = phys >= 0;
                    }
                }
                if (!done) {
                    if (phys < 0) {
                        mbar_arrive(full + at);
                    } else {
                        unsigned char* dst = smem + (size_t)at * S::STAGE;
                        const size_t row = ((size_t)phys * pv.H + it.h) * PAGE;
                        // (the zeroing of scales below carries its own proxy fence)
                        mbar_expect_tx(full + at, (S::WHOLE ? 2 : 1) * PAGE * (code_row + scale_row));
                        bulk_g2s(dst, (kv ? cache.codes[1] : cache.codes[0]) + row * code_row, off_scale, full + at);
                        bulk_g2s(dst + off_scale, (kv ? cache.scales[1] : cache.scales[0]) + row * scale_row, PAGE * scale_row, full + at);
                        if (S::WHOLE) {
                            bulk_g2s(dst + S::HALF, cache.codes[1] + row * code_row, off_scale, full + at);
                            bulk_g2s(dst + S::HALF + off_scale, cache.scales[1] + row * scale_row, PAGE * scale_row, full + at);
                        }
                    }
                    if (kv || S::WHOLE) {                             // what comes next
                        ++n;
                        if (tile == 0 && it.slot >= 0 && (it.slot & 1))
                            paged_note_shared(wk, tab, it, x, w, paged_unit_first<0>(pb, it.u, S::ROWS), paged_unit_rows<0>(pb, it.u, it.q.n, S::ROWS));
                        if (++tile >= ntile) {
                            x += it.steps;
                            if (x < end) begin();
                        } else {
                            entry = table_entry(it.p0 + tile);
                        }
                    }
                    ++part;
                    if (++place == S::STAGES) { place = 0; parity ^= 1u; }
                }
            }
            if (__any_sync(0xffffffffu, go)) idle = 0;
            else if (++idle > W4_IDLE_LIMIT) break;
            else __nanosleep(W4_NAP);
        }
        if (!done) latch_error(pb.status, TRIMKV_E_TIMEOUT);          // a warp gave up
        // The copies in flight land before this warp leaves (bounded), also where all were issued: the warp that wants them may have given up.
        for (unsigned k = part > S::STAGES ? part - S::STAGES : 0; k < part; ++k) mbar_wait_bounded(full + c * S::STAGES + k % S::STAGES, (k / S::STAGES) & 1u);
        return;
    }

    // ---- the warps that compute
    const unsigned char* ring = smem + (size_t)warp * S::STAGES * S::STAGE;
    full += warp * S::STAGES;
    empty += warp * S::STAGES;
    desc += warp * W4_AHEAD;
    // this thread's places in a tile: codes and scales of K (entry of row gq, channels tq d / 4 ..), of V (entries of rows 2 tq and + 1, channels gq d / 8 ..)
    const int k_codes = w4_entry(gq) * code_row + tq * (D / 8), k_scales = off_scale + w4_entry(gq) * scale_row + tq * (D / 64);
    const int v_codes[2] = {w4_entry(2 * tq) * code_row + gq * (D / 16), w4_entry(2 * tq + 1) * code_row + gq * (D / 16)};
    const int v_scales[2] = {off_scale + w4_entry(2 * tq) * scale_row + gq * D / 128, off_scale + w4_entry(2 * tq + 1) * scale_row + gq * D / 128};
    int row_first = 0, rows = 0, pos0 = 0, len = 0, all_lo = 0, all_hi = 0, all_end = 0;       // of the stretch; pos0: position of its request's first token

    uint32_t bq[NT][PARTS][KS][2];
    float o[NT][KS][4];
    float m_run[NT][2], l_run[NT][2], to_log2[NT][2];

    unsigned stage = 0, parity = 0;
    bool ok = true;
    for (unsigned tile_n = 0;; ++tile_n) {
        for (unsigned k = 0; (ok = (int)(told[warp] - tile_n) > 0) == false && k < W4_IDLE_LIMIT; ++k) __nanosleep(W4_NAP);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        __syncwarp();                                                 // the description is read after the count
        const Tile4& it = desc[tile_n % W4_AHEAD];
        const int flags = it.flags, e0 = it.e0;
        if (flags & TILE_END) return;
        if (flags & TILE_FIRST) {
            row_first = it.row_first;
            rows = it.rows;
            len = it.len;
            pos0 = it.len - it.n;
            const int ksh = p4_shift(cache, 0, it.h);
            // ---- Q fragments (B operand: k = channel, n = row): row gq of a column tile, channels tq d / 4 ..
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int row = nt * 8 + gq, qr = row_first + row;
                const int qt = row < rows ? pb.by_g.div(qr) : 0, qj = row < rows ? qr - qt * g : 0;
                const T* p = q + (size_t)(it.row0 + qt) * pb.q_stride + (size_t)(it.h * g + qj) * d + tq * (D / 4);
                float top = 0.f;
                auto load = [&](float (&v)[8], int c) {
                    if (row < rows && tq * (D / 4) + c < d) w4_load8(v, p + c);
                    else
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = 0.f;
                };
#pragma unroll
                for (int c = 0; c < D / 4; c += 8) {
                    float v[8];
                    load(v, c);
#pragma unroll
                    for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(v[e]));
                }
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                const int up = top > 0.f ? max(-60, min(60, 137 - (int)(__float_as_uint(top) >> 23))) : 0;
                const float f = p4_pow2(up);
#pragma unroll
                for (int c = 0; c < D / 4; c += 8) {
                    float v[8];
                    load(v, c);
#pragma unroll
                    for (int e = 0; e < 8; e += 2) {
                        const float x0 = v[e] * f, x1 = v[e + 1] * f;
                        const uint32_t hi = p4_f16x2(x0, x1);
                        bq[nt][0][c / 4 + e / 4][(e >> 1) & 1] = hi;
                        if constexpr (F32) {
                            const float2 b = p4_float2(hi);
                            bq[nt][1][c / 4 + e / 4][(e >> 1) & 1] = p4_f16x2(x0 - b.x, x1 - b.y);
                        }
                    }
                }
                const float back = p4_to_log2(scale_log2, ksh - up);      // of row gq; this thread's columns are 2 tq, + 1
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    to_log2[nt][c] = __shfl_sync(0xffffffffu, back, (2 * tq + c) * 4);
                    m_run[nt][c] = -INFINITY;
                    l_run[nt][c] = 0.f;
                }
#pragma unroll
                for (int dt = 0; dt < KS; ++dt) o[nt][dt][0] = o[nt][dt][1] = o[nt][dt][2] = o[nt][dt][3] = 0.f;
            }
            // entries that every row of the unit sees, from its first and last row
            all_hi = max(pos0 + pb.by_g.div(row_first) + 1, 0);
            all_end = pos0 + pb.by_g.div(row_first + rows - 1) + 1;        // none sees an entry from here on
            all_lo = pb.window > 0 ? max(all_end - pb.window, 0) : 0;
        }

        ok = w4_wait(full + stage, parity);
        if (!ok) break;
        const unsigned k_stage = stage;
        if (!S::WHOLE && ++stage == S::STAGES) { stage = 0; parity ^= 1u; }
        const unsigned char* k_tile = ring + k_stage * S::STAGE;
        unsigned char* v_tile = const_cast<unsigned char*>(ring) + stage * S::STAGE + (S::WHOLE ? S::HALF : 0);
        bool v_here = false;
        const bool any = it.real != 0;
#pragma unroll 1
        for (int at = 0; at < PAGE; at += S::STEP) {
            const int es = e0 + at;                                   // entries es .. es + 31
            const bool work = any && es < all_end;
            float sacc[MT][NT][4];
            if (work) {
                const unsigned char *kc = k_tile + k_codes + at * code_row, *ks_at = k_tile + k_scales + at * scale_row;
                // ---- S^T[entry][row] = K Q^T
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) sacc[mt][nt][0] = sacc[mt][nt][1] = sacc[mt][nt][2] = sacc[mt][nt][3] = 0.f;
                    uint32_t kw[2][KW], ks[2][(KW + 3) / 4 * 2];           // rows gq and gq + 8: codes; scales, both halves of a register alike
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const unsigned char* cp = kc + (mt * 16 + i * 8) * code_row;
                        const unsigned char* sp = ks_at + (mt * 16 + i * 8) * scale_row;
#pragma unroll
                        for (int c = 0; c < KW; c += 4) {                 // (KW = 2 for heads of 64)
                            uint32_t two = 0u;
                            if (EXACT || tq * (D / 4) + c * 8 < d) {
                                w4_load<KW == 2 ? 8 : 16>(&kw[i][c], cp + c * 4);
                                two = KW == 2 ? (uint32_t)sp[0] : (uint32_t)*reinterpret_cast<const uint16_t*>(sp + c / 2);
                            } else                                        // missing channels: Q has zeros there
#pragma unroll
                                for (int x = 0; x < 4 && c + x < KW; ++x) kw[i][c + x] = 0u;
                            const uint32_t sc = p4_scales(two);
                            ks[i][c / 2] = p4_both_low(sc);
                            if (KW > 2) ks[i][c / 2 + 1] = p4_both_high(sc);
                        }
                    }
#pragma unroll
                    for (int x = 0; x < KW; ++x) {                        // a word of each row: two products
                        uint32_t r0[4], r1[4];
                        p4_codes(kw[0][x], r0);
                        p4_codes(kw[1][x], r1);
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            uint32_t a[4];
                            a[0] = p4_mul(r0[2 * j], ks[0][x / 2]);
                            a[1] = p4_mul(r1[2 * j], ks[1][x / 2]);
                            a[2] = p4_mul(r0[2 * j + 1], ks[0][x / 2]);
                            a[3] = p4_mul(r1[2 * j + 1], ks[1][x / 2]);
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                for (int part = 0; part < PARTS; ++part) w4_mma(sacc[mt][nt], a, bq[nt][part][2 * x + j][0], bq[nt][part][2 * x + j][1]);
                        }
                    }
                }
            }
            if (!S::WHOLE && at + S::STEP >= PAGE) {                  // K is done with
                __syncwarp();
                if (lane == 0) mbar_arrive(empty + k_stage);
            }
            if (!v_here) {
                if (!S::WHOLE) ok = w4_wait(full + stage, parity);
                if (!ok) break;
                v_here = true;
                const int held = len - e0;                            // entries of the page, if it is not full
                if (any && held < PAGE) {
                    for (int i = max(held, 0) * scale_row + lane; i < PAGE * scale_row; i += 32) v_tile[off_scale + i] = 0;
                    fence_proxy_async_smem();                         // before a later copy into this stage
                    __syncwarp();
                }
            }
            if (!work) continue;
            const unsigned char *vc0 = v_tile + v_codes[0] + at * code_row, *vc1 = v_tile + v_codes[1] + at * code_row, *vs0 = v_tile + v_scales[0] + at * scale_row,
                                *vs1 = v_tile + v_scales[1] + at * scale_row;
            // ---- softmax over the entries; this thread owns rows 2 tq, + 1 of each column tile.  The reference of a row's
            // weights is raised only when some logit exceeds it by 2^8: until then a tile needs one vote and no exchange.
            const bool edge = es + S::STEP > all_hi || es < all_lo;
            float mx[NT][2];
            bool raise = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                if (edge) {                                           // rows of the column's token see entries lo .. pos
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int col = nt * 8 + 2 * tq + c;
                        const int pos = col < rows ? pos0 + pb.by_g.div(row_first + col) : -1;
                        const int lo = pb.window > 0 ? pos + 1 - pb.window : 0;
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                            for (int i = c; i < 4; i += 2) {
                                const int e = es + mt * 16 + w4_entry(gq) + (i >> 1) * 8;
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
                    mx[nt][c] *= to_log2[nt][c];                      // > 0
                    raise |= mx[nt][c] > m_run[nt][c] + W4_RESCALE_STEP;
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
                        const float f = m == -INFINITY ? 1.f : w4_exp2(m_run[nt][c] - m, Exact{});      // (0 the first time)
                        m_run[nt][c] = m;
                        l_run[nt][c] *= f;
#pragma unroll
                        for (int dt = 0; dt < KS; ++dt) { o[nt][dt][c] *= f; o[nt][dt][c + 2] *= f; }
                    }
            }
            uint32_t pf[MT][NT][PARTS][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                // (a row that has seen nothing: every weight is 2^-inf = 0)
                const float ref0 = m_run[nt][0] == -INFINITY ? 0.f : W4_OFFSET - m_run[nt][0], ref1 = m_run[nt][1] == -INFINITY ? 0.f : W4_OFFSET - m_run[nt][1];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    const float* sc = sacc[mt][nt];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float p0 = w4_exp2(fmaf(sc[2 * i], to_log2[nt][0], ref0), Exact{}), p1 = w4_exp2(fmaf(sc[2 * i + 1], to_log2[nt][1], ref1), Exact{});
                        l_run[nt][0] += p0;
                        l_run[nt][1] += p1;
                        const uint32_t hi = p4_f16x2(p0, p1);
                        pf[mt][nt][0][i] = movmatrix_trans(hi);
                        if constexpr (F32) {
                            const float2 b = p4_float2(hi);
                            pf[mt][nt][PARTS - 1][i] = movmatrix_trans(p4_f16x2(p0 - b.x, p1 - b.y));
                        }
                    }
                }
            }
            // ---- O^T[channel][row] += V^T P^T: this thread's channels are gq d / 8 .., its entries 2 tq, 2 tq + 1 and 8 further
            const bool v_on = EXACT || gq * (D / 8) < d;              // otherwise these channels are missing: nothing is written from them
            float acc[F32 ? NT : 1][F32 ? KS : 1][4];
            if constexpr (F32)
#pragma unroll
                for (int i = 0; i < NT * KS * 4; ++i) (&acc[0][0][0])[i] = 0.f;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                uint32_t a[2][VW], b[2][VW], sp[2][(VW + 1) / 2];     // rows 2 tq + 8 i, and 2 tq + 8 i + 1: codes; scales of both
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (v_on) {
                        w4_load<VW * 4>(a[i], vc0 + (mt * 16 + i * 8) * code_row);
                        w4_load<VW * 4>(b[i], vc1 + (mt * 16 + i * 8) * code_row);
                    } else
#pragma unroll
                        for (int x = 0; x < VW; ++x) a[i][x] = b[i][x] = 0u;
#pragma unroll
                    for (int x = 0; x < (VW + 1) / 2; ++x) {
                        const uint32_t s0 = v_on ? vs0[(mt * 16 + i * 8) * scale_row + x] : 0, s1 = v_on ? vs1[(mt * 16 + i * 8) * scale_row + x] : 0;
                        sp[i][x] = p4_scales(__byte_perm(s0, s1, 0x0040));
                    }
                }
#pragma unroll
                for (int x = 0; x < VW; ++x) {
                    uint32_t r[4][4];                                 // even channels of both entries, odd ones; the same 8 entries on
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        p4_codes((a[i][x] & 0x0f0f0f0fu) | ((b[i][x] << 4) & 0xf0f0f0f0u), r[2 * i]);
                        p4_codes(((a[i][x] >> 4) & 0x0f0f0f0fu) | (b[i][x] & 0xf0f0f0f0u), r[2 * i + 1]);
                    }
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const uint32_t af[4] = {p4_mul(r[0][c], sp[0][x / 2]), p4_mul(r[1][c], sp[0][x / 2]), p4_mul(r[2][c], sp[1][x / 2]), p4_mul(r[3][c], sp[1][x / 2])};
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int part = 0; part < PARTS; ++part) {
                                if constexpr (F32) w4_mma(acc[nt][4 * x + c], af, pf[mt][nt][part][0], pf[mt][nt][part][1]);
                                else w4_mma(o[nt][4 * x + c], af, pf[mt][nt][part][0], pf[mt][nt][part][1]);
                            }
                    }
                }
            }
            if constexpr (F32)                                        // a tile's sum apart: short chains
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int dt = 0; dt < KS; ++dt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[nt][dt][i] += acc[nt][dt][i];
        }
        if (!ok) break;
        const int row0 = it.row0, h = it.h, slot = it.slot;
        __syncwarp();                                                 // all lanes are done with V, and with the description
        if (lane == 0) mbar_arrive(empty + stage);
        if (++stage == S::STAGES) { stage = 0; parity ^= 1u; }
        if (!(flags & TILE_LAST)) continue;

        // ---- the unit's result, or this worker's part of it.  o[nt][4 x + b]: channels 8 x + 2 b (c) and + 1 (c + 2) of the thread's
        const float v_up = p4_pow2(p4_shift(cache, 1, h));
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float l = l_run[nt][c];
#pragma unroll
                for (int off = 4; off < 32; off <<= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
                const int col = nt * 8 + 2 * tq + c;
                if (col >= rows) continue;
                const float f = slot < 0 ? (l > 0.f ? v_up / l : (l == 0.f ? 0.f : l)) : v_up;
                const int qt = pb.by_g.div(row_first + col), qj = row_first + col - qt * g;
                T* op = out + ((size_t)(row0 + qt) * pb.Hq + (size_t)(h * g + qj)) * d + gq * (D / 8);
                const size_t pr = (size_t)(slot < 0 ? 0 : slot) * S::ROWS + col;
                float* po = wk.part_o + pr * d + gq * (D / 8);
                if (gq * (D / 8) < d) {
#pragma unroll
                    for (int x = 0; x < VW; ++x) {
                        float v[8];
#pragma unroll
                        for (int b = 0; b < 4; ++b) {
                            v[2 * b] = o[nt][4 * x + b][c] * f;
                            v[2 * b + 1] = o[nt][4 * x + b][c + 2] * f;
                        }
                        if (slot < 0) w4_store8(op + 8 * x, v);
                        else w4_store8(po + 8 * x, v);
                    }
                }
                if (slot >= 0 && gq == 0) { wk.part_ml[pr * 2] = m_run[nt][c]; wk.part_ml[pr * 2 + 1] = l; }
            }
    }
    if (!ok && lane == 0) latch_error(pb.status, TRIMKV_E_TIMEOUT);   // (who brings the tiles waits for the copies in flight)
}

template <int D, int NT, bool EXACT, typename T>
cudaError_t run_warp4(const Paged4View& c, const PagedBatch& pb, const void* q, void* out, float scale, const PagedWork& w, int max_rows, cudaStream_t st) {
    using S = Warp4Shape<D, NT, sizeof(T) == 4>;
    static std::atomic<unsigned long long> done{0};
    cudaError_t e = paged_allow_smem(reinterpret_cast<const void*>(paged4_attn_warp_kernel<D, NT, EXACT, T>), S::SMEM, done);
    if (e != cudaSuccess) return e;
    e = paged_launch(paged4_attn_warp_kernel<D, NT, EXACT, T>, dim3(PAGED_SMS), dim3((S::WARPS + S::FEED) * 32), S::SMEM, 1, true, st, c, pb, (const T*)q, (T*)out, scale * LOG2E, w,
                     max_rows);
    if (e != cudaSuccess || paged_always_whole(pb, c.pv.H, S::ROWS, PAGED_SMS * S::WARPS, W4_JOIN_STEPS)) return e;
    return launch_paged_join(c.pv, pb, sizeof(T) == 2, out, w, S::ROWS, PAGED_SMS * S::WARPS, st, NT == 1 ? PAGED_SMS * 2 : 0);
}

}  // namespace

cudaError_t launch_paged4_attention_warp(const Paged4View& c, const PagedBatch& pb, int is_bf16, const void* q, void* out, float scale, const PagedWork& w,
                                         int tile_rows, int max_rows, cudaStream_t st) {
    auto go = [&](auto d, auto nt) {
        constexpr int D = decltype(d)::value, NT = decltype(nt)::value;
        if (c.pv.d == D) return is_bf16 ? run_warp4<D, NT, true, __nv_bfloat16>(c, pb, q, out, scale, w, max_rows, st) : run_warp4<D, NT, true, float>(c, pb, q, out, scale, w, max_rows, st);
        return is_bf16 ? run_warp4<D, NT, false, __nv_bfloat16>(c, pb, q, out, scale, w, max_rows, st) : run_warp4<D, NT, false, float>(c, pb, q, out, scale, w, max_rows, st);
    };
    auto two256 = [&] {
        return c.pv.d == 256 ? run_warp4<256, 2, true, __nv_bfloat16>(c, pb, q, out, scale, w, max_rows, st) : run_warp4<256, 2, false, __nv_bfloat16>(c, pb, q, out, scale, w, max_rows, st);
    };
    auto rows = [&](auto d) {
        return tile_rows <= 8 ? go(d, std::integral_constant<int, 1>{}) : go(d, std::integral_constant<int, 2>{});
    };
    return c.pv.d <= 64    ? rows(std::integral_constant<int, 64>{})
           : c.pv.d <= 128 ? rows(std::integral_constant<int, 128>{})
                           // 16 rows of 256 spill: they pay for chunks, whose passes over the cache they halve (2 x 512 tokens over 8K, 4 x 4 heads:
                           // 930 to 724 us), not for 32 rows (80 to 87)
                           : is_bf16 && tile_rows > 8 ? two256() : go(std::integral_constant<int, 256>{}, std::integral_constant<int, 1>{});
}

}  // namespace tkv
