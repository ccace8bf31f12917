// Attention over the caller-owned paged cache for many query rows, on tcgen05: bf16, head size 64 or 128.
//
// A unit is 256 (token, query head) rows of one KV head in two groups of 128 that share every K/V tile; a tile is one page
// (64 entries).  One persistent CTA per SM takes an equal share of the line of page steps (paged.cuh) and meets a stretch of a
// unit at a time.  TMA copies the page's K and V as 64-column planes with the 128-byte swizzle: K planes are K-major operands
// of S = Q K^T, V planes MN-major operands of O += P V.  Warps 0-3 / 4-7 are the softmax warps of group 0 / 1 (a thread owns a
// row: S from tensor memory, masked, exponentiated, P back to tensor memory as the A operand of P V), warp 8 issues the
// copies, warps 9 and 10 the products of a group each; S is double-buffered and issued two tiles ahead of the P V that needs the
// softmax.  The maximum is only raised (and O rescaled) when it grows by more than 2^8.  A third of the exponentials are
// evaluated on the FMA pipe.  A unit of 128 rows or fewer leaves group 1 idle.  V rows behind a request's last entry are zeroed
// in shared memory before the product reads them (they may hold NaN).  Every wait is bounded; one that runs out latches
// TRIMKV_E_TIMEOUT.
#include "paged.cuh"
#include "tcgen05_attn.cuh"

namespace tkv {

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr int T_ROWS = 128, T_UNIT = PAGED_TC_ROWS;
constexpr int T_PLANE = PAGE * 128;                                   // 64 entries x 64 columns
constexpr int T_QPLANE = T_ROWS * 128;
constexpr int T_THREADS = 352;
constexpr int T_TMEM_COLS = 512;      // group g: S of even / odd tiles at columns 128 g, 128 g + 64 (P over the first half); O at 256 + 128 g
constexpr int T_POLY_EVERY = 3;
constexpr float T_RESCALE_STEP = 8.0f;
constexpr int T_E0 = 16;              // ring of the tiles' first entries: more than a stage count and two tiles

template <int D>
struct TcShape {
    static constexpr int PLANES = D / 64;
    static constexpr int STAGE = 2 * PLANES * T_PLANE;
    static constexpr int STAGES = D == 128 ? 4 : 6;
    static constexpr int Q_BYTES = 2 * PLANES * T_QPLANE;
    static constexpr int OFF_Q = STAGES * STAGE;
    static constexpr int OFF_BAR = OFF_Q + Q_BYTES;
    static constexpr int OFF_E0 = OFF_BAR + 256;
    static constexpr int OFF_TAB = OFF_E0 + T_E0 * 4;
    static constexpr int SMEM = OFF_TAB + (int)sizeof(PagedTableMem) + 1024;      // 1024: alignment slack
    // D fp32, A and B bf16, M = 128.  S: both K-major, N = 64.  P V: B (V) MN-major, N = D.
    static constexpr uint32_t IDESC_S = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(64 >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
    static constexpr uint32_t IDESC_PV = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
};

template <int D>
__global__ void __launch_bounds__(T_THREADS, 1)
paged_attn_tc_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, PagedView pv, PagedBatch pb,
                     const __nv_bfloat16* __restrict__ q, __nv_bfloat16* __restrict__ out, float scale_log2, PagedWork wk, int min_rows) {
    using S = TcShape<D>;
    extern __shared__ unsigned char t_smem_raw[];
    const uint32_t raw = a_smem(t_smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    unsigned char* gen = t_smem_raw + (base - raw);
    const uint32_t bars = base + S::OFF_BAR;
    const uint32_t full0 = bars, empty0 = bars + 8 * S::STAGES, s_ready0 = empty0 + 8 * S::STAGES /* [group][tile parity] */,
                   p_ready0 = s_ready0 + 32, pv_done0 = p_ready0 + 16;
    volatile uint32_t* s_tmem = reinterpret_cast<volatile uint32_t*>(gen + S::OFF_BAR + 240);
    volatile int* s_fail = reinterpret_cast<volatile int*>(gen + S::OFF_BAR + 248);
    volatile int* s_e0 = reinterpret_cast<volatile int*>(gen + S::OFF_E0);
    PagedTableMem* table_mem = reinterpret_cast<PagedTableMem*>(gen + S::OFF_TAB);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = pb.g;
    static_assert(16 * S::STAGES + 64 <= 240, "barriers fit");

    if (threadIdx.x == 0) {
        for (int s = 0; s < S::STAGES; ++s) { a_bar_init(full0 + 8 * s, 1); a_bar_init(empty0 + 8 * s, 2); }   // both issuers free a stage
        for (int gq = 0; gq < 2; ++gq) {
            a_bar_init(s_ready0 + 16 * gq, 1);
            a_bar_init(s_ready0 + 16 * gq + 8, 1);
            a_bar_init(p_ready0 + 8 * gq, 4);
            a_bar_init(pv_done0 + 8 * gq, 1);
        }
        *s_fail = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        a_prefetch_map(&map_k);
        a_prefetch_map(&map_v);
    }
    grid_dependency_wait();
    PagedTable tab;
    paged_build_table(tab, pb, pv.H, T_UNIT, min_rows, INT_MAX, (int)gridDim.x, 4, table_mem, wk.prefix);
    grid_dependents_may_launch();
    const int w = blockIdx.x;
    if (w >= tab.workers) return;                                     // the whole block, before it holds tensor memory
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(a_smem((const void*)s_tmem)), "r"(T_TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    a_fence_before();
    __syncthreads();
    a_fence_after();
    const uint32_t tmem = *s_tmem;
    const int grp = (warp >> 2) & 1, wl = warp & 3;
    const int r = wl * 32 + lane, R = grp * T_ROWS + r;               // a softmax thread's row: lane of tensor memory, row of the unit

    const long long end = tab.share(w + 1);
    // tiles of the stretches before this one: of the ring, and of group 1, whose barriers rest while it has no rows
    unsigned ct = 0, ct1 = 0;
    for (long long x = tab.share(w); x < end;) {
        const PagedItem it = paged_item(tab, pb, x, end, w);
        x += it.steps;
        const int ntile = it.p1 - it.p0;
        const int row_first = it.u * T_UNIT, rows = min(T_UNIT, it.q.n * g - row_first);
        const bool both = rows > T_ROWS;
        const bool valid = warp < 8 && R < rows;
        const int tok = valid ? (row_first + R) / g : 0, head = valid ? (row_first + R) % g : 0;
        const int pos = it.q.len - it.q.n + tok;
        const int see_hi = valid ? max(pos + 1, 0) : 0;               // entries the row sees: see_lo .. see_hi - 1
        const int see_lo = valid && pb.window > 0 ? max(pos + 1 - pb.window, 0) : 0;
        if (ntile > 0) {
            if (warp < 8 && (grp == 0 || both)) {
                const uint4* src = reinterpret_cast<const uint4*>(q + (size_t)(it.q.row0 + tok) * pb.q_stride + (size_t)(it.h * g + head) * D);
                unsigned char* qdst = gen + S::OFF_Q + grp * S::PLANES * T_QPLANE + r * 128;
#pragma unroll
                for (int c = 0; c < D / 8; ++c) {
                    const uint4 v = valid ? src[c] : make_uint4(0u, 0u, 0u, 0u);
                    *reinterpret_cast<uint4*>(qdst + (c >> 3) * T_QPLANE + (((c & 7) ^ (r & 7)) << 4)) = v;
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // Q and the barriers, before the async proxy uses them
            a_fence_before();
            __syncthreads();
            a_fence_after();

            if (warp == 8) {
                // ---- TMA producer: lane l holds the page of tile l of the current run of 32
                int phys = 0;
                for (int i = 0; i < ntile; ++i) {
                    if ((i & 31) == 0) phys = i + lane < ntile ? paged_physical(pb, pv, it.r, it.p0 + i + lane) : -1;
                    const int page = __shfl_sync(0xffffffffu, phys, i & 31);
                    const unsigned c = ct + i, s = c % S::STAGES;
                    int ok = 1;
                    if (lane == 0) {
                        if (c >= S::STAGES) ok = a_bar_wait(empty0 + 8 * s, ((c / S::STAGES) - 1) & 1) ? 1 : 0;
                        if (ok) {
                            // a page that does not exist: the copy reads page 0 and every row masks the tile
                            s_e0[c % T_E0] = page < 0 ? INT_MAX / 2 : (it.p0 + i) * PAGE;
                            const uint32_t dst = base + s * S::STAGE;
                            const int krow = (max(page, 0) * pv.H + it.h) * PAGE;
                            a_bar_expect_tx(full0 + 8 * s, S::STAGE);
                            a_tma_3d(dst, &map_k, 0, krow, 0, full0 + 8 * s);
                            a_tma_3d(dst + S::PLANES * T_PLANE, &map_v, 0, krow, 0, full0 + 8 * s);
                        }
                    }
                    if (__shfl_sync(0xffffffffu, ok, 0) == 0) {
                        if (lane == 0) *s_fail = 1;
                        // the copies already issued land before the block leaves (bounded)
                        for (unsigned k = c >= S::STAGES ? c - S::STAGES : 0; k < c; ++k) a_bar_wait(full0 + 8 * (k % S::STAGES), (k / S::STAGES) & 1);
                        break;
                    }
                }
            } else if (warp >= 9) {
                const int gq = warp - 9;
                bool ok = true;
                if (gq == 1 && !both) {
                    // ---- no rows in this group: its share of freeing the stages
                    for (int i = 0; i < ntile && ok; ++i) {
                        const unsigned c = ct + i, s = c % S::STAGES;
                        ok = a_bar_wait(full0 + 8 * s, (c / S::STAGES) & 1);
                        if (ok && lane == 0) a_bar_arrive(empty0 + 8 * s);
                        __syncwarp();
                    }
                } else {
                    // ---- MMA issuer of group gq: S of tiles i + 1 and i + 2 are issued before P V of tile i
                    const uint32_t d_s0 = tmem + 128 * gq, d_o = tmem + 256 + 128 * gq;
                    const uint32_t qb = base + S::OFF_Q + gq * S::PLANES * T_QPLANE;
                    const unsigned gt = gq ? ct1 : ct;
                    auto issue_s = [&](int i) {                       // S = Q K^T of tile i into buffer (gt + i) & 1
                        const unsigned c = ct + i, s = c % S::STAGES, b = (gt + i) & 1;
                        ok = __all_sync(0xffffffffu, a_bar_wait(full0 + 8 * s, (c / S::STAGES) & 1));
                        if (!ok) return;
                        a_fence_after();
                        if (lane == 0) {
                            const uint32_t st = base + s * S::STAGE, d_s = d_s0 + 64 * b;
#pragma unroll
                            for (int p = 0; p < S::PLANES; ++p) {
                                const uint64_t qd = a_desc(qb + p * T_QPLANE, 16), kd = a_desc(st + p * T_PLANE, 16);
#pragma unroll
                                for (int j = 0; j < 4; ++j)           // 16 channels per instruction, 32 bytes along the row
                                    a_umma(d_s, qd + (uint64_t)(j * 32 >> 4), kd + (uint64_t)(j * 32 >> 4), S::IDESC_S, (p | j) != 0);
                            }
                            a_commit(s_ready0 + 16 * gq + 8 * b);
                        }
                        __syncwarp();
                    };
                    auto issue_pv = [&](int i) {                      // O += P V of tile i
                        const unsigned c = ct + i, s = c % S::STAGES, b = (gt + i) & 1;
                        const uint32_t st = base + s * S::STAGE, a_p = d_s0 + 64 * b;
                        const int held = it.q.len - s_e0[c % T_E0];   // (<= 0 for a page that does not exist: all of its V is zeroed)
                        if (held < PAGE) {
                            unsigned char* vg = gen + s * S::STAGE + S::PLANES * T_PLANE;
                            for (int e = max(held, 0) * 8 + lane; e < PAGE * 8; e += 32)
#pragma unroll
                                for (int p = 0; p < S::PLANES; ++p) *reinterpret_cast<uint4*>(vg + p * T_PLANE + e * 16) = make_uint4(0u, 0u, 0u, 0u);
                            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        }
                        ok = __all_sync(0xffffffffu, a_bar_wait(p_ready0 + 8 * gq, b));
                        if (!ok) return;
                        a_fence_after();
                        if (lane == 0) {
                            const uint64_t vd = a_desc(st + S::PLANES * T_PLANE, T_PLANE);    // the next 64 channels: one plane further
#pragma unroll
                            for (int j = 0; j < PAGE / 16; ++j)       // 16 entries per instruction: P +8 columns, V +2 row groups
                                a_umma_ts(d_o, a_p + j * 8, vd + (uint64_t)(j * 2048 >> 4), S::IDESC_PV, (i | j) != 0);
                            a_commit(pv_done0 + 8 * gq);
                            a_commit(empty0 + 8 * s);                 // this group is done with the stage
                        }
                        __syncwarp();
                    };
                    issue_s(0);
                    if (ok && ntile > 1) issue_s(1);
                    for (int i = 0; i < ntile && ok; ++i) {
                        issue_pv(i);
                        if (ok && i + 2 < ntile) issue_s(i + 2);
                    }
                }
                if (!ok && lane == 0) *s_fail = 1;
            }
        }
        if (warp < 8 && (grp == 0 || both)) {
            // ---- softmax warps
            const uint32_t lane_addr = tmem + ((uint32_t)(wl * 32) << 16);
            const uint32_t s_col0 = (uint32_t)(128 * grp), o_col = (uint32_t)(256 + 128 * grp);
            float m_used = -INFINITY, l = 0.f;
            bool ok = true;
            const unsigned gt = grp ? ct1 : ct;
            for (int i = 0; i < ntile; ++i) {
                const unsigned c = gt + i;                            // of the group's tiles
                ok = __all_sync(0xffffffffu, a_bar_wait(s_ready0 + 16 * grp + 8 * (c & 1), (c >> 1) & 1));
                if (!ok) break;
                const uint32_t s_col = s_col0 + 64u * (c & 1u);
                a_fence_after();
                uint32_t sv[64];
                a_tmem_ld32(lane_addr + s_col, sv);
                a_tmem_ld32(lane_addr + s_col + 32, sv + 32);
                asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                const int e0 = s_e0[(ct + i) % T_E0];
                if (e0 + PAGE > see_hi || e0 < see_lo) {              // the tile crosses the row's limits
#pragma unroll
                    for (int e = 0; e < 64; ++e)
                        if (e0 + e >= see_hi || e0 + e < see_lo) sv[e] = 0xff800000u;        // -inf
                }
                float mq[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int e = 0; e < 64; e += 8) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) mq[k] = a_max3(mq[k], __uint_as_float(sv[e + 2 * k]), __uint_as_float(sv[e + 2 * k + 1]));
                }
                const float mx = fmaxf(fmaxf(mq[0], mq[1]), fmaxf(mq[2], mq[3]));
                const float m_new = mx * scale_log2;                  // scale_log2 > 0
                const bool resc = __any_sync(0xffffffffu, m_new > m_used + T_RESCALE_STEP);
                float alpha = 1.0f;
                if (resc) {
                    const float mn = fmaxf(m_used, m_new);
                    alpha = (m_used == -INFINITY) ? 0.0f : exp2f(m_used - mn);
                    m_used = mn;
                }
                const float mref = (m_used == -INFINITY) ? 0.0f : m_used;
                const uint64_t sc2 = a_pack2(scale_log2, scale_log2), nm2 = a_pack2(-mref, -mref);
                uint64_t sq[4] = {0ull, 0ull, 0ull, 0ull};
                uint32_t pk[32];
#pragma unroll
                for (int e = 0; e < 64; e += 2) {
                    const uint64_t x2 = a_fma2(a_pack2(__uint_as_float(sv[e]), __uint_as_float(sv[e + 1])), sc2, nm2);
                    float p0, p1;
                    if ((e >> 1) % T_POLY_EVERY == T_POLY_EVERY - 1) {
                        a_exp2_fma2(x2, p0, p1);
                    } else {
                        float x0, x1;
                        a_unpack2(x2, x0, x1);
                        p0 = a_ex2(x0);
                        p1 = a_ex2(x1);
                    }
                    sq[(e >> 1) & 3] = a_add2(sq[(e >> 1) & 3], a_pack2(p0, p1));
                    pk[e >> 1] = a_bf16x2(p0, p1);
                }
                float a0, a1;
                a_unpack2(a_add2(a_add2(sq[0], sq[1]), a_add2(sq[2], sq[3])), a0, a1);
                l = l * alpha + (a0 + a1);
                if (i > 0) {                                          // O complete up to the previous tile
                    ok = __all_sync(0xffffffffu, a_bar_wait(pv_done0 + 8 * grp, (c - 1) & 1));
                    if (!ok) break;
                    a_fence_after();
                    if (resc) {
#pragma unroll
                        for (int k = 0; k < D / 32; ++k) {
                            uint32_t ov[32];
                            a_tmem_ld32(lane_addr + o_col + k * 32, ov);
                            asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
                            for (int e = 0; e < 32; ++e) ov[e] = __float_as_uint(__uint_as_float(ov[e]) * alpha);
                            a_tmem_st32(lane_addr + o_col + k * 32, ov);
                        }
                        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                    }
                }
                a_tmem_st32(lane_addr + s_col, pk);
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                a_fence_before();
                __syncwarp();
                if (lane == 0) a_bar_arrive(p_ready0 + 8 * grp);
            }
            if (ok && ntile > 0) ok = __all_sync(0xffffffffu, a_bar_wait(pv_done0 + 8 * grp, (gt + ntile - 1) & 1));
            if (!ok) {
                if (lane == 0) *s_fail = 1;
            } else {
                a_fence_after();
                if (m_used == -INFINITY && !(l != l)) l = 0.f;        // a row that sees nothing (the polynomial gives masked entries 2^-125)
                const float inv = l > 0.f ? 1.0f / l : (l == 0.f ? 0.f : l);
                uint4* op = reinterpret_cast<uint4*>(out + ((size_t)(it.q.row0 + tok) * pb.Hq + (size_t)(it.h * g + head)) * D);
                const size_t pr = (size_t)(it.slot < 0 ? 0 : it.slot) * T_UNIT + R;
                float4* po = reinterpret_cast<float4*>(wk.part_o + pr * D);
                const bool zero = l == 0.f;                           // (also a stretch without tiles, whose O was never written)
#pragma unroll
                for (int k = 0; k < D / 32; ++k) {
                    uint32_t ov[32];
                    if (ntile > 0) {
                        a_tmem_ld32(lane_addr + o_col + k * 32, ov);
                        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                    }
#pragma unroll
                    for (int e = 0; e < 32; ++e) ov[e] = zero ? 0u : ov[e];
                    if (!valid) continue;
                    if (it.slot < 0) {
#pragma unroll
                        for (int e = 0; e < 32; e += 8) {
                            uint32_t v[4];
#pragma unroll
                            for (int k2 = 0; k2 < 4; ++k2)
                                v[k2] = a_bf16x2(__uint_as_float(ov[e + 2 * k2]) * inv, __uint_as_float(ov[e + 2 * k2 + 1]) * inv);
                            op[k * 4 + (e >> 3)] = make_uint4(v[0], v[1], v[2], v[3]);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; e += 4)
                            po[k * 8 + (e >> 2)] = make_float4(__uint_as_float(ov[e]), __uint_as_float(ov[e + 1]), __uint_as_float(ov[e + 2]), __uint_as_float(ov[e + 3]));
                    }
                }
                if (valid && it.slot >= 0) {
                    wk.part_ml[pr * 2] = m_used;
                    wk.part_ml[pr * 2 + 1] = l;
                }
            }
        }
        ct += (unsigned)ntile;
        if (both) ct1 += (unsigned)ntile;
        a_fence_before();
        __syncthreads();                                              // Q and tensor memory are free for the next stretch
        a_fence_after();
        if (*s_fail) break;
    }
    __syncthreads();
    if (warp == 9) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(T_TMEM_COLS) : "memory");
    if (threadIdx.x == 0 && *s_fail) latch_error(pb.status, TRIMKV_E_TIMEOUT);
}

template <int D>
cudaError_t run_tc(const PagedView& pv, const PagedBatch& pb, const void* q, void* out, float scale, const PagedWork& w, int min_rows, cudaStream_t st) {
    using S = TcShape<D>;
    static std::atomic<unsigned long long> done{0};
    cudaError_t e = paged_allow_smem(reinterpret_cast<const void*>(paged_attn_tc_kernel<D>), S::SMEM, done);
    if (e != cudaSuccess) return e;
    CUtensorMap mk, mv;
    e = paged_tensor_map(&mk, pv.k, pv, PAGE);
    if (e == cudaSuccess) e = paged_tensor_map(&mv, pv.v, pv, PAGE);
    if (e != cudaSuccess) return e;
    e = paged_launch(paged_attn_tc_kernel<D>, dim3(PAGED_SMS), dim3(T_THREADS), S::SMEM, 1, st, mk, mv, pv, pb, (const __nv_bfloat16*)q, (__nv_bfloat16*)out,
                     scale * LOG2E, w, min_rows);
    return e != cudaSuccess ? e : launch_paged_join(pv, pb, 1, out, w, T_UNIT, min_rows, INT_MAX, true, st);
}

}  // namespace

cudaError_t launch_paged_attention_tc(const PagedView& pv, const PagedBatch& pb, const void* q, void* out, float scale, const PagedWork& w,
                                      int min_rows, cudaStream_t st) {
    return pv.d == 64 ? run_tc<64>(pv, pb, q, out, scale, w, min_rows, st) : run_tc<128>(pv, pb, q, out, scale, w, min_rows, st);
}

}  // namespace tkv
