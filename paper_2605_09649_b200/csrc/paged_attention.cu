// Attention of new tokens over the caller-owned paged cache: the fp32 form, and the kernel that joins partial results.
//
// fp32 form.  A CTA of 256 threads holds 16 (token, query head) rows of one KV head and walks its share of the pages
// (paged_item), a page at a time: cp.async brings K and V into one of two buffers while the page before is worked on (rows
// behind the last entry are filled with zeros).  The products run on the tensor cores in three TF32 parts: a value is split
// x = hi + lo with hi and lo rounded to 11 bits, and hi hi + hi lo + lo hi leaves out 2^-22 of a product, as fp32 does; the
// parts go to accumulators of their own (short chains) and are added up at the end of a page.  S = Q K^T: a warp has 8 keys
// x 16 rows, its K fragments come by ldmatrix and Q waits in registers (head sizes up to 128); the running maximum and sum of
// the softmax with two rows per warp; O += P V: a warp has an eighth of the columns.  Plain fp32 FMAs were bound by shared
// memory (a 16-byte read per 4 products: 5100 cycles a page at d = 64); this is bound by the latency of a page's three phases, each
// behind a block barrier: a prompt of 512 tokens, 4 heads of 64, 22.6 us with the join (38 with plain FMAs); single tokens of 8 requests of
// up to 32 K, 8 x 4 heads of 128, 760 us for 2.15 GB, 0.44 of the measured copy rate.
#include "mma_sync.cuh"
#include "paged.cuh"

namespace tkv {

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr int F_THREADS = 256, F_ROWS = PAGED_F32_ROWS, F_JOIN_STEPS = 4;

// DP: head size rounded up to 64, 128 or 256.  Row strides: ldmatrix reads 8 rows of 16 bytes (16 bytes apart modulo 128), the V
// fragments 4 rows of 8 words (8 words apart modulo 32).
template <int DP>
struct F32Shape {
    static constexpr int KS = DP + 4, VS = DP + 8, QS = DP + 4, PS = PAGE + 4;
    static constexpr int STAGE = PAGE * (KS + VS);                // floats
    static constexpr int STAGES = DP == 256 ? 1 : 2;
    static constexpr bool Q_REG = DP <= 128;
    static constexpr int SMEM = (int)sizeof(float) * (STAGES * STAGE + 2 * F_ROWS * QS + F_ROWS * PS + 3 * F_ROWS);
    static constexpr int CTAS = DP == 64 ? 2 : 1;                 // per SM
};

// 16 bytes, or zeros (src is not read).
__device__ __forceinline__ void f32_copy16(void* dst, const void* src, bool on) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ uint32_t f32_tf32(float x) {
    uint32_t r;
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ void f32_split(uint32_t x, uint32_t& hi, uint32_t& lo) {
    hi = f32_tf32(__uint_as_float(x));
    lo = f32_tf32(__uint_as_float(x) - __uint_as_float(hi));
}
__device__ __forceinline__ void f32_mma(float (&c)[4], const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <int DP>
__global__ void __launch_bounds__(F_THREADS, F32Shape<DP>::CTAS)
paged_attn_f32_kernel(PagedView pv, PagedBatch pb, const float* q, float* out, float scale_log2, PagedWork wk) {
    using S = F32Shape<DP>;
    constexpr int KSTEPS = DP / 8, NT = DP / 64;                  // k steps of S; 8-column tiles of O per warp
    extern __shared__ __align__(16) float s_f32[];
    __shared__ PagedTableMem s_tab;
    float* s_qh = s_f32 + S::STAGES * S::STAGE;                   // [16][QS]: the two parts of Q
    float* s_ql = s_qh + F_ROWS * S::QS;
    float* s_p = s_ql + F_ROWS * S::QS;                          // [16][PS]
    float* s_m = s_p + F_ROWS * S::PS;                           // running maximum, sum, factor of this step
    float* s_l = s_m + F_ROWS;
    float* s_a = s_l + F_ROWS;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, d = pv.d, g = pb.g;
    const int cpr = d / 4;

    grid_dependency_wait();
    PagedTable tab;
    const int unit_rows = pb.top > 0 ? pb.sub_rows : F_ROWS;
    paged_build_table<-1>(tab, pb, pv.H, F_ROWS, 1, INT_MAX, (int)gridDim.x, 2, F_JOIN_STEPS, &s_tab);
    grid_dependents_may_launch();
    const int w = blockIdx.x;
    if (tid == 0) paged_note_none(wk, w);
    if (w >= tab.workers) return;
    const long long end = tab.share(w + 1);
    const int lrow = (lane & 7) + ((lane >> 3) & 1) * 8, lcol = (lane >> 4) * 4;      // this lane's row and column of an A fragment's ldmatrix

    for (long long x = tab.share(w); x < end;) {
        const PagedItem it = paged_item<-1>(tab, pb, x, end, w);
        x += it.steps;
        const int row_first = paged_unit_first<-1>(pb, it.u, F_ROWS), rows = paged_unit_rows<-1>(pb, it.u, it.q.n, F_ROWS);
        auto load_page = [&](int p) {                            // place p of the unit's pages into buffer (p - p0) % STAGES
            float* s_k = s_f32 + (p - it.p0) % S::STAGES * S::STAGE;
            float* s_v = s_k + PAGE * S::KS;
            const int page = pb.top > 0 ? pb.selected[((size_t)(it.q.row0 + it.tok0) * pv.H + it.h) * pb.top + p] : p;
            const int phys = paged_physical(pb, pv, it.r, page);
            const int held = phys < 0 ? 0 : it.q.len - page * PAGE;      // what lies behind the last entry is not read
            const size_t off = ((size_t)max(phys, 0) * pv.H + it.h) * PAGE * d;
            for (int i = tid; i < PAGE * cpr; i += F_THREADS) {
                const int e = i / cpr, c = (i - e * cpr) * 4;
                f32_copy16(s_k + e * S::KS + c, reinterpret_cast<const float*>(pv.k) + off + (size_t)e * d + c, e < held);
                f32_copy16(s_v + e * S::VS + c, reinterpret_cast<const float*>(pv.v) + off + (size_t)e * d + c, e < held);
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            return phys < 0 ? INT_MAX / 2 : page * PAGE;         // first entry; of a page that does not exist: seen by no row
        };
        __syncthreads();                                          // the last unit's buffers and rows are done with
        int e_next = it.p0 < it.p1 ? load_page(it.p0) : 0;
        for (int i = tid; i < F_ROWS * cpr; i += F_THREADS) {
            const int rr = i / cpr, c = (i - rr * cpr) * 4;
            uint4 v = make_uint4(0u, 0u, 0u, 0u), hi, lo;
            if (rr < rows) {
                const int row = row_first + rr;
                const int qt = pb.by_g.div(row);
                v = *reinterpret_cast<const uint4*>(q + (size_t)(it.q.row0 + qt) * pb.q_stride + (size_t)(it.h * g + row - qt * g) * d + c);
            }
            f32_split(v.x, hi.x, lo.x); f32_split(v.y, hi.y, lo.y); f32_split(v.z, hi.z, lo.z); f32_split(v.w, hi.w, lo.w);
            *reinterpret_cast<uint4*>(s_qh + rr * S::QS + c) = hi;
            *reinterpret_cast<uint4*>(s_ql + rr * S::QS + c) = lo;
        }
        if (tid < F_ROWS) { s_m[tid] = -INFINITY; s_l[tid] = 0.f; }
        float o[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) o[nt][0] = o[nt][1] = o[nt][2] = o[nt][3] = 0.f;
        // S: this thread has rows lane / 4 and + 8, keys 8 warp + 2 (lane % 4) and + 1 of a page; the entries its rows see
        int see_hi[2], see_lo[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int rr = (lane >> 2) + 8 * i;
            const int pos = rr < rows ? it.q.len - it.q.n + pb.by_g.div(row_first + rr) : -1;
            see_hi[i] = pos;
            see_lo[i] = pb.window > 0 ? pos + 1 - pb.window : 0;
        }
        uint32_t qh[S::Q_REG ? KSTEPS : 1][4], ql[S::Q_REG ? KSTEPS : 1][4];
        auto load_q = [&](int ks, uint32_t (&h)[4], uint32_t (&l)[4]) {
            const int at = lrow * S::QS + ks * 8 + lcol;
            ldsm_x4(h, (uint32_t)__cvta_generic_to_shared(s_qh + at));
            ldsm_x4(l, (uint32_t)__cvta_generic_to_shared(s_ql + at));
        };
        if (S::Q_REG) {
            __syncthreads();
#pragma unroll
            for (int ks = 0; ks < KSTEPS; ++ks)
                if (ks * 8 < d) load_q(ks, qh[S::Q_REG ? ks : 0], ql[S::Q_REG ? ks : 0]);
        }

        for (int p = it.p0; p < it.p1; ++p) {
            const int e0 = e_next;
            const float* s_k = s_f32 + (p - it.p0) % S::STAGES * S::STAGE;
            const float* s_v = s_k + PAGE * S::KS;
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            __syncthreads();                                      // the page is here, and the page before is done with
            if (S::STAGES > 1 && p + 1 < it.p1) e_next = load_page(p + 1);
            {
                float acc[3][2][4];                               // hi hi, lo hi, hi lo; even and odd steps
#pragma unroll
                for (int i = 0; i < 24; ++i) (&acc[0][0][0])[i] = 0.f;
                const uint32_t kaddr = (uint32_t)__cvta_generic_to_shared(s_k + (warp * 8 + (lane & 7)) * S::KS + (lane >> 3) * 4);
#pragma unroll
                for (int ks = 0; ks < KSTEPS; ks += 2) {
                    if (ks * 8 >= d) break;
                    uint32_t kb[4];                               // k 0-3, 4-7 of this step and of the next
                    ldsm_x4(kb, kaddr + ks * 32);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        if ((ks + e) * 8 >= d) break;
                        uint32_t h0, l0, h1, l1, th[4], tl[4];
                        f32_split(kb[2 * e], h0, l0);
                        f32_split(kb[2 * e + 1], h1, l1);
                        if (!S::Q_REG) load_q(ks + e, th, tl);
                        const uint32_t* ah = S::Q_REG ? qh[S::Q_REG ? ks + e : 0] : th;
                        const uint32_t* al = S::Q_REG ? ql[S::Q_REG ? ks + e : 0] : tl;
                        f32_mma(acc[0][e], ah, h0, h1);
                        f32_mma(acc[1][e], al, h0, h1);
                        f32_mma(acc[2][e], ah, l0, l1);
                    }
                }
                const int key = warp * 8 + 2 * (lane & 3);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int at = e0 + key + (i & 1), rr = (lane >> 2) + 8 * (i >> 1);
                    const float v = (acc[0][0][i] + acc[0][1][i]) + ((acc[1][0][i] + acc[1][1][i]) + (acc[2][0][i] + acc[2][1][i]));
                    s_p[rr * S::PS + key + (i & 1)] = at <= see_hi[i >> 1] && at >= see_lo[i >> 1] ? v * scale_log2 : -INFINITY;
                }
            }
            __syncthreads();
            {
                float a[2], b[2], mx[2], sum[2], m0[2], ref[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int rr = warp * 2 + i;
                    a[i] = s_p[rr * S::PS + lane];
                    b[i] = s_p[rr * S::PS + 32 + lane];
                    m0[i] = s_m[rr];
                    mx[i] = fmaxf(a[i], b[i]);
                }
#pragma unroll
                for (int off = 16; off > 0; off >>= 1)
#pragma unroll
                    for (int i = 0; i < 2; ++i) mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], off));
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    mx[i] = fmaxf(m0[i], mx[i]);
                    ref[i] = mx[i] == -INFINITY ? 0.f : mx[i];           // a row that has seen nothing yet: every weight is 0
                    a[i] = exp2f(a[i] - ref[i]);
                    b[i] = exp2f(b[i] - ref[i]);
                    sum[i] = a[i] + b[i];
                    s_p[(warp * 2 + i) * S::PS + lane] = a[i];
                    s_p[(warp * 2 + i) * S::PS + 32 + lane] = b[i];
                }
#pragma unroll
                for (int off = 16; off > 0; off >>= 1)
#pragma unroll
                    for (int i = 0; i < 2; ++i) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], off);
                if (lane < 2) {
                    const int rr = warp * 2 + lane;
                    const float f = exp2f((lane ? m0[1] : m0[0]) - (lane ? ref[1] : ref[0]));
                    s_a[rr] = f;
                    s_l[rr] = s_l[rr] * f + (lane ? sum[1] : sum[0]);
                    s_m[rr] = lane ? mx[1] : mx[0];
                }
            }
            __syncthreads();
            {
                float acc[NT][3][4];
#pragma unroll
                for (int i = 0; i < NT * 12; ++i) (&acc[0][0][0])[i] = 0.f;
                const uint32_t paddr = (uint32_t)__cvta_generic_to_shared(s_p + lrow * S::PS + lcol);
                const float* vb = s_v + (lane & 3) * S::VS + warp * (DP / 8) + (lane >> 2);
#pragma unroll
                for (int ks = 0; ks < PAGE / 8; ++ks) {
                    uint32_t pr[4], ph[4], pl[4];
                    ldsm_x4(pr, paddr + ks * 32);
#pragma unroll
                    for (int i = 0; i < 4; ++i) f32_split(pr[i], ph[i], pl[i]);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        uint32_t h0, l0, h1, l1;
                        f32_split(__float_as_uint(vb[ks * 8 * S::VS + nt * 8]), h0, l0);
                        f32_split(__float_as_uint(vb[(ks * 8 + 4) * S::VS + nt * 8]), h1, l1);
                        f32_mma(acc[nt][0], ph, h0, h1);
                        f32_mma(acc[nt][1], pl, h0, h1);
                        f32_mma(acc[nt][2], ph, l0, l1);
                    }
                }
                const float f0 = s_a[lane >> 2], f1 = s_a[(lane >> 2) + 8];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[nt][i] = fmaf(o[nt][i], i < 2 ? f0 : f1, acc[nt][0][i] + (acc[nt][1][i] + acc[nt][2][i]));
            }
            if (S::STAGES == 1 && p + 1 < it.p1) {
                __syncthreads();                                  // the only buffer is free
                e_next = load_page(p + 1);
            }
        }
        __syncthreads();                                          // the last sums are written
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int rr = (lane >> 2) + 8 * i;
            if (rr >= rows) continue;
            const int row = row_first + rr, qt = pb.by_g.div(row);
            const float l = s_l[rr], inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
            float* op = out + ((size_t)(it.q.row0 + qt) * pb.Hq + (size_t)(it.h * g + row - qt * g)) * d;
            const size_t pr = (size_t)(it.slot < 0 ? 0 : it.slot) * unit_rows + rr;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int col = warp * (DP / 8) + nt * 8 + 2 * (lane & 3);
                if (col >= d) continue;
                if (it.slot < 0) *reinterpret_cast<float2*>(op + col) = make_float2(o[nt][2 * i] * inv, o[nt][2 * i + 1] * inv);
                else *reinterpret_cast<float2*>(wk.part_o + pr * d + col) = make_float2(o[nt][2 * i], o[nt][2 * i + 1]);
            }
            if (it.slot >= 0 && warp == 0 && (lane & 3) == 0) { wk.part_ml[pr * 2] = s_m[rr]; wk.part_ml[pr * 2 + 1] = l; }
        }
        if (it.slot >= 0 && (it.slot & 1) && tid == 0) paged_note_shared(wk, tab, it, x - it.steps, w, row_first, rows);
    }
}

// ---------------------------------------------------------------- joining the partials
// A unit that several workers shared: M = max m, out = sum e^(m - M) O / sum e^(m - M) l over its parts, in worker order, so
// the result does not depend on timing.  Block (w, y): rows y * chunk .. of the unit that worker w began.  Bound by latency, and short
// enough to be paced by fetching its code: one loop takes up to J_BATCH parts at a time, m, l and O in flight together, with a running
// maximum; a row of many parts is dealt out over several warps.  5 to 6 us for a decode step, 18 us for the 38 MB of parts of 4 x
// 512 tokens x 32 heads.  (Every row searching for its request and its workers by itself took 7 to 11 and 31 us.)
constexpr int J_THREADS = 512, J_WARPS = J_THREADS / 32, J_BATCH = 6, J_NOTES = 16;

__device__ __forceinline__ void join_store(__nv_bfloat16* o, const float4& v, float f) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(v.x * f, v.y * f), b = __floats2bfloat162_rn(v.z * f, v.w * f);
    *reinterpret_cast<uint2*>(o) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}
__device__ __forceinline__ void join_store(float* o, const float4& v, float f) { *reinterpret_cast<float4*>(o) = make_float4(v.x * f, v.y * f, v.z * f, v.w * f); }
__device__ __forceinline__ void join_add(float4& s, float e, const float4& v) {
    s.x = fmaf(e, v.x, s.x); s.y = fmaf(e, v.y, s.y); s.z = fmaf(e, v.z, s.z); s.w = fmaf(e, v.w, s.w);
}
__device__ __forceinline__ float join_factor(float l) { return l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l); }      // rows that see nothing: 0; NaN stays

// FEWER: blocks than workers, J_NOTES of them for each at most.
template <typename T, bool FEWER>
__global__ void __launch_bounds__(J_THREADS, 2)
paged_join_kernel(T* out, PagedWork wk, FastDiv by_g, int Hq, int d, int unit_rows, int chunk, int workers) {
    extern __shared__ __align__(16) float4 s_sum[];               // [J_WARPS][d / 4]
    __shared__ float2 s_ml[J_WARPS];
    __shared__ int4 s_unit[FEWER ? J_NOTES : 1];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = (int)by_g.d;
    grid_dependents_may_launch();
    grid_dependency_wait();
    if constexpr (FEWER) {                                        // the notes of workers blockIdx.x, + gridDim.x, ..., all at once
        const int at = (int)(blockIdx.x + threadIdx.x * gridDim.x);
        if (threadIdx.x < J_NOTES) s_unit[threadIdx.x] = at < workers ? wk.shared[at] : make_int4(0, 0, 0, 0);
        __syncthreads();
    }
    for (int w = blockIdx.x, note = 0; FEWER ? w < workers : note == 0; w += (int)gridDim.x, ++note) {
        const int4 unit = FEWER ? s_unit[note] : wk.shared[w];
        const int r0 = (int)blockIdx.y * chunk, nr = min(chunk, (unit.z & 4095) - r0), n = unit.z >> 12;
        if (nr <= 0) continue;
        int shift = 0;                                                // 2^shift warps per row
        while ((2 << shift) * nr <= J_WARPS && (J_BATCH << shift) < n) ++shift;
        const int way = warp & ((1 << shift) - 1), i_lo = n * way >> shift, i_hi = n * (way + 1) >> shift;
        for (int rr = warp >> shift; rr < nr; rr += J_WARPS >> shift) {       // (several warps per row: one round)
            const int row = unit.y + r0 + rr, t = by_g.div(row);
            T* o = out + ((size_t)(unit.x + t) * Hq + (size_t)(unit.w * g + row - t * g)) * d;
#pragma unroll 1
            for (int c0 = lane * 4; c0 < d; c0 += 128) {
                float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
                float M = -INFINITY, L = 0.f;
#pragma unroll 1
                for (int i0 = i_lo; i0 < i_hi; i0 += J_BATCH) {
                    float4 v[J_BATCH];
                    float2 ml[J_BATCH];
                    float top = M;
#pragma unroll
                    for (int i = 0; i < J_BATCH; ++i) {
                        // part 0: worker w began the unit and did not end it; the others did not begin it
                        const size_t p = (size_t)(2 * (w + i0 + i) + (i0 + i == 0)) * unit_rows + r0 + rr;
                        v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                        ml[i] = make_float2(-INFINITY, 0.f);
                        if (i0 + i < i_hi) {
                            v[i] = *reinterpret_cast<const float4*>(wk.part_o + p * d + c0);
                            ml[i] = *reinterpret_cast<const float2*>(wk.part_ml + p * 2);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < J_BATCH; ++i) top = fmaxf(top, ml[i].x);
                    const float ref = top == -INFINITY ? 0.f : top, keep = exp2f(M - ref);
                    M = top;
                    L *= keep;
                    sum.x *= keep; sum.y *= keep; sum.z *= keep; sum.w *= keep;
#pragma unroll
                    for (int i = 0; i < J_BATCH; ++i) {
                        const float e = exp2f(ml[i].x - ref);
                        L = fmaf(e, ml[i].y, L);
                        join_add(sum, e, v[i]);
                    }
                }
                if (shift == 0) join_store(o + c0, sum, join_factor(L));
                else {
                    s_sum[warp * (d / 4) + c0 / 4] = sum;
                    s_ml[warp] = make_float2(M, L);
                }
            }
        }
        if (shift == 0) continue;
        __syncthreads();
        const int rr = warp >> shift;
        if (way == 0 && rr < nr) {
            const int row = unit.y + r0 + rr, t = by_g.div(row);
            T* o = out + ((size_t)(unit.x + t) * Hq + (size_t)(unit.w * g + row - t * g)) * d;
            float M = -INFINITY, L = 0.f;
            for (int x = 0; x < 1 << shift; ++x) M = fmaxf(M, s_ml[warp + x].x);
            const float ref = M == -INFINITY ? 0.f : M;
            for (int x = 0; x < 1 << shift; ++x) L = fmaf(exp2f(s_ml[warp + x].x - ref), s_ml[warp + x].y, L);
            for (int c0 = lane * 4; c0 < d; c0 += 128) {
                float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
                for (int x = 0; x < 1 << shift; ++x) join_add(sum, exp2f(s_ml[warp + x].x - ref), s_sum[(warp + x) * (d / 4) + c0 / 4]);
                join_store(o + c0, sum, join_factor(L));
            }
        }
        if constexpr (FEWER) __syncthreads();                         // the sums are read
    }
}

template <int DP>
cudaError_t run_f32(const PagedView& pv, const PagedBatch& pb, const void* q, void* out, float scale, const PagedWork& w, cudaStream_t st) {
    using S = F32Shape<DP>;
    static_assert(S::CTAS <= PAGED_F32_CTAS, "the workspace holds the workers' partial results");
    static_assert((S::SMEM + (int)sizeof(PagedTableMem) + 1024) * S::CTAS <= 228 * 1024, "shared memory of one SM");
    static std::atomic<unsigned long long> done{0};
    const cudaError_t e = paged_allow_smem(reinterpret_cast<const void*>(paged_attn_f32_kernel<DP>), S::SMEM, done);
    if (e != cudaSuccess) return e;
    const int workers = PAGED_SMS * S::CTAS;
    const cudaError_t e2 = paged_launch(paged_attn_f32_kernel<DP>, dim3(workers), dim3(F_THREADS), S::SMEM, 1, true, st, pv, pb, (const float*)q, (float*)out,
                                        scale * LOG2E, w);
    if (e2 != cudaSuccess || paged_always_whole(pb, pv.H, F_ROWS, workers, F_JOIN_STEPS)) return e2;
    return launch_paged_join(pv, pb, 0, out, w, pb.top > 0 ? pb.sub_rows : F_ROWS, workers, st);
}

}  // namespace

cudaError_t launch_paged_join(const PagedView& pv, const PagedBatch& pb, int is_bf16, void* out, const PagedWork& w, int unit_rows,
                              int workers, cudaStream_t st, int blocks) {
    // Units of few rows are those with many parts: four rows leave four warps to each (measured for 4 requests x 4 heads of 7 rows in
    // 37 parts: 25.9 us with the kernel before it, eight rows to a block 28.6); otherwise two rows per warp.
    const int chunk = std::min(unit_rows, unit_rows <= 8 ? 4 : 2 * J_WARPS);
    if (blocks <= 0 || blocks * J_NOTES < workers) blocks = workers;
    const dim3 grid((unsigned)std::min(blocks, workers), (unsigned)((unit_rows + chunk - 1) / chunk)), block(J_THREADS);
    const size_t smem = (size_t)J_WARPS * pv.d * sizeof(float);
    auto go = [&](auto kernel, auto* o) { return paged_launch(kernel, grid, block, smem, 1, true, st, o, w, pb.by_g, pb.Hq, pv.d, unit_rows, chunk, workers); };
    if (blocks < workers) return is_bf16 ? go(paged_join_kernel<__nv_bfloat16, true>, (__nv_bfloat16*)out) : go(paged_join_kernel<float, true>, (float*)out);
    return is_bf16 ? go(paged_join_kernel<__nv_bfloat16, false>, (__nv_bfloat16*)out) : go(paged_join_kernel<float, false>, (float*)out);
}

cudaError_t launch_paged_attention_f32(const PagedView& pv, const PagedBatch& pb, const void* q, void* out, float scale, const PagedWork& w,
                                       cudaStream_t st) {
    return pv.d <= 64    ? run_f32<64>(pv, pb, q, out, scale, w, st)
           : pv.d <= 128 ? run_f32<128>(pv, pb, q, out, scale, w, st)
                         : run_f32<256>(pv, pb, q, out, scale, w, st);
}

}  // namespace tkv
