// Attention of new tokens over the caller-owned paged cache: the form for any head size and type, and the kernel that joins
// partial results.
//
// Plain form.  A CTA of 256 threads holds 16 (token, query head) rows of one KV head and walks its share of the pages
// (paged_item), a page at a time: cp.async brings K and V as they are stored into one of two buffers while the page before
// is worked on (rows behind the last entry are filled with zeros); S = Q K^T in fp32 with one key and four rows per thread -- a
// warp has 8 keys x 16 rows, so that a 16-byte read of K serves 16 FMAs and the reads of Q are broadcasts --, the running
// maximum and sum of the softmax with two rows per warp, then O += P V with a column and 4 to 16 rows of O per thread.  All
// sums are fp32.  fp32 caches and head sizes other than 64 and 128 run here; bound by shared-memory reads (about 2200 cycles a
// page at d = 64) beyond a few rows per page, by the page loads below that.
#include "mma_sync.cuh"
#include "paged.cuh"

namespace tkv {

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr int PL_THREADS = 256, PL_ROWS = PAGED_PLAIN_ROWS;

// DP: head size rounded up to 64, 128 or 256
template <typename T, int DP>
struct PlainShape {
    static constexpr int E = 16 / (int)sizeof(T);
    static constexpr int KS = DP + E;                             // row stride of K (elements): rows 16 bytes apart modulo 128
    static constexpr int QS = DP + 4;                             // row stride of Q (floats)
    static constexpr int COLS = DP, RG = PL_THREADS / COLS;       // columns, row groups of O over the threads
    static constexpr int RPT = PL_ROWS / RG;                      // rows of O per thread
    static constexpr int STAGE = PAGE * (KS + DP) * (int)sizeof(T);
    static constexpr int STAGES = STAGE <= 100 * 1024 ? 2 : 1;
    static constexpr int SMEM = STAGES * STAGE + (int)sizeof(float) * (PL_ROWS * QS + PL_ROWS * PAGE + 3 * PL_ROWS);
    static constexpr int CTAS = SMEM <= 100 * 1024 ? 2 : 1;       // per SM
};

template <typename T>
__device__ __forceinline__ float4 plain_load4(const T* p);
template <>
__device__ __forceinline__ float4 plain_load4<float>(const float* p) { return *reinterpret_cast<const float4*>(p); }
template <>
__device__ __forceinline__ float4 plain_load4<__nv_bfloat16>(const __nv_bfloat16* p) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u));
}
// 16 bytes, or zeros (src is not read).
__device__ __forceinline__ void plain_copy16(void* dst, const void* src, bool on) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "r"(on ? 16 : 0) : "memory");
}

template <typename T, int DP>
__global__ void __launch_bounds__(PL_THREADS, PlainShape<T, DP>::CTAS)
paged_attn_plain_kernel(PagedView pv, PagedBatch pb, const T* __restrict__ q, T* __restrict__ out, float scale_log2, PagedWork wk) {
    using S = PlainShape<T, DP>;
    extern __shared__ __align__(16) unsigned char s_pl[];
    __shared__ PagedTableMem s_tab;
    float* s_q = reinterpret_cast<float*>(s_pl + S::STAGES * S::STAGE);   // [16][QS]
    float* s_p = s_q + PL_ROWS * S::QS;                           // [16][64]
    float* s_m = s_p + PL_ROWS * PAGE;                            // running maximum, sum, factor of this step
    float* s_l = s_m + PL_ROWS;
    float* s_a = s_l + PL_ROWS;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, d = pv.d, g = pb.g;
    const int cpr = d / S::E;

    grid_dependency_wait();
    PagedTable tab;
    const int unit_rows = pb.top > 0 ? g : PL_ROWS;               // rows of a unit (top > 0: one token)
    paged_build_table(tab, pb, pv.H, PL_ROWS, 1, INT_MAX, (int)gridDim.x, 2, 2, &s_tab, wk.prefix);
    grid_dependents_may_launch();
    const int w = blockIdx.x;
    if (w >= tab.workers) return;
    const long long end = tab.share(w + 1);

    for (long long x = tab.share(w); x < end;) {
        const PagedItem it = paged_item(tab, pb, x, end, w);
        x += it.steps;
        const int row_first = pb.top > 0 ? it.u * g : it.u * PL_ROWS;    // of the request's n * g rows
        const int unit_n = min(unit_rows, it.q.n * g - row_first);
        auto load_page = [&](int p) {                            // place p of the unit's pages into buffer (p - p0) % STAGES
            T* s_k = reinterpret_cast<T*>(s_pl + (p - it.p0) % S::STAGES * S::STAGE);
            T* s_v = s_k + PAGE * S::KS;
            const int page = pb.top > 0 ? pb.selected[((size_t)(it.q.row0 + it.u) * pv.H + it.h) * pb.top + p] : p;
            const int phys = paged_physical(pb, pv, it.r, page);
            const int held = phys < 0 ? 0 : it.q.len - page * PAGE;      // what lies behind the last entry is not read
            const size_t off = ((size_t)max(phys, 0) * pv.H + it.h) * PAGE * d;
            for (int i = tid; i < PAGE * cpr; i += PL_THREADS) {
                const int e = i / cpr, c = (i - e * cpr) * S::E;
                plain_copy16(s_k + e * S::KS + c, reinterpret_cast<const T*>(pv.k) + off + (size_t)e * d + c, e < held);
                plain_copy16(s_v + e * DP + c, reinterpret_cast<const T*>(pv.v) + off + (size_t)e * d + c, e < held);
            }
            return phys < 0 ? INT_MAX / 2 : page * PAGE;         // first entry; of a page that does not exist: seen by no row
        };
        for (int b0 = 0; b0 < unit_n; b0 += PL_ROWS) {           // a token with more than 16 query heads: 16 at a time
            const int rows = min(PL_ROWS, unit_n - b0);
            __syncthreads();
            int e_next = it.p0 < it.p1 ? load_page(it.p0) : 0;
            asm volatile("cp.async.commit_group;" ::: "memory");
            for (int i = tid; i < PL_ROWS * cpr; i += PL_THREADS) {
                const int rr = i / cpr, c = (i - rr * cpr) * S::E;
                uint4 val = make_uint4(0u, 0u, 0u, 0u);
                if (rr < rows) {
                    const int row = row_first + b0 + rr;
                    val = *reinterpret_cast<const uint4*>(q + (size_t)(it.q.row0 + row / g) * pb.q_stride + (size_t)(it.h * g + row % g) * d + c);
                }
                const T* p = reinterpret_cast<const T*>(&val);
#pragma unroll
                for (int e = 0; e < S::E; ++e) s_q[rr * S::QS + c + e] = to_f32<T>(p[e]);
            }
            if (tid < PL_ROWS) { s_m[tid] = -INFINITY; s_l[tid] = 0.f; }
            float acc[S::RPT];
#pragma unroll
            for (int i = 0; i < S::RPT; ++i) acc[i] = 0.f;
            // S: this thread's key and first row; the entries its rows see
            const int key = warp * 8 + (lane & 7), rh = (lane >> 3) * 4;
            int see_hi[4], see_lo[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int pos = rh + i < rows ? it.q.len - it.q.n + (row_first + b0 + rh + i) / g : -1;
                see_hi[i] = pos;
                see_lo[i] = pb.window > 0 ? pos + 1 - pb.window : 0;
            }
            const int col = tid % S::COLS, r0 = (tid / S::COLS) * S::RPT;

            for (int p = it.p0; p < it.p1; ++p) {
                const int e0 = e_next;
                const T* s_k = reinterpret_cast<const T*>(s_pl + (p - it.p0) % S::STAGES * S::STAGE);
                const T* s_v = s_k + PAGE * S::KS;
                if (S::STAGES > 1 && p + 1 < it.p1) e_next = load_page(p + 1);
                asm volatile("cp.async.commit_group;" ::: "memory");
                if (S::STAGES > 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
                else asm volatile("cp.async.wait_group 0;" ::: "memory");
                __syncthreads();
                {
                    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
                    for (int c = 0; c < d; c += 4) {
                        const float4 kk = plain_load4<T>(s_k + key * S::KS + c);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float4 qq = *reinterpret_cast<const float4*>(s_q + (rh + i) * S::QS + c);
                            s[i] = fmaf(qq.x, kk.x, fmaf(qq.y, kk.y, fmaf(qq.z, kk.z, fmaf(qq.w, kk.w, s[i]))));
                        }
                    }
                    const int at = e0 + key;
#pragma unroll
                    for (int i = 0; i < 4; ++i) s_p[(rh + i) * PAGE + key] = at <= see_hi[i] && at >= see_lo[i] ? s[i] * scale_log2 : -INFINITY;
                }
                __syncthreads();
                {
                    float a[2], b[2], mx[2], sum[2], m0[2], ref[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int rr = warp * 2 + i;
                        a[i] = s_p[rr * PAGE + lane];
                        b[i] = s_p[rr * PAGE + 32 + lane];
                        m0[i] = s_m[rr];
                        mx[i] = fmaxf(a[i], b[i]);
                    }
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
                        for (int i = 0; i < 2; ++i) mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], o));
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        mx[i] = fmaxf(m0[i], mx[i]);
                        ref[i] = mx[i] == -INFINITY ? 0.f : mx[i];       // a row that has seen nothing yet: every weight is 0
                        a[i] = exp2f(a[i] - ref[i]);
                        b[i] = exp2f(b[i] - ref[i]);
                        sum[i] = a[i] + b[i];
                        s_p[(warp * 2 + i) * PAGE + lane] = a[i];
                        s_p[(warp * 2 + i) * PAGE + 32 + lane] = b[i];
                    }
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
                        for (int i = 0; i < 2; ++i) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
                    if (lane < 2) {
                        const int rr = warp * 2 + lane;
                        const float f = exp2f((lane ? m0[1] : m0[0]) - (lane ? ref[1] : ref[0]));
                        s_a[rr] = f;
                        s_l[rr] = s_l[rr] * f + (lane ? sum[1] : sum[0]);
                        s_m[rr] = lane ? mx[1] : mx[0];
                    }
                }
                __syncthreads();
#pragma unroll
                for (int i = 0; i < S::RPT; ++i) acc[i] *= s_a[r0 + i];
#pragma unroll 4
                for (int e = 0; e < PAGE; e += 4) {
                    float vv[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) vv[u] = to_f32<T>(s_v[(e + u) * DP + col]);
#pragma unroll
                    for (int i = 0; i < S::RPT; ++i) {
                        const float4 pp = *reinterpret_cast<const float4*>(s_p + (r0 + i) * PAGE + e);
                        acc[i] = fmaf(pp.x, vv[0], fmaf(pp.y, vv[1], fmaf(pp.z, vv[2], fmaf(pp.w, vv[3], acc[i]))));
                    }
                }
                __syncthreads();                                  // the buffer and the weights are free
                if (S::STAGES == 1 && p + 1 < it.p1) {
                    e_next = load_page(p + 1);
                    asm volatile("cp.async.commit_group;" ::: "memory");
                }
            }
            __syncthreads();
            if (col < d) {
#pragma unroll
                for (int i = 0; i < S::RPT; ++i) {
                    if (r0 + i >= rows) continue;
                    const int row = row_first + b0 + r0 + i;
                    const float l = s_l[r0 + i], inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
                    if (it.slot < 0) {
                        out[((size_t)(it.q.row0 + row / g) * pb.Hq + (size_t)(it.h * g + row % g)) * d + col] = from_f32<T>(acc[i] * inv);
                    } else {
                        const size_t pr = (size_t)it.slot * unit_rows + b0 + r0 + i;
                        wk.part_o[pr * d + col] = acc[i];
                        if (col == 0) { wk.part_ml[pr * 2] = s_m[r0 + i]; wk.part_ml[pr * 2 + 1] = l; }
                    }
                }
            }
        }
    }
}

// ---------------------------------------------------------------- joining the partials
// The rows of a (token, KV head) whose unit was shared between workers: M = max m, out = sum e^(m - M) O / sum e^(m - M) l,
// in worker order, so the result does not depend on timing.  SPLIT warps per row (units with many parts, few rows in all)
// or SPLIT = 1: a warp walks all g rows of its (token, KV head).  Bound by latency: the request is found by a warp-wide
// search before the wait for the kernel that wrote the partials.
template <typename T, int SPLIT>
__global__ void __launch_bounds__(128)
paged_join_kernel(PagedView pv, PagedBatch pb, T* __restrict__ out, PagedWork wk, int tile_rows, int min_rows, int max_rows) {
    __shared__ float4 s_sum[SPLIT > 1 ? SPLIT : 1][64];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, d = pv.d, g = pb.g;
    const long long item = SPLIT > 1 ? (long long)blockIdx.x : (long long)blockIdx.x * 4 + warp;
    const int heads = SPLIT > 1 ? pb.Hq : pv.H;
    const int t = (int)(item / heads), rest = (int)(item % heads);
    const int h = SPLIT > 1 ? rest / g : rest;
    // cu_new and lens are older than the kernel before this one, which has waited for them
    PagedReq rq;
    const int r = paged_find_request(pb, min(t, pb.T - 1), rq);
    const int j = t - rq.row0;
    const PagedCost c = paged_cost(pb, rq, tile_rows, min_rows, max_rows);
    grid_dependents_may_launch();
    grid_dependency_wait();
    const int workers = (int)wk.prefix[pb.R + 1];                 // 0: the workers had whole units
    if (workers == 0 || t >= pb.T || j < 0 || j >= rq.n || c.U == 0) return;      // (U = 0: another kernel's request)
    const long long total = wk.prefix[pb.R], before = wk.prefix[r];
    const int unit_rows = pb.top > 0 ? g : tile_rows;
    int u_now = -1, w0 = 0, n = 0;
    auto locate = [&](int u) {                                    // the unit's first worker and number of parts
        if (u == u_now) return;
        const long long a = before + (long long)(h * c.U + paged_unfold(u, c.U)) * c.C;
        w0 = paged_owner(total, workers, a);
        n = paged_owner(total, workers, a + c.C - 1) - w0 + 1;
        u_now = u;
    };
    if (SPLIT == 1 && pb.top == 0 && (j * g) / tile_rows == (j * g + g - 1) / tile_rows) {
        // the rows of one unit, in few parts: half a warp per row and every load of the row in flight at once
        locate(j * g / tile_rows);
        if (n == 1) return;
        if (n <= 4) {
            const int l16 = lane & 15;
            for (int j0 = 0; j0 < g; j0 += 2) {
                const int jj = j0 + (lane >> 4);
                const bool on = jj < g;
                const int rr = j * g + jj - u_now * tile_rows;
                float m[4], l[4];
                float4 v[4][4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    m[i] = -INFINITY; l[i] = 0.f;
                    if (on && i < n) {
                        const size_t pr = (size_t)(i == 0 ? 2 * w0 + 1 : 2 * (w0 + i)) * unit_rows + rr;
                        const float2 ml = *reinterpret_cast<const float2*>(wk.part_ml + pr * 2);
                        m[i] = ml.x; l[i] = ml.y;
#pragma unroll
                        for (int x = 0; x < 4; ++x)
                            if (l16 * 4 + x * 64 < d) v[i][x] = *reinterpret_cast<const float4*>(wk.part_o + pr * d + l16 * 4 + x * 64);
                    }
                }
                const float M = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])), ref = M == -INFINITY ? 0.f : M;
                float e[4], L = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) { e[i] = exp2f(m[i] - ref); L = fmaf(e[i], l[i], L); }
                const float inv = L > 0.f ? 1.f / L : (L == 0.f ? 0.f : L);
                T* o = out + ((size_t)t * pb.Hq + (size_t)h * g + jj) * d + l16 * 4;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    if (!on || l16 * 4 + x * 64 >= d) continue;
                    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (i < n) {
                            sum.x = fmaf(e[i], v[i][x].x, sum.x); sum.y = fmaf(e[i], v[i][x].y, sum.y);
                            sum.z = fmaf(e[i], v[i][x].z, sum.z); sum.w = fmaf(e[i], v[i][x].w, sum.w);
                        }
                    o[x * 64] = from_f32<T>(sum.x * inv); o[x * 64 + 1] = from_f32<T>(sum.y * inv);
                    o[x * 64 + 2] = from_f32<T>(sum.z * inv); o[x * 64 + 3] = from_f32<T>(sum.w * inv);
                }
            }
            return;
        }
    }
    for (int jj = SPLIT > 1 ? rest % g : 0; jj < g; ++jj) {
        const int row = j * g + jj, u = pb.top > 0 ? j : row / tile_rows, rr = row - u * unit_rows;
        locate(u);
        if (n > 1) {
            // i-th part: worker w0 began the unit and did not end it (its slot 2 w + 1), the others did not begin it
            auto slot_row = [&](int i) { return (size_t)(i == 0 ? 2 * w0 + 1 : 2 * (w0 + i)) * unit_rows + rr; };
            float M = -INFINITY, L = 0.f;
            for (int i0 = 0; i0 < n; i0 += 32) {
                float m = -INFINITY, l = 0.f;
                if (i0 + lane < n) {
                    const float2 v = *reinterpret_cast<const float2*>(wk.part_ml + slot_row(i0 + lane) * 2);
                    m = v.x; l = v.y;
                }
                float mx = m;
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
                const float Mn = fmaxf(M, mx), ref = Mn == -INFINITY ? 0.f : Mn;
                float s = exp2f(m - ref) * l;
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
                L = L * exp2f(M - ref) + s;
                M = Mn;
            }
            const float ref = M == -INFINITY ? 0.f : M, inv = L > 0.f ? 1.f / L : (L == 0.f ? 0.f : L);
            T* o = out + ((size_t)t * pb.Hq + (size_t)h * g + jj) * d;
            // warp x of SPLIT takes the parts [n x / SPLIT, n (x + 1) / SPLIT)
            const int i_lo = SPLIT > 1 ? n * warp / SPLIT : 0, i_hi = SPLIT > 1 ? n * (warp + 1) / SPLIT : n;
            for (int c0 = lane * 4; c0 < d; c0 += 128) {
                float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
                for (int i0 = i_lo; i0 < i_hi; i0 += 8) {
                    float4 v[8];
                    float f[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                        f[i] = -INFINITY;
                        if (i0 + i < i_hi) {
                            v[i] = *reinterpret_cast<const float4*>(wk.part_o + slot_row(i0 + i) * d + c0);
                            f[i] = wk.part_ml[slot_row(i0 + i) * 2];
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float e = exp2f(f[i] - ref);
                        sum.x = fmaf(e, v[i].x, sum.x); sum.y = fmaf(e, v[i].y, sum.y);
                        sum.z = fmaf(e, v[i].z, sum.z); sum.w = fmaf(e, v[i].w, sum.w);
                    }
                }
                if (SPLIT > 1) s_sum[warp][c0 / 4] = sum;
                else {
                    o[c0] = from_f32<T>(sum.x * inv); o[c0 + 1] = from_f32<T>(sum.y * inv);
                    o[c0 + 2] = from_f32<T>(sum.z * inv); o[c0 + 3] = from_f32<T>(sum.w * inv);
                }
            }
            if (SPLIT > 1) {                                      // n is the same for the whole block
                __syncthreads();
                for (int cc = threadIdx.x; cc < d; cc += 128) {
                    float sum = 0.f;
#pragma unroll
                    for (int x = 0; x < SPLIT; ++x) sum += reinterpret_cast<const float*>(s_sum[x])[cc];
                    o[cc] = from_f32<T>(sum * inv);
                }
            }
        }
        if (SPLIT > 1) break;
    }
}

template <typename T, int DP>
cudaError_t run_plain(const PagedView& pv, const PagedBatch& pb, const void* q, void* out, float scale, const PagedWork& w,
                      cudaStream_t st) {
    using S = PlainShape<T, DP>;
    static std::atomic<unsigned long long> done{0};
    cudaError_t e = paged_allow_smem(reinterpret_cast<const void*>(paged_attn_plain_kernel<T, DP>), S::SMEM, done);
    if (e != cudaSuccess) return e;
    static_assert(S::CTAS <= PAGED_PLAIN_CTAS, "the workspace holds the workers' partial results");
    return paged_launch(paged_attn_plain_kernel<T, DP>, dim3(PAGED_SMS * S::CTAS), dim3(PL_THREADS), S::SMEM, 1, true, st, pv, pb, (const T*)q, (T*)out,
                        scale * LOG2E, w);
}

template <typename T>
cudaError_t run_plain_d(const PagedView& pv, const PagedBatch& pb, const void* q, void* out, float scale, const PagedWork& w,
                        cudaStream_t st) {
    if (pv.d <= 64) return run_plain<T, 64>(pv, pb, q, out, scale, w, st);
    if (pv.d <= 128) return run_plain<T, 128>(pv, pb, q, out, scale, w, st);
    return run_plain<T, 256>(pv, pb, q, out, scale, w, st);
}

}  // namespace

cudaError_t launch_paged_join(const PagedView& pv, const PagedBatch& pb, int is_bf16, void* out, const PagedWork& w, int tile_rows,
                              int min_rows, int max_rows, cudaStream_t st) {
    // A block per row while the GPU holds them all at once; beyond that the parts per row are few and a warp walks a
    // token's rows (measured for 256 tokens x 32 heads in 5 parts: 13 us, a block per row 35).
    const bool split = (long long)pb.T * pb.Hq <= PAGED_SMS * 16;
    const long long items = (long long)pb.T * (split ? pb.Hq : pv.H);
    const dim3 grid((unsigned)(split ? items : (items + 3) / 4)), block(128);
    auto go = [&](auto kernel, auto* o) { return paged_launch(kernel, grid, block, 0, 1, true, st, pv, pb, o, w, tile_rows, min_rows, max_rows); };
    if (is_bf16) return split ? go(paged_join_kernel<__nv_bfloat16, 4>, (__nv_bfloat16*)out) : go(paged_join_kernel<__nv_bfloat16, 1>, (__nv_bfloat16*)out);
    return split ? go(paged_join_kernel<float, 4>, (float*)out) : go(paged_join_kernel<float, 1>, (float*)out);
}

cudaError_t launch_paged_attention_plain(const PagedView& pv, const PagedBatch& pb, int is_bf16, const void* q, void* out,
                                         float scale, const PagedWork& w, cudaStream_t st) {
    const cudaError_t e = is_bf16 ? run_plain_d<__nv_bfloat16>(pv, pb, q, out, scale, w, st)
                                  : run_plain_d<float>(pv, pb, q, out, scale, w, st);
    return e != cudaSuccess ? e : launch_paged_join(pv, pb, is_bf16, out, w, PL_ROWS, 1, INT_MAX, st);
}

}  // namespace tkv
