// Attention of new tokens over the caller-owned paged cache: the form for any head size and type, and the kernel that joins
// partial results.
//
// Plain form.  A CTA of 128 threads holds 16 (token, query head) rows of one KV head and walks its share of the pages
// (paged_item): 64 keys at a time, widened to fp32 in shared memory; S = Q K^T with one key per thread and 8 rows in
// registers, the running maximum and sum of the softmax per row, then O += P V with a column of O per thread.  All sums are
// fp32.  fp32 caches and head sizes other than 64 and 128 run here; bound by shared-memory reads and FMAs beyond a few
// rows per page, by the page loads below that.
#include "mma_sync.cuh"
#include "paged.cuh"

namespace tkv {

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr int PL_THREADS = 128, PL_ROWS = PAGED_PLAIN_ROWS;

// DP: head size rounded up to 64, 128 or 256
template <typename T, int DP>
struct PlainShape {
    static constexpr int KS = DP + 4;                             // row stride of K and Q in shared memory (floats)
    static constexpr int COLS = DP < PL_THREADS ? DP : PL_THREADS;
    static constexpr int RG = PL_THREADS / COLS, CPT = DP / COLS; // row groups, columns of O per thread
    static constexpr int RPT = PL_ROWS / RG;                      // rows of O per thread
    static constexpr int SMEM = (int)sizeof(float) * (PAGE * KS + PAGE * DP + PL_ROWS * KS + PL_ROWS * PAGE) + 3 * PL_ROWS * 4;
};

template <typename T, int DP>
__global__ void __launch_bounds__(PL_THREADS)
paged_attn_plain_kernel(PagedView pv, PagedBatch pb, const T* __restrict__ q, T* __restrict__ out, float scale_log2, PagedWork wk,
                        int max_workers) {
    using S = PlainShape<T, DP>;
    extern __shared__ __align__(16) float s_f[];
    __shared__ long long s_grp[PAGED_GROUPS + 1];
    float* s_k = s_f;                                             // [64][KS]
    float* s_v = s_k + PAGE * S::KS;                              // [64][DP]
    float* s_q = s_v + PAGE * DP;                                 // [16][KS]
    float* s_p = s_q + PL_ROWS * S::KS;                           // [16][64]
    float* s_m = s_p + PL_ROWS * PAGE;                            // running maximum, sum, factor of this step
    float* s_l = s_m + PL_ROWS;
    float* s_a = s_l + PL_ROWS;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, d = pv.d, g = pb.g;
    constexpr int E = 16 / (int)sizeof(T);
    const int cpr = d / E;

    grid_dependency_wait();
    PagedTable tab;
    const int unit_rows = pb.top > 0 ? g : PL_ROWS;               // rows of a unit (top > 0: one token)
    paged_build_table(tab, pb, pv.H, PL_ROWS, 1, INT_MAX, max_workers, 2, s_grp, wk.prefix);
    grid_dependents_may_launch();
    const int w = blockIdx.x;
    if (w >= tab.workers) return;
    const long long end = paged_share(tab.total, tab.workers, w + 1);
    for (int i = tid; i < PL_ROWS * S::KS; i += PL_THREADS) s_q[i] = 0.f;
    for (int i = tid; i < PAGE * S::KS; i += PL_THREADS) s_k[i] = 0.f;
    for (int i = tid; i < PAGE * DP; i += PL_THREADS) s_v[i] = 0.f;

    for (long long x = paged_share(tab.total, tab.workers, w); x < end;) {
        const PagedItem it = paged_item(tab, pb, x, end, w);
        x += it.steps;
        const int row_first = pb.top > 0 ? it.u * g : it.u * PL_ROWS;    // of the request's n * g rows
        const int unit_n = min(unit_rows, it.q.n * g - row_first);
        for (int b0 = 0; b0 < unit_n; b0 += PL_ROWS) {           // a token with more than 16 query heads: 16 at a time
            const int rows = min(PL_ROWS, unit_n - b0);
            __syncthreads();
            for (int i = tid; i < PL_ROWS * cpr; i += PL_THREADS) {
                const int rr = i / cpr, c = (i - rr * cpr) * E;
                uint4 val = make_uint4(0u, 0u, 0u, 0u);
                if (rr < rows) {
                    const int row = row_first + b0 + rr;
                    val = *reinterpret_cast<const uint4*>(q + (size_t)(it.q.row0 + row / g) * pb.q_stride + (size_t)(it.h * g + row % g) * d + c);
                }
                const T* p = reinterpret_cast<const T*>(&val);
#pragma unroll
                for (int e = 0; e < E; ++e) s_q[rr * S::KS + c + e] = to_f32<T>(p[e]);
            }
            if (tid < PL_ROWS) { s_m[tid] = -INFINITY; s_l[tid] = 0.f; }
            float acc[S::CPT][S::RPT];
#pragma unroll
            for (int c = 0; c < S::CPT; ++c)
#pragma unroll
                for (int i = 0; i < S::RPT; ++i) acc[c][i] = 0.f;

            for (int p = it.p0; p < it.p1; ++p) {
                const int page = pb.top > 0 ? pb.selected[((size_t)(it.q.row0 + it.u) * pv.H + it.h) * pb.top + p] : p;
                const int phys = paged_physical(pb, pv, it.r, page);
                if (phys < 0) continue;                          // the same for every thread
                const int e0 = page * PAGE, held = min(PAGE, it.q.len - e0);   // rows of the page that hold entries
                __syncthreads();                                  // the last page's products are done
                const T* kp = reinterpret_cast<const T*>(pv.k) + ((size_t)phys * pv.H + it.h) * PAGE * d;
                const T* vp = reinterpret_cast<const T*>(pv.v) + ((size_t)phys * pv.H + it.h) * PAGE * d;
                for (int i = tid; i < PAGE * cpr; i += PL_THREADS) {
                    const int e = i / cpr, c = (i - e * cpr) * E;
                    uint4 kv = make_uint4(0u, 0u, 0u, 0u), vv = kv;           // what lies behind the last entry is not read
                    if (e < held) {
                        kv = *reinterpret_cast<const uint4*>(kp + (size_t)e * d + c);
                        vv = *reinterpret_cast<const uint4*>(vp + (size_t)e * d + c);
                    }
                    const T* pk = reinterpret_cast<const T*>(&kv);
                    const T* pvv = reinterpret_cast<const T*>(&vv);
#pragma unroll
                    for (int u = 0; u < E; ++u) { s_k[e * S::KS + c + u] = to_f32<T>(pk[u]); s_v[e * DP + c + u] = to_f32<T>(pvv[u]); }
                }
                __syncthreads();
                {                                                 // S: key tid & 63, rows 8 (tid / 64) ..
                    const int key = tid & 63, rh = (tid >> 6) * (PL_ROWS / 2);
                    float s[PL_ROWS / 2];
#pragma unroll
                    for (int i = 0; i < PL_ROWS / 2; ++i) s[i] = 0.f;
                    for (int c = 0; c < d; c += 4) {
                        const float4 kk = *reinterpret_cast<const float4*>(s_k + key * S::KS + c);
#pragma unroll
                        for (int i = 0; i < PL_ROWS / 2; ++i) {
                            const float4 qq = *reinterpret_cast<const float4*>(s_q + (rh + i) * S::KS + c);
                            s[i] = fmaf(qq.x, kk.x, fmaf(qq.y, kk.y, fmaf(qq.z, kk.z, fmaf(qq.w, kk.w, s[i]))));
                        }
                    }
#pragma unroll
                    for (int i = 0; i < PL_ROWS / 2; ++i) {
                        const int pos = it.q.len - it.q.n + (row_first + b0 + rh + i) / g, at = e0 + key;
                        const bool on = rh + i < rows && at <= pos && (pb.window <= 0 || at > pos - pb.window);
                        s_p[(rh + i) * PAGE + key] = on ? s[i] * scale_log2 : -INFINITY;
                    }
                }
                __syncthreads();
                for (int rr = warp; rr < PL_ROWS; rr += PL_THREADS / 32) {
                    const float a = s_p[rr * PAGE + lane], b = s_p[rr * PAGE + 32 + lane];
                    float mx = fmaxf(a, b);
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
                    const float m0 = s_m[rr], mn = fmaxf(m0, mx);
                    const float ref = mn == -INFINITY ? 0.f : mn; // a row that has seen nothing yet: every weight is 0
                    const float pa = exp2f(a - ref), pbv = exp2f(b - ref);
                    float sum = pa + pbv;
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                    s_p[rr * PAGE + lane] = pa;
                    s_p[rr * PAGE + 32 + lane] = pbv;
                    __syncwarp();
                    if (lane == 0) {
                        const float f = exp2f(m0 - ref);
                        s_a[rr] = f;
                        s_l[rr] = s_l[rr] * f + sum;
                        s_m[rr] = mn;
                    }
                    __syncwarp();
                }
                __syncthreads();
                {
                    const int col = tid % S::COLS, r0 = (tid / S::COLS) * S::RPT;
#pragma unroll
                    for (int i = 0; i < S::RPT; ++i) {
                        const float f = s_a[r0 + i];
#pragma unroll
                        for (int c = 0; c < S::CPT; ++c) acc[c][i] *= f;
                    }
                    for (int e = 0; e < PAGE; e += 4) {
                        float vv[S::CPT][4];
#pragma unroll
                        for (int u = 0; u < 4; ++u)
#pragma unroll
                            for (int c = 0; c < S::CPT; ++c) vv[c][u] = s_v[(e + u) * DP + col + c * S::COLS];
#pragma unroll
                        for (int i = 0; i < S::RPT; ++i) {
                            const float4 pp = *reinterpret_cast<const float4*>(s_p + (r0 + i) * PAGE + e);
#pragma unroll
                            for (int c = 0; c < S::CPT; ++c)
                                acc[c][i] = fmaf(pp.x, vv[c][0], fmaf(pp.y, vv[c][1], fmaf(pp.z, vv[c][2], fmaf(pp.w, vv[c][3], acc[c][i]))));
                        }
                    }
                }
            }
            __syncthreads();
            const int col = tid % S::COLS, r0 = (tid / S::COLS) * S::RPT;
#pragma unroll
            for (int i = 0; i < S::RPT; ++i) {
                if (r0 + i >= rows) continue;
                const int row = row_first + b0 + r0 + i;
                const float l = s_l[r0 + i], inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
#pragma unroll
                for (int c = 0; c < S::CPT; ++c) {
                    const int dd = col + c * S::COLS;
                    if (dd >= d) continue;
                    if (it.slot < 0)
                        out[((size_t)(it.q.row0 + row / g) * pb.Hq + (size_t)(it.h * g + row % g)) * d + dd] = from_f32<T>(acc[c][i] * inv);
                    else
                        wk.part_o[((size_t)it.slot * unit_rows + b0 + r0 + i) * d + dd] = acc[c][i];
                }
                if (it.slot >= 0 && col == 0) {
                    float* ml = wk.part_ml + ((size_t)it.slot * unit_rows + b0 + r0 + i) * 2;
                    ml[0] = s_m[r0 + i];
                    ml[1] = l;
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
    if (t >= pb.T) return;
    PagedReq rq;
    const int r = paged_find_request(pb, t, rq);
    const int j = t - rq.row0;
    if (j < 0 || j >= rq.n) return;
    const PagedCost c = paged_cost(pb, rq, tile_rows, min_rows, max_rows);
    if (c.U == 0) return;                                         // another kernel's request
    grid_dependency_wait();
    const long long total = wk.prefix[pb.R], before = wk.prefix[r];
    const int workers = (int)wk.prefix[pb.R + 1];
    const int unit_rows = pb.top > 0 ? g : tile_rows;
    int u_now = -1, w0 = 0, n = 0;
    for (int jj = SPLIT > 1 ? rest % g : 0; jj < g; ++jj) {
        const int row = j * g + jj, u = pb.top > 0 ? j : row / tile_rows, rr = row - u * unit_rows;
        if (u != u_now) {
            const long long a = before + ((long long)h * c.U + paged_unfold(u, c.U)) * c.C;
            w0 = paged_owner(total, workers, a);
            n = paged_owner(total, workers, a + c.C - 1) - w0 + 1;
            u_now = u;
        }
        if (SPLIT == 1 && n > 1 && n <= 4) {                      // few parts: every load of the row in flight at once
            float m[4], l[4];
            float4 v[4][2];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                m[i] = -INFINITY; l[i] = 0.f;
                v[i][0] = v[i][1] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (i < n) {
                    const size_t pr = (size_t)(i == 0 ? 2 * w0 + 1 : 2 * (w0 + i)) * unit_rows + rr;
                    const float2 ml = *reinterpret_cast<const float2*>(wk.part_ml + pr * 2);
                    m[i] = ml.x; l[i] = ml.y;
#pragma unroll
                    for (int x = 0; x < 2; ++x)
                        if (lane * 4 + x * 128 < d) v[i][x] = *reinterpret_cast<const float4*>(wk.part_o + pr * d + lane * 4 + x * 128);
                }
            }
            const float M = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])), ref = M == -INFINITY ? 0.f : M;
            float e[4], L = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) { e[i] = exp2f(m[i] - ref); L = fmaf(e[i], l[i], L); }
            const float inv = L > 0.f ? 1.f / L : (L == 0.f ? 0.f : L);
            T* o = out + ((size_t)t * pb.Hq + (size_t)h * g + jj) * d + lane * 4;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                if (lane * 4 + x * 128 >= d) continue;
                float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    sum.x = fmaf(e[i], v[i][x].x, sum.x); sum.y = fmaf(e[i], v[i][x].y, sum.y);
                    sum.z = fmaf(e[i], v[i][x].z, sum.z); sum.w = fmaf(e[i], v[i][x].w, sum.w);
                }
                o[x * 128] = from_f32<T>(sum.x * inv); o[x * 128 + 1] = from_f32<T>(sum.y * inv);
                o[x * 128 + 2] = from_f32<T>(sum.z * inv); o[x * 128 + 3] = from_f32<T>(sum.w * inv);
            }
        } else if (n > 1) {
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
                      bool dependent, cudaStream_t st) {
    using S = PlainShape<T, DP>;
    static std::atomic<unsigned long long> done{0};
    cudaError_t e = paged_allow_smem(reinterpret_cast<const void*>(paged_attn_plain_kernel<T, DP>), S::SMEM, done);
    if (e != cudaSuccess) return e;
    const int workers = PAGED_SMS * PAGED_PLAIN_CTAS;
    count_launch();
    const dim3 grid(workers), block(PL_THREADS);
    if (dependent)
        return launch_dependent(paged_attn_plain_kernel<T, DP>, grid, block, S::SMEM, st, pv, pb, (const T*)q, (T*)out, scale * LOG2E, w, workers);
    paged_attn_plain_kernel<T, DP><<<grid, block, S::SMEM, st>>>(pv, pb, (const T*)q, (T*)out, scale * LOG2E, w, workers);
    return cudaGetLastError();
}

template <typename T>
cudaError_t run_plain_d(const PagedView& pv, const PagedBatch& pb, const void* q, void* out, float scale, const PagedWork& w,
                        bool dependent, cudaStream_t st) {
    if (pv.d <= 64) return run_plain<T, 64>(pv, pb, q, out, scale, w, dependent, st);
    if (pv.d <= 128) return run_plain<T, 128>(pv, pb, q, out, scale, w, dependent, st);
    return run_plain<T, 256>(pv, pb, q, out, scale, w, dependent, st);
}

}  // namespace

cudaError_t launch_paged_join(const PagedView& pv, const PagedBatch& pb, int is_bf16, void* out, const PagedWork& w, int tile_rows,
                              int min_rows, int max_rows, bool many_rows, cudaStream_t st) {
    // A block per row while the GPU holds them all at once; beyond that the parts per row are few and a warp walks a
    // token's rows.
    const bool split = !many_rows && (long long)pb.T * pb.Hq <= PAGED_SMS * 16;
    const long long items = (long long)pb.T * (split ? pb.Hq : pv.H);
    const dim3 grid((unsigned)(split ? items : (items + 3) / 4)), block(128);
    count_launch();
    auto go = [&](auto kernel, auto* o) { return launch_dependent(kernel, grid, block, 0, st, pv, pb, o, w, tile_rows, min_rows, max_rows); };
    if (is_bf16) return split ? go(paged_join_kernel<__nv_bfloat16, 4>, (__nv_bfloat16*)out) : go(paged_join_kernel<__nv_bfloat16, 1>, (__nv_bfloat16*)out);
    return split ? go(paged_join_kernel<float, 4>, (float*)out) : go(paged_join_kernel<float, 1>, (float*)out);
}

cudaError_t launch_paged_attention_plain(const PagedView& pv, const PagedBatch& pb, int is_bf16, const void* q, void* out,
                                         float scale, const PagedWork& w, bool dependent, cudaStream_t st) {
    const cudaError_t e = is_bf16 ? run_plain_d<__nv_bfloat16>(pv, pb, q, out, scale, w, dependent, st)
                                  : run_plain_d<float>(pv, pb, q, out, scale, w, dependent, st);
    return e != cudaSuccess ? e : launch_paged_join(pv, pb, is_bf16, out, w, PL_ROWS, 1, INT_MAX, false, st);
}

}  // namespace tkv
