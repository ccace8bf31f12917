// Which pages of the caller-owned cache a token reads: the pages whose key bounds allow the largest logits.
//
// For token t and KV head h, U(page) = max over the group's query heads of sum_c max(q_c lo_c, q_c hi_c): no key of the
// page has a larger q . k.  The first `sink` and the newest `recent` pages up to the token's own are always read; the
// rest of the `top` places go to the largest U, ties to the lower page.  Only full pages before the token's own are ever
// scored, so the bounds of a page that is still being filled are not looked at.
//
// The order of the scores decides which pages are read, so a rounding could change the result altogether: the sums are
// held in 64 bits.  The term max(q lo, q hi) is q hi where q > 0 and q lo elsewhere: a select and one fp64 fma.  Products of
// bf16 values are exact there, and the sum's error (128 x 2^-53) is far below the distance of different scores.
//
// One cluster of 1, 2, 4 or 8 CTAs per (token, KV head) -- as many as keep the GPU busy -- shares the pages; eight lanes
// take a page (16 bytes of lo and of hi per lane and step), the queries wait in shared memory as doubles laid out so that
// the eight lanes read 128 consecutive bytes.  The first CTA collects the 64-bit order keys in its shared memory and finds
// the m-th largest by radix descent, eight bits at a time, ending early once a bin holds exactly the places left.
#include <cooperative_groups.h>

#include <atomic>

#include "mma_sync.cuh"
#include "paged.cuh"

namespace tkv {

namespace {

namespace cg = cooperative_groups;

constexpr int SEL_THREADS = 256;

// Larger score, larger key; NaN above everything (what cannot be bounded is read).
__device__ __forceinline__ u64 score_key(double s) {
    if (s != s) return ~0ull;
    const u64 u = (u64)__double_as_longlong(s + 0.0);
    return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}

template <typename T>
__device__ __forceinline__ void widen16(const uint4& v, double (&x)[16 / sizeof(T)]) {
    const T* p = reinterpret_cast<const T*>(&v);
#pragma unroll
    for (int i = 0; i < (int)(16 / sizeof(T)); ++i) x[i] = (double)to_f32<T>(p[i]);
}

// grid = T * H clusters.  Shared memory: queries [g][chunks][E / 2][8] double2, then keys [W], then the flags of the pages.
template <typename T>
__global__ void __launch_bounds__(SEL_THREADS)
paged_select_kernel(PagedView pv, PagedBatch pb, const T* __restrict__ q, int32_t* __restrict__ selected, int nclust, int chunks) {
    extern __shared__ __align__(16) unsigned char s_raw[];
    constexpr int E = 16 / (int)sizeof(T);                        // channels of a 16-byte chunk
    __shared__ int s_hist[256];
    __shared__ int s_digit, s_need, s_count, s_warp[SEL_THREADS / 32];
    const int rank = (int)blockIdx.x % nclust, unit = (int)blockIdx.x / nclust;
    const int t = unit / pv.H, h = unit % pv.H;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int32_t* sel = selected + (size_t)unit * pb.top;

    // the token's request: last r with cu_new[r] <= t
    int lo = 0, hi = pb.R - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (pb.cu_new[mid] <= t) lo = mid; else hi = mid - 1;
    }
    const int r = lo;
    const PagedReq rq = paged_request(pb, r);
    const int j = t - rq.row0;
    const bool mine = rq.n > 0 && j >= 0 && j < rq.n;             // else: a row behind the last request, left as it is
    const int pos = mine ? rq.len - rq.n + j : -1;
    const int np = pos < 0 ? 0 : pos / PAGE + 1;
    if (!mine || np <= pb.top) {                                  // the same for every CTA of the cluster
        if (mine && rank == 0)
            for (int i = tid; i < pb.top; i += SEL_THREADS) sel[i] = i < np ? i : -1;
        return;
    }
    const int g = pb.g, d = pv.d;
    double2* s_q = reinterpret_cast<double2*>(s_raw);
    u64* s_key = reinterpret_cast<u64*>(s_raw + (size_t)g * chunks * 8 * E * sizeof(double));
    const int first = pb.sink, ncand = np - pb.recent - pb.sink;  // candidates: pages first .. first + ncand - 1
    // channel chunk i * 8 + l of a head: pair e at [head][i][e][l]
    for (int idx = tid; idx < g * chunks * (E / 2) * 8; idx += SEL_THREADS) {
        const int l = idx & 7, e = (idx >> 3) % (E / 2), i = (idx >> 3) / (E / 2) % chunks, head = (idx >> 3) / (E / 2) / chunks;
        const int c = (i * 8 + l) * E + 2 * e;
        double2 v = make_double2(0.0, 0.0);
        if (c < d) {
            const T* p = q + (size_t)t * pb.q_stride + (size_t)(h * g + head) * d + c;
            v = make_double2((double)to_f32<T>(p[0]), (double)to_f32<T>(p[1]));
        }
        s_q[idx] = v;
    }
    __syncthreads();
    cg::cluster_group cluster = cg::this_cluster();
    u64* key0 = nclust > 1 ? cluster.map_shared_rank(s_key, 0) : s_key;
    if (nclust > 1) cluster.sync();                               // every CTA runs: its shared memory can be written
    {
        const int l = lane & 7, pg = lane >> 3;
        const int stride = nclust * (SEL_THREADS / 32) * 4;
        for (int c0 = (rank * (SEL_THREADS / 32) + warp) * 4; c0 < ncand; c0 += stride) {
            const int cand = c0 + pg, page = first + cand;
            const int phys = cand < ncand ? paged_physical(pb, pv, r, page) : -1;
            const T* b = reinterpret_cast<const T*>(pv.bounds) + ((size_t)max(phys, 0) * pv.H + h) * 2 * d;
            double best = -INFINITY;
            bool nan = false;
            for (int h0 = 0; h0 < g; h0 += 4) {                   // four heads per walk over the bounds
                double acc[4] = {0.0, 0.0, 0.0, 0.0};
                for (int i = 0; i < chunks; ++i) {
                    const int c = (i * 8 + l) * E;
                    uint4 vlo = make_uint4(0u, 0u, 0u, 0u), vhi = vlo;
                    if (c < d && phys >= 0) {
                        vlo = *reinterpret_cast<const uint4*>(b + c);
                        vhi = *reinterpret_cast<const uint4*>(b + d + c);
                    }
                    double xlo[E], xhi[E];
                    widen16<T>(vlo, xlo);
                    widen16<T>(vhi, xhi);
#pragma unroll
                    for (int hh = 0; hh < 4; ++hh) {
                        if (h0 + hh >= g) break;
                        const double2* qp = s_q + (((size_t)(h0 + hh) * chunks + i) * (E / 2)) * 8 + l;
#pragma unroll
                        for (int e = 0; e < E / 2; ++e) {
                            const double2 qq = qp[e * 8];
                            acc[hh] = fma(qq.x, qq.x > 0.0 ? xhi[2 * e] : xlo[2 * e], acc[hh]);
                            acc[hh] = fma(qq.y, qq.y > 0.0 ? xhi[2 * e + 1] : xlo[2 * e + 1], acc[hh]);
                        }
                    }
                }
#pragma unroll
                for (int hh = 0; hh < 4; ++hh) {
                    if (h0 + hh >= g) break;
#pragma unroll
                    for (int o = 1; o < 8; o <<= 1) acc[hh] += __shfl_xor_sync(0xffffffffu, acc[hh], o);
                    nan |= acc[hh] != acc[hh];
                    best = fmax(best, acc[hh]);
                }
            }
            if (l == 0 && cand < ncand) key0[cand] = phys < 0 ? 0ull : score_key(nan ? (double)NAN : best);
        }
    }
    if (nclust > 1) cluster.sync(); else __syncthreads();
    if (rank != 0) return;

    // ---- the `need` largest of ncand keys: radix descent to the smallest key taken
    const int m = pb.top - pb.sink - pb.recent;
    u64 prefix = 0, mask = 0;
    int need = m;                                                 // places left among the keys that match the prefix
    bool all = m == 0;                                            // true: every key that matches is taken
    for (int shift = 56; shift >= 0 && !all; shift -= 8) {
        for (int i = tid; i < 256; i += SEL_THREADS) s_hist[i] = 0;
        __syncthreads();
        for (int i = tid; i < ncand; i += SEL_THREADS)
            if ((s_key[i] & mask) == prefix) atomicAdd(&s_hist[(int)(s_key[i] >> shift) & 255], 1);
        __syncthreads();
        if (warp == 0) {                                          // lane l: bins 255 - 8 l down to 248 - 8 l
            int c[8], sum = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) { c[i] = s_hist[255 - lane * 8 - i]; sum += c[i]; }
            int incl = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += v;
            }
            int run = incl - sum;
            if (run < need && need <= incl) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (run < need && need <= run + c[i]) { s_digit = 255 - lane * 8 - i; s_need = need - run; s_count = c[i]; }
                    run += c[i];
                }
            }
        }
        __syncthreads();
        prefix |= (u64)s_digit << shift;
        mask |= 255ull << shift;
        need = s_need;
        all = s_count == need;
        __syncthreads();
    }
    // ---- pages in ascending order: taken if the key is above the prefix's range, or matches it and a place is left
    if (m > 0) {
        int taken = 0, equal_before = 0;                          // of the candidates before this block of 256
        for (int i0 = 0; i0 < ncand; i0 += SEL_THREADS) {
            const int i = i0 + tid;
            const u64 k = i < ncand ? s_key[i] : 0ull;
            const bool above = i < ncand && (k & mask) > prefix, equal = i < ncand && (k & mask) == prefix;
            const unsigned eq = __ballot_sync(0xffffffffu, equal);
            if (lane == 0) s_warp[warp] = __popc(eq);
            __syncthreads();
            int before = equal_before, total = 0;
            for (int w = 0; w < SEL_THREADS / 32; ++w) { if (w < warp) before += s_warp[w]; total += s_warp[w]; }
            equal_before += total;
            before += __popc(eq & ((1u << lane) - 1u));
            const bool take = above || (equal && before < need);
            __syncthreads();
            const unsigned tk = __ballot_sync(0xffffffffu, take);
            if (lane == 0) s_warp[warp] = __popc(tk);
            __syncthreads();
            int at = taken;
            total = 0;
            for (int w = 0; w < SEL_THREADS / 32; ++w) { if (w < warp) at += s_warp[w]; total += s_warp[w]; }
            taken += total;
            if (take) sel[pb.sink + at + __popc(tk & ((1u << lane) - 1u))] = first + i;
            __syncthreads();
        }
    }
    for (int i = tid; i < pb.sink; i += SEL_THREADS) sel[i] = i;
    for (int i = tid; i < pb.recent; i += SEL_THREADS) sel[pb.top - pb.recent + i] = np - pb.recent + i;
}

template <typename T>
cudaError_t run_select(const PagedView& pv, const PagedBatch& pb, const void* q, int32_t* selected, cudaStream_t st) {
    constexpr int E = 16 / (int)sizeof(T);
    const int chunks = (pv.d / E + 7) / 8;
    // Pages of one (token, head) are shared out only while there are few of them: a CTA for every SM and some to spare
    // is enough, and more CTAs per unit only wait for the first one.
    const long long units = (long long)pb.T * pv.H;
    int nclust = 1;
    while (nclust < 8 && units * nclust < 2 * PAGED_SMS && pb.W > 64 * nclust) nclust *= 2;
    const size_t smem = (size_t)pb.g * chunks * 8 * E * sizeof(double) + (size_t)pb.W * sizeof(u64);
    static std::atomic<unsigned long long> done{0};
    const cudaError_t e = paged_allow_smem(reinterpret_cast<const void*>(paged_select_kernel<T>), PAGED_SELECT_SMEM, done);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(units * nclust));
    cfg.blockDim = dim3(SEL_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = nclust;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    count_launch();
    return cudaLaunchKernelEx(&cfg, paged_select_kernel<T>, pv, pb, (const T*)q, selected, nclust, chunks);
}

}  // namespace

size_t paged_select_smem(int W, int g, int d, int is_bf16) {
    const int E = is_bf16 ? 8 : 4, chunks = (d / E + 7) / 8;
    return (size_t)g * chunks * 8 * E * sizeof(double) + (size_t)W * sizeof(u64);
}

cudaError_t launch_paged_select(const PagedView& pv, const PagedBatch& pb, int is_bf16, const void* q, int32_t* selected,
                                cudaStream_t st) {
    return is_bf16 ? run_select<__nv_bfloat16>(pv, pb, q, selected, st) : run_select<float>(pv, pb, q, selected, st);
}

}  // namespace tkv
