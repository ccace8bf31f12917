// Which pages of the caller-owned cache a token reads: the pages whose key bounds allow the largest logits.
//
// For token t and KV head h, U(page) = max over the group's query heads of sum_c max(q_c lo_c, q_c hi_c): no key of the
// page has a larger q . k.  The first `sink` and the newest `recent` pages up to the token's own are always read; the
// rest of the `top` places go to the largest U, ties to the lower page.  Only full pages before the token's own are ever
// scored, so the bounds of a page that is still being filled are not looked at.
//
// The order of the scores decides which pages are read, so a rounding could change the result altogether: U is settled in
// 64 bits, where products of bf16 values are exact and a sum's error (128 x 2^-53) is far below the distance of different
// scores.  max(q lo, q hi) = min(q, 0) lo + max(q, 0) hi, so U is a product of the page's 2 d bounds, which lie side by
// side in memory, with the clamped query.
//
// bf16 (paged_select_mma_kernel): the tensor cores compute U for 16 pages x 8 rows at a time in fp32, and beside it the
// sum of the terms' magnitudes A, the same product of absolute values.  An fp32 sum of 2 d exact products is off by less than
// E = A 2 d 2^-23 whatever the order and the rounding of its additions (each off by 2^-23 of a partial sum at most).  The
// m-th largest fp32 score is bracketed to [a, b], by bisection on scores in registers or, for very many, by one histogram;
// pages above b + 2 E are in, pages below a - 2 E are out (E: the largest error of the token's pages), and the few in
// between are scored again in 64 bits.  If all are in
// between (equal bounds, infinities, NaN) all are, and a descent over 64-bit keys decides.  Bound by the latency of its
// chain (request, table, bounds, descent: 33000 cycles for one token with the scores in shared memory, 26000 in registers); the
// bounds are read once per group of tokens.  18 us for one token over 2048 pages x 8 heads, 16 us for 32 tokens over up to 256
// pages (33 MB of bounds: 5 us), 30 us for 232 tokens over up to 133.
//
// fp32 (paged_select_kernel): fp64 sums for every page, eight lanes per page.
//
// In both, a cluster of 1, 2, 4 or 8 CTAs per unit of tokens and KV head -- as many as fill the GPU -- shares the pages, and
// its first CTA collects the scores in its shared memory.
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
paged_select_kernel(PagedView pv, PagedBatch pb, const T* q, int32_t* selected, int nclust, int chunks) {
    extern __shared__ __align__(16) unsigned char s_raw[];
    constexpr int E = 16 / (int)sizeof(T);                        // channels of a 16-byte chunk
    __shared__ int s_hist[256];
    __shared__ int s_digit, s_need, s_count, s_warp[SEL_THREADS / 32];
    const int rank = (int)blockIdx.x % nclust, unit = (int)blockIdx.x / nclust;
    const int t = unit / pv.H, h = unit % pv.H;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int32_t* sel = selected + (size_t)unit * pb.top;
    grid_dependency_wait();
    grid_dependents_may_launch();

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

// ---------------------------------------------------------------- bf16: tensor cores, then 64 bits where it matters
constexpr int SEL_TOKENS = 4;                 // tokens of one unit, at most
constexpr int SEL_KPL = 8;                    // a block alone settles one with up to 8 per thread in registers
constexpr int SEL_WARP_MAX = 512;             // a warp alone settles a token with up to this many candidates
constexpr int SEL_WARP_LIST = 32, SEL_LIST = 512;   // pages between the thresholds that are ranked by counting (warp, block)
constexpr int SEL_BINS = 1024;

__device__ __forceinline__ uint32_t clamp_neg(uint32_t v) {
    const __nv_bfloat162 z = __float2bfloat162_rn(0.f), x = __hmin2_nan(*reinterpret_cast<const __nv_bfloat162*>(&v), z);
    return *reinterpret_cast<const uint32_t*>(&x);
}
__device__ __forceinline__ uint32_t clamp_pos(uint32_t v) {
    const __nv_bfloat162 z = __float2bfloat162_rn(0.f), x = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&v), z);
    return *reinterpret_cast<const uint32_t*>(&x);
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k); }

// The 64-bit key of one page, by a whole warp: eight lanes per head, 8 channels per lane and step, four sums per lane (an
// fp64 fma waits long for the one before it).  The bounds are loaded once, all at the same time.
__device__ __noinline__ u64 exact_key(const __nv_bfloat16* b, const __nv_bfloat16* q, int g, int d) {
    const int lane = threadIdx.x & 31, c0 = (lane & 7) * 8;
    uint4 vlo[4], vhi[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        vlo[i] = vhi[i] = make_uint4(0u, 0u, 0u, 0u);
        if (c0 + i * 64 < d) {
            vlo[i] = *reinterpret_cast<const uint4*>(b + c0 + i * 64);
            vhi[i] = *reinterpret_cast<const uint4*>(b + d + c0 + i * 64);
        }
    }
    double best = -INFINITY;
    bool nan = false;
    for (int h0 = 0; h0 < g; h0 += 4) {
        const int head = h0 + (lane >> 3);
        double s[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i * 64 >= d) break;
            const uint4 vq = head < g && c0 + i * 64 < d ? *reinterpret_cast<const uint4*>(q + (size_t)head * d + c0 + i * 64) : make_uint4(0u, 0u, 0u, 0u);
            const __nv_bfloat16 *xq = reinterpret_cast<const __nv_bfloat16*>(&vq), *xlo = reinterpret_cast<const __nv_bfloat16*>(&vlo[i]),
                                *xhi = reinterpret_cast<const __nv_bfloat16*>(&vhi[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = __bfloat162float(xq[e]);
                s[e & 3] = fma((double)x, (double)__bfloat162float(x > 0.f ? xhi[e] : xlo[e]), s[e & 3]);
            }
        }
        double sum = (s[0] + s[1]) + (s[2] + s[3]);
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (head < g) {
            nan |= sum != sum;
            best = fmax(best, sum);
        }
    }
#pragma unroll
    for (int o = 8; o < 32; o <<= 1) best = fmax(best, __shfl_xor_sync(0xffffffffu, best, o));
    return score_key(__any_sync(0xffffffffu, nan) ? (double)NAN : best);
}

// Sum over the block of each thread's value, and the sum over the threads before it.
__device__ __forceinline__ int block_before(int v, int* s_warp, int& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int incl = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += x;
    }
    __syncthreads();
    if (lane == 31) s_warp[warp] = incl;
    __syncthreads();
    int before = incl - v;
    total = 0;
#pragma unroll
    for (int w = 0; w < SEL_THREADS / 32; ++w) {
        if (w < warp) before += s_warp[w];
        total += s_warp[w];
    }
    return before;
}

// One digit of a radix descent: the bin, from the top, in which the count reaches `need`; need and the bin's count by reference.
__device__ __forceinline__ int pick_digit(const int* s_hist, int* s_pick, int& need, int& count) {
    const int lane = threadIdx.x & 31;
    if (threadIdx.x < 32) {                                       // lane l: bins 255 - 8 l down to 248 - 8 l
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
                if (run < need && need <= run + c[i]) { s_pick[0] = 255 - lane * 8 - i; s_pick[1] = need - run; s_pick[2] = c[i]; }
                run += c[i];
            }
        }
    }
    __syncthreads();
    need = s_pick[1];
    count = s_pick[2];
    return s_pick[0];
}

// One token's selection: n candidates (pages sink ..), of which m < n are taken; scores c[n]; the places of the pages
// taken go to sel[0 .. m), ascending.
struct SelTask {
    const __nv_bfloat16* bounds;  // of the KV head, page 0
    const int32_t* table;         // the request's row
    int32_t* status;
    int n_pages, page_stride;     // pages; elements from one page's bounds to the next
    int first, n, m, g, d;        // first candidate page
    const __nv_bfloat16* q;       // the token's group of query heads
    float* c;
    float mass;                   // largest A of the candidates
    int32_t* sel;
    __device__ __forceinline__ u64 key(int x) const {
        const int phys = table[first + x];
        if (phys >= 0 && phys < n_pages) return exact_key(bounds + (size_t)phys * page_stride, q, g, d);
        latch_error(status, TRIMKV_E_ARG);
        return 0ull;
    }
};
// The band around the m-th largest fp32 score in which 64 bits decide; above it a page is in, below it out.
struct SelBand {
    float below, above;
    bool everything;              // scores that cannot be bounded: all pages are in the band
    __device__ __forceinline__ bool holds(float v) const { return everything || (v <= above && v >= below); }
    __device__ __forceinline__ bool in(float v) const { return !everything && v > above; }
};
// Twice the error of a score, see above; one addition more pays for the rounding of `mass` itself, 1e-33 for products that underflow.
__device__ __forceinline__ float sel_slack(float mass, int d) { return __fadd_ru(__fmul_ru(mass, (float)(2 * d + 1) * (2.0f / 8388608.0f)), 1e-33f); }

// By one warp, KPL scores per lane in registers (n <= 32 KPL).  false: too many pages in the band, nothing written.
template <int KPL>
__device__ __forceinline__ bool select_by_warp(const SelTask& k, int* list, u64* lkey) {
    const int lane = threadIdx.x & 31;
    if (!(k.mass < INFINITY)) return false;
    const float e2 = sel_slack(k.mass, k.d);
    float v[KPL];
    uint32_t key[KPL];
    // [a, b] holds the m-th largest; three pivots a step until it is narrower than the slack
    uint32_t a = ~0u, b = 0u;
#pragma unroll
    for (int i = 0; i < KPL; ++i) {
        const int x = i * 32 + lane;
        v[i] = x < k.n ? k.c[x] : 0.f;
        key[i] = x < k.n ? orderable_key(v[i]) : 0u;              // 0: below every pivot (a score's key is greater)
        if (x < k.n) { a = min(a, key[i]); b = max(b, key[i]); }
    }
    a = __reduce_min_sync(0xffffffffu, a);
    b = __reduce_max_sync(0xffffffffu, b);
    while (a < b && !(key_value(b) - key_value(a) <= e2)) {
        const uint32_t quarter = (b - a) / 4 + 1, p1 = a + quarter, p2 = min(b, p1 - 1 + quarter) + 1, p3 = min(b, p2 - 1 + quarter) + 1;
        uint32_t n123 = 0;                                        // keys >= p1, >= p2, >= p3: ten bits each
#pragma unroll
        for (int i = 0; i < KPL; ++i) n123 += (key[i] >= p1 ? 1u : 0u) + (key[i] >= p2 ? 1u << 10 : 0u) + (key[i] >= p3 ? 1u << 20 : 0u);
        n123 = __reduce_add_sync(0xffffffffu, n123);
        if ((int)(n123 >> 20) >= k.m) a = p3;
        else if ((int)((n123 >> 10) & 1023u) >= k.m) { a = p2; b = p3 - 1; }
        else if ((int)(n123 & 1023u) >= k.m) { a = p1; b = p2 - 1; }
        else b = p1 - 1;
    }
    const SelBand band = {__fadd_rd(key_value(a), -e2), __fadd_ru(key_value(b), e2), false};
    unsigned in[KPL], hold[KPL];                                  // the pages in for certain, the pages of the band
    int sure = 0, held = 0;
#pragma unroll
    for (int i = 0; i < KPL; ++i) {
        const bool real = i * 32 + lane < k.n;
        in[i] = __ballot_sync(0xffffffffu, real && band.in(v[i]));
        hold[i] = __ballot_sync(0xffffffffu, real && band.holds(v[i]));
        sure += __popc(in[i]);
        held += __popc(hold[i]);
    }
    const int left = k.m - sure;
    if (left < held) {
        if (held > SEL_WARP_LIST) return false;
        int at = 0;
#pragma unroll
        for (int i = 0; i < KPL; ++i) {
            if ((hold[i] >> lane) & 1u) list[at + __popc(hold[i] & ((1u << lane) - 1u))] = i * 32 + lane;
            at += __popc(hold[i]);
        }
        __syncwarp();
        for (int i = 0; i < held; ++i) {
            const u64 x = k.key(list[i]);
            if (lane == 0) lkey[i] = x;
        }
        __syncwarp();
        bool take = false;
        if (lane < held) {                                        // the list ascends: among equal keys the lower page comes first
            const u64 x = lkey[lane];
            int above = 0;
            for (int i = 0; i < held; ++i) above += lkey[i] > x || (lkey[i] == x && i < lane);
            take = above < left;
        }
        // bit j of `taken`: the j-th page of the band
        const unsigned taken = __ballot_sync(0xffffffffu, take);
        at = 0;
#pragma unroll
        for (int i = 0; i < KPL; ++i) {
            const int j = at + __popc(hold[i] & ((1u << lane) - 1u));
            at += __popc(hold[i]);
            in[i] |= __ballot_sync(0xffffffffu, ((hold[i] >> lane) & 1u) && ((taken >> (j & 31)) & 1u));
        }
    } else {
#pragma unroll
        for (int i = 0; i < KPL; ++i) in[i] |= hold[i];
    }
    int at = 0;
#pragma unroll
    for (int i = 0; i < KPL; ++i) {
        if ((in[i] >> lane) & 1u) k.sel[at + __popc(in[i] & ((1u << lane) - 1u))] = i * 32 + lane + k.first;
        at += __popc(in[i]);
    }
    return true;
}

struct SelShared {
    int hist[SEL_BINS], pick[3], warp[SEL_THREADS / 32], nlist, list[SEL_LIST];
    uint2 range[2][SEL_THREADS / 32];
    u64 lkey[SEL_LIST];
};

// By the block, KPL scores per thread in registers (n <= KPL x SEL_THREADS): the same bisection, its counts summed over the warps in
// shared memory.  A warp has a run of neighbouring candidates.  false, for the whole block: as above.
template <int KPL>
__device__ __forceinline__ bool select_in_registers(const SelTask& k, SelShared& sh) {
    constexpr int WARPS = SEL_THREADS / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (!(k.mass < INFINITY)) return false;
    const float e2 = sel_slack(k.mass, k.d);
    const int per = (k.n + SEL_THREADS - 1) / SEL_THREADS, x0 = warp * per * 32 + lane;
    float v[KPL];
    uint32_t key[KPL];
    uint32_t a = ~0u, b = 0u;
#pragma unroll
    for (int i = 0; i < KPL; ++i) {
        const bool real = i < per && x0 + i * 32 < k.n;
        v[i] = real ? k.c[x0 + i * 32] : 0.f;
        key[i] = real ? orderable_key(v[i]) : 0u;
        if (real) { a = min(a, key[i]); b = max(b, key[i]); }
    }
    a = __reduce_min_sync(0xffffffffu, a);
    b = __reduce_max_sync(0xffffffffu, b);
    if (lane == 0) sh.range[0][warp] = make_uint2(a, b);
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WARPS; ++w) { a = min(a, sh.range[0][w].x); b = max(b, sh.range[0][w].y); }
    // (two buffers in turn: whoever writes one again has passed the barrier behind which everybody has read it)
    for (int turn = 1; a < b && !(key_value(b) - key_value(a) <= e2); turn ^= 1) {
        const uint32_t quarter = (b - a) / 4 + 1, p1 = a + quarter, p2 = min(b, p1 - 1 + quarter) + 1, p3 = min(b, p2 - 1 + quarter) + 1;
        uint32_t n12 = 0, n3 = 0;                                 // keys >= p1 and >= p2, 16 bits each; >= p3
#pragma unroll
        for (int i = 0; i < KPL; ++i) {
            if (i >= per) break;
            n12 += (key[i] >= p1 ? 1u : 0u) + (key[i] >= p2 ? 1u << 16 : 0u);
            n3 += key[i] >= p3 ? 1u : 0u;
        }
        n12 = __reduce_add_sync(0xffffffffu, n12);
        n3 = __reduce_add_sync(0xffffffffu, n3);
        if (lane == 0) sh.range[turn][warp] = make_uint2(n12, n3);
        __syncthreads();
        n12 = n3 = 0;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) { n12 += sh.range[turn][w].x; n3 += sh.range[turn][w].y; }
        if ((int)n3 >= k.m) a = p3;
        else if ((int)(n12 >> 16) >= k.m) { a = p2; b = p3 - 1; }
        else if ((int)(n12 & 0xffffu) >= k.m) { a = p1; b = p2 - 1; }
        else b = p1 - 1;
    }
    const SelBand band = {__fadd_rd(key_value(a), -e2), __fadd_ru(key_value(b), e2), false};
    unsigned in[KPL], hold[KPL];
    int sure = 0, held = 0, before = 0;
#pragma unroll
    for (int i = 0; i < KPL; ++i) {
        const bool real = i < per && x0 + i * 32 < k.n;
        in[i] = __ballot_sync(0xffffffffu, real && band.in(v[i]));
        hold[i] = __ballot_sync(0xffffffffu, real && band.holds(v[i]));
        sure += __popc(in[i]);
        held += __popc(hold[i]);
    }
    __syncthreads();
    if (lane == 0) sh.range[0][warp] = make_uint2((unsigned)sure, (unsigned)held);
    __syncthreads();
    sure = held = 0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
        if (w == warp) before = held;
        sure += (int)sh.range[0][w].x;
        held += (int)sh.range[0][w].y;
    }
    const int left = k.m - sure;
    const bool some = left < held;
    if (some) {
        if (held > SEL_LIST) return false;
        int at = before;
#pragma unroll
        for (int i = 0; i < KPL; ++i) {
            if ((hold[i] >> lane) & 1u) sh.list[at + __popc(hold[i] & ((1u << lane) - 1u))] = x0 + i * 32;
            at += __popc(hold[i]);
        }
        __syncthreads();
        for (int x = warp; x < held; x += WARPS) {
            const u64 y = k.key(sh.list[x]);
            if (lane == 0) sh.lkey[x] = y;
        }
        __syncthreads();
        for (int x = tid; x < held; x += SEL_THREADS) {           // the list ascends: among equal keys the lower page comes first
            const u64 y = sh.lkey[x];
            int above = 0;
            for (int i = 0; i < held; ++i) above += sh.lkey[i] > y || (sh.lkey[i] == y && i < x);
            sh.hist[x] = above < left;
        }
        __syncthreads();
    }
    int at = before, mine = 0;
#pragma unroll
    for (int i = 0; i < KPL; ++i) {
        if (hold[i]) {
            const bool h = (hold[i] >> lane) & 1u;
            in[i] |= some ? __ballot_sync(0xffffffffu, h && sh.hist[at + __popc(hold[i] & ((1u << lane) - 1u))]) : hold[i];
            at += __popc(hold[i]);
        }
        mine += __popc(in[i]);
    }
    if (lane == 0) sh.warp[warp] = mine;
    __syncthreads();
    at = 0;
    for (int w = 0; w < warp; ++w) at += sh.warp[w];
#pragma unroll
    for (int i = 0; i < KPL; ++i) {
        if ((in[i] >> lane) & 1u) k.sel[at + __popc(in[i] & ((1u << lane) - 1u))] = x0 + i * 32 + k.first;
        at += __popc(in[i]);
    }
    return true;
}

// By the block; keys: [n] 64-bit words of shared memory.
__device__ __noinline__ void select_by_block(const SelTask& k, SelShared& sh, u64* keys) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    SelBand band = {-INFINITY, INFINITY, !(k.mass < INFINITY)};
    __syncthreads();
    for (int i = tid; i < SEL_BINS; i += SEL_THREADS) sh.hist[i] = 0;
    if (tid == 0) sh.nlist = 0;
    if (!band.everything) {
        // one histogram over [min, max]: the bin in which the count from the top reaches m, widened by the slack
        uint32_t kmin = ~0u, kmax = 0u;
        for (int x = tid; x < k.n; x += SEL_THREADS) {
            const uint32_t v = orderable_key(k.c[x]);
            kmin = min(kmin, v);
            kmax = max(kmax, v);
        }
        kmin = __reduce_min_sync(0xffffffffu, kmin);
        kmax = __reduce_max_sync(0xffffffffu, kmax);
        if (lane == 0) sh.range[0][warp] = make_uint2(kmin, kmax);
        __syncthreads();
#pragma unroll
        for (int w = 0; w < SEL_THREADS / 32; ++w) { kmin = min(kmin, sh.range[0][w].x); kmax = max(kmax, sh.range[0][w].y); }
        // the bin of a key: monotone in the key, exact integers
        const uint32_t span = kmax - kmin;
        const int shift = max(0, 32 - __clz((int)span) - 10);     // span >> shift < 1024 (span = 0: shift 0)
        for (int x = tid; x < k.n; x += SEL_THREADS) atomicAdd(&sh.hist[(orderable_key(k.c[x]) - kmin) >> shift], 1);
        __syncthreads();
        int c[4], sum = 0, total;                                 // thread t: bins 1023 - 4 t down to 1020 - 4 t
#pragma unroll
        for (int i = 0; i < 4; ++i) { c[i] = sh.hist[SEL_BINS - 1 - 4 * tid - i]; sum += c[i]; }
        int run = block_before(sum, sh.warp, total);
        if (run < k.m && k.m <= run + sum) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (run < k.m && k.m <= run + c[i]) sh.pick[0] = SEL_BINS - 1 - 4 * tid - i;
                run += c[i];
            }
        }
        __syncthreads();
        const uint32_t a = kmin + ((uint32_t)sh.pick[0] << shift), b = min(kmax, a + ((1u << shift) - 1u));
        const float e2 = sel_slack(k.mass, k.d);
        band.below = __fadd_rd(key_value(a), -e2);
        band.above = __fadd_ru(key_value(b), e2);
    } else
        __syncthreads();
    int sure = 0, held = 0;
    for (int x = tid; x < k.n; x += SEL_THREADS) {
        const float v = k.c[x];
        if (band.holds(v)) {
            ++held;
            const int at = atomicAdd(&sh.nlist, 1);
            if (at < SEL_LIST) sh.list[at] = x;
        } else if (band.in(v)) ++sure;
    }
    int all_sure, all_held;
    block_before(sure | (held << 16), sh.warp, all_sure);         // n <= 16384: both fit
    all_held = all_sure >> 16;
    all_sure &= 0xffff;
    const int left = k.m - all_sure;                              // places for the pages of the band; marked +inf (taken) or -inf
    if (left >= all_held) {
        for (int x = tid; x < k.n; x += SEL_THREADS)
            if (band.holds(k.c[x])) k.c[x] = INFINITY;
    } else if (all_held <= SEL_LIST) {
        for (int x = warp; x < all_held; x += SEL_THREADS / 32) {
            const u64 key = k.key(sh.list[x]);
            if (lane == 0) sh.lkey[x] = key;
        }
        __syncthreads();
        for (int x = tid; x < all_held; x += SEL_THREADS) {
            const u64 key = sh.lkey[x];
            const int at = sh.list[x];
            int above = 0;
            for (int y = 0; y < all_held; ++y) above += sh.lkey[y] > key || (sh.lkey[y] == key && sh.list[y] < at);
            k.c[at] = above < left ? INFINITY : -INFINITY;
        }
    } else {
        for (int x = warp; x < k.n; x += SEL_THREADS / 32) {
            if (!band.holds(k.c[x])) continue;
            const u64 key = k.key(x);
            if (lane == 0) keys[x] = key;
        }
        u64 kp = 0, km = 0;
        int kn = left, kc = 0;
        bool all = false;                                         // every key that matches the prefix is taken
        for (int shift = 56; shift >= 0 && !all; shift -= 8) {
            __syncthreads();
            for (int x = tid; x < 256; x += SEL_THREADS) sh.hist[x] = 0;
            __syncthreads();
            for (int x = tid; x < k.n; x += SEL_THREADS)
                if (band.holds(k.c[x]) && (keys[x] & km) == kp) atomicAdd(&sh.hist[(int)(keys[x] >> shift) & 255], 1);
            __syncthreads();
            kp |= (u64)pick_digit(sh.hist, sh.pick, kn, kc) << shift;
            km |= 255ull << shift;
            all = kc == kn;
        }
        // equal keys: the lower pages; a thread takes a run of neighbouring pages, so one sum over the block counts those before
        const int per = (k.n + SEL_THREADS - 1) / SEL_THREADS, x0 = min(k.n, tid * per), x1 = min(k.n, x0 + per);
        int equal = 0, total;
        for (int x = x0; x < x1; ++x) equal += band.holds(k.c[x]) && (keys[x] & km) == kp;
        int before = block_before(equal, sh.warp, total);
        for (int x = x0; x < x1; ++x) {
            if (!band.holds(k.c[x])) continue;
            const u64 key = keys[x] & km;
            bool take = key > kp;
            if (key == kp) { take = before < kn; ++before; }
            k.c[x] = take ? INFINITY : -INFINITY;
        }
    }
    __syncthreads();
    // ---- the pages taken, ascending: a warp has a run of neighbouring pages
    const int per = ((k.n + SEL_THREADS - 1) / SEL_THREADS) * 32, x0 = min(k.n, warp * per), x1 = min(k.n, x0 + per);
    int mine = 0;
    for (int x = x0; x < x1; x += 32) {
        const bool t = x + lane < x1 && (band.in(k.c[x + lane]) || k.c[x + lane] == INFINITY);
        mine += __popc(__ballot_sync(0xffffffffu, t));
    }
    if (lane == 0) sh.warp[warp] = mine;
    __syncthreads();
    int at = 0;
    for (int w = 0; w < warp; ++w) at += sh.warp[w];
    for (int x = x0; x < x1; x += 32) {
        const bool t = x + lane < x1 && (band.in(k.c[x + lane]) || k.c[x + lane] == INFINITY);
        const unsigned votes = __ballot_sync(0xffffffffu, t);
        if (t) k.sel[at + __popc(votes & ((1u << lane) - 1u))] = k.first + x + lane;
        at += __popc(votes);
    }
}

// grid = ceil(T / ntok) * H clusters.  Dynamic shared memory: 64-bit keys [W], then scores [ntok][W] fp32.
// DK: ceil(d / 32).  NTOK: 1, or up to SEL_TOKENS.  NC: column tiles (8 rows of q each) per walk over the bounds.
template <int DK, int NTOK, int NC>
__global__ void __launch_bounds__(SEL_THREADS, DK <= 4 ? 2 : 1)
paged_select_mma_kernel(PagedView pv, PagedBatch pb, const __nv_bfloat16* q, int32_t* selected, int nclust, int ntok) {
    extern __shared__ __align__(16) unsigned char s_raw[];
    __shared__ int s_req[NTOK], s_np[NTOK], s_hard[NTOK];         // request of each token (-1: none), pages up to its own
    __shared__ unsigned s_err[NTOK];
    __shared__ SelShared sh;
    grid_dependency_wait();
    grid_dependents_may_launch();
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)blockIdx.x % nclust, unit = (int)blockIdx.x / nclust;
    const int unit_t = pb.by_h.div(unit), t0 = unit_t * ntok, h = unit - unit_t * pv.H;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = pb.g, d = pv.d, W = pb.W;
    u64* s_key = reinterpret_cast<u64*>(s_raw);
    float* s_c = reinterpret_cast<float*>(s_raw + (size_t)W * sizeof(u64));
    if (warp < ntok) {
        const int t = t0 + warp;
        int req = -1, np = 0;
        if (t < pb.T) {
            PagedReq rq;
            const int r = paged_find_request(pb, t, rq);
            const int j = t - rq.row0;
            if (j >= 0 && j < rq.n) {                             // else: a row behind the last request, left as it is
                req = r;
                const int pos = rq.len - rq.n + j;
                np = pos < 0 ? 0 : pos / PAGE + 1;
            }
        }
        if (lane == 0) { s_req[warp] = req; s_np[warp] = np; s_err[warp] = 0u; }
    }
    __syncthreads();
    int most = 0;
    for (int i = 0; i < ntok; ++i) most = max(most, s_np[i]);
    if (most > pb.top) {                                          // the same for every CTA of the cluster
        float* c0 = s_c;
        unsigned* err0 = s_err;
        if (nclust > 1) {
            c0 = cluster.map_shared_rank(s_c, 0);
            err0 = cluster.map_shared_rank(s_err, 0);
            cluster.barrier_arrive();                             // this CTA runs and has cleared its errors
        }
        bool arrived = nclust == 1;                               // nothing is written to the first CTA before all have arrived
        auto all_run = [&]() { if (!arrived) { cluster.barrier_wait(); arrived = true; } };
        const int quad = lane & 3, row = lane >> 2;
        for (int i0 = 0; i0 < ntok;) {                            // runs of tokens of one request
            const int r = s_req[i0];
            int i1 = i0 + 1;
            while (i1 < ntok && s_req[i1] == r) ++i1;
            int np = 0;
            for (int i = i0; i < i1; ++i) np = max(np, s_np[i]);
            const int ncand = np > pb.top ? np - pb.recent - pb.sink : 0, ncol = (i1 - i0) * g;
            float worst[NTOK];
#pragma unroll
            for (int i = 0; i < NTOK; ++i) worst[i] = 0.f;
            // Row n of the columns: token t0 + i0 + n / g, head n % g.  The lanes of a quad take 8 channels (16 bytes) each of a
            // 32-channel block: words x and y are the two k pairs of one product, z and w of the next; q is dealt out alike.
            uint4 qv[NC][DK];
            auto load_q = [&](int cb) {
#pragma unroll
                for (int nc = 0; nc < NC; ++nc) {
                    const int n = cb + nc * 8 + row;
                    const int tk = NTOK == 1 || n >= ncol ? 0 : pb.by_g.div(n), head = n >= ncol ? 0 : n - tk * g;
                    const __nv_bfloat16* p = q + (size_t)(t0 + i0 + tk) * pb.q_stride + (size_t)(h * g + head) * d + quad * 8;
#pragma unroll
                    for (int k = 0; k < DK; ++k)
                        qv[nc][k] = n < ncol && k * 32 + quad * 8 < d ? *reinterpret_cast<const uint4*>(p + k * 32) : make_uint4(0u, 0u, 0u, 0u);
                }
            };
            const int tile0 = rank * (SEL_THREADS / 32) + warp;
            if (tile0 * 16 < ncand) load_q(0);
            for (int tile = tile0; tile * 16 < ncand; tile += nclust * (SEL_THREADS / 32)) {
                const int cand = tile * 16 + (lane & 15);
                const int phys = cand < ncand ? paged_physical(pb, pv, r, pb.sink + cand) : -1;
                const int pa = __shfl_sync(0xffffffffu, phys, row), pc = __shfl_sync(0xffffffffu, phys, row + 8);
                const __nv_bfloat16* b = reinterpret_cast<const __nv_bfloat16*>(pv.bounds) + (size_t)h * 2 * d + quad * 8;
                const __nv_bfloat16 *ba = b + (size_t)max(pa, 0) * pv.H * 2 * d, *bc = b + (size_t)max(pc, 0) * pv.H * 2 * d;
                float best[NTOK][2], mass[NTOK][2];
#pragma unroll
                for (int i = 0; i < NTOK; ++i) { best[i][0] = best[i][1] = -INFINITY; mass[i][0] = mass[i][1] = 0.f; }
                for (int cb = 0; cb < ncol; cb += NC * 8) {
                    if (ncol > NC * 8) load_q(cb);
                    float s[NC][4], m[NC][4];
#pragma unroll
                    for (int nc = 0; nc < NC; ++nc)
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[nc][e] = m[nc][e] = 0.f;
                    uint4 va[2][DK], vc[2][DK];                   // lo, hi of the two pages of this lane's rows
#pragma unroll
                    for (int part = 0; part < 2; ++part)
#pragma unroll
                        for (int k = 0; k < DK; ++k) {
                            const bool on = k * 32 + quad * 8 < d;
                            va[part][k] = on && pa >= 0 ? *reinterpret_cast<const uint4*>(ba + part * d + k * 32) : make_uint4(0u, 0u, 0u, 0u);
                            vc[part][k] = on && pc >= 0 ? *reinterpret_cast<const uint4*>(bc + part * d + k * 32) : make_uint4(0u, 0u, 0u, 0u);
                        }
#pragma unroll
                    for (int part = 0; part < 2; ++part)          // lo with min(q, 0), hi with max(q, 0)
#pragma unroll
                        for (int k = 0; k < DK; ++k) {
                            const uint4 xa = va[part][k], xc = vc[part][k];
                            const uint32_t a0[4] = {xa.x, xc.x, xa.y, xc.y}, a1[4] = {xa.z, xc.z, xa.w, xc.w};
                            uint32_t z0[4], z1[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) { z0[e] = a0[e] & 0x7fff7fffu; z1[e] = a1[e] & 0x7fff7fffu; }
#pragma unroll
                            for (int nc = 0; nc < NC; ++nc) {
                                const uint4 x = qv[nc][k];
                                const uint32_t b0 = part ? clamp_pos(x.x) : clamp_neg(x.x), b1 = part ? clamp_pos(x.y) : clamp_neg(x.y);
                                const uint32_t b2 = part ? clamp_pos(x.z) : clamp_neg(x.z), b3 = part ? clamp_pos(x.w) : clamp_neg(x.w);
                                mma_bf16(s[nc], a0, b0, b1);
                                mma_bf16(s[nc], a1, b2, b3);
                                mma_bf16(m[nc], z0, b0 & 0x7fff7fffu, b1 & 0x7fff7fffu);
                                mma_bf16(m[nc], z1, b2 & 0x7fff7fffu, b3 & 0x7fff7fffu);
                            }
                        }
#pragma unroll
                    for (int nc = 0; nc < NC; ++nc)
#pragma unroll
                        for (int cc = 0; cc < 2; ++cc) {          // column 2 quad + cc; elements cc, cc + 2: page rows row, row + 8
                            const int n = cb + nc * 8 + 2 * quad + cc;
                            if (n >= ncol) continue;
                            const int tk = NTOK == 1 ? 0 : pb.by_g.div(n);
#pragma unroll
                            for (int i = 0; i < NTOK; ++i)
                                if (NTOK == 1 || i == tk)
#pragma unroll
                                    for (int e = 0; e < 2; ++e) {
                                        best[i][e] = fmaxf(best[i][e], s[nc][cc + 2 * e]);
                                        // what is not finite cannot be bounded
                                        mass[i][e] = fmaxf(mass[i][e], m[nc][cc + 2 * e] < 3.0e38f ? m[nc][cc + 2 * e] : INFINITY);
                                    }
                        }
                }
                all_run();
#pragma unroll
                for (int i = 0; i < NTOK; ++i) {
                    if (i >= i1 - i0) break;
#pragma unroll
                    for (int o = 1; o < 4; o <<= 1)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            best[i][e] = fmaxf(best[i][e], __shfl_xor_sync(0xffffffffu, best[i][e], o));
                            mass[i][e] = fmaxf(mass[i][e], __shfl_xor_sync(0xffffffffu, mass[i][e], o));
                        }
                    if (quad < 2) {                               // lane 0 of the quad writes page `row`, lane 1 page `row + 8`
                        const int cd = tile * 16 + row + 8 * quad;
                        const int ph = quad ? pc : pa;
                        if (cd < ncand) {
                            c0[(size_t)(i0 + i) * W + cd] = ph < 0 ? -INFINITY : quad ? best[i][1] : best[i][0];
                            if (ph >= 0 && cd < s_np[i0 + i] - pb.recent - pb.sink) worst[i] = fmaxf(worst[i], quad ? mass[i][1] : mass[i][0]);
                        }
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < NTOK; ++i) {
                if (i >= i1 - i0) break;
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) worst[i] = fmaxf(worst[i], __shfl_xor_sync(0xffffffffu, worst[i], o));
                if (lane == 0 && worst[i] > 0.f) atomicMax(err0 + i0 + i, __float_as_uint(worst[i]));     // both >= 0: ordered as integers
            }
            i0 = i1;
        }
        all_run();
        if (nclust > 1) cluster.sync(); else __syncthreads();
    }
    if (rank != 0) return;

    auto task = [&](int i) {
        SelTask k;
        k.bounds = reinterpret_cast<const __nv_bfloat16*>(pv.bounds) + (size_t)h * 2 * d;
        k.table = pb.table + (size_t)s_req[i] * W;
        k.status = pb.status;
        k.n_pages = pv.n_pages;
        k.page_stride = pv.H * 2 * d;
        k.first = pb.sink;
        k.g = g; k.d = d;
        k.n = s_np[i] - pb.recent - pb.sink;
        k.m = pb.top - pb.sink - pb.recent;
        k.q = q + (size_t)(t0 + i) * pb.q_stride + (size_t)h * g * d;
        k.c = s_c + (size_t)i * W;
        k.mass = __uint_as_float(s_err[i]);
        k.sel = selected + ((size_t)(t0 + i) * pv.H + h) * pb.top + pb.sink;
        return k;
    };
    // pages that are always read; whether any are left to choose
    auto always = [&](int i, int x0, int step) {
        const int np = s_np[i];
        int32_t* sel = selected + ((size_t)(t0 + i) * pv.H + h) * pb.top;
        if (np <= pb.top) {
            for (int x = x0; x < pb.top; x += step) sel[x] = x < np ? x : -1;
            return false;
        }
        for (int x = x0; x < pb.sink; x += step) sel[x] = x;
        for (int x = x0; x < pb.recent; x += step) sel[pb.top - pb.recent + x] = np - pb.recent + x;
        return pb.top > pb.sink + pb.recent;
    };
    if (NTOK == 1) {                                              // the block has one token
        if (s_req[0] < 0 || !always(0, tid, SEL_THREADS)) return;
        const SelTask k = task(0);
        if (k.n > SEL_KPL * SEL_THREADS || !select_in_registers<SEL_KPL>(k, sh)) select_by_block(k, sh, s_key);
        return;
    }
    // a warp per token; what is too much for a warp is left to the block
    if (warp < ntok) {
        bool hard = false;
        if (s_req[warp] >= 0 && always(warp, lane, 32)) {
            const SelTask k = task(warp);
            hard = k.n > SEL_WARP_MAX || !(k.n <= 256 ? select_by_warp<8>(k, sh.list + warp * SEL_WARP_LIST, sh.lkey + warp * SEL_WARP_LIST)
                                                      : select_by_warp<16>(k, sh.list + warp * SEL_WARP_LIST, sh.lkey + warp * SEL_WARP_LIST));
        }
        if (lane == 0) s_hard[warp] = hard;
    }
    __syncthreads();
    for (int i = 0; i < ntok; ++i)
        if (s_hard[i]) select_by_block(task(i), sh, s_key);
}

cudaError_t run_select_mma(const PagedView& pv, const PagedBatch& pb, const void* q, int32_t* selected, cudaStream_t st) {
    // Several tokens of one unit share the walk over the bounds: as many as fill 16 columns, if requests have that many and
    // enough units are left for the GPU.  Few units: a cluster shares the pages.
    int ntok = 1;
    while (ntok < SEL_TOKENS && ntok * 2 * pb.g <= 16 && ntok * 2 <= pb.T / pb.R && (long long)pb.T * pv.H / (ntok * 2) >= 2 * PAGED_SMS &&
           (size_t)pb.W * (sizeof(u64) + ntok * 2 * sizeof(float)) <= (size_t)PAGED_SELECT_SMEM / 4) ntok *= 2;
    const long long units = (long long)(pb.T + ntok - 1) / ntok * pv.H;
    int nclust = 1;
    while (nclust < 8 && units * nclust * 2 <= 2 * PAGED_SMS && pb.W > 128 * nclust) nclust *= 2;
    const size_t smem = (size_t)pb.W * (sizeof(u64) + ntok * sizeof(float));
    // Not placed early: its CTAs, waiting, take the registers that the CTAs of the kernel before would free (measured as a dependent
    // launch: 42 instead of 35 us for one token over 128 K, 82 instead of 78 for 32 requests over 16 K).
    auto go = [&](auto kernel, std::atomic<unsigned long long>& done) {
        const cudaError_t e = paged_allow_smem(reinterpret_cast<const void*>(kernel), PAGED_SELECT_SMEM, done);
        if (e != cudaSuccess) return e;
        return paged_launch(kernel, dim3((unsigned)(units * nclust)), dim3(SEL_THREADS), smem, nclust, false, st, pv, pb, (const __nv_bfloat16*)q, selected, nclust, ntok);
    };
    auto by_width = [&](auto dk) {
        constexpr int DK = decltype(dk)::value;
        static std::atomic<unsigned long long> done[3];
        if (ntok > 1) return go(paged_select_mma_kernel<DK, SEL_TOKENS, 2>, done[0]);
        return pb.g <= 8 ? go(paged_select_mma_kernel<DK, 1, 1>, done[1]) : go(paged_select_mma_kernel<DK, 1, 2>, done[2]);
    };
    if (pv.d <= 64) return by_width(std::integral_constant<int, 2>{});
    if (pv.d <= 128) return by_width(std::integral_constant<int, 4>{});
    return by_width(std::integral_constant<int, 8>{});
}

// ---------------------------------------------------------------- fp32
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
    return paged_launch(paged_select_kernel<T>, dim3((unsigned)(units * nclust)), dim3(SEL_THREADS), smem, nclust, false, st, pv, pb, (const T*)q, selected, nclust, chunks);
}

}  // namespace

size_t paged_select_smem(int W, int g, int d, int is_bf16) {
    if (is_bf16) return (size_t)W * (sizeof(u64) + sizeof(float));
    return (size_t)g * ((d / 4 + 7) / 8) * 8 * 4 * sizeof(double) + (size_t)W * sizeof(u64);
}

cudaError_t launch_paged_select(const PagedView& pv, const PagedBatch& pb, int is_bf16, const void* q, int32_t* selected,
                                cudaStream_t st) {
    return is_bf16 ? run_select_mma(pv, pb, q, selected, st) : run_select<float>(pv, pb, q, selected, st);
}

}  // namespace tkv
