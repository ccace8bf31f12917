// Rows of a block table that share pages: forks, growth and release by reference counts, and dropping entries by keep bits.
//
// Both are one launch of one cluster of 16 CTAs, 512 warps.  Page numbers are dealt out in (row, place) order, so the result is a pure function of
// the inputs although the counts are kept with atomics: counts are sums of whole numbers, and who of several rows keeps or
// returns a page is settled by a minimum over row numbers, taken in the count itself (a count of 0 becomes negative while it is
// in dispute).  The cluster barrier orders the steps; per-row and per-stretch counts go to every CTA's shared memory
// through the cluster, and every CTA computes the prefix sums that place things for itself.
//
// Share: refs_out = refs - the rows' old holds + those that go on; a partly filled page that a row will write stays with the lowest such
// row if no other holds it, the others take a fresh page and list its rows to be copied; pages left without a holder go
// on the stack; fresh pages come from its top.
// Compact: a row's pages up to the first dropped entry's stay, the entries kept from there on are listed to be moved to fresh pages, the old pages are
// released.  Fresh pages are taken before any is released, so no listed source is a destination.
// Both are bound by latency, five to six cluster barriers and the way to memory between them: a share of 64 beams of 2.3 K entries 13.2 us, of 128
// samples of 8 prompts of up to 16 K 16.0 us (losses and gains apart, rows and tokens by the same warps as stretches, lists summed one by
// one: 17.9 and 21.0; three barriers more: 20.4 and 24.7); a compact of one request of 4 K entries 10.1 us, of 32 of up to 32 K (1 MB of
// listed rows) 22.0 us.  (A warp to each row's bits, and 32 words at a time in exchanges of registers: 15.9 and 34.8.)
#include <cooperative_groups.h>

#include <algorithm>

#include "paged.cuh"
#include "paged_share.cuh"

namespace tkv {

namespace {

namespace cg = cooperative_groups;

constexpr int SH_CTAS = 16, SH_THREADS = 1024, SH_WARPS = SH_CTAS * SH_THREADS / 32;
constexpr int SH_TASKS = 512;                 // stretches of rows, if there are fewer rows than that: one for each warp
// Kept entries of a word of 64 up to which lanes look for theirs: 32 rows of 32 K entries, an eighth kept, 21.4 us that way and 26.7 with a
// word after another; a quarter 25.6 and 26.8; 0.4 30.5 and 26.8.
constexpr int SH_SPARSE = 16;
constexpr int SH_FIRST = 2 * PAGED_MAX_REQ;   // see the dispute over pages that nobody holds

__device__ __forceinline__ int sh_pages(int n) { return (int)(((unsigned)n + PAGE - 1u) / PAGE); }
__device__ __forceinline__ int sh_ld(const int32_t* p) { return __ldcg(p); }      // written by other CTAs

// A row's table places are cut into nseg stretches of seg places (a multiple of 32); stretch t belongs to row t / nseg.
struct ShareCut { int nseg, seg, tasks; };
__host__ __device__ inline ShareCut share_cut(int R, int W) {
    ShareCut c;
    const int most = (W + 31) / 32;
    int n = R >= SH_TASKS ? 1 : SH_TASKS / R;
    n = n < most ? n : most;
    c.seg = ((W + n - 1) / n + 31) / 32 * 32;
    c.nseg = (W + c.seg - 1) / c.seg;
    c.tasks = R * c.nseg;
    return c;
}

// Up to four lists at once, a quarter of the block each: v[0 .. n] = sums before each of v[0 .. n - 1]; the block calls it.  Sums fit 32
// bits.  w: 32 ints of shared memory.
struct ShareList { int* v; int n; };          // null: none
__device__ __forceinline__ void share_scan(int* w, ShareList a, ShareList b = {nullptr, 0}, ShareList c = {nullptr, 0}, ShareList d = {nullptr, 0}) {
    constexpr int QUARTER = SH_THREADS / 4;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, q = threadIdx.x / QUARTER, id = threadIdx.x % QUARTER;
    const ShareList mine_of = q == 0 ? a : q == 1 ? b : q == 2 ? c : d;
    int* v = mine_of.v;
    const int n = v ? mine_of.n : 0, per = (n + QUARTER - 1) / QUARTER, i0 = min(n, id * per), i1 = min(n, i0 + per);
    int mine = 0;
    for (int i = i0; i < i1; ++i) mine += v[i];
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += u;
    }
    if (lane == 31) w[warp] = incl;
    __syncthreads();
    int run = incl - mine;                    // and the quarter's warps before this one
    for (int k = q * (QUARTER / 32); k < warp; ++k) run += w[k];
    for (int i = i0; i < i1; ++i) { const int x = v[i]; v[i] = run; run += x; }
    if (id == QUARTER - 1 && v) v[n] = run;
    __syncthreads();
}

// Last r with at[r] <= x (at ascending, at[0] = 0, x < at[n]); rows without any are passed over.
__device__ __forceinline__ int share_find(const int* at, int n, int x) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (at[mid] <= x) lo = mid; else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ void share_tell(cg::cluster_group& cluster, int* slot, int v) {      // *slot = v in every CTA
    for (int i = 0; i < SH_CTAS; ++i) *cluster.map_shared_rank(slot, i) = v;
}

// Counts and the live part of the stack, where they are kept apart from the inputs.
__device__ __forceinline__ void share_copy(const ShareArgs& a, int fc, int gt, int GT) {
    if (a.refs_out != a.refs)
        for (int i = gt; i < a.n_pages; i += GT) a.refs_out[i] = a.refs[i];
    if (a.free_out != a.free_pages)
        for (int i = gt; i < min(max(fc, 0), a.n_pages); i += GT) a.free_out[i] = a.free_pages[i];
}

__device__ __forceinline__ void share_none_moved(const ShareArgs& a, int from, int gt, int GT) {
    for (int i = from + gt; i < a.max_moves; i += GT) { a.move_src[i] = -1; a.move_dst[i] = -1; }
    if (gt == 0) *a.move_count = from;
}

// ---------------------------------------------------------------- share

// What row r of a share is.
struct ShareRow {
    int source, old, keep, now;
    int stay;                                 // pages that it goes on holding without writing them
    bool writes;                              // page keep / 64 of its source is partly filled and will be written
};
__device__ __forceinline__ ShareRow share_row(const ShareArgs& a, int r) {
    ShareRow s;
    s.source = a.source[r]; s.old = a.old_lens[r]; s.keep = a.keep_lens[r]; s.now = a.new_lens[r];
    s.writes = s.keep % PAGE != 0 && s.now > s.keep;
    s.stay = s.writes ? s.keep / PAGE : sh_pages(s.keep);
    return s;
}

__global__ void __launch_bounds__(SH_THREADS, 1)
paged_share_kernel(ShareArgs a) {
    extern __shared__ int s_share[];
    __shared__ int s_w[32], s_bad;
    __shared__ long long s_total;
    const int R = a.R, W = a.W;
    const ShareCut cut = share_cut(R, W);
    int* s_tok = s_share;                     // [R + 1] each: per row, then sums before it
    int* s_take = s_tok + R + 1;
    int* s_move = s_take + R + 1;
    int* s_back = s_move + R + 1;             // [tasks + 1]
    cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, lane = tid & 31, rank = (int)cluster.block_rank();
    const int gt = rank * SH_THREADS + tid, GT = SH_CTAS * SH_THREADS, gw = rank * (SH_THREADS / 32) + (tid >> 5);
    const int gt_row = GT - 1 - gt, gt_move = gt ^ (GT / 2);      // rows and tokens, and moves, go to warps without stretches first
    if (tid == 0) { s_bad = 0; s_total = 0; }
    grid_dependency_wait();
    grid_dependents_may_launch();
    __syncthreads();
    const int fc = *a.free_count;

    // ---- lengths
    const int cap = W * PAGE;
    long long tokens_mine = 0;
    for (int r = tid; r < R; r += SH_THREADS) {
        const int src = a.source[r], o = a.old_lens[r], k = a.keep_lens[r], n = a.new_lens[r];
        const int so = src >= 0 && src < R ? a.old_lens[src] : 0;
        if (src < -1 || src >= R || o < 0 || o > cap || n < 0 || n > cap || k < 0 || k > so || k > n) { s_bad = TRIMKV_E_ARG; continue; }
        tokens_mine += n - k;
        s_tok[r] = n - k;
        s_take[r] = sh_pages(n) - sh_pages(k);        // and one more where a page is copied
        s_move[r] = 0;
    }
    for (int o = 16; o > 0; o >>= 1) tokens_mine += __shfl_xor_sync(0xffffffffu, tokens_mine, o);
    if (lane == 0 && tokens_mine) atomicAdd(reinterpret_cast<unsigned long long*>(&s_total), (unsigned long long)tokens_mine);
    share_copy(a, fc, gt, GT);
    __syncthreads();
    int bad = s_bad;
    if (!bad && (fc < 0 || fc > a.n_pages || s_total > a.max_tokens)) bad = TRIMKV_E_ARG;
    cluster.sync();                           // copies are made, every CTA's shared memory is set up
    bool wrong = false;                       // a page that does not exist
    auto page_at = [&](int r, int j) {
        const int p = a.table[(size_t)r * W + j];
        return p >= 0 && p < a.n_pages ? p : -1;
    };
    // places of row r that it lets go of: those it holds and does not go on with
    auto each_dropped = [&](auto&& f) {
        for (int t = gw; t < cut.tasks; t += SH_WARPS) {
            const int r = t / cut.nseg, j0 = (t - r * cut.nseg) * cut.seg;
            const ShareRow s = share_row(a, r);
            const int from = s.source == r ? s.stay : 0, to = sh_pages(s.old);
            f(t, r, max(j0, from / 32 * 32), from, min(to, j0 + cut.seg));
        }
    };
    auto add = [&](int sign) {                // holds let go of, and holds of a page of another row
        each_dropped([&](int t, int r, int, int from, int to) {
            const ShareRow s = share_row(a, r);
            const int j0 = (t - r * cut.nseg) * cut.seg, gains = s.source < 0 || s.source == r ? 0 : min(s.stay, j0 + cut.seg);
            for (int j = j0 + lane; j < max(to, gains); j += 32) {
                const bool loss = j >= from && j < to, gain = j < gains;
                const int p = loss ? page_at(r, j) : -1, u = gain ? page_at(s.source, j) : -1;
                if (p >= 0) atomicAdd(a.refs_out + p, -sign);
                if (u >= 0) atomicAdd(a.refs_out + u, sign);
                wrong |= (loss && p < 0) || (gain && u < 0);
            }
        });
    };
    if (!bad) {
        add(1);
        __threadfence();
        cluster.sync();
        // ---- counts are now of the holders that do not write.  Pages that nobody holds are in dispute: among the rows that will write one, and
        // if there is none among those that let go of it; the lowest of either gets it, and writers go first by SH_FIRST.
        for (int r = gt_row; r < R; r += GT) {
            const ShareRow s = share_row(a, r);
            const int p = s.writes ? page_at(s.source, s.keep / PAGE) : -1;
            if (p >= 0 && sh_ld(a.refs_out + p) <= 0) atomicMin(a.refs_out + p, r - R - SH_FIRST);
        }
        each_dropped([&](int, int r, int j0, int from, int to) {
            for (int j = j0 + lane; j < to; j += 32) {
                const int p = j >= from ? page_at(r, j) : -1;
                if (p >= 0 && sh_ld(a.refs_out + p) <= 0) atomicMin(a.refs_out + p, r - R);
            }
        });
        __threadfence();
        cluster.sync();
        for (int r = gt_row; r < R; r += GT) {
            const ShareRow s = share_row(a, r);
            const int p = s.writes ? page_at(s.source, s.keep / PAGE) : -1;
            if (p < 0) { wrong |= s.writes; continue; }
            if (sh_ld(a.refs_out + p) == r - R - SH_FIRST) {
                a.refs_out[p] = 1;            // (others who read it now see this or the minimum: not theirs)
            } else {
                share_tell(cluster, s_take + r, sh_pages(s.now) - sh_pages(s.keep) + 1);
                share_tell(cluster, s_move + r, s.keep % PAGE);
            }
        }
        // ---- pages that are given back, by the lowest row that let go of them
        each_dropped([&](int t, int r, int j0, int from, int to) {
            int n = 0;
            for (int j = j0; j < to; j += 32) {
                const int p = j + lane >= from && j + lane < to ? page_at(r, j + lane) : -1;
                n += __popc(__ballot_sync(0xffffffffu, p >= 0 && sh_ld(a.refs_out + p) == r - R));
            }
            if (lane < SH_CTAS) *cluster.map_shared_rank(s_back + t, lane) = n;
        });
        __threadfence();
        cluster.sync();
        share_scan(s_w, {s_tok, R}, {s_take, R}, {s_move, R}, {s_back, cut.tasks});
        if (fc + s_back[cut.tasks] > a.n_pages || s_move[R] > a.max_moves) bad = TRIMKV_E_ARG;
        else if (fc + s_back[cut.tasks] < s_take[R]) bad = TRIMKV_E_NOMEM;
        if (bad) {                            // the counts as they were
            each_dropped([&](int, int r, int j0, int from, int to) {
                for (int j = j0 + lane; j < to; j += 32) {
                    const int p = j >= from ? page_at(r, j) : -1;
                    if (p >= 0 && sh_ld(a.refs_out + p) == r - R) a.refs_out[p] = 0;
                }
            });
            __threadfence();
            cluster.sync();
            for (int r = gt; r < R; r += GT) {
                const ShareRow s = share_row(a, r);
                const int p = s.writes && s_move[r + 1] == s_move[r] ? page_at(s.source, s.keep / PAGE) : -1;
                if (p >= 0) atomicAdd(a.refs_out + p, -1);
            }
            add(-1);
        }
    }
    if (bad) {                                // nothing changes hands; the call's tokens are none
        for (int t = gw; t < cut.tasks; t += SH_WARPS) {
            const int r = t / cut.nseg, j0 = (t - r * cut.nseg) * cut.seg;
            for (int j = j0 + lane; j < min(min(sh_pages(max(a.old_lens[r], 0)), W), j0 + cut.seg); j += 32) a.table_out[(size_t)r * W + j] = a.table[(size_t)r * W + j];
        }
        for (int r = gt; r <= R; r += GT) {
            a.cu_new[r] = 0;
            if (r < R) a.lens_out[r] = a.old_lens[r];
        }
        for (int i = gt; i < a.max_tokens; i += GT) { a.slot_map[i] = -1; if (a.positions) a.positions[i] = -1; }
        share_none_moved(a, 0, gt, GT);
        if (gt == 0) { *a.free_count_out = fc; latch_error(a.status, bad); }      // (a barrier ago everyone had read the free count)
        return;
    }
    const int back = s_back[cut.tasks], taken = s_take[R], tokens = s_tok[R], moves = s_move[R];
    // ---- given back, in (row, place) order
    each_dropped([&](int t, int r, int j0, int from, int to) {
        int at = fc + s_back[t];
        for (int j = j0; j < to; j += 32) {
            const int p = j + lane >= from && j + lane < to ? page_at(r, j + lane) : -1;
            const bool mine = p >= 0 && sh_ld(a.refs_out + p) == r - R;
            const unsigned all = __ballot_sync(0xffffffffu, mine);
            const int i = at + __popc(all & ((1u << lane) - 1u));
            if (mine) {
                if (i < a.n_pages) a.free_out[i] = p;
                a.refs_out[p] = 0;
            }
            at += __popc(all);
        }
    });
    __threadfence();
    cluster.sync();
    auto fresh = [&](int i) {                 // the i-th page taken from the top of the stack
        const int p = sh_ld(a.free_out + (fc + back - 1 - i));
        return p >= 0 && p < a.n_pages ? p : -1;
    };
    auto new_page = [&](int r, int j) {       // page j of row r as it is now
        const int begin = sh_pages(a.new_lens[r]) - (s_take[r + 1] - s_take[r]);
        return j < begin ? page_at(a.source[r], j) : fresh(s_take[r] + j - begin);
    };
    // ---- the new rows: what they go on with, then fresh pages from the top of the stack
    for (int t = gw; t < cut.tasks; t += SH_WARPS) {
        const int r = t / cut.nseg, j0 = (t - r * cut.nseg) * cut.seg;
        const ShareRow s = share_row(a, r);
        const int has = sh_pages(s.now), begin = has - (s_take[r + 1] - s_take[r]);
        for (int j = j0 + lane; j < min(has, j0 + cut.seg); j += 32) {
            int p;
            if (j < begin) {
                p = page_at(s.source, j);
            } else {
                p = fresh(s_take[r] + j - begin);
                if (p >= 0) a.refs_out[p] = 1;
            }
            wrong |= p < 0;
            a.table_out[(size_t)r * W + j] = p;
        }
    }
    for (int r = gt_row; r <= R; r += GT) {
        a.cu_new[r] = s_tok[r];
        if (r < R) a.lens_out[r] = a.new_lens[r];
    }
    if (gt == 0) *a.free_count_out = fc + back - taken;
    for (int i = gt_row; i < a.max_tokens; i += GT) {
        int slot = -1, pos = -1;
        if (i < tokens) {
            const int r = share_find(s_tok, R, i);
            pos = a.keep_lens[r] + (i - s_tok[r]);
            const int p = new_page(r, pos / PAGE);
            if (p >= 0) slot = p * PAGE + pos % PAGE;
        }
        a.slot_map[i] = slot;
        if (a.positions) a.positions[i] = pos;
    }
    for (int i = gt_move; i < moves; i += GT) {
        const int r = share_find(s_move, R, i), e = i - s_move[r], page = a.keep_lens[r] / PAGE;
        const int from = page_at(a.source[r], page), to = new_page(r, page);
        a.move_src[i] = to >= 0 ? from * PAGE + e : -1;
        a.move_dst[i] = to >= 0 ? to * PAGE + e : -1;
    }
    share_none_moved(a, moves, gt, GT);
    if (wrong) latch_error(a.status, TRIMKV_E_ARG);
}

// ---------------------------------------------------------------- compact

__global__ void __launch_bounds__(SH_THREADS, 1)
paged_compact_kernel(ShareArgs a, const u64* keep_bits) {
    extern __shared__ int s_share[];
    __shared__ int s_w[32], s_bad, s_cnt[SH_THREADS / 32], s_first[SH_THREADS / 32], s_last[SH_THREADS / 32];
    __shared__ uint4 s_word[SH_THREADS / 32][32][2];      // see the entries that move
    const int R = a.R, W = a.W;
    const ShareCut cut = share_cut(R, W);
    int* s_len = s_share;                     // [R]: entries kept
    int* s_stay = s_len + R;                  // [R]: pages that stay
    int* s_take = s_stay + R;                 // [R + 1] each: per row, then sums before it
    int* s_move = s_take + R + 1;
    int* s_back = s_move + R + 1;             // [tasks + 1]
    cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, lane = tid & 31, rank = (int)cluster.block_rank();
    const int gt = rank * SH_THREADS + tid, GT = SH_CTAS * SH_THREADS, gw = rank * (SH_THREADS / 32) + (tid >> 5);
    if (tid == 0) s_bad = 0;
    grid_dependency_wait();
    grid_dependents_may_launch();
    __syncthreads();
    const int fc = *a.free_count;
    for (int r = tid; r < R; r += SH_THREADS) {
        const int n = a.old_lens[r];
        if (n < 0 || n > W * PAGE) s_bad = TRIMKV_E_ARG;
    }
    share_copy(a, fc, gt, GT);
    __syncthreads();
    int bad = s_bad;
    if (!bad && (fc < 0 || fc > a.n_pages)) bad = TRIMKV_E_ARG;
    cluster.sync();                           // copies are made, every CTA's shared memory is set up
    // Word w of row r: which of its entries are kept, and which are dropped.
    auto kept = [&](int r, int w, int n) {
        const u64 in = n - w * PAGE >= PAGE ? ~0ull : n > w * PAGE ? (1ull << (n - w * PAGE)) - 1ull : 0ull;
        return keep_bits[(size_t)r * W + w] & in;
    };
    bool wrong = false;
    auto page_at = [&](int r, int j) {
        const int p = a.table[(size_t)r * W + j];
        return p >= 0 && p < a.n_pages ? p : -1;
    };
    if (!bad) {
        // ---- of each row: entries kept, the first dropped, the last kept
        auto look = [&](int r, int n, int id, int step, int& cnt, int& first, int& last) {
#pragma unroll 4
            for (int w = id; w < sh_pages(n); w += step) {
                const u64 k = kept(r, w, n), gone = ~k;
                cnt += __popcll(k);
                if (k) last = w * PAGE + 63 - __clzll((long long)k);
                const int f = gone ? w * PAGE + __ffsll((long long)gone) - 1 : n;
                first = min(first, f);
            }
            cnt = __reduce_add_sync(0xffffffffu, cnt);
            first = __reduce_min_sync(0xffffffffu, first);
            last = __reduce_max_sync(0xffffffffu, last);
        };
        auto tell = [&](int r, int to, int cnt, int first, int last) {        // CTA `to`
            const bool moves = last > first;
            const int stay = moves ? first / PAGE : sh_pages(cnt);
            *cluster.map_shared_rank(s_len + r, to) = cnt;
            *cluster.map_shared_rank(s_stay + r, to) = stay;
            *cluster.map_shared_rank(s_take + r, to) = sh_pages(cnt) - stay;
            *cluster.map_shared_rank(s_move + r, to) = moves ? cnt - stay * PAGE : 0;
        };
        // a CTA takes every 16th row, `team` warps each: as many as there are, or as find four words a lane
        const int mine = (R - rank + SH_CTAS - 1) / SH_CTAS, most = min(max(mine, 1), SH_THREADS / 32);
        const int team = min(SH_THREADS / 32 / most, (W + 127) / 128), teams = SH_THREADS / 32 / team, warp = tid >> 5, tm = warp / team;
        for (int i0 = 0; i0 < mine; i0 += teams) {
            const int i = i0 + tm, r = rank + i * SH_CTAS;
            const bool on = tm < teams && i < mine;
            const int n = on ? a.old_lens[r] : 0;
            int cnt = 0, first = n, last = -1;
            if (team > 1) {
                if (on && warp == tm * team && lane == 0) { s_cnt[tm] = 0; s_first[tm] = n; s_last[tm] = -1; }
                __syncthreads();
            }
            if (on) look(r, n, tid - tm * team * 32, team * 32, cnt, first, last);
            if (team > 1) {
                if (on && lane == 0) {
                    atomicAdd(&s_cnt[tm], cnt);
                    atomicMin(&s_first[tm], first);
                    atomicMax(&s_last[tm], last);
                }
                __syncthreads();
                if (on && warp == tm * team) { cnt = s_cnt[tm]; first = s_first[tm]; last = s_last[tm]; }
            }
            if (on && warp == tm * team && lane < SH_CTAS) tell(r, lane, cnt, first, last);
        }
        cluster.sync();
        share_scan(s_w, {s_take, R}, {s_move, R});
        if (s_move[R] > a.max_moves) bad = TRIMKV_E_ARG;
        else if (s_take[R] > fc) bad = TRIMKV_E_NOMEM;
    }
    if (bad) {                                // nothing changes hands
        for (int t = gw; t < cut.tasks; t += SH_WARPS) {
            const int r = t / cut.nseg, j0 = (t - r * cut.nseg) * cut.seg;
            for (int j = j0 + lane; j < min(min(sh_pages(max(a.old_lens[r], 0)), W), j0 + cut.seg); j += 32) a.table_out[(size_t)r * W + j] = a.table[(size_t)r * W + j];
        }
        for (int r = gt; r < R; r += GT) a.lens_out[r] = a.old_lens[r];
        share_none_moved(a, 0, gt, GT);
        if (gt == 0) { *a.free_count_out = fc; latch_error(a.status, bad); }      // (a barrier ago everyone had read the free count)
        return;
    }
    const int taken = s_take[R], moves = s_move[R];
    auto each_dropped = [&](auto&& f) {
        for (int t = gw; t < cut.tasks; t += SH_WARPS) {
            const int r = t / cut.nseg, j0 = (t - r * cut.nseg) * cut.seg, from = s_stay[r];
            f(t, r, max(j0, from / 32 * 32), from, min(sh_pages(a.old_lens[r]), j0 + cut.seg));
        }
    };
    // ---- the new rows, and one holder less for what they leave
    for (int t = gw; t < cut.tasks; t += SH_WARPS) {
        const int r = t / cut.nseg, j0 = (t - r * cut.nseg) * cut.seg, has = sh_pages(s_len[r]), stay = s_stay[r];
        for (int j = j0 + lane; j < min(has, j0 + cut.seg); j += 32) {
            int p;
            if (j < stay) {
                p = page_at(r, j);
            } else {
                p = a.free_pages[fc - 1 - (s_take[r] + j - stay)];
                if (p < 0 || p >= a.n_pages) p = -1;
                else if (a.refs_out) a.refs_out[p] = 1;
            }
            wrong |= p < 0;
            a.table_out[(size_t)r * W + j] = p;
        }
    }
    each_dropped([&](int, int r, int j0, int from, int to) {
        for (int j = j0 + lane; j < to; j += 32) {
            const int p = j >= from ? page_at(r, j) : -1;
            if (p >= 0 && a.refs_out) atomicAdd(a.refs_out + p, -1);
            wrong |= j >= from && p < 0;
        }
    });
    __threadfence();
    cluster.sync();
    if (a.refs_out) {
        each_dropped([&](int, int r, int j0, int from, int to) {
            for (int j = j0 + lane; j < to; j += 32) {
                const int p = j >= from ? page_at(r, j) : -1;
                if (p >= 0 && sh_ld(a.refs_out + p) <= 0) atomicMin(a.refs_out + p, r - R);
            }
        });
        __threadfence();
        cluster.sync();
    }
    auto returns = [&](int r, int p) { return p >= 0 && (!a.refs_out || sh_ld(a.refs_out + p) == r - R); };
    each_dropped([&](int t, int r, int j0, int from, int to) {
        int n = 0;
        for (int j = j0; j < to; j += 32) {
            const int p = j + lane >= from && j + lane < to ? page_at(r, j + lane) : -1;
            n += __popc(__ballot_sync(0xffffffffu, returns(r, p)));
        }
        if (lane < SH_CTAS) *cluster.map_shared_rank(s_back + t, lane) = n;
    });
    cluster.sync();
    share_scan(s_w, {s_back, cut.tasks});
    each_dropped([&](int t, int r, int j0, int from, int to) {
        int at = fc - taken + s_back[t];
        for (int j = j0; j < to; j += 32) {
            const int p = j + lane >= from && j + lane < to ? page_at(r, j + lane) : -1;
            const bool mine = returns(r, p);
            const unsigned all = __ballot_sync(0xffffffffu, mine);
            const int i = at + __popc(all & ((1u << lane) - 1u));
            if (mine) {
                if (i < a.n_pages) a.free_out[i] = p;
                if (a.refs_out) a.refs_out[p] = 0;
            }
            at += __popc(all);
        }
    });
    for (int r = gt; r < R; r += GT) a.lens_out[r] = s_len[r];
    if (gt == 0) {                            // more than there are pages: some have two holders, and nobody counted
        const int live = fc - taken + s_back[cut.tasks];
        *a.free_count_out = min(live, a.n_pages);
        wrong |= live > a.n_pages;
    }
    // ---- the entries that move: a warp takes up to 32 words of a row, a lane describes one; then a lane looks for the word and bit of an
    // entry, or, of many, all lanes list those of a word after another
    const int span = (int)min(32ll, max(2ll, ((long long)R * W + SH_WARPS - 1) / SH_WARPS)), per_row = (W + span - 1) / span;
    uint4(*desc)[2] = s_word[tid >> 5];
    for (long long t = gw; t < (long long)R * per_row; t += SH_WARPS) {
        const int r = (int)(t / per_row), w0 = (int)(t - (long long)r * per_row) * span, stay = s_stay[r];
        const int n = a.old_lens[r], count = s_move[r + 1] - s_move[r], end = min(w0 + span, sh_pages(n));
        if (count == 0 || end <= stay || w0 >= end) continue;
        int before = 0;                       // entries kept in the row's earlier words
#pragma unroll 4
        for (int w = lane; w < w0; w += 32) before += __popcll(kept(r, w, n));
        const int w = w0 + lane;
        const u64 bits = w < end ? kept(r, w, n) : 0ull;
        int sum = __popcll(bits);
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += u;
        }
        const int base = __reduce_add_sync(0xffffffffu, before) + sum - __popcll(bits);
        if (bits && w >= stay) {              // its entries go to one page, or to two
            const int32_t* to = a.table_out + (size_t)r * W + base / PAGE;
            const int from = page_at(r, w), to0 = sh_ld(to), to1 = base % PAGE + __popcll(bits) > PAGE ? sh_ld(to + 1) : -1;
            auto slot = [&](int page, int other) { return page >= 0 && other >= 0 ? page * PAGE : -1; };
            desc[lane][0] = make_uint4((uint32_t)bits, (uint32_t)(bits >> 32), (uint32_t)(s_move[r] + base - stay * PAGE), (uint32_t)(base % PAGE));
            desc[lane][1] = make_uint4((uint32_t)slot(from, to0), (uint32_t)slot(to0, from), (uint32_t)slot(from, to1), (uint32_t)slot(to1, from));
        }
        __syncwarp();
        const unsigned words = __ballot_sync(0xffffffffu, bits && w >= stay);
        const int base0 = words ? __shfl_sync(0xffffffffu, base, __ffs(words) - 1) : 0, listed = words ? __shfl_sync(0xffffffffu, base + __popcll(bits), 31) - base0 : 0;
        if (listed <= SH_SPARSE * __popc(words)) {            // few entries a word: a lane finds the word and the bit of its entry
            const int at = w >= stay ? base - base0 : 0;      // entries listed of the words before (words before `stay` come first)
            for (int i0 = 0; i0 < listed; i0 += 32) {
                const int i = i0 + lane;
                int k = 0;
#pragma unroll
                for (int step = 16; step; step >>= 1)         // the last word with at <= i
                    if (__shfl_sync(0xffffffffu, at, k + step) <= i) k += step;
                int nth = i - __shfl_sync(0xffffffffu, at, k);
                if (i < listed) {
                    const uint4 d0 = desc[k][0], d1 = desc[k][1];
                    const int to = (int)d0.w + nth, m = (int)d0.z + nth, low = __popc(d0.x);
                    unsigned rest = nth < low ? d0.x : d0.y;
                    int bit = nth < low ? 0 : 32;
                    nth -= nth < low ? 0 : low;
#pragma unroll
                    for (int half = 16; half; half >>= 1) {   // the nth bit of a word
                        const int c = __popc(rest & ((1u << half) - 1u));
                        if (nth >= c) { nth -= c; bit += half; rest >>= half; }
                    }
                    a.move_src[m] = (int)(to < PAGE ? d1.x : d1.z) | bit;
                    a.move_dst[m] = (int)(to < PAGE ? d1.y : d1.w) | (to % PAGE);
                }
            }
        }
        for (unsigned todo = listed <= SH_SPARSE * __popc(words) ? 0u : words; todo; todo &= todo - 1) {
            const uint4 d0 = desc[__ffs(todo) - 1][0], d1 = desc[__ffs(todo) - 1][1];
            const unsigned below = (1u << lane) - 1u;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const unsigned word = half ? d0.y : d0.x;
                const int k = __popc(word & below) + (half ? __popc(d0.x) : 0), at = (int)d0.w + k, m = (int)d0.z + k;
                if ((word >> lane) & 1u) {    // (-1 with any row is -1)
                    a.move_src[m] = (int)(at < PAGE ? d1.x : d1.z) | (half * 32 + lane);
                    a.move_dst[m] = (int)(at < PAGE ? d1.y : d1.w) | (at % PAGE);
                }
            }
        }
        __syncwarp();
    }
    share_none_moved(a, moves, gt, GT);
    if (wrong) latch_error(a.status, TRIMKV_E_ARG);
}

size_t share_ints(int R, int W) { return (size_t)4 * R + 4 + share_cut(R, W).tasks + 1; }
constexpr int SH_MOST_SMEM = (5 * PAGED_MAX_REQ + 8) * (int)sizeof(int);          // (fewer tasks than rows above SH_TASKS rows)
static_assert(PAGED_MAX_REQ >= SH_TASKS, "tasks are at most the larger of the two");

}  // namespace

cudaError_t launch_paged_share(const ShareArgs& a, cudaStream_t st) {
    static std::atomic<unsigned long long> ready{0};
    const cudaError_t e = paged_allow_smem(reinterpret_cast<const void*>(paged_share_kernel), SH_MOST_SMEM, ready, true);
    if (e != cudaSuccess) return e;
    return paged_launch(paged_share_kernel, dim3(SH_CTAS), dim3(SH_THREADS), share_ints(a.R, a.W) * sizeof(int), SH_CTAS, true, st, a);
}

cudaError_t launch_paged_compact(const ShareArgs& a, const unsigned long long* keep_bits, cudaStream_t st) {
    static std::atomic<unsigned long long> ready{0};
    const cudaError_t e = paged_allow_smem(reinterpret_cast<const void*>(paged_compact_kernel), SH_MOST_SMEM, ready, true);
    if (e != cudaSuccess) return e;
    return paged_launch(paged_compact_kernel, dim3(SH_CTAS), dim3(SH_THREADS), share_ints(a.R, a.W) * sizeof(int), SH_CTAS, true, st, a, keep_bits);
}

}  // namespace tkv
