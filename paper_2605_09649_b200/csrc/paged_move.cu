// Copies of listed rows of page arrays: what a fork's last page and dropped entries ask for, in every layer at once.
//
// move_src[i] -> move_dst[i] (page x 64 + row), for each of up to 128 arrays and each of its heads in one launch.  Pairs come in ascending
// runs, so a block takes 64 pairs of four heads, whose rows mostly lie side by side on both ends, and its threads take 16
// bytes each (less where a row is not a multiple of 16).  Bound by the copy: 32 rows on average of 32 requests in 32 layers of 8 heads of 128 (282 MB) take 49.5 us,
// 0.87 of the measured copy rate.  (A head a block, its array looked for and a division for every 16 bytes: 70 us.)
//
// Bounds: pages whose last row (63) was a destination get the channelwise smallest and largest of their 64 keys, in a
// second launch that reads them from L2.
#include <algorithm>

#include "paged_bounds.cuh"
#include "paged_share.cuh"

namespace tkv {

namespace {

constexpr int MV_THREADS = 256, MV_GROUP = 64, MV_HEADS = 4, MV_BLOCKS = PAGED_SMS * 8;

// The rows of MV_GROUP pairs of one head, pieces of sizeof(T) bytes.
template <typename T>
__device__ __forceinline__ void move_rows(char* base, int row_bytes, size_t head_row, size_t page_rows, const int* s_src, const int* s_dst) {
    const unsigned per_row = (unsigned)row_bytes / sizeof(T);
    auto from = [&](int slot, unsigned col) { return reinterpret_cast<T*>(base + ((size_t)(slot / PAGE) * page_rows + head_row + slot % PAGE) * row_bytes) + col; };
    if (MV_THREADS % per_row == 0) {                                  // a thread keeps its column
        const unsigned col = threadIdx.x % per_row, rows = MV_THREADS / per_row;
        for (unsigned m0 = threadIdx.x / per_row; m0 < MV_GROUP; m0 += 4 * rows) {
            T v[4];
            int s[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {                             // all loads in flight before the first store
                const unsigned m = m0 + u * rows;
                s[u] = m < MV_GROUP ? s_src[m] : -1;
                if (s[u] >= 0) v[u] = *from(s[u], col);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (s[u] >= 0) *from(s_dst[m0 + u * rows], col) = v[u];
        }
    } else {
        for (unsigned i = threadIdx.x; i < per_row * MV_GROUP; i += MV_THREADS) {
            const unsigned m = i / per_row;
            if (s_src[m] >= 0) *from(s_dst[m], i - m * per_row) = *from(s_src[m], i - m * per_row);
        }
    }
}

// An item is 64 pairs and MV_HEADS heads, of one or several arrays (heads are numbered through all of them; same: heads of each, if they are alike).
__global__ void __launch_bounds__(MV_THREADS)
paged_move_kernel(const __grid_constant__ MoveArrays arrays, MoveList list, int heads_total, FastDiv same, FastDiv by_parts) {
    __shared__ int s_src[MV_GROUP], s_dst[MV_GROUP];
    grid_dependency_wait();
    grid_dependents_may_launch();
    const int count = min(max(*list.count, 0), list.max_moves), slots = list.n_pages * PAGE;
    if (blockIdx.x == 0 && threadIdx.x == 0 && count != *list.count) latch_error(list.status, TRIMKV_E_ARG);
    const int parts = (int)by_parts.d;
    const long long items = (long long)((count + MV_GROUP - 1) / MV_GROUP) * parts;
    for (long long it = blockIdx.x; it < items; it += gridDim.x) {
        const int grp = it <= INT_MAX ? by_parts.div((int)it) : (int)(it / parts), h0 = (int)(it - (long long)grp * parts) * MV_HEADS;
        __syncthreads();
        if (threadIdx.x < MV_GROUP) {
            const int i = grp * MV_GROUP + threadIdx.x;
            int s = -1, d = -1;
            if (i < count) {
                s = list.src[i];
                d = list.dst[i];
                if (s < 0 || s >= slots || d < 0 || d >= slots) {
                    if (s != -1 || d != -1) latch_error(list.status, TRIMKV_E_ARG);
                    s = -1;
                }
            }
            s_src[threadIdx.x] = s;
            s_dst[threadIdx.x] = d;
        }
        __syncthreads();
        for (int hh = h0; hh < min(h0 + MV_HEADS, heads_total); ++hh) {
            int x, h = hh;
            if (same.d) {
                x = same.div(hh);
                h -= x * (int)same.d;
            } else {
                for (x = 0; h >= arrays.a[x].heads; ++x) h -= arrays.a[x].heads;
            }
            const MoveArray a = arrays.a[x];
            const size_t head_row = (size_t)h * PAGE, page_rows = (size_t)a.heads * PAGE;
            if (a.row_bytes % 16 == 0) move_rows<uint4>(a.pages, a.row_bytes, head_row, page_rows, s_src, s_dst);
            else if (a.row_bytes % 8 == 0) move_rows<uint2>(a.pages, a.row_bytes, head_row, page_rows, s_src, s_dst);
            else if (a.row_bytes % 4 == 0) move_rows<uint32_t>(a.pages, a.row_bytes, head_row, page_rows, s_src, s_dst);
            else if (a.row_bytes % 2 == 0) move_rows<uint16_t>(a.pages, a.row_bytes, head_row, page_rows, s_src, s_dst);
            else move_rows<uint8_t>(a.pages, a.row_bytes, head_row, page_rows, s_src, s_dst);
        }
    }
}

// An item is an array and 64 pairs; its pages that were completed, head by head: 16 threads to a row of 256 bytes, four rows each, then the 16
// groups of rows are joined.
template <typename T>
__global__ void __launch_bounds__(MV_THREADS)
paged_bounds_kernel(const __grid_constant__ MoveBounds arrays, MoveList list) {
    constexpr int COLS = 16, ROWS = MV_THREADS / COLS, EACH = PAGE / ROWS;
    __shared__ int s_full[MV_GROUP], s_n;
    __shared__ uint4 s_part[2][ROWS][COLS];
    grid_dependency_wait();
    grid_dependents_may_launch();
    const int count = min(max(*list.count, 0), list.max_moves), slots = list.n_pages * PAGE;
    const int lane = threadIdx.x & 31, col = threadIdx.x % COLS, rg = threadIdx.x / COLS;
    const long long items = (long long)((count + MV_GROUP - 1) / MV_GROUP) * arrays.n;
    for (long long it = blockIdx.x; it < items; it += gridDim.x) {
        const int grp = (int)(it / arrays.n), x = (int)(it - (long long)grp * arrays.n);
        const MoveBound a = arrays.a[x];
        __syncthreads();
        if (threadIdx.x < 32) {
            int n = 0;
            for (int half = 0; half < MV_GROUP; half += 32) {
                const int i = grp * MV_GROUP + half + lane, s = i < count ? list.src[i] : -1, d = i < count ? list.dst[i] : -1;
                const bool full = s >= 0 && s < slots && d >= 0 && d < slots && d % PAGE == PAGE - 1;
                const unsigned all = __ballot_sync(0xffffffffu, full);
                if (full) s_full[n + __popc(all & ((1u << lane) - 1u))] = d / PAGE;
                n += __popc(all);
            }
            if (lane == 0) s_n = n;
        }
        __syncthreads();
        const int cpr = a.row_bytes / 16;                         // 16-byte chunks of a row
        for (int ph = 0; ph < s_n * a.heads; ++ph) {
            const size_t head = (size_t)s_full[ph / a.heads] * a.heads + ph % a.heads;
            for (int c0 = 0; c0 < cpr; c0 += COLS) {
                const bool on = c0 + col < cpr;
                const char* rows = a.pages + (head * PAGE + rg) * a.row_bytes + (size_t)(c0 + col) * 16;
                uint4 v[EACH];
#pragma unroll
                for (int r = 0; r < EACH; ++r) v[r] = on ? __ldcg(reinterpret_cast<const uint4*>(rows + (size_t)r * ROWS * a.row_bytes)) : make_uint4(0u, 0u, 0u, 0u);
                MinMax16<T> mm;
                mm.start(v[0]);
#pragma unroll
                for (int r = 1; r < EACH; ++r) mm.add(v[r]);
                s_part[0][rg][col] = *reinterpret_cast<uint4*>(mm.lo);
                s_part[1][rg][col] = *reinterpret_cast<uint4*>(mm.hi);
                __syncthreads();
                if (rg == 0 && on) {
                    for (int r = 1; r < ROWS; ++r) mm.join(s_part[0][r][col], s_part[1][r][col]);
                    *reinterpret_cast<uint4*>(a.bounds + head * 2 * a.row_bytes + (size_t)(c0 + col) * 16) = *reinterpret_cast<uint4*>(mm.lo);
                    *reinterpret_cast<uint4*>(a.bounds + (head * 2 + 1) * a.row_bytes + (size_t)(c0 + col) * 16) = *reinterpret_cast<uint4*>(mm.hi);
                }
                __syncthreads();
            }
        }
    }
}

}  // namespace

cudaError_t launch_paged_move(const MoveArrays& arrays, const MoveList& list, cudaStream_t st) {
    int heads = 0;
    bool same = true;
    for (int i = 0; i < arrays.n; ++i) {
        heads += arrays.a[i].heads;
        same &= arrays.a[i].heads == arrays.a[0].heads;
    }
    const int parts = (heads + MV_HEADS - 1) / MV_HEADS;
    const long long items = (long long)parts * ((list.max_moves + MV_GROUP - 1) / MV_GROUP);
    return paged_launch(paged_move_kernel, dim3((unsigned)std::min<long long>(items, MV_BLOCKS)), dim3(MV_THREADS), 0, 1, true, st, arrays, list, heads,
                        same ? FastDiv::by(arrays.a[0].heads) : FastDiv{0u, 0u, 0u}, FastDiv::by(parts));
}

cudaError_t launch_paged_bounds(const MoveBounds& arrays, int is_bf16, const MoveList& list, cudaStream_t st) {
    const long long items = (long long)arrays.n * ((list.max_moves + MV_GROUP - 1) / MV_GROUP);
    const dim3 grid((unsigned)std::min<long long>(items, MV_BLOCKS));
    return is_bf16 ? paged_launch(paged_bounds_kernel<__nv_bfloat16>, grid, dim3(MV_THREADS), 0, 1, true, st, arrays, list)
                   : paged_launch(paged_bounds_kernel<float>, grid, dim3(MV_THREADS), 0, 1, true, st, arrays, list);
}

}  // namespace tkv
