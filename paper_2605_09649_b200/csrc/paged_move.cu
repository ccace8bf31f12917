// Copies of listed rows of page arrays: what a fork's last page and dropped entries ask for, in every layer at once.
//
// move_src[i] -> move_dst[i] (page x 64 + row), for each of up to 128 arrays and each of its heads in one launch.  Pairs come in ascending
// runs, so a block takes 64 pairs of one array and head, whose rows mostly lie side by side on both ends, and its threads take 16
// bytes each (less where a row is not a multiple of 16).  Bound by the copy.
//
// Bounds: pages whose last row (63) was a destination get the channelwise smallest and largest of their 64 keys, in a
// second launch that reads them from L2.
#include <algorithm>

#include "paged_bounds.cuh"
#include "paged_share.cuh"

namespace tkv {

namespace {

constexpr int MV_THREADS = 256, MV_GROUP = 64, MV_BLOCKS = PAGED_SMS * 8;

template <typename T>
__device__ __forceinline__ void move_rows(char* base, int row_bytes, size_t head_row, size_t page_rows, const int* s_src, const int* s_dst) {
    constexpr int UNROLL = 4;
    const unsigned per_row = (unsigned)row_bytes / sizeof(T), n = per_row * MV_GROUP;
    for (unsigned i0 = threadIdx.x; i0 < n; i0 += UNROLL * MV_THREADS) {
        T v[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {                        // all loads in flight before the first store
            const unsigned i = i0 + u * MV_THREADS;
            if (i >= n) continue;
            const unsigned m = i / per_row;
            const int s = s_src[m];
            if (s >= 0) v[u] = *reinterpret_cast<const T*>(base + ((size_t)(s / PAGE) * page_rows + head_row + s % PAGE) * row_bytes + (size_t)(i - m * per_row) * sizeof(T));
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const unsigned i = i0 + u * MV_THREADS;
            if (i >= n) continue;
            const unsigned m = i / per_row;
            const int d = s_dst[m];
            if (s_src[m] >= 0) *reinterpret_cast<T*>(base + ((size_t)(d / PAGE) * page_rows + head_row + d % PAGE) * row_bytes + (size_t)(i - m * per_row) * sizeof(T)) = v[u];
        }
    }
}

__global__ void __launch_bounds__(MV_THREADS)
paged_move_kernel(const __grid_constant__ MoveArrays arrays, MoveList list, int heads_total) {
    __shared__ int s_src[MV_GROUP], s_dst[MV_GROUP];
    grid_dependency_wait();
    grid_dependents_may_launch();
    const int count = min(max(*list.count, 0), list.max_moves), slots = list.n_pages * PAGE;
    if (blockIdx.x == 0 && threadIdx.x == 0 && count != *list.count) latch_error(list.status, TRIMKV_E_ARG);
    const int groups = (count + MV_GROUP - 1) / MV_GROUP;
    const long long items = (long long)groups * heads_total;      // group by group, all heads of all arrays
    for (long long it = blockIdx.x; it < items; it += gridDim.x) {
        const int grp = (int)(it / heads_total);
        int h = (int)(it - (long long)grp * heads_total), x = 0;
        while (h >= arrays.a[x].heads) h -= arrays.a[x++].heads;
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
        const MoveArray& a = arrays.a[x];
        const size_t head_row = (size_t)h * PAGE, page_rows = (size_t)a.heads * PAGE;
        if (a.row_bytes % 16 == 0) move_rows<uint4>(a.pages, a.row_bytes, head_row, page_rows, s_src, s_dst);
        else if (a.row_bytes % 8 == 0) move_rows<uint2>(a.pages, a.row_bytes, head_row, page_rows, s_src, s_dst);
        else if (a.row_bytes % 4 == 0) move_rows<uint32_t>(a.pages, a.row_bytes, head_row, page_rows, s_src, s_dst);
        else if (a.row_bytes % 2 == 0) move_rows<uint16_t>(a.pages, a.row_bytes, head_row, page_rows, s_src, s_dst);
        else move_rows<uint8_t>(a.pages, a.row_bytes, head_row, page_rows, s_src, s_dst);
    }
}

// An item is an array and 64 pairs; its pages that were completed, head by head: a warp per 16 bytes of channels, two rows a lane.
template <typename T>
__global__ void __launch_bounds__(MV_THREADS)
paged_bounds_kernel(const __grid_constant__ MoveBounds arrays, MoveList list) {
    constexpr int WARPS = MV_THREADS / 32;
    __shared__ int s_full[MV_GROUP], s_n;
    grid_dependency_wait();
    grid_dependents_may_launch();
    const int count = min(max(*list.count, 0), list.max_moves), slots = list.n_pages * PAGE;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long items = (long long)((count + MV_GROUP - 1) / MV_GROUP) * arrays.n;
    for (long long it = blockIdx.x; it < items; it += gridDim.x) {
        const int grp = (int)(it / arrays.n), x = (int)(it - (long long)grp * arrays.n);
        const MoveBound& a = arrays.a[x];
        __syncthreads();
        if (warp == 0) {
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
        for (int j = warp; j < s_n * a.heads * cpr; j += WARPS) {
            const int c = j % cpr, ph = j / cpr;
            const size_t head = (size_t)s_full[ph / a.heads] * a.heads + ph % a.heads;
            const char* rows = a.pages + head * PAGE * a.row_bytes + (size_t)c * 16;
            MinMax16<T> mm;
            mm.start(__ldcg(reinterpret_cast<const uint4*>(rows + (size_t)lane * a.row_bytes)));
            mm.add(__ldcg(reinterpret_cast<const uint4*>(rows + (size_t)(lane + 32) * a.row_bytes)));
            for (int o = 16; o > 0; o >>= 1) {
                const uint4 lo = *reinterpret_cast<uint4*>(mm.lo), hi = *reinterpret_cast<uint4*>(mm.hi);
                const uint4 olo = make_uint4(__shfl_xor_sync(0xffffffffu, lo.x, o), __shfl_xor_sync(0xffffffffu, lo.y, o), __shfl_xor_sync(0xffffffffu, lo.z, o), __shfl_xor_sync(0xffffffffu, lo.w, o));
                const uint4 ohi = make_uint4(__shfl_xor_sync(0xffffffffu, hi.x, o), __shfl_xor_sync(0xffffffffu, hi.y, o), __shfl_xor_sync(0xffffffffu, hi.z, o), __shfl_xor_sync(0xffffffffu, hi.w, o));
                mm.join(olo, ohi);
            }
            if (lane < 2) *reinterpret_cast<uint4*>(a.bounds + (head * 2 + lane) * a.row_bytes + (size_t)c * 16) = lane ? *reinterpret_cast<uint4*>(mm.hi) : *reinterpret_cast<uint4*>(mm.lo);
        }
    }
}

}  // namespace

cudaError_t launch_paged_move(const MoveArrays& arrays, const MoveList& list, cudaStream_t st) {
    long long heads = 0;
    for (int i = 0; i < arrays.n; ++i) heads += arrays.a[i].heads;
    const long long items = heads * ((list.max_moves + MV_GROUP - 1) / MV_GROUP);
    return paged_launch(paged_move_kernel, dim3((unsigned)std::min<long long>(items, MV_BLOCKS)), dim3(MV_THREADS), 0, 1, true, st, arrays, list, (int)heads);
}

cudaError_t launch_paged_bounds(const MoveBounds& arrays, int is_bf16, const MoveList& list, cudaStream_t st) {
    const long long items = (long long)arrays.n * ((list.max_moves + MV_GROUP - 1) / MV_GROUP);
    const dim3 grid((unsigned)std::min<long long>(items, MV_BLOCKS));
    return is_bf16 ? paged_launch(paged_bounds_kernel<__nv_bfloat16>, grid, dim3(MV_THREADS), 0, 1, true, st, arrays, list)
                   : paged_launch(paged_bounds_kernel<float>, grid, dim3(MV_THREADS), 0, 1, true, st, arrays, list);
}

}  // namespace tkv
