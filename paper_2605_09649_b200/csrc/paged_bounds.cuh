// Channelwise smallest and largest keys, 16 bytes of a row at a time.
#pragma once

#include <cuda_bf16.h>

namespace tkv {

template <typename T>
struct MinMax16;                              // channelwise bounds of 16 bytes of keys; NaN in a channel stays NaN
template <>
struct MinMax16<__nv_bfloat16> {
    __nv_bfloat162 lo[4], hi[4];
    __device__ __forceinline__ void start(const uint4& v) {
        const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&v);
#pragma unroll
        for (int i = 0; i < 4; ++i) lo[i] = hi[i] = p[i];
    }
    __device__ __forceinline__ void add(const uint4& v) {
        const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&v);
#pragma unroll
        for (int i = 0; i < 4; ++i) { lo[i] = __hmin2_nan(lo[i], p[i]); hi[i] = __hmax2_nan(hi[i], p[i]); }
    }
    __device__ __forceinline__ void join(const uint4& vlo, const uint4& vhi) {
        const __nv_bfloat162 *a = reinterpret_cast<const __nv_bfloat162*>(&vlo), *b = reinterpret_cast<const __nv_bfloat162*>(&vhi);
#pragma unroll
        for (int i = 0; i < 4; ++i) { lo[i] = __hmin2_nan(lo[i], a[i]); hi[i] = __hmax2_nan(hi[i], b[i]); }
    }
};
template <>
struct MinMax16<float> {
    float lo[4], hi[4];
    static __device__ __forceinline__ float mn(float a, float b) { float d; asm("min.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b)); return d; }
    static __device__ __forceinline__ float mx(float a, float b) { float d; asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b)); return d; }
    __device__ __forceinline__ void start(const uint4& v) {
        const float* p = reinterpret_cast<const float*>(&v);
#pragma unroll
        for (int i = 0; i < 4; ++i) lo[i] = hi[i] = p[i];
    }
    __device__ __forceinline__ void add(const uint4& v) {
        const float* p = reinterpret_cast<const float*>(&v);
#pragma unroll
        for (int i = 0; i < 4; ++i) { lo[i] = mn(lo[i], p[i]); hi[i] = mx(hi[i], p[i]); }
    }
    __device__ __forceinline__ void join(const uint4& vlo, const uint4& vhi) {
        const float *a = reinterpret_cast<const float*>(&vlo), *b = reinterpret_cast<const float*>(&vhi);
#pragma unroll
        for (int i = 0; i < 4; ++i) { lo[i] = mn(lo[i], a[i]); hi[i] = mx(hi[i], b[i]); }
    }
};

}  // namespace tkv
