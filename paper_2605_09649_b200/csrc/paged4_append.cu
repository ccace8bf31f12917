// Rounding of keys and values into the 4-bit paged cache, and reading them back.
//
// Append.  A block is 16 channels x of one entry and KV head, x' = x 2^-shift.  Its scale is s = e4m3(max |x'| / 6) (to nearest
// even, at most 448), its codes are e2m1(x' / s): nearest, ties to the even code, at most 6; magnitude 0 where s = 0, the sign always that of x; s = NaN
// where the block holds one.  A thread takes two blocks: it reads 32 channels and writes 16 bytes of codes and two of scales.
//   The quotient.  bf16: x' has 8 significant bits, the halfway points m s (m of three bits, s of four) have 7, so a quotient is
// a halfway point or at least 2^-9 of it away; x' times the rounded reciprocal of s is off by 2^-22 and, rounded to 16
// bits, is the halfway point itself where the quotient is one.  fp32: x' is compared with the seven halfway points m s,
// which are exact.
// 2 x 2 bytes per channel in, 2 x 0.5625 out: 12 K tokens of 8 heads of 128 in 15.7 us, 64 MB, 0.62 of the measured copy rate; fp32 30.8 us, 0.57; 32 tokens
// in 2.4 us.  (Half a block per thread, so that every access is contiguous: 29 us, the quotients are computed twice.)
//
// Read.  The way back: every value is exact in bf16 (6 significant bits) and fp32.  12 K tokens in 11.0 us, 0.89 of the copy rate: four items' loads in
// flight per thread and whole sectors stored.  fp32 37.4 us, 0.47: it stores half a sector at a time.
#include <algorithm>

#include "paged4.cuh"

namespace tkv {

namespace {

constexpr int A4_THREADS = 256, R4_UNROLL = 4;

__device__ __forceinline__ float max_nan(float a, float b) { float d; asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b)); return d; }
__device__ __forceinline__ uint32_t a4_scale(float amax) {                // of max |x'|
    const float s = __fdiv_rn(amax, 6.0f);
    uint32_t r;
    asm("{\n\t.reg .b16 x;\n\tcvt.rn.satfinite.e4m3x2.f32 x, %1, %1;\n\tcvt.u32.u16 %0, x;\n\t}" : "=r"(r) : "f"(s));
    return r & 0xffu;
}
__device__ __forceinline__ uint32_t a4_pair(float lo, float hi) {         // e2m1 of two quotients, in one byte
    uint32_t r;
    asm("{\n\t.reg .b8 x;\n\t.reg .b32 z;\n\tcvt.rn.satfinite.e2m1x2.f32 x, %2, %1;\n\tmov.b32 %0, {x, x, x, x};\n\t}" : "=r"(r) : "f"(lo), "f"(hi));
    return r & 0xffu;
}
__device__ __forceinline__ float a4_16_bits(float y) { return __uint_as_float((__float_as_uint(y) + 0x80u) & 0xffffff00u); }
__device__ __forceinline__ uint32_t a4_code(float x, float s) {           // by comparison
    const float t = fabsf(x);
    const uint32_t n = (t > 0.25f * s) + (t >= 0.75f * s) + (t > 1.25f * s) + (t >= 1.75f * s) + (t > 2.5f * s) + (t >= 3.5f * s) + (t > 5.0f * s);
    return (s > 0.f ? n : 0u) | (__float_as_uint(x) >> 31 << 3);
}

template <typename T>
struct Load32;                                // 32 channels
template <>
struct Load32<__nv_bfloat16> {
    uint4 v[4];
    __device__ __forceinline__ void load(const void* p) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = reinterpret_cast<const uint4*>(p)[i];
    }
    __device__ __forceinline__ float operator[](int i) const {
        const uint32_t w = reinterpret_cast<const uint32_t*>(v)[i >> 1];
        return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
    }
};
template <>
struct Load32<float> {
    uint4 v[8];
    __device__ __forceinline__ void load(const void* p) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = reinterpret_cast<const uint4*>(p)[i];
    }
    __device__ __forceinline__ float operator[](int i) const { return __uint_as_float(reinterpret_cast<const uint32_t*>(v)[i]); }
};

// Item i: 32 channels of token i / (H d / 32); the grid's second dimension is K or V.
template <typename T>
__global__ void __launch_bounds__(A4_THREADS)
paged4_append_kernel(Paged4View c, uint8_t* k_codes, uint8_t* k_scales, uint8_t* v_codes, uint8_t* v_scales, long long items, const T* k, long long k_stride,
                     const T* v, long long v_stride, const int32_t* slot_map, int32_t* status) {
    const int kv = blockIdx.y, H = c.pv.H, d = c.pv.d, per_head = d / 32, per_tok = H * per_head;
    const T* x = kv ? v : k;
    const long long stride = kv ? v_stride : k_stride;
    uint8_t* codes = kv ? v_codes : k_codes;
    uint8_t* scales = kv ? v_scales : k_scales;
    grid_dependency_wait();
    grid_dependents_may_launch();
    for (long long i = (long long)blockIdx.x * A4_THREADS + threadIdx.x; i < items; i += (long long)gridDim.x * A4_THREADS) {
        const int tok = (int)(i / per_tok), rest = (int)(i - (long long)tok * per_tok), h = rest / per_head, part = rest - h * per_head;
        const int slot = slot_map[tok];
        if (slot < 0 || slot >= c.pv.n_pages * PAGE) {
            if (slot != -1 && rest == 0) latch_error(status, TRIMKV_E_ARG);
            continue;
        }
        Load32<T> in;
        in.load(x + (long long)tok * stride + (long long)h * d + part * 32);
        const float down = p4_pow2(-p4_shift(c, kv, h));
        uint32_t word[4], scale2 = 0;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            float amax = 0.f;
#pragma unroll
            for (int e = 0; e < 16; ++e) amax = max_nan(amax, fabsf(in[b * 16 + e]));
            const uint32_t s8 = a4_scale(amax * down);
            const float s = p4_float2(p4_scales(s8)).x;
            scale2 |= s8 << (8 * b);
            const float inv = s > 0.f ? __frcp_rn(s) * down : (s == 0.f ? 0.f : s);        // (a power of two: exact)
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                uint32_t r = 0;
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float x0 = in[b * 16 + w * 8 + e], x1 = in[b * 16 + w * 8 + e + 1];
                    if constexpr (sizeof(T) == 2) r |= a4_pair(a4_16_bits(x0 * inv), a4_16_bits(x1 * inv)) << (4 * e);
                    else r |= (a4_code(x0 * down, s) | a4_code(x1 * down, s) << 4) << (4 * e);
                }
                word[b * 2 + w] = r;
            }
        }
        const long long row = ((long long)(slot / PAGE) * H + h) * PAGE + slot % PAGE;
        *reinterpret_cast<uint4*>(codes + row * (d / 2) + part * 16) = make_uint4(word[0], word[1], word[2], word[3]);
        *reinterpret_cast<uint16_t*>(scales + row * (d / 16) + part * 2) = (uint16_t)scale2;
    }
}

// 32 bytes, a whole sector.
__device__ __forceinline__ void r4_store32(void* p, const uint32_t* v) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]),
                 "r"(v[7])
                 : "memory");
}
__device__ __forceinline__ void r4_store(__nv_bfloat16* p, const float2 (&v)[8]) {       // 16 values
    uint32_t w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(v[e].x, v[e].y);
        w[e] = *reinterpret_cast<const uint32_t*>(&b);
    }
    if ((reinterpret_cast<uintptr_t>(p) & 31u) == 0) {
        r4_store32(p, w);
    } else {
        reinterpret_cast<uint4*>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4*>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
}
__device__ __forceinline__ void r4_store(float* p, const float2 (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) reinterpret_cast<float4*>(p)[i] = make_float4(v[2 * i].x, v[2 * i].y, v[2 * i + 1].x, v[2 * i + 1].y);
}

template <typename T>
__global__ void __launch_bounds__(A4_THREADS)
paged4_read_kernel(Paged4View c, long long items, const int32_t* slot_map, T* k, T* v, int32_t* status) {
    const int kv = blockIdx.y, H = c.pv.H, d = c.pv.d, per_head = d / 32, per_tok = H * per_head;
    const uint8_t* codes = kv ? c.codes[1] : c.codes[0];
    const uint8_t* scales = kv ? c.scales[1] : c.scales[0];
    T* out = kv ? v : k;
    const long long step = (long long)gridDim.x * A4_THREADS;
    grid_dependency_wait();
    grid_dependents_may_launch();
    for (long long i0 = (long long)blockIdx.x * A4_THREADS + threadIdx.x; i0 < items; i0 += R4_UNROLL * step) {
        uint4 code[R4_UNROLL];
        uint32_t scale[R4_UNROLL];
        int head[R4_UNROLL];
        bool wrong = false;
#pragma unroll
        for (int u = 0; u < R4_UNROLL; ++u) {                             // all loads in flight
            const long long i = i0 + u * step;
            const int tok = (unsigned long long)i >> 32 ? (int)(i / per_tok) : (int)((unsigned)i / (unsigned)per_tok);
            const unsigned rest = (unsigned)(i - (long long)tok * per_tok);
            head[u] = (int)(rest / (unsigned)per_head);
            const int part = (int)(rest - (unsigned)head[u] * (unsigned)per_head);
            const int slot = i < items ? slot_map[tok] : -1;
            code[u] = make_uint4(0u, 0u, 0u, 0u);                         // a slot that is none: zeros
            scale[u] = 0u;
            if (slot >= 0 && slot < c.pv.n_pages * PAGE) {
                const long long row = ((long long)(slot / PAGE) * H + head[u]) * PAGE + slot % PAGE;
                code[u] = *reinterpret_cast<const uint4*>(codes + row * (d / 2) + part * 16);
                scale[u] = *reinterpret_cast<const uint16_t*>(scales + row * (d / 16) + part * 2);
            } else {
                wrong |= slot != -1;
            }
        }
        if (wrong) latch_error(status, TRIMKV_E_ARG);
#pragma unroll
        for (int u = 0; u < R4_UNROLL; ++u) {
            const long long i = i0 + u * step;
            if (i >= items) continue;
            const uint32_t s2 = p4_scales(scale[u]);
            const float up = p4_pow2(p4_shift(c, kv, head[u]));
            const uint32_t word[4] = {code[u].x, code[u].y, code[u].z, code[u].w};
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const uint32_t by = b ? p4_both_high(s2) : p4_both_low(s2);
                float2 val[8];
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    uint32_t r[4];
                    p4_codes(word[2 * b + w], r);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float2 f = p4_float2(p4_mul(r[e], by));
                        val[w * 4 + e] = make_float2(f.x * up, f.y * up);
                    }
                }
                r4_store(out + i * 32 + b * 16, val);                     // (items lie in the output's order)
            }
        }
    }
}

unsigned a4_blocks(long long items, int each) {      // `each` items per thread, fewer while that leaves the GPU unfilled
    const long long one = (items + A4_THREADS - 1) / A4_THREADS;
    return (unsigned)std::max<long long>(std::min<long long>(one, PAGED_SMS * 4), std::min<long long>((one + each - 1) / each, PAGED_SMS * 64));
}

}  // namespace

cudaError_t launch_paged4_append(const Paged4View& c, int is_bf16, int T, const void* k, long long k_stride, const void* v, long long v_stride,
                                 const int32_t* slot_map, int32_t* status, cudaStream_t st) {
    const long long items = (long long)T * c.pv.H * (c.pv.d / 32);
    auto go = [&](auto kernel, auto* type) {
        return paged_launch(kernel, dim3(a4_blocks(items, 1), 2), dim3(A4_THREADS), 0, 1, true, st, c, const_cast<uint8_t*>(c.codes[0]), const_cast<uint8_t*>(c.scales[0]),
                            const_cast<uint8_t*>(c.codes[1]), const_cast<uint8_t*>(c.scales[1]), items, (decltype(type))k, k_stride, (decltype(type))v, v_stride,
                            slot_map, status);
    };
    return is_bf16 ? go(paged4_append_kernel<__nv_bfloat16>, (const __nv_bfloat16*)nullptr) : go(paged4_append_kernel<float>, (const float*)nullptr);
}

cudaError_t launch_paged4_read(const Paged4View& c, int is_bf16, int n, const int32_t* slot_map, void* k, void* v, int32_t* status, cudaStream_t st) {
    const long long items = (long long)n * c.pv.H * (c.pv.d / 32);
    auto go = [&](auto kernel, auto* type) {
        return paged_launch(kernel, dim3(a4_blocks(items, R4_UNROLL), 2), dim3(A4_THREADS), 0, 1, true, st, c, items, slot_map, (decltype(type))k, (decltype(type))v, status);
    };
    return is_bf16 ? go(paged4_read_kernel<__nv_bfloat16>, (__nv_bfloat16*)nullptr) : go(paged4_read_kernel<float>, (float*)nullptr);
}

}  // namespace tkv
