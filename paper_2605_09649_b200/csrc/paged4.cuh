// The paged cache held in 4 bits: layout, number formats, launchers.  Not part of the public ABI.
//
// k_codes, v_codes [n_pages][H][64][d / 2]: channel 2 i of an entry in the low half of byte i, 2 i + 1 in the high half; each
// half an e2m1 number (sign, two bits of exponent, one of mantissa: 0, 0.5, 1, 1.5, 2, 3, 4, 6).  k_scales, v_scales
// [n_pages][H][64][d / 16]: an e4m3 number per 16 channels.  k_shift, v_shift [H] or null: value = code x scale x 2^shift.
// Why e2m1 x e4m3: the product of the two has at most 6 significant bits and lies in 2^-10 .. 2688, so it is exact in fp16 (and
// in bf16), and the tensor cores see the cache's values without a rounding; one instruction turns a byte of codes into two fp16.
#pragma once

#include <float.h>

#include <cuda_fp16.h>

#include "paged.cuh"

namespace tkv {

constexpr int P4_BLOCK = 16;                  // channels that share a scale
constexpr int P4_MAX_SHIFT = 64;

struct Paged4View {
    PagedView pv;                             // n_pages, H, d; no pointers
    const uint8_t* codes[2];                  // K, V
    const uint8_t* scales[2];
    const int32_t* shift[2];                  // or null
};

__device__ __forceinline__ int p4_shift(const Paged4View& c, int kv, int h) {
    const int32_t* shift = kv ? c.shift[1] : c.shift[0];      // (an index known only at run time would copy the view to local memory)
    return shift ? max(-P4_MAX_SHIFT, min(P4_MAX_SHIFT, shift[h])) : 0;
}
__device__ __forceinline__ float p4_pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }      // 2^e, -126 <= e <= 127

// From a row's products to logits in log2 units, scale_log2 2^e.  A scale, a shift and a row's own power of two may together leave fp32's
// range; a factor of 0 or infinity would make masked (-inf) or zero products NaN.  At the lower end logits are below 2^-95 either way.
__device__ __forceinline__ float p4_to_log2(float scale_log2, int e) {
    return fminf(fmaxf(scale_log2 * p4_pow2(max(-126, min(127, e))), FLT_MIN), FLT_MAX);
}

// Four bytes of codes as eight fp16: r[i] = {low half of byte i, high half}.
__device__ __forceinline__ void p4_codes(uint32_t b, uint32_t (&r)[4]) {
    asm("{\n\t.reg .b8 x, y, z, w;\n\tmov.b32 {x, y, z, w}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, x;\n\tcvt.rn.f16x2.e2m1x2 %1, y;\n\tcvt.rn.f16x2.e2m1x2 %2, z;\n\tcvt.rn.f16x2.e2m1x2 %3, w;\n\t}"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
        : "r"(b));
}
// Two scales (the low 16 bits) as two fp16.
__device__ __forceinline__ uint32_t p4_scales(uint32_t two) {
    uint32_t r;
    asm("{\n\t.reg .b16 x;\n\tcvt.u16.u32 x, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, x;\n\t}" : "=r"(r) : "r"(two));
    return r;
}
__device__ __forceinline__ uint32_t p4_mul(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t p4_both_low(uint32_t a) { return __byte_perm(a, a, 0x1010); }
__device__ __forceinline__ uint32_t p4_both_high(uint32_t a) { return __byte_perm(a, a, 0x3232); }
__device__ __forceinline__ uint32_t p4_f16x2(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ float2 p4_float2(uint32_t a) { return __half22float2(*reinterpret_cast<const __half2*>(&a)); }

cudaError_t launch_paged4_append(const Paged4View& c, int is_bf16, int T, const void* k, long long k_stride, const void* v, long long v_stride,
                                 const int32_t* slot_map, int32_t* status, cudaStream_t st);
cudaError_t launch_paged4_read(const Paged4View& c, int is_bf16, int n, const int32_t* slot_map, void* k, void* v, int32_t* status, cudaStream_t st);

// Warp kernel: workers per SM and the most rows that they hold in all (workers x rows of a unit).
constexpr int P4_WARPS = 16;
constexpr int P4_WORKER_ROWS = PAGED_SMS * 11 * 16;
constexpr size_t P4_SHARED_BYTES = (size_t)PAGED_SMS * P4_WARPS * 16;
static_assert(P4_SHARED_BYTES % 256 == 0, "partial results are aligned");
// Units of tile_rows = 8 or 16 rows (fp32 and head sizes above 128: 8) of the requests of up to max_rows rows.
cudaError_t launch_paged4_attention_warp(const Paged4View& c, const PagedBatch& pb, int is_bf16, const void* q, void* out, float scale, const PagedWork& w,
                                         int tile_rows, int max_rows, cudaStream_t st);
// Tensor-core kernel, bf16 and head sizes up to PAGED_TC_HEAD: units of PAGED_TC_ROWS rows of the requests of more than min_rows - 1.
cudaError_t launch_paged4_attention_tc(const Paged4View& c, const PagedBatch& pb, const void* q, void* out, float scale, const PagedWork& w, int min_rows,
                                       cudaStream_t st);

}  // namespace tkv
