// Device helpers of the two kernels from rows to codes.
#pragma once

#include <float.h>
#include <stdint.h>

#include "fp4_common.cuh"

namespace fq {

// cudaErrorNotSupported where the rows do not fit it or are too few; the caller then uses the kernel that keeps rows in registers.
cudaError_t launch_row_quantize_ring(const RowQuant& q, cudaStream_t stream);

namespace {

// Eight e2m1 codes, element 0 in the lowest nibble.
__device__ __forceinline__ uint32_t pack_e2m1(const float* v) {
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r)
        : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}
// e4m3 of a non-negative number, and what it stands for.
__device__ __forceinline__ uint32_t to_e4m3(float v, float* back) {
    uint16_t b;
    uint32_t h2;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(b) : "f"(0.0f), "f"(v));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h2) : "h"(b));
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.f32.f16 %0, l;\n\t}" : "=f"(*back) : "r"(h2));
    return b & 0xffu;
}

// Step of a row and its inverse for q = 127 or 7 (a row below the smallest normal step is the zero token).
__device__ __forceinline__ float int_step(float m, float clip, float inv_qmax, float* inv) {
    const float d = __fmul_rn(__fmul_rn(clip, m), inv_qmax);
    *inv = d >= FLT_MIN ? __fdiv_rn(1.0f, d) : 0.0f;
    return d >= FLT_MIN ? d : 0.0f;
}
// The same of a row of e2m1 with e4m3 scales (the zero token: below 2^-100).
__device__ __forceinline__ float nv_step(float m, float* inv) {
    const float d = __fmul_rn(m, 1.0f / 2688.0f);
    const bool live = d >= 7.888609052e-31f;
    *inv = live ? __fdiv_rn(1.0f, d) : 0.0f;
    return live ? d : 0.0f;
}
// Scale byte of a block with largest magnitude m, and what its channels are multiplied by.
__device__ __forceinline__ uint32_t nv_scale(float m, float inv, float* q) {
    float s;
    const uint32_t byte = to_e4m3(__fmul_rn(__fmul_rn(m, inv), 0.166666672f), &s);
    *q = s > 0.0f ? __fdiv_rn(inv, s) : 0.0f;
    return byte;
}
__device__ __forceinline__ uint32_t mx_scale(float m, float* q) {
    const int e = max((int)(__float_as_uint(m) >> 23) - 2, 0);
    *q = __uint_as_float((uint32_t)(254 - e) << 23);
    return (uint32_t)e;
}
// Step of a row with largest magnitude m, ahead of the norm.
template <int FMT>
__device__ __forceinline__ float row_step(float m, float clip) {
    float inv;
    return FMT == 3 ? 1.0f : FMT == 4 ? nv_step(m, &inv) : int_step(m, clip, 1.0f / (FMT == 0 ? 7.0f : 127.0f), &inv);
}
// 1 / sqrt(sum / K + eps); the sum in binary32.  (0 for a sum of 0 without eps; a sum that is NaN stays it.)
__device__ __forceinline__ float inverse_rms(float total, int K, float eps) {
    const float ms = __fadd_rn(__fdiv_rn(total, (float)K), eps);
    return ms == 0.0f ? 0.0f : __fdiv_rn(1.0f, __fsqrt_rn(ms));
}
// Rows whose squares leave binary32 have them added up in binary64, and their step divided there: 1 / rms may leave binary32 where
// the step does not.  A step of 1 / rms that does (e2m1 with e8m0 scales, whose codes are then all but zeros) makes the zero token; an
// infinite sum, of a row that is not finite, a NaN.
__device__ __forceinline__ bool squares_leave_range(float total, float m, float eps) { return total > 1e37f || (m > 0.0f && total < 1e-30f && eps < 1e-20f); }
template <int FMT>
__device__ __forceinline__ float wide_step(float m, float clip, double sum, int K, float eps) {
    const double s = (double)row_step<FMT>(m, clip) / sqrt(sum / K + (double)eps);
    return FMT == 3 && s > (double)FLT_MAX ? 0.0f : (float)(s + (sum - sum));
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

}  // namespace
}  // namespace fq
