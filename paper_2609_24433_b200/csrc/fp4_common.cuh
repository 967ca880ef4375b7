// Internal declarations of the projections in microscaled 4-bit floating point and of the row quantiser that they share with
// the RMS norm.
#pragma once

#include "fq_common.cuh"

namespace fq {

constexpr int fp4_block(fq_fp4_format f) { return f == FQ_NVFP4 ? 16 : 32; }
// Tiles of 512 scale bytes (128 rows x 4 blocks) across K.
inline int64_t fp4_scale_tiles(int64_t K, fq_fp4_format f) { return (K / fp4_block(f) + 3) / 4; }
inline size_t fp4_scale_bytes(int64_t rows, int64_t K, fq_fp4_format f) { return (size_t)((rows + 127) / 128) * (size_t)fp4_scale_tiles(K, f) * 512; }

struct Fp4Weights {
    int64_t N = 0, K = 0;
    int block = 0;
    fq_fp4_format format = FQ_NVFP4;
    int device = 0;
    uint8_t* codes = nullptr;    // [N, K/2]
    uint8_t* scales = nullptr;   // tiles
    float* w_scale = nullptr;    // [N]
    float* bias = nullptr;       // [N]
    float* mult_g = nullptr;     // [K]
    bool mult_const = false;     // block^-1/2 in every entry
    CUtensorMap map_codes, map_scales;
};

// Codes of rows: an optional residual and norm ahead of transform and quantiser.
enum class RowFmt : int { Int4 = 0, Int8 = 1, Mx = 3, Nv = 4 };
struct RowQuant {
    const void* x;
    const void* residual;        // with h
    void* h;
    fq_dtype xt;
    int64_t rows, K, ldx, ldr, ldh;
    bool norm;
    float eps;
    const float* mult;           // or null: cnorm
    float cnorm, clip_ratio;
    int block;
    RowFmt fmt;
    uint8_t* codes;
    uint8_t* scales;             // Mx, Nv
    float* delta;
    bool mult_ready;             // see kMultReady
};
cudaError_t launch_row_quantize(const RowQuant& q, cudaStream_t stream);

// Zeros in the places of the scale tiles past the last row or block.
cudaError_t launch_fp4_clear_pads(uint8_t* scales, int64_t rows, int64_t K, fq_fp4_format f, cudaStream_t stream);
cudaError_t launch_fill(float* p, float v, int64_t n, cudaStream_t stream);

bool fp4_weight_maps(Fp4Weights& W);
fq_status launch_gemm_fp4(const uint8_t* codes, const uint8_t* scales, const float* delta, int64_t M, const Fp4Weights& W, void* y,
                          fq_dtype yt, int64_t ldy, cudaStream_t stream);

}  // namespace fq
