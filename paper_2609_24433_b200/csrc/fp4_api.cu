// C ABI of the projections in microscaled 4-bit floating point and of the RMS norm that ends in codes (see include/fq.h):
// argument checks on the host, handles, dispatch.
#include <math.h>
#include <new>

#include "fp4_common.cuh"

using namespace fq;

namespace {

constexpr int64_t kMaxRowK = 32768;              // one thread block works on a row: 1024 threads of 32 channels
constexpr int64_t kMaxRows = 0x7fff0000;         // rows of one call (indexes of tiles are 32-bit)
constexpr int64_t kMaxN = 1ll << 28;             // channels of one handle

bool aligned(const void* p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
bool aligned16(const void* p) { return aligned(p, 16); }
bool valid_format(fq_fp4_format f) { return f == FQ_MXFP4 || f == FQ_NVFP4; }
bool valid_dtype(fq_dtype t) { return t == FQ_F32 || t == FQ_BF16; }
bool valid_block(int block, int64_t K) { return block >= 1 && block <= 256 && (block & (block - 1)) == 0 && K % block == 0; }
float block_norm(int block) { return (float)(1.0 / sqrt((double)block)); }

fq_status check_arch() {
    const int major = device_cc_major();
    if (major < 0) return FQ_ERR_CUDA;
    return major == 10 ? FQ_OK : FQ_ERR_ARCH;
}
fq_status check_width(int64_t K, int block) {
    if (K <= 0) return FQ_ERR_INVALID_ARG;
    return valid_block(block, K) && K % 32 == 0 && K <= kMaxRowK ? FQ_OK : FQ_ERR_UNSUPPORTED;
}
fq_status check_rows(const void* x, fq_dtype xt, int64_t M, int64_t K, int64_t ld) {
    if (!valid_dtype(xt)) return FQ_ERR_INVALID_ARG;
    if (M == 0) return FQ_OK;
    if (M > kMaxRows) return FQ_ERR_UNSUPPORTED;
    if (!x || ld < K) return FQ_ERR_INVALID_ARG;
    return aligned16(x) && ld % 8 == 0 ? FQ_OK : FQ_ERR_ALIGNMENT;
}
fq_status check_codes(const void* codes, const void* scales, const float* delta) {
    if (!codes || !scales || !delta) return FQ_ERR_INVALID_ARG;
    return aligned16(codes) && aligned16(scales) && aligned(delta, 4) ? FQ_OK : FQ_ERR_ALIGNMENT;
}
fq_status check_y(const void* y, fq_dtype yt, int64_t ldy, int64_t N) {
    if (!y || !valid_dtype(yt) || ldy < N) return FQ_ERR_INVALID_ARG;
    return aligned16(y) && ldy % 8 == 0 ? FQ_OK : FQ_ERR_ALIGNMENT;
}
// A handle's memory lies on the device that was current when it was made.
fq_status check_place(const Fp4Weights* w) {
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) {
        (void)cudaGetLastError();
        return FQ_ERR_CUDA;
    }
    return dev == w->device ? FQ_OK : FQ_ERR_INVALID_ARG;
}
fq_status done(cudaError_t e) { return e == cudaSuccess ? FQ_OK : FQ_ERR_CUDA; }

void release(Fp4Weights* w) {
    cudaFree(w->codes); cudaFree(w->scales); cudaFree(w->w_scale); cudaFree(w->bias); cudaFree(w->mult_g);
    delete w;
}
fq_status make_handle(int64_t N, int64_t K, int block, fq_fp4_format f, Fp4Weights** out) {
    Fp4Weights* w = new (std::nothrow) Fp4Weights();
    if (!w) return FQ_ERR_NOMEM;
    w->N = N; w->K = K; w->block = block; w->format = f;
    cudaGetDevice(&w->device);
    const size_t n = (size_t)(N > 0 ? N : 4), scales = fp4_scale_bytes(N, K, f);
    const bool ok = cudaMalloc(&w->codes, n * (size_t)K / 2) == cudaSuccess && cudaMalloc(&w->scales, scales ? scales : 16) == cudaSuccess &&
                    cudaMalloc(&w->w_scale, sizeof(float) * n) == cudaSuccess && cudaMalloc(&w->bias, sizeof(float) * n) == cudaSuccess &&
                    cudaMalloc(&w->mult_g, sizeof(float) * (size_t)K) == cudaSuccess;
    if (!ok) {
        (void)cudaGetLastError();
        release(w);
        return FQ_ERR_NOMEM;
    }
    *out = w;
    return FQ_OK;
}
fq_status check_handle(int64_t N, int64_t K, int block, fq_fp4_format f) {
    if (N < 0 || !valid_format(f)) return FQ_ERR_INVALID_ARG;
    const fq_status st = check_width(K, block);
    if (st != FQ_OK) return st;
    return N % 8 == 0 && N <= kMaxN ? FQ_OK : FQ_ERR_UNSUPPORTED;
}
// A vector of a handle: the caller's or a constant.
bool vector(float* dst, const float* src, float otherwise, int64_t n, cudaStream_t s) {
    if (n == 0) return true;
    if (src) return cudaMemcpyAsync(dst, src, sizeof(float) * (size_t)n, cudaMemcpyDeviceToDevice, s) == cudaSuccess;
    return launch_fill(dst, otherwise, n, s) == cudaSuccess;
}

struct Workspace {
    uint8_t* codes;
    uint8_t* scales;
    float* delta;
};
size_t code_part(int64_t M, int64_t K) { return align_up((size_t)M * (size_t)K / 2, 256); }
size_t scale_part(int64_t M, int64_t K, fq_fp4_format f) { return align_up(fp4_scale_bytes(M, K, f), 256); }

fq_status rmsnorm(const void* x, const void* residual, fq_dtype xt, int64_t M, int64_t K, int64_t ldx, int64_t ldr, float eps, void* h, int64_t ldh,
                  const float* mult_g, int block, RowFmt fmt, float clip_ratio, void* codes, void* scales, float* delta, cudaStream_t stream) {
    const bool fp4 = fmt == RowFmt::Mx || fmt == RowFmt::Nv;
    if (M < 0 || !(eps >= 0.0f) || !(eps <= 3.402823466e38f)) return FQ_ERR_INVALID_ARG;
    fq_status st = check_width(K, block);
    if (st == FQ_OK) st = check_rows(x, xt, M, K, ldx);
    if (st != FQ_OK || M == 0) return st;
    if ((residual != nullptr) != (h != nullptr)) return FQ_ERR_INVALID_ARG;
    if (residual) {
        if ((st = check_rows(residual, xt, M, K, ldr)) != FQ_OK || (st = check_rows(h, xt, M, K, ldh)) != FQ_OK) return st;
        if ((h == x && ldh != ldx && M > 1) || (h == residual && ldh != ldr && M > 1)) return FQ_ERR_INVALID_ARG;
    }
    if ((st = check_codes(codes, fp4 ? scales : codes, delta)) != FQ_OK) return st;
    if (mult_g && !aligned16(mult_g)) return FQ_ERR_ALIGNMENT;
    if ((st = check_arch()) != FQ_OK) return st;
    RowQuant q = {};
    q.x = x; q.residual = residual; q.h = h;
    q.xt = xt; q.rows = M; q.K = K; q.ldx = ldx; q.ldr = ldr; q.ldh = ldh;
    q.norm = true; q.eps = eps;
    q.mult = mult_g; q.cnorm = block_norm(block); q.clip_ratio = clip_ratio; q.block = block;
    q.fmt = fmt;
    q.codes = static_cast<uint8_t*>(codes); q.scales = static_cast<uint8_t*>(scales); q.delta = delta;
    return done(launch_row_quantize(q, stream));
}

}  // namespace

extern "C" {

size_t fq_fp4_scale_bytes(int64_t rows, int64_t K, fq_fp4_format format) {
    if (rows <= 0 || rows > kMaxRows || !valid_format(format) || K <= 0 || K % 32 != 0 || K > kMaxRowK) return 0;
    return fp4_scale_bytes(rows, K, format);
}

fq_status fq_fold_weights_fp4(const void* Wsrc, fq_dtype wt, int64_t N, int64_t K, int64_t ldw, const float* smooth, const float* bias,
                              int hadamard_block, fq_fp4_format format, void* stream, fq_fp4_weights** out) {
    if (!out) return FQ_ERR_INVALID_ARG;
    *out = nullptr;
    fq_status st = check_handle(N, K, hadamard_block, format);
    if (st == FQ_OK) st = check_rows(Wsrc, wt, N, K, ldw);
    if (st != FQ_OK) return st;
    if ((smooth && !aligned16(smooth)) || (bias && !aligned(bias, 4))) return FQ_ERR_ALIGNMENT;
    if ((st = check_arch()) != FQ_OK) return st;
    Fp4Weights* w = nullptr;
    if ((st = make_handle(N, K, hadamard_block, format, &w)) != FQ_OK) return st;
    float* mult_w = nullptr;                     // s_c block^-1/2, needed here only
    if (cudaMalloc(&mult_w, sizeof(float) * (size_t)K) != cudaSuccess) {
        (void)cudaGetLastError();
        release(w);
        return FQ_ERR_NOMEM;
    }
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    w->mult_const = smooth == nullptr;
    bool ok = launch_multipliers(smooth, K, block_norm(hadamard_block), mult_w, w->mult_g, s) == cudaSuccess;
    RowQuant q = {};
    q.x = Wsrc; q.xt = wt; q.rows = N; q.K = K; q.ldx = ldw;
    q.mult = mult_w; q.cnorm = block_norm(hadamard_block); q.clip_ratio = 1.0f; q.block = hadamard_block;
    q.fmt = format == FQ_NVFP4 ? RowFmt::Nv : RowFmt::Mx;
    q.codes = w->codes; q.scales = w->scales; q.delta = w->w_scale;
    ok = ok && launch_row_quantize(q, s) == cudaSuccess && vector(w->bias, bias, 0.0f, N, s);
    ok = cudaStreamSynchronize(s) == cudaSuccess && ok;
    cudaFree(mult_w);
    if (!ok || !fp4_weight_maps(*w)) {
        release(w);
        return FQ_ERR_CUDA;
    }
    *out = reinterpret_cast<fq_fp4_weights*>(w);
    return FQ_OK;
}

fq_status fq_fp4_weights_import(const void* codes, const void* scales, const float* w_scale, const float* mult_g, const float* bias, int64_t N,
                                int64_t K, int hadamard_block, fq_fp4_format format, void* stream, fq_fp4_weights** out) {
    if (!out) return FQ_ERR_INVALID_ARG;
    *out = nullptr;
    fq_status st = check_handle(N, K, hadamard_block, format);
    if (st != FQ_OK) return st;
    if (N > 0 && (!codes || !scales)) return FQ_ERR_INVALID_ARG;
    if (!aligned(w_scale, 4) || !aligned(mult_g, 4) || !aligned(bias, 4)) return FQ_ERR_ALIGNMENT;
    if ((st = check_arch()) != FQ_OK) return st;
    Fp4Weights* w = nullptr;
    if ((st = make_handle(N, K, hadamard_block, format, &w)) != FQ_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    w->mult_const = mult_g == nullptr;
    bool ok = true;
    if (N > 0) {
        ok = cudaMemcpyAsync(w->codes, codes, (size_t)N * (size_t)K / 2, cudaMemcpyDeviceToDevice, s) == cudaSuccess &&
             cudaMemcpyAsync(w->scales, scales, fp4_scale_bytes(N, K, format), cudaMemcpyDeviceToDevice, s) == cudaSuccess &&
             launch_fp4_clear_pads(w->scales, N, K, format, s) == cudaSuccess;
    }
    ok = ok && vector(w->w_scale, w_scale, 1.0f, N, s) && vector(w->bias, bias, 0.0f, N, s) && vector(w->mult_g, mult_g, block_norm(hadamard_block), K, s);
    ok = cudaStreamSynchronize(s) == cudaSuccess && ok;
    if (!ok || !fp4_weight_maps(*w)) {
        release(w);
        return FQ_ERR_CUDA;
    }
    *out = reinterpret_cast<fq_fp4_weights*>(w);
    return FQ_OK;
}

fq_status fq_fp4_weights_export(const fq_fp4_weights* wp, void* codes, void* scales, float* w_scale, float* mult_g, float* bias, void* stream) {
    const Fp4Weights* w = reinterpret_cast<const Fp4Weights*>(wp);
    if (!w) return FQ_ERR_INVALID_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    auto copy = [s](void* dst, const void* src, size_t n) { return !dst || n == 0 || cudaMemcpyAsync(dst, src, n, cudaMemcpyDeviceToDevice, s) == cudaSuccess; };
    const size_t n = (size_t)w->N;
    const bool ok = copy(codes, w->codes, n * (size_t)w->K / 2) && copy(scales, w->scales, fp4_scale_bytes(w->N, w->K, w->format)) &&
                    copy(w_scale, w->w_scale, 4 * n) && copy(mult_g, w->mult_g, 4 * (size_t)w->K) && copy(bias, w->bias, 4 * n);
    return ok ? FQ_OK : FQ_ERR_CUDA;
}

fq_status fq_fp4_weights_info(const fq_fp4_weights* wp, int64_t* N, int64_t* K, int* hadamard_block, fq_fp4_format* format) {
    const Fp4Weights* w = reinterpret_cast<const Fp4Weights*>(wp);
    if (!w) return FQ_ERR_INVALID_ARG;
    if (N) *N = w->N;
    if (K) *K = w->K;
    if (hadamard_block) *hadamard_block = w->block;
    if (format) *format = w->format;
    return FQ_OK;
}

const float* fq_fp4_weights_multiplier(const fq_fp4_weights* wp) {
    const Fp4Weights* w = reinterpret_cast<const Fp4Weights*>(wp);
    return w ? w->mult_g : nullptr;
}

fq_status fq_fp4_weights_destroy(fq_fp4_weights* wp) {
    if (wp) release(reinterpret_cast<Fp4Weights*>(wp));
    return FQ_OK;
}

fq_status fq_quantize_act_fp4(const void* x, fq_dtype xt, int64_t M, int64_t K, int64_t ldx, const float* mult_g, int hadamard_block,
                              fq_fp4_format format, void* codes_out, void* scales_out, float* delta_out, void* stream) {
    if (M < 0 || !valid_format(format)) return FQ_ERR_INVALID_ARG;
    fq_status st = check_width(K, hadamard_block);
    if (st == FQ_OK) st = check_rows(x, xt, M, K, ldx);
    if (st != FQ_OK || M == 0) return st;
    if ((st = check_codes(codes_out, scales_out, delta_out)) != FQ_OK) return st;
    if (mult_g && !aligned16(mult_g)) return FQ_ERR_ALIGNMENT;
    if ((st = check_arch()) != FQ_OK) return st;
    RowQuant q = {};
    q.x = x; q.xt = xt; q.rows = M; q.K = K; q.ldx = ldx;
    q.mult = mult_g; q.cnorm = block_norm(hadamard_block); q.clip_ratio = 1.0f; q.block = hadamard_block;
    q.fmt = format == FQ_NVFP4 ? RowFmt::Nv : RowFmt::Mx;
    q.codes = static_cast<uint8_t*>(codes_out); q.scales = static_cast<uint8_t*>(scales_out); q.delta = delta_out;
    return done(launch_row_quantize(q, static_cast<cudaStream_t>(stream)));
}

fq_status fq_gemm_fp4(const void* a_codes, const void* a_scales, const float* a_delta, int64_t M, const fq_fp4_weights* Wp, void* y, fq_dtype yt,
                      int64_t ldy, void* stream) {
    const Fp4Weights* W = reinterpret_cast<const Fp4Weights*>(Wp);
    if (!W || M < 0) return FQ_ERR_INVALID_ARG;
    if (M == 0 || W->N == 0) return FQ_OK;
    if (M > kMaxRows) return FQ_ERR_UNSUPPORTED;
    fq_status st = check_codes(a_codes, a_scales, a_delta);
    if (st == FQ_OK) st = check_y(y, yt, ldy, W->N);
    if (st == FQ_OK) st = check_arch();
    if (st == FQ_OK) st = check_place(W);
    if (st != FQ_OK) return st;
    return launch_gemm_fp4(static_cast<const uint8_t*>(a_codes), static_cast<const uint8_t*>(a_scales), a_delta, M, *W, y, yt, ldy,
                           static_cast<cudaStream_t>(stream));
}

size_t fq_linear_fp4_workspace_bytes(int64_t M, int64_t K, fq_fp4_format format) {
    if (M <= 0 || M > kMaxRows || !valid_format(format) || K <= 0 || K % 32 != 0 || K > kMaxRowK) return 0;
    return code_part(M, K) + scale_part(M, K, format) + align_up(sizeof(float) * (size_t)M, 256);
}

fq_status fq_linear_fp4(const void* x, fq_dtype xt, int64_t M, int64_t ldx, const fq_fp4_weights* Wp, void* y, fq_dtype yt, int64_t ldy,
                        void* workspace, size_t ws_bytes, void* stream) {
    const Fp4Weights* W = reinterpret_cast<const Fp4Weights*>(Wp);
    if (!W || M < 0) return FQ_ERR_INVALID_ARG;
    fq_status st = check_rows(x, xt, M, W->K, ldx);
    if (st != FQ_OK || M == 0 || W->N == 0) return st;
    if ((st = check_y(y, yt, ldy, W->N)) != FQ_OK) return st;
    if (!workspace) return FQ_ERR_INVALID_ARG;
    if (!aligned(workspace, 256)) return FQ_ERR_ALIGNMENT;
    if (ws_bytes < fq_linear_fp4_workspace_bytes(M, W->K, W->format)) return FQ_ERR_NOMEM;
    if ((st = check_arch()) != FQ_OK || (st = check_place(W)) != FQ_OK) return st;
    uint8_t* codes = static_cast<uint8_t*>(workspace);
    uint8_t* scales = codes + code_part(M, W->K);
    float* delta = reinterpret_cast<float*>(scales + scale_part(M, W->K, W->format));
    RowQuant q = {};
    q.x = x; q.xt = xt; q.rows = M; q.K = W->K; q.ldx = ldx;
    q.mult = W->mult_const ? nullptr : W->mult_g; q.cnorm = block_norm(W->block); q.clip_ratio = 1.0f; q.block = W->block;
    q.fmt = W->format == FQ_NVFP4 ? RowFmt::Nv : RowFmt::Mx;
    q.codes = codes; q.scales = scales; q.delta = delta;
    q.mult_ready = true;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (launch_row_quantize(q, s) != cudaSuccess) return FQ_ERR_CUDA;
    return launch_gemm_fp4(codes, scales, delta, M, *W, y, yt, ldy, s);
}

fq_status fq_rmsnorm_quantize_act(const void* x, const void* residual, fq_dtype xt, int64_t M, int64_t K, int64_t ldx, int64_t ldr, float eps,
                                  void* h, int64_t ldh, const float* mult_g, int hadamard_block, int bits, float clip_ratio, void* codes_out,
                                  float* delta_out, void* stream) {
    if ((bits != 4 && bits != 8) || !(clip_ratio > 0.0f && clip_ratio <= 1.0f)) return FQ_ERR_INVALID_ARG;
    return rmsnorm(x, residual, xt, M, K, ldx, ldr, eps, h, ldh, mult_g, hadamard_block, bits == 4 ? RowFmt::Int4 : RowFmt::Int8, clip_ratio,
                   codes_out, nullptr, delta_out, static_cast<cudaStream_t>(stream));
}

fq_status fq_rmsnorm_quantize_act_fp4(const void* x, const void* residual, fq_dtype xt, int64_t M, int64_t K, int64_t ldx, int64_t ldr, float eps,
                                      void* h, int64_t ldh, const float* mult_g, int hadamard_block, fq_fp4_format format, void* codes_out,
                                      void* scales_out, float* delta_out, void* stream) {
    if (!valid_format(format)) return FQ_ERR_INVALID_ARG;
    return rmsnorm(x, residual, xt, M, K, ldx, ldr, eps, h, ldh, mult_g, hadamard_block, format == FQ_NVFP4 ? RowFmt::Nv : RowFmt::Mx, 1.0f,
                   codes_out, scales_out, delta_out, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
