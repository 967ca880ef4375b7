// Rows to codes: [h = x + residual, RMS norm,] per-channel multiplier, block FWHT, quantiser to 4- or 8-bit integers with a step
// per row or to e2m1 with block scales (formulas: include/fq.h).
//
// The norm needs no pass of its own: the quantiser is positively homogeneous, so the codes of h / rms are those of h and only
// the step is divided by rms.  Largest magnitude and sum of squares are then two reductions behind one barrier.
//
// A thread owns E consecutive channels of a row, a row is spread over whole warps, and the row stays in registers between the
// reduction and the quantiser: x (and the residual) are read once.  Butterflies of strides below E run in registers on pairs
// (channel p, channel p + E/2), two IEEE operations per packed instruction; strides E .. block/2 go across lanes.
#include <cuda_bf16.h>
#include <float.h>

#include "act_common.cuh"
#include "fp4_common.cuh"
#include "ptx_sm100.cuh"
#include "row_quant.cuh"

namespace fq {
namespace {

struct RowParams {
    const void* x;
    const void* residual;
    void* h;
    int64_t rows, rows_pad, ldx, ldr, ldh;
    int K, block, tpr, rpc;
    float eps, cnorm, clip_ratio, qmax;
    const float* mult;
    uint8_t* codes;
    uint8_t* scales;
    int scale_tiles;
    float* delta;
    int mult_ready, early;
};

// Eight values of two bytes or four of four as they lie in memory.
template <typename XT, int E>
struct Raw {
    static constexpr int kVecs = E * (int)sizeof(XT) / 16;
    uint4 q[kVecs];
    __device__ __forceinline__ void load(const XT* p, bool ok) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) q[i] = ld_global_v4(reinterpret_cast<const uint4*>(p) + i, ok);
    }
    __device__ __forceinline__ void store(XT* p) const {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) reinterpret_cast<uint4*>(p)[i] = q[i];
    }
    __device__ __forceinline__ uint32_t word(int i) const {
        const uint4 v = q[i / 4];
        return i % 4 == 0 ? v.x : i % 4 == 1 ? v.y : i % 4 == 2 ? v.z : v.w;
    }
    __device__ __forceinline__ float get(int c) const {
        if (sizeof(XT) == 4) return __uint_as_float(word(c));
        return __uint_as_float(c & 1 ? word(c / 2) & 0xffff0000u : word(c / 2) << 16);
    }
    __device__ __forceinline__ void add(const Raw& r) {          // rounded once, to XT
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (sizeof(XT) == 4) {
                    w[j] = __float_as_uint(__fadd_rn(get(4 * i + j), r.get(4 * i + j)));
                } else {
                    const int c = 8 * i + 2 * j;
                    const float2 s = f2_add(make_float2(get(c), get(c + 1)), make_float2(r.get(c), r.get(c + 1)));
                    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[j]) : "f"(s.y), "f"(s.x));
                }
            }
            q[i] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
};

// CACHE: the multiplier's slice stays in registers and the next row is requested while this one is worked on (at most 512
// threads); otherwise both are read where they are needed.
template <typename XT, int E, int FMT, bool NORM, bool CACHE>
__global__ void __launch_bounds__(CACHE ? 512 : 1024) row_quantize_kernel(const RowParams p) {
    constexpr bool kFp4 = FMT >= 3, kMx = FMT == 3;
    constexpr bool kReduce = NORM || !kMx;                    // a row's largest magnitude or sum of squares is needed
    constexpr int kHalf = E / 2;
    __shared__ float2 s_part[2][32];                          // per warp: largest magnitude, sum of squares; double buffered

    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int r_in_cta = threadIdx.x / p.tpr, t_in_row = threadIdx.x - r_in_cta * p.tpr;
    const int wpr = p.tpr >> 5;
    const int col0 = t_in_row * E;
    const bool col_ok = col0 < p.K;
    const XT* x = static_cast<const XT*>(p.x) + col0;
    const XT* res = NORM && p.residual ? static_cast<const XT*>(p.residual) + col0 : nullptr;
    XT* h = NORM ? static_cast<XT*>(p.h) + col0 : nullptr;

    float2 g[CACHE ? kHalf : 1];
    auto load_g = [&]() {
#pragma unroll
        for (int i = 0; i < kHalf / 4; ++i) {
            const float4 a = ld_global_f4(p.mult + col0 + 4 * i, col_ok), b = ld_global_f4(p.mult + col0 + kHalf + 4 * i, col_ok);
            g[(4 * i + 0) % (CACHE ? kHalf : 1)] = make_float2(a.x, b.x);
            g[(4 * i + 1) % (CACHE ? kHalf : 1)] = make_float2(a.y, b.y);
            g[(4 * i + 2) % (CACHE ? kHalf : 1)] = make_float2(a.z, b.z);
            g[(4 * i + 3) % (CACHE ? kHalf : 1)] = make_float2(a.w, b.w);
        }
    };
    if (p.early) griddep_launch_dependents();
    if (CACHE) {
        if (!p.mult) {
#pragma unroll
            for (int i = 0; i < kHalf; ++i) g[i % (CACHE ? kHalf : 1)] = make_float2(p.cnorm, p.cnorm);
        } else if (p.mult_ready) {
            load_g();
        }
    }
    griddep_wait();
    if (!p.early) griddep_launch_dependents();
    if (CACHE && p.mult && !p.mult_ready) load_g();

    const int64_t step = (int64_t)gridDim.x * p.rpc;
    int64_t row = (int64_t)blockIdx.x * p.rpc + r_in_cta;
    Raw<XT, E> nx, nr;
    if (CACHE) {
        nx.load(x + row * p.ldx, col_ok && row < p.rows);
        if (NORM && res) nr.load(res + row * p.ldr, col_ok && row < p.rows);
    }
    int buf = 0;
    for (int64_t rb = (int64_t)blockIdx.x * p.rpc; rb < p.rows_pad; rb += step, row += step, buf ^= 1) {
        // place of this row's scales in its tile
        uint8_t* sc = nullptr;
        constexpr int kLanesPerWord = (kMx ? 128 : 64) / E;    // threads that share the four scales of a tile's row
        const int tile = (t_in_row * E) / (kMx ? 128 : 64);
        const bool sc_ok = kFp4 && row < p.rows_pad && tile < p.scale_tiles && lane % kLanesPerWord == 0;
        if (kFp4) sc = p.scales + ((row >> 7) * p.scale_tiles + tile) * 512 + (row & 31) * 16 + ((row & 127) >> 5) * 4;
        if (kFp4 && rb >= p.rows) {                            // rows that only pad the last tile
            if (sc_ok) *reinterpret_cast<uint32_t*>(sc) = 0u;
            continue;
        }
        const bool row_ok = col_ok && row < p.rows;
        Raw<XT, E> in;
        float2 v[kHalf];
        float ss = 0.0f;
        if (CACHE) {
            in = nx;
            if (NORM && res) in.add(nr);
            const int64_t next = row + step;
            const bool ok = col_ok && next < p.rows;
            nx.load(x + next * p.ldx, ok);
            if (NORM && res) nr.load(res + next * p.ldr, ok);
        } else {
            in.load(x + row * p.ldx, row_ok);
            if (NORM && res) {
                nr.load(res + row * p.ldr, row_ok);
                in.add(nr);
            }
        }
        if (NORM && res && row_ok) in.store(h + row * p.ldh);
#pragma unroll
        for (int i = 0; i < kHalf; ++i) v[i] = make_float2(in.get(i), in.get(i + kHalf));
        if (NORM) {
            float2 s2 = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int i = 0; i < kHalf; ++i) s2 = f2_fma(v[i], v[i], s2);
            ss = s2.x + s2.y;
        }
        if (CACHE) {
#pragma unroll
            for (int i = 0; i < kHalf; ++i) v[i] = f2_mul(v[i], g[i % (CACHE ? kHalf : 1)]);
        } else if (p.mult) {
#pragma unroll
            for (int i = 0; i < kHalf / 4; ++i) {
                const float4 a = ld_global_f4(p.mult + col0 + 4 * i, col_ok), b = ld_global_f4(p.mult + col0 + kHalf + 4 * i, col_ok);
                v[4 * i + 0] = f2_mul(v[4 * i + 0], make_float2(a.x, b.x));
                v[4 * i + 1] = f2_mul(v[4 * i + 1], make_float2(a.y, b.y));
                v[4 * i + 2] = f2_mul(v[4 * i + 2], make_float2(a.z, b.z));
                v[4 * i + 3] = f2_mul(v[4 * i + 3], make_float2(a.w, b.w));
            }
        } else {
#pragma unroll
            for (int i = 0; i < kHalf; ++i) v[i] = f2_mul(v[i], make_float2(p.cnorm, p.cnorm));
        }
        // strides 1 .. E/4: both halves at once (a - b as b * -1 + a: exact product, the same rounding)
#pragma unroll
        for (int s = 1; s < kHalf; s <<= 1) {
            if (s < p.block) {
#pragma unroll
                for (int i = 0; i < kHalf; ++i) {
                    if ((i & s) == 0) {
                        const float2 a = v[i], b = v[i + s];
                        v[i] = f2_add(a, b);
                        v[i + s] = f2_fma(b, make_float2(-1.0f, -1.0f), a);
                    }
                }
            }
        }
        if (kHalf < p.block) {
#pragma unroll
            for (int i = 0; i < kHalf; ++i) v[i] = make_float2(__fadd_rn(v[i].x, v[i].y), __fsub_rn(v[i].x, v[i].y));
        }
        // strides E .. block/2: the lane with the bit keeps partner - own
        for (int s = E; s < p.block; s <<= 1) {
            const int lm = s / E;
            const float sgn = (lane & lm) ? -1.0f : 1.0f;
#pragma unroll
            for (int i = 0; i < kHalf; ++i) {
                const float2 o = make_float2(__shfl_xor_sync(0xffffffffu, v[i].x, lm), __shfl_xor_sync(0xffffffffu, v[i].y, lm));
                v[i] = f2_fma(v[i], make_float2(sgn, sgn), o);
            }
        }
        // largest magnitudes: of the thread's halves (a block of 16 channels each where E is 32), of the row
        float mlo = 0.0f, mhi = 0.0f;
#pragma unroll
        for (int i = 0; i < kHalf; ++i) {
            mlo = fmaxf(mlo, fabsf(v[i].x));
            mhi = fmaxf(mhi, fabsf(v[i].y));
        }
        float m = fmaxf(mlo, mhi);
        const float mine = m;
        float total = ss;
        if (kReduce) {
            m = warp_max_nonneg(m);
            if (NORM) total = warp_sum(total);
            if (wpr > 1) {
                if (lane == 0) s_part[buf][warp] = make_float2(m, total);
                __syncthreads();
                const float2 t = lane < wpr ? s_part[buf][r_in_cta * wpr + lane] : make_float2(0.0f, 0.0f);
                m = warp_max_nonneg(t.x);
                if (NORM && t_in_row < 32) total = warp_sum(t.y);
            }
        }
        // 1 / rms of the row, for its first warp, or (wide) the step behind the norm
        float rinv = 1.0f;
        bool wide = false;
        if (NORM && t_in_row < 32) {
            if (row < p.rows && squares_leave_range(total, m, p.eps)) {
                // squares out of binary32's range: the row once more, in binary64 (the stream was written ahead of the barrier;
                // rows of a single warp have it ordered by the warp's own)
                __syncwarp();
                const XT* src = (res ? h + row * p.ldh : x + row * p.ldx) - col0;      // the whole row's first channel
                double s = 0.0;
                for (int c = lane; c < p.K; c += 32) {
                    const double e = sizeof(XT) == 2 ? (double)__uint_as_float(ld_global_u16(src + c) << 16) : (double)ld_global_f32(reinterpret_cast<const float*>(src) + c);
                    s += e * e;
                }
                for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
                rinv = wide_step<FMT>(m, p.clip_ratio, s, p.K, p.eps);
                wide = true;
            } else {
                rinv = inverse_rms(total, p.K, p.eps);
            }
        }

        if (kFp4) {
            uint32_t w[E / 8], word = 0u;
            float d = 1.0f;
            float qlo, qhi;
            if (kMx) {
                // a block of 32 channels: E = 32 a thread's own, E = 16 two lanes'
                float mb = mine;
                if (E == 16) mb = fmaxf(mb, __shfl_xor_sync(0xffffffffu, mb, 1));
                const uint32_t byte = mx_scale(mb, &qlo);
                qhi = qlo;
                constexpr int kThreads = E == 16 ? 2 : 1;      // threads of a block
                if (col_ok && lane % kThreads == 0) word = byte << (8 * ((lane / kThreads) & 3));
            } else {
                float inv;
                d = nv_step(m, &inv);
                if (E == 16) {
                    word = nv_scale(mine, inv, &qlo) << (8 * (lane & 3));
                    qhi = qlo;
                } else {
                    word = nv_scale(mlo, inv, &qlo);
                    word |= nv_scale(mhi, inv, &qhi) << 8;
                    word <<= 16 * (lane & 1);
                }
                if (!col_ok) word = 0u;
            }
#pragma unroll
            for (int o = 1; o < kLanesPerWord; o <<= 1) word |= __shfl_xor_sync(0xffffffffu, word, o);
            if (sc_ok) *reinterpret_cast<uint32_t*>(sc) = row < p.rows ? word : 0u;
            const float2 q2 = make_float2(qlo, qhi);
#pragma unroll
            for (int j = 0; j < kHalf / 8; ++j) {
                float lo[8], hi[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float2 t = f2_mul(v[8 * j + i], q2);
                    lo[i] = t.x;
                    hi[i] = t.y;
                }
                w[j] = pack_e2m1(lo);
                w[kHalf / 8 + j] = pack_e2m1(hi);
            }
            if (row_ok) {
                uint8_t* dst = p.codes + row * (int64_t)(p.K / 2) + col0 / 2;
                if (E == 16) *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
                else *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2 % (E / 8)], w[3 % (E / 8)]);
                if (t_in_row == 0) p.delta[row] = NORM ? (wide ? rinv : __fmul_rn(d, rinv)) : d;
            }
        } else {
            float inv;
            const float d = int_step(m, p.clip_ratio, 1.0f / (FMT == 0 ? 7.0f : 127.0f), &inv);
            // round to nearest even: the low bits of t + 1.5 * 2^23 hold the two's-complement integer
            uint32_t b[E];
#pragma unroll
            for (int i = 0; i < kHalf; ++i) {
                float2 t = f2_mul(v[i], make_float2(inv, inv));
                if (p.clip_ratio < 1.0f) {
                    t.x = fminf(fmaxf(t.x, -p.qmax), p.qmax);
                    t.y = fminf(fmaxf(t.y, -p.qmax), p.qmax);
                }
                // (as a packed FMA by 1: a packed multiply ahead of a packed add may be fused, which rounds ties differently)
                t = f2_fma(t, make_float2(1.0f, 1.0f), make_float2(12582912.0f, 12582912.0f));
                b[i] = __float_as_uint(t.x);
                b[i + kHalf] = __float_as_uint(t.y);
            }
            if (row_ok) {
                constexpr int kPer = FMT == 0 ? 8 : 4, kWords = E / kPer;
                uint32_t w[kWords];
#pragma unroll
                for (int j = 0; j < kWords; ++j) w[j] = pack_word<FMT == 0 ? 0 : 1>(b + j * kPer);
                uint8_t* dst = p.codes + (row * (int64_t)p.K + col0) / (FMT == 0 ? 2 : 1);
                if (kWords == 2) *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
                else {
#pragma unroll
                    for (int j = 0; j < kWords / 4; ++j)
                        reinterpret_cast<uint4*>(dst)[j] = make_uint4(w[4 * j], w[(4 * j + 1) % kWords], w[(4 * j + 2) % kWords], w[(4 * j + 3) % kWords]);
                }
                if (t_in_row == 0) p.delta[row] = NORM ? (wide ? rinv : __fmul_rn(d, rinv)) : d;
            }
        }
    }
}

template <typename XT, int E, int FMT, bool NORM, bool CACHE>
cudaError_t go(RowParams& p, cudaStream_t stream) {
    auto kern = row_quantize_kernel<XT, E, FMT, NORM, CACHE>;
    p.tpr = (p.K / E + 31) / 32 * 32;
    p.rpc = p.tpr >= 128 ? 1 : 128 / p.tpr;
    const int threads = p.tpr * p.rpc;
    int64_t blocks = (p.rows_pad + p.rpc - 1) / p.rpc;
    const int sms = device_sm_count();
    if (blocks > sms) {
        const int64_t most = (int64_t)sms * max_resident_blocks(reinterpret_cast<const void*>(kern), threads);
        if (blocks > most) blocks = most;
    }
    return launch_pdl(kern, (unsigned)blocks, (unsigned)threads, 0, stream, 1u, p);
}
// 16 channels a thread; rows past 8192 channels take up to 1024 threads of 64 registers, which hold no next row, and only the longest
// 32 channels a thread, which spill with a norm or in binary32 (2948 x 11296 binary32 with residual 183 us against 101).
template <typename XT, int FMT, bool NORM>
cudaError_t by_width(RowParams& p, cudaStream_t stream) {
    if (p.K <= 8192) return go<XT, 16, FMT, NORM, true>(p, stream);
    if (p.K <= 16384) return go<XT, 16, FMT, NORM, false>(p, stream);
    return go<XT, 32, FMT, NORM, false>(p, stream);
}
template <typename XT>
cudaError_t by_format(RowParams& p, const RowQuant& q, cudaStream_t stream) {
    switch (q.fmt) {
        case RowFmt::Int4: return q.norm ? by_width<XT, 0, true>(p, stream) : cudaErrorInvalidValue;
        case RowFmt::Int8: return q.norm ? by_width<XT, 1, true>(p, stream) : cudaErrorInvalidValue;
        case RowFmt::Mx: return q.norm ? by_width<XT, 3, true>(p, stream) : by_width<XT, 3, false>(p, stream);
        case RowFmt::Nv: return q.norm ? by_width<XT, 4, true>(p, stream) : by_width<XT, 4, false>(p, stream);
    }
    return cudaErrorInvalidValue;
}

__global__ void clear_pads_kernel(uint8_t* scales, int64_t rows, int blocks, int tiles, int64_t words) {
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= words) return;
    const int64_t t = i / 128, at = i % 128;                 // a word: the four blocks of one row of a tile
    const int64_t row = t / tiles * 128 + (at & 3) * 32 + at / 4;
    const int left = blocks - (int)(t % tiles) * 4;
    uint32_t* w = reinterpret_cast<uint32_t*>(scales) + i;
    if (row >= rows) *w = 0u;
    else if (left < 4) *w &= (1u << (8 * left)) - 1u;
}
__global__ void fill_kernel(float* p, float v, int64_t n) {
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i < n) p[i] = v;
}

}  // namespace

cudaError_t launch_row_quantize(const RowQuant& q, cudaStream_t stream) {
    if (q.rows == 0) return cudaSuccess;
    {   // batches of some length stream through a ring of rows in shared memory
        const cudaError_t e = launch_row_quantize_ring(q, stream);
        if (e != cudaErrorNotSupported) return e;
    }
    const bool fp4 = q.fmt == RowFmt::Mx || q.fmt == RowFmt::Nv;
    RowParams p = {};
    p.x = q.x; p.residual = q.residual; p.h = q.h;
    p.rows = q.rows;
    p.rows_pad = fp4 ? (q.rows + 127) / 128 * 128 : q.rows;
    p.ldx = q.ldx; p.ldr = q.ldr; p.ldh = q.ldh;
    p.K = (int)q.K; p.block = q.block;
    p.eps = q.eps; p.cnorm = q.cnorm; p.clip_ratio = q.clip_ratio; p.qmax = q.fmt == RowFmt::Int4 ? 7.0f : 127.0f;
    p.mult = q.mult; p.codes = q.codes; p.scales = q.scales; p.delta = q.delta;
    p.scale_tiles = fp4 ? (int)fp4_scale_tiles(q.K, q.fmt == RowFmt::Nv ? FQ_NVFP4 : FQ_MXFP4) : 0;
    p.mult_ready = q.mult_ready ? 1 : 0;
    p.early = q.rows <= 64 ? 1 : 0;
    return q.xt == FQ_F32 ? by_format<float>(p, q, stream) : by_format<__nv_bfloat16>(p, q, stream);
}

cudaError_t launch_fp4_clear_pads(uint8_t* scales, int64_t rows, int64_t K, fq_fp4_format f, cudaStream_t stream) {
    const int64_t words = (int64_t)(fp4_scale_bytes(rows, K, f) / 4);
    if (words == 0) return cudaSuccess;
    clear_pads_kernel<<<(unsigned)((words + 255) / 256), 256, 0, stream>>>(scales, rows, (int)(K / fp4_block(f)), (int)fp4_scale_tiles(K, f), words);
    return cudaGetLastError();
}

cudaError_t launch_fill(float* p, float v, int64_t n, cudaStream_t stream) {
    if (n == 0) return cudaSuccess;
    fill_kernel<<<(unsigned)((n + 255) / 256), 256, 0, stream>>>(p, v, n);
    return cudaGetLastError();
}

}  // namespace fq
