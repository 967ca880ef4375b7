// Attention in binary32 on the CUDA cores: every product, statistic and sum in 32 bits.  Takes binary32 queries, which the
// tensor cores would round, on either kind of keys.
//
// Softmax in one pass over the keys: for each row the running maximum m of the scores (times log2 e), the sum l of
// 2^(s - m) and o = sum 2^(s - m) v, the last two rescaled by 2^(m_old - m_new) when m rises.  A CTA takes `ROWS` rows --
// (token, head of a group) pairs of one kv head, so that its keys are read once for the whole group -- and `chunk` keys.
// A thread has 4 x 4 scores and 4 rows x 4 .. 16 channels of o, and takes four steps of either contraction to a 16-byte read of shared
// memory.  Bound by issue slots and those reads: 16 x 256 queries x 1024 keys, 16 heads of 64, 665 us = 26 TFLOP/s, from the cache 575
// (with values read one by one, and a key's place looked up for each of them, 1055 and 1032).
#include "attention_common.cuh"

#include <float.h>

namespace fq {
namespace {

constexpr int kThreads = 256;
constexpr int kKeys = 64;

template <bool CACHED, int ROWS, int DP>
__global__ void __launch_bounds__(kThreads) attention_simt_kernel(const Attention a) {
    constexpr int RT = ROWS / 16;                       // rows per thread
    constexpr int KP = DP + 4;                          // pitch of queries and keys (16-byte reads down a column meet no conflict)
    constexpr int DT = DP / 16;                         // channels per thread
    extern __shared__ __align__(16) float smem[];
    float* qs = smem;                                   // [ROWS][KP]
    float* ks = qs + ROWS * KP;                         // [kKeys][KP]
    float* vs = ks + kKeys * KP;                        // [kKeys][DP]
    float* ps = vs + kKeys * DP;                        // [ROWS][PP]
    constexpr int PP = kKeys + 4;
    __shared__ int64_t places[kKeys];                   // row of a key, or (page, head); -1 where it is masked
    griddep_wait();
    const int b = blockIdx.z / a.kv_heads, hk = blockIdx.z % a.kv_heads, c = blockIdx.y;
    const Sequence s = sequence_of(a, b);
    const int D = a.head_dim, G = a.group;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    for (int64_t tile = blockIdx.x; tile * ROWS < s.queries * G; tile += gridDim.x) {
        const TileKeys tk = tile_keys(a, s, tile, ROWS);
        const int64_t k0 = (int64_t)c * a.chunk, k1 = min(tk.end, k0 + a.chunk);
        if (c > 0 && k0 >= tk.end) continue;
        __syncthreads();
        for (int e = threadIdx.x; e < ROWS * (DP / 4); e += kThreads) {
            const int r = e / (DP / 4), d = (e % (DP / 4)) * 4;
            const int64_t row = tile * ROWS + r;
            float4 f = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (row < s.queries * G && d < D)
                f = load4(static_cast<const float*>(a.q) + (s.q0 + row / G) * a.ldq + (int64_t)(hk * G + row % G) * D + d);
            *reinterpret_cast<float4*>(qs + r * KP + d) = f;
        }
        float m[RT], l[RT], o[RT][DT];
        int64_t limit[RT];
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            m[i] = -INFINITY;
            l[i] = 0.0f;
            limit[i] = row_limit(a, s, tile * ROWS + ty * RT + i);
#pragma unroll
            for (int j = 0; j < DT; ++j) o[i][j] = 0.0f;
        }
        for (int64_t j0 = k0; j0 < k1; j0 += kKeys) {
            __syncthreads();
            if (threadIdx.x < kKeys) {
                const KeyPlace p = key_place<CACHED>(a, s, b, hk, j0 + threadIdx.x, k1);
                places[threadIdx.x] = p.valid ? p.row : -1;
            }
            __syncthreads();
            if (!CACHED) {
                for (int e = threadIdx.x; e < kKeys * (DP / 4); e += kThreads) {
                    const int t = e / (DP / 4), d = (e % (DP / 4)) * 4;
                    const int64_t row = places[t];
                    float4 kf = make_float4(0.0f, 0.0f, 0.0f, 0.0f), vf = kf;
                    if (row >= 0 && d < D) {
                        kf = load4(static_cast<const float*>(a.k) + row * a.ldk + (int64_t)hk * D + d);
                        vf = load4(static_cast<const float*>(a.v) + row * a.ldv + (int64_t)hk * D + d);
                    }
                    *reinterpret_cast<float4*>(ks + t * KP + d) = kf;
                    *reinterpret_cast<float4*>(vs + t * DP + d) = vf;
                }
            } else {                                    // 16 channels of a key, 16 keys of a channel
                const int P = a.cache.page;
                for (int e = threadIdx.x; e < kKeys * (DP / 16); e += kThreads) {
                    const int t = e / (DP / 16), d = (e % (DP / 16)) * 16;
                    const int64_t at = places[t];
                    const bool ok = at >= 0 && d < D;
                    const uint4 w = ld_global_v4(a.cache.k + (ok ? (at * P + ((j0 + t) & (P - 1))) * D + d : 0), ok);
                    const float f = ok ? ld_global_f32(a.cache.k_scale + at) : 0.0f;
                    const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        *reinterpret_cast<float4*>(ks + t * KP + d + 4 * x) = make_float4((float)(int8_t)words[x] * f, (float)(int8_t)(words[x] >> 8) * f,
                                                                                          (float)(int8_t)(words[x] >> 16) * f, (float)(int8_t)(words[x] >> 24) * f);
                }
                for (int e = threadIdx.x; e < kKeys / 16 * DP; e += kThreads) {
                    const int t = e / DP * 16, d = e % DP;
                    const int64_t at = places[t];       // (keys of a run are of one page; where it ends inside, the first one is there)
                    const bool ok = at >= 0 && d < D;
                    const uint4 w = ld_global_v4(a.cache.v + (ok ? (at * D + d) * P + ((j0 + t) & (P - 1)) : 0), ok);
                    const float f = ok ? ld_global_f32(a.cache.v_scale + at) : 0.0f;
                    const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                    for (int x = 0; x < 16; ++x) vs[(t + x) * DP + d] = (float)(int8_t)(words[x / 4] >> (8 * (x % 4))) * f;
                }
            }
            __syncthreads();
            float acc[RT][4];
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = 0.0f;
            for (int d = 0; d < DP; d += 4) {
                float4 kf[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) kf[j] = *reinterpret_cast<const float4*>(ks + (tx + 16 * j) * KP + d);
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    const float4 qf = *reinterpret_cast<const float4*>(qs + (ty * RT + i) * KP + d);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        acc[i][j] = fmaf(qf.x, kf[j].x, acc[i][j]);
                        acc[i][j] = fmaf(qf.y, kf[j].y, acc[i][j]);
                        acc[i][j] = fmaf(qf.z, kf[j].z, acc[i][j]);
                        acc[i][j] = fmaf(qf.w, kf[j].w, acc[i][j]);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                float top = -INFINITY;                  // (stays so to a row that sees nothing, and to no other)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int t = tx + 16 * j;
                    const bool seen = places[t] >= 0 && j0 + t <= limit[i];
                    acc[i][j] = seen ? acc[i][j] * a.scale_log2 : -INFINITY;
                    if (seen) top = fmaxf(fmaxf(top, -FLT_MAX), acc[i][j]);
                }
#pragma unroll
                for (int x = 8; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
                const float now = fmaxf(m[i], top);
                const float base = now == -INFINITY ? 0.0f : now;      // nothing seen yet: every term below is 2^-inf = 0
                const float keep = exp2f(m[i] - base);
                m[i] = now;
                float sum = 0.0f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float p = exp2f(acc[i][j] - base);
                    sum += p;
                    ps[(ty * RT + i) * PP + tx + 16 * j] = p;
                }
#pragma unroll
                for (int x = 8; x > 0; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
                l[i] = fmaf(l[i], keep, sum);
#pragma unroll
                for (int j = 0; j < DT; ++j) o[i][j] *= keep;
            }
            __syncwarp();                               // a row's probabilities are written and read by one half of a warp
            for (int t = 0; t < kKeys; t += 4) {
                float4 p[RT];
#pragma unroll
                for (int i = 0; i < RT; ++i) p[i] = *reinterpret_cast<const float4*>(ps + (ty * RT + i) * PP + t);
#pragma unroll
                for (int x = 0; x < 4; ++x) {
#pragma unroll
                    for (int j = 0; j < DT; j += 4) {
                        const float4 vf = *reinterpret_cast<const float4*>(vs + (t + x) * DP + 16 * j + 4 * tx);
#pragma unroll
                        for (int i = 0; i < RT; ++i) {
                            const float w = x == 0 ? p[i].x : x == 1 ? p[i].y : x == 2 ? p[i].z : p[i].w;
                            o[i][j] = fmaf(w, vf.x, o[i][j]);
                            o[i][j + 1] = fmaf(w, vf.y, o[i][j + 1]);
                            o[i][j + 2] = fmaf(w, vf.z, o[i][j + 2]);
                            o[i][j + 3] = fmaf(w, vf.w, o[i][j + 3]);
                        }
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const int64_t row = tile * ROWS + ty * RT + i;
            if (row >= s.queries * G) continue;
            const int64_t token = s.q0 + row / G, head = hk * G + row % G;
            if (tk.chunks <= 1) {
                const float inv = reciprocal_sum(m[i], l[i]);
                float* y = static_cast<float*>(a.y) + token * a.ldy + head * D;
#pragma unroll
                for (int j = 0; j < DT; j += 4)
                    if (16 * j + 4 * tx < D) store4(y + 16 * j + 4 * tx, o[i][j] * inv, o[i][j + 1] * inv, o[i][j + 2] * inv, o[i][j + 3] * inv);
            } else {
                const int64_t at = (token * a.q_heads + head) * a.chunks + c;
#pragma unroll
                for (int j = 0; j < DT; j += 4)
                    if (16 * j + 4 * tx < D) *reinterpret_cast<float4*>(a.part + at * D + 16 * j + 4 * tx) = make_float4(o[i][j], o[i][j + 1], o[i][j + 2], o[i][j + 3]);
                if (tx == 0) {
                    a.part_ml[2 * at] = m[i];
                    a.part_ml[2 * at + 1] = l[i];
                }
            }
        }
    }
}

// Joins the chunks of the rows that have more than one, WARPS warps to a row.
template <typename T, int WARPS>
__global__ void __launch_bounds__(128) attention_join_kernel(const Attention a) {
    griddep_wait();
    const int b = blockIdx.y;
    const Sequence s = sequence_of(a, b);
    const int64_t rows = s.queries * a.q_heads;
    constexpr int kRows = 4 / WARPS;
    for (int64_t r0 = (int64_t)blockIdx.x * kRows; r0 < rows; r0 += (int64_t)gridDim.x * kRows) {
        const int64_t r = r0 + threadIdx.x / 32 / WARPS;         // (WARPS == 4: the same for the whole CTA)
        if (r >= rows) continue;
        const int64_t token = r / a.q_heads, head = r % a.q_heads;
        const int64_t tile = (token * a.group + head % a.group) / a.tile_rows;
        const int n = tile_keys(a, s, tile, a.tile_rows).chunks;
        if (n <= 1) continue;
        const int64_t at = ((s.q0 + token) * a.q_heads + head) * a.chunks;
        join_row<T, WARPS>(a, n, [&](int c) { return at + c; }, static_cast<T*>(a.y) + (s.q0 + token) * a.ldy + head * a.head_dim);
    }
}

template <bool CACHED, int ROWS, int DP>
cudaError_t launch(const Attention& a, dim3 grid, cudaStream_t stream) {
    const size_t smem = sizeof(float) * ((size_t)(ROWS + kKeys) * (DP + 4) + (size_t)kKeys * DP + (size_t)ROWS * (kKeys + 4));
    auto* kern = attention_simt_kernel<CACHED, ROWS, DP>;
    const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kern), smem);
    return e != cudaSuccess ? e : launch_pdl3(kern, grid, kThreads, smem, stream, a);
}
template <bool CACHED, int ROWS>
cudaError_t by_width(const Attention& a, dim3 grid, cudaStream_t stream) {
    if (a.head_dim <= 64) return launch<CACHED, ROWS, 64>(a, grid, stream);
    if (a.head_dim <= 128) return launch<CACHED, ROWS, 128>(a, grid, stream);
    return launch<CACHED, ROWS, 256>(a, grid, stream);
}

}  // namespace

cudaError_t launch_attention_simt(const Attention& a, cudaStream_t stream) {
    const dim3 grid((unsigned)row_tiles(a), (unsigned)a.chunks, (unsigned)(a.batch * a.kv_heads));
    if (a.cached) return by_width<true, 64>(a, grid, stream);           // (16 rows and fewer take the kernel of few queries)
    return a.tile_rows == 16 ? by_width<false, 16>(a, grid, stream) : by_width<false, 64>(a, grid, stream);
}

template <typename T>
static cudaError_t join_by_chunks(const Attention& a, cudaStream_t stream) {
    const int warps = a.chunks > 4 ? 4 : 1;
    int64_t ctas = (a.max_q * a.q_heads * warps + 3) / 4;
    if (ctas > 65535) ctas = 65535;
    const dim3 grid((unsigned)(ctas > 0 ? ctas : 1), (unsigned)a.batch);
    return warps == 4 ? launch_pdl3(attention_join_kernel<T, 4>, grid, 128, 0, stream, a) : launch_pdl3(attention_join_kernel<T, 1>, grid, 128, 0, stream, a);
}
cudaError_t launch_attention_join(const Attention& a, cudaStream_t stream) {
    return a.dt == FQ_BF16 ? join_by_chunks<__nv_bfloat16>(a, stream) : join_by_chunks<float>(a, stream);
}

}  // namespace fq
