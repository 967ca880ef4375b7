// Attention in binary32 on the CUDA cores: every product, statistic and sum in 32 bits.  Takes binary32 queries, which the
// tensor cores would round, on either kind of keys; and is the plain kernel that the others are measured against.
//
// Softmax in one pass over the keys: for each row the running maximum m of the scores (times log2 e), the sum l of
// 2^(s - m) and o = sum 2^(s - m) v, the last two rescaled by 2^(m_old - m_new) when m rises.  A CTA takes `ROWS` rows --
// (token, head of a group) pairs of one kv head, so that its keys are read once for the whole group -- and `chunk` keys.
#include "attention_common.cuh"

namespace fq {
namespace {

constexpr int kThreads = 256;
constexpr int kKeys = 64;

template <typename T, bool CACHED, int ROWS, int DP>
__global__ void __launch_bounds__(kThreads) attention_simt_kernel(const Attention a) {
    constexpr int RT = ROWS / 16;                       // rows per thread
    constexpr int KP = DP + 4;                          // pitch of queries and keys (16-byte reads down a column meet no conflict)
    constexpr int DT = DP / 16;                         // channels per thread
    extern __shared__ float smem[];
    float* qs = smem;                                   // [ROWS][KP]
    float* ks = qs + ROWS * KP;                         // [kKeys][KP]
    float* vs = ks + kKeys * KP;                        // [kKeys][DP]
    float* ps = vs + kKeys * DP;                        // [ROWS][kKeys + 1]
    __shared__ int valid[kKeys];
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
                f = load4(static_cast<const T*>(a.q) + (s.q0 + row / G) * a.ldq + (int64_t)(hk * G + row % G) * D + d);
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
            for (int e = threadIdx.x; e < kKeys * (DP / 4); e += kThreads) {
                const int t = e / (DP / 4), d = (e % (DP / 4)) * 4;
                const KeyPlace p = key_place<CACHED>(a, s, b, hk, j0 + t, k1);
                float4 kf = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (p.valid && d < D) kf = load_key4<T, CACHED>(a, p, hk, d);
                *reinterpret_cast<float4*>(ks + t * KP + d) = kf;
                if (d == 0) valid[t] = p.valid;
            }
            // (cached values keep tokens innermost: neighbouring threads then take neighbouring tokens)
            for (int e = threadIdx.x; e < kKeys * DP; e += kThreads) {
                const int t = CACHED ? e % kKeys : e / DP, d = CACHED ? e / kKeys : e % DP;
                const KeyPlace p = key_place<CACHED>(a, s, b, hk, j0 + t, k1);
                vs[t * DP + d] = p.valid && d < D ? load_value<T, CACHED>(a, p, hk, d) : 0.0f;
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
                float top = -INFINITY;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int t = tx + 16 * j;
                    const bool seen = valid[t] && j0 + t <= limit[i];
                    acc[i][j] = seen ? acc[i][j] * a.scale_log2 : -INFINITY;
                    top = fmaxf(top, acc[i][j]);
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
                    ps[(ty * RT + i) * (kKeys + 1) + tx + 16 * j] = p;
                }
#pragma unroll
                for (int x = 8; x > 0; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
                l[i] = fmaf(l[i], keep, sum);
#pragma unroll
                for (int j = 0; j < DT; ++j) o[i][j] *= keep;
            }
            __syncwarp();                               // a row's probabilities are written and read by one half of a warp
            for (int t = 0; t < kKeys; ++t) {
                float vf[DT];
#pragma unroll
                for (int j = 0; j < DT; ++j) vf[j] = vs[t * DP + tx + 16 * j];
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    const float p = ps[(ty * RT + i) * (kKeys + 1) + t];
#pragma unroll
                    for (int j = 0; j < DT; ++j) o[i][j] = fmaf(p, vf[j], o[i][j]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const int64_t row = tile * ROWS + ty * RT + i;
            if (row >= s.queries * G) continue;
            const int64_t token = s.q0 + row / G, head = hk * G + row % G;
            if (tk.chunks <= 1) {
                const float inv = l[i] > 0.0f ? 1.0f / l[i] : 0.0f;
                T* y = static_cast<T*>(a.y) + token * a.ldy + head * D;
#pragma unroll
                for (int j = 0; j < DT; ++j)
                    if (tx + 16 * j < D) store1(y + tx + 16 * j, o[i][j] * inv);
            } else {
                const int64_t at = (token * a.q_heads + head) * a.chunks + c;
#pragma unroll
                for (int j = 0; j < DT; ++j)
                    if (tx + 16 * j < D) a.part[at * D + tx + 16 * j] = o[i][j];
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

template <typename T, bool CACHED, int ROWS, int DP>
cudaError_t launch(const Attention& a, dim3 grid, cudaStream_t stream) {
    const size_t smem = sizeof(float) * ((size_t)(ROWS + kKeys) * (DP + 4) + (size_t)kKeys * DP + (size_t)ROWS * (kKeys + 1));
    auto* kern = attention_simt_kernel<T, CACHED, ROWS, DP>;
    const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kern), smem);
    return e != cudaSuccess ? e : launch_pdl3(kern, grid, kThreads, smem, stream, a);
}
template <typename T, bool CACHED, int ROWS>
cudaError_t by_width(const Attention& a, dim3 grid, cudaStream_t stream) {
    if (a.head_dim <= 64) return launch<T, CACHED, ROWS, 64>(a, grid, stream);
    if (a.head_dim <= 128) return launch<T, CACHED, ROWS, 128>(a, grid, stream);
    return launch<T, CACHED, ROWS, 256>(a, grid, stream);
}
template <typename T>
cudaError_t by_rows(const Attention& a, dim3 grid, cudaStream_t stream) {
    if (a.cached) return a.tile_rows == 16 ? by_width<T, true, 16>(a, grid, stream) : by_width<T, true, 64>(a, grid, stream);
    return a.tile_rows == 16 ? by_width<T, false, 16>(a, grid, stream) : by_width<T, false, 64>(a, grid, stream);
}

}  // namespace

cudaError_t launch_attention_simt(const Attention& a, cudaStream_t stream) {
    const dim3 grid((unsigned)row_tiles(a), (unsigned)a.chunks, (unsigned)(a.batch * a.kv_heads));
    return a.dt == FQ_BF16 ? by_rows<__nv_bfloat16>(a, grid, stream) : by_rows<float>(a, grid, stream);
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
