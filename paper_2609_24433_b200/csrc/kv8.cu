// Appends keys and values of new tokens to the paged cache of 8-bit codes with one scale for each (page, head).
//
// For one page and head, x the page's new tokens, s the scale of what it holds (nothing is read, s = 0, where the new tokens
// start the page):  a = max|x|,  c = a/127 (0 below the smallest normal number),  s' = max(s, c),
//   new codes  round(x 127 / a) where c >= s, else round(x / s);   held codes  round(code s / s') where s' > s.
// Each is the rounding of the exact quotient, ties to even, so a code does not depend on how the division was done: the
// kernel multiplies by a binary32 reciprocal and divides (in binary64) only where that lands within 2^-13 of a border, which
// is more than its error (|code| <= 127, three roundings of 2^-24 each: below 2^-15).
//
// Bound by memory: D (e + 1) bytes per token, head and operand.  One CTA per (page, operand, head) reads its tokens twice --
// the second time out of L1/L2 -- and turns the values' codes, whose pages keep tokens innermost, in shared memory.
#include "fq_common.cuh"
#include "layer_common.cuh"
#include "ptx_sm100.cuh"

namespace fq {
namespace {

constexpr int kThreads = 256;

struct AppendArgs {
    const void* x[2];                   // keys, values
    int64_t ld[2];
    int8_t* codes[2];
    float* scales[2];
    int64_t pages, tokens;
    int heads, head_dim, page, batch, table_width;
    const int32_t* table;
    int64_t ld_table;
    const int32_t* kv_len;
    const int32_t* offsets;
};

template <typename T>
__device__ __forceinline__ void load8(const T* p, float* f);
template <>
__device__ __forceinline__ void load8<float>(const float* p, float* f) {
    const float4 a = ld_global_f4(p), b = ld_global_f4(p + 4);
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
template <>
__device__ __forceinline__ void load8<__nv_bfloat16>(const __nv_bfloat16* p, float* f) {
    const uint4 v = ld_global_v4(p);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

// round(x num / den) of the exact quotient, to [-127, 127]; inv = num / den in binary32.
__device__ __forceinline__ int code_of(float x, float inv, double num, double den) {
    const float r = x * inv;
    float c = rintf(r);
    if (fabsf(r - c) > 0.5f - 0x1p-13f) c = (float)rint((double)x * num / den);
    return (int)fminf(fmaxf(c, -127.0f), 127.0f);
}
__device__ __forceinline__ uint32_t pack4(int a, int b, int c, int d) {
    return (uint32_t)(a & 255) | (uint32_t)(b & 255) << 8 | (uint32_t)(c & 255) << 16 | (uint32_t)(d & 255) << 24;
}
__device__ __forceinline__ uint32_t requantize4(uint32_t w, float ratio, double was, double now) {
    int c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = code_of((float)(int8_t)(w >> (8 * i)), ratio, was, now);
    return pack4(c[0], c[1], c[2], c[3]);
}

template <typename T>
__global__ void __launch_bounds__(kThreads) kv8_append_kernel(const AppendArgs a) {
    extern __shared__ uint32_t turned[];                // values: [head_dim][page / 4 + 1] words of four tokens
    __shared__ float warp_max[kThreads / 32];
    griddep_wait();
    const int b = blockIdx.z, which = blockIdx.y & 1, head = blockIdx.y >> 1;
    int64_t row0, n;
    sequence_rows(a.offsets, b, a.batch, a.tokens, &row0, &n);
    const int64_t held = max((int64_t)a.kv_len[b], (int64_t)0);
    const int64_t end = min(held + n, (int64_t)a.table_width * a.page);
    const int D = a.head_dim, P = a.page;
    for (int64_t i = held / P + blockIdx.x; i * P < end; i += gridDim.x) {
        const int first = (int)max(held - i * P, (int64_t)0), last = (int)min(end - i * P, (int64_t)P), m = last - first;
        const int64_t id = a.table[b * a.ld_table + i];
        if (m <= 0 || id < 0 || id >= a.pages) continue;
        const T* x = static_cast<const T*>(a.x[which]) + (row0 + i * P + first - held) * a.ld[which] + (int64_t)head * D;
        float* scale = a.scales[which] + id * a.heads + head;
        const float was = first > 0 ? ld_global_f32(scale) : 0.0f;
        // ---- the largest magnitude
        const int per_row = D / 8;
        float most = 0.0f;
        for (int e = threadIdx.x; e < m * per_row; e += kThreads) {
            const int t = e / per_row, c = (e - t * per_row) * 8;
            float f[8];
            load8(x + t * a.ld[which] + c, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(f[j]));
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
        __syncthreads();                                // (the last page's readers of warp_max, turned and the old scale)
        if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = most;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) most = fmaxf(most, warp_max[w]);
        float cand = __fdiv_rn(most, 127.0f);
        if (cand < 1.17549435e-38f) cand = 0.0f;
        const float now = fmaxf(was, cand);
        const bool sets = cand >= was, grown = first > 0 && now > was;
        const double num = sets ? 127.0 : 1.0, den = sets ? (double)most : (double)was;
        const float inv = now > 0.0f ? (sets ? __fdiv_rn(127.0f, most) : __fdiv_rn(1.0f, was)) : 0.0f;
        const float ratio = grown ? __fdiv_rn(was, now) : 1.0f;
        int8_t* page = a.codes[which] + (id * a.heads + head) * (int64_t)P * D;
        // ---- the codes
        const int words = P / 4 + 1;
        for (int e = threadIdx.x; e < m * per_row; e += kThreads) {
            const int t = e / per_row, c = (e - t * per_row) * 8;
            float f[8];
            load8(x + t * a.ld[which] + c, f);
            int q[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) q[j] = now > 0.0f ? code_of(f[j], inv, num, den) : 0;
            if (which == 0) {
                *reinterpret_cast<uint2*>(page + (int64_t)(first + t) * D + c) = make_uint2(pack4(q[0], q[1], q[2], q[3]), pack4(q[4], q[5], q[6], q[7]));
            } else {
                int8_t* to = reinterpret_cast<int8_t*>(turned);
#pragma unroll
                for (int j = 0; j < 8; ++j) to[(c + j) * words * 4 + first + t] = (int8_t)q[j];
            }
        }
        if (which == 0) {
            if (grown) {
                uint32_t* w = reinterpret_cast<uint32_t*>(page);
                for (int e = threadIdx.x; e < first * D / 4; e += kThreads) w[e] = requantize4(w[e], ratio, was, now);
            }
        } else {
            __syncthreads();
            const int w0 = grown ? 0 : first / 4, count = (last + 3) / 4 - w0;
            uint32_t* w = reinterpret_cast<uint32_t*>(page);
            for (int e = threadIdx.x; e < count * D; e += kThreads) {
                const int d = e / count, k = w0 + e - d * count, t = k * 4;
                uint32_t keep = 0;                      // bytes of tokens that are not new
#pragma unroll
                for (int j = 0; j < 4; ++j) keep |= t + j < first || t + j >= last ? 0xffu << (8 * j) : 0u;
                uint32_t v = turned[d * words + k];
                if (keep) {
                    const uint32_t old = w[d * (P / 4) + k];
                    uint32_t held_bytes = 0;
#pragma unroll
                    for (int j = 0; j < 4; ++j) held_bytes |= t + j < first ? 0xffu << (8 * j) : 0u;
                    const uint32_t kept = grown ? (requantize4(old, ratio, was, now) & held_bytes) | (old & ~held_bytes) : old;
                    v = (v & ~keep) | (kept & keep);
                }
                w[d * (P / 4) + k] = v;
            }
        }
        if (threadIdx.x == 0) *scale = now;
    }
}

}  // namespace

cudaError_t launch_kv8_append(const Kv8Append& r, cudaStream_t stream) {
    AppendArgs a = {};
    a.x[0] = r.k; a.x[1] = r.v; a.ld[0] = r.ldk; a.ld[1] = r.ldv;
    a.codes[0] = r.cache.k; a.codes[1] = r.cache.v; a.scales[0] = r.cache.k_scale; a.scales[1] = r.cache.v_scale;
    a.pages = r.cache.pages; a.tokens = r.tokens; a.heads = r.cache.heads; a.head_dim = r.cache.head_dim; a.page = r.cache.page;
    a.batch = r.batch; a.table_width = r.table_width; a.table = r.table; a.ld_table = r.ld_table;
    a.kv_len = r.kv_len; a.offsets = r.offsets;
    const int64_t most = r.max_new < r.tokens ? r.max_new : r.tokens;
    int64_t pages = (most + r.cache.page - 2) / r.cache.page + 1;      // that a run of `most` tokens touches, wherever it starts
    if (pages > r.table_width) pages = r.table_width;
    const dim3 grid((unsigned)(pages > 0 ? pages : 1), (unsigned)(2 * r.cache.heads), (unsigned)r.batch);
    const size_t smem = (size_t)r.cache.head_dim * (r.cache.page / 4 + 1) * 4;
    return r.xt == FQ_BF16 ? launch_pdl3(kv8_append_kernel<__nv_bfloat16>, grid, kThreads, smem, stream, a)
                           : launch_pdl3(kv8_append_kernel<float>, grid, kThreads, smem, stream, a);
}

}  // namespace fq
