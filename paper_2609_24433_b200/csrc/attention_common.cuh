// What the attention kernels share: where a sequence's queries and keys are, how far a tile's rows see.
#pragma once

#include "fq_common.cuh"
#include "layer_common.cuh"
#include "ptx_sm100.cuh"

namespace fq {

constexpr int kTokensBlock = 256;       // keys of a block of work of the few-queries kernel

inline int64_t row_tiles(const Attention& a) {
    const int64_t n = (a.max_q * a.group + a.tile_rows - 1) / a.tile_rows;
    return n < 1 ? 1 : n > 0x7fffffff ? 0x7fffffff : n;
}
cudaError_t launch_attention_widen(const Attention& a, cudaStream_t stream);
cudaError_t launch_attention_tiles(const Attention& a, cudaStream_t stream);
cudaError_t launch_attention_tokens(const Attention& a, cudaStream_t stream);
cudaError_t launch_attention_simt(const Attention& a, cudaStream_t stream);
int tokens_ctas(const Attention& a);             // of the few-queries kernel, resident at once
cudaError_t launch_attention_join(const Attention& a, cudaStream_t stream);

#ifdef __CUDACC__
namespace {

struct Sequence {
    int64_t q0, queries;                // rows of its queries
    int64_t k0, keys;                   // rows of its keys (cached: k0 unused)
};
__device__ __forceinline__ Sequence sequence_of(const Attention& a, int b) {
    Sequence s;
    sequence_rows(a.q_offsets, b, a.batch, a.q_rows, &s.q0, &s.queries);
    s.k0 = 0;
    s.keys = a.max_kv;
    if (!a.cached) {
        int64_t n;
        sequence_rows(a.kv_offsets, b, a.batch, a.kv_rows, &s.k0, &n);
        s.keys = min(s.keys, n);
    }
    if (a.kv_len) s.keys = min(s.keys, max((int64_t)ld_global_s32(a.kv_len + b), (int64_t)0));
    return s;
}
// The last key that a row -- (token, head of the group) -- sees, -1 for none.
__device__ __forceinline__ int64_t row_limit(const Attention& a, const Sequence& s, int64_t row) {
    return a.causal ? s.keys - s.queries + row / a.group : s.keys - 1;
}
// Keys that the rows of a tile see, and the chunks that they lie in (at least one, which then writes the zeros).
struct TileKeys {
    int64_t end;
    int chunks;
};
__device__ __forceinline__ TileKeys tile_keys(const Attention& a, const Sequence& s, int64_t tile, int tile_rows) {
    TileKeys t;
    const int64_t last = min((tile + 1) * tile_rows, s.queries * a.group) - 1;
    t.end = max(min(s.keys, row_limit(a, s, last) + 1), (int64_t)0);
    t.chunks = max((int)((t.end + a.chunk - 1) / a.chunk), 1);
    return t;
}

struct KeyPlace {
    bool valid;
    int64_t row;                        // of the keys, or page * kv_heads + head
};
// Key j of sequence b (j < end where it may be read at all).
template <bool CACHED>
__device__ __forceinline__ KeyPlace key_place(const Attention& a, const Sequence& s, int b, int hk, int64_t j, int64_t end) {
    KeyPlace p;
    p.valid = j < end;
    p.row = 0;
    if (!p.valid) return p;
    if (CACHED) {
        const int64_t id = ld_global_s32(a.table + b * a.ld_table + j / a.cache.page);
        p.valid = id >= 0 && id < a.cache.pages;
        p.row = id * a.kv_heads + hk;
    } else {
        p.row = s.k0 + j;
        p.valid = !a.key_mask || a.key_mask[p.row] != 0;
    }
    return p;
}

__device__ __forceinline__ float4 load4(const float* p) { return ld_global_f4(p); }
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p) {
    uint32_t x, y;
    asm volatile("ld.global.v2.b32 {%0, %1}, [%2];" : "=r"(x), "=r"(y) : "l"(p));
    return make_float4(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u), __uint_as_float(y << 16), __uint_as_float(y & 0xffff0000u));
}

__device__ __forceinline__ void store4(float* p, float x, float y, float z, float w) { *reinterpret_cast<float4*>(p) = make_float4(x, y, z, w); }
__device__ __forceinline__ void store4(__nv_bfloat16* p, float x, float y, float z, float w) { *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(x, y), pack_bf16(z, w)); }

// 1 / l of a row with the maximum m and the sum l: 0 for a row that sees no key (m = -inf, which no seen score leaves: a maximum is
// -FLT_MAX at least).  NaN where the scores that it sees are all -inf or there is a +inf, so that no term is left, as in the formula.
__device__ __forceinline__ float reciprocal_sum(float m, float l) { return l == 0.0f ? (m == -INFINITY ? 0.0f : __int_as_float(0x7fffffff)) : 1.0f / l; }

// Joins n partial results of a row, at(c) their places: o = sum_c 2^(m_c - m) o_c / sum_c 2^(m_c - m) l_c.  (The maximum passes over
// a NaN among the m_c, whose weight carries it on.)  WARPS warps (1, or
// all 4 of the CTA) take them in turn, four at a time under way each: a lone sequence has few rows and many chunks (16384 keys,
// 32 heads of 128 in 64 chunks: the whole call 51 us with one warp a row and one chunk at a time, 17 so).  Fixed order of sums.
template <typename T, int WARPS, typename At>
__device__ __forceinline__ void join_row(const Attention& a, int n, At at, T* y) {
    __shared__ float4 seats[4][64];
    __shared__ float sums[4];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, part = warp % WARPS;
    float m = -INFINITY;
    for (int c = lane; c < n; c += 32) m = fmaxf(m, ld_global_f32(a.part_ml + 2 * at(c)));
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
    const float base = m == -INFINITY ? 0.0f : m;
    const bool low = 4 * lane < a.head_dim, high = 128 + 4 * lane < a.head_dim;
    float l = 0.0f;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f), p = o;       // channels 4 lane .., 128 + 4 lane ..
    for (int c0 = part; c0 < n; c0 += 32 * WARPS) {              // (a lane looks up the weight of one of 32 chunks)
        const int own = c0 + WARPS * lane;
        const float mine = own < n ? exp2f(ld_global_f32(a.part_ml + 2 * at(own)) - base) : 0.0f;
        if (own < n) l = fmaf(mine, ld_global_f32(a.part_ml + 2 * at(own) + 1), l);
        for (int i = 0; i < 32 && c0 + WARPS * i < n; i += 4) {
            float4 x[4], z[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int c = c0 + WARPS * (i + k);
                const float* from = a.part + at(c) * a.head_dim + 4 * lane;
                x[k] = c < n && low ? ld_global_f4(from) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                z[k] = c < n && high ? ld_global_f4(from + 128) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float w = __shfl_sync(0xffffffffu, mine, i + k);
                o.x = fmaf(w, x[k].x, o.x); o.y = fmaf(w, x[k].y, o.y); o.z = fmaf(w, x[k].z, o.z); o.w = fmaf(w, x[k].w, o.w);
                p.x = fmaf(w, z[k].x, p.x); p.y = fmaf(w, z[k].y, p.y); p.z = fmaf(w, z[k].z, p.z); p.w = fmaf(w, z[k].w, p.w);
            }
        }
    }
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
    if (WARPS > 1) {
        __syncthreads();                                         // (the last row's seats are read)
        seats[warp][lane] = o;
        seats[warp][32 + lane] = p;
        if (lane == 0) sums[warp] = l;
        __syncthreads();
        if (part > 1) return;                                    // warp 0 has the low channels, warp 1 the high ones
        l = 0.0f;
        o = p = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            const float4 x = seats[w][32 * part + lane];
            l += sums[w];
            o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
        }
        if (part == 1) p = o;
    }
    const float inv = reciprocal_sum(m, l);
    if (low && part == 0) store4(y + 4 * lane, o.x * inv, o.y * inv, o.z * inv, o.w * inv);
    if (high && part == (WARPS > 1 ? 1 : 0)) store4(y + 128 + 4 * lane, p.x * inv, p.y * inv, p.z * inv, p.w * inv);
}

}  // namespace
#endif

}  // namespace fq
