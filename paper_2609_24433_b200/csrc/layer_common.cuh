// Internal declarations of the operators between a layer's projections: head norms with rotary positions, the 8-bit
// paged cache, attention.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "fq.h"

namespace fq {

// launch_pdl with a three-dimensional grid and no cluster.
template <typename... Params, typename... Args>
inline cudaError_t launch_pdl3(void (*kern)(Params...), dim3 grid, unsigned block, size_t smem, cudaStream_t stream, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(block, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kern, args...);
}

struct QkNormRope {
    const void* x;
    fq_dtype xt, yt;
    int64_t M, ldx;
    int q_heads, k_heads, head_dim, rotary;
    bool interleaved;
    const float* q_gain;
    const float* k_gain;
    float eps, amplitude;
    const int32_t* positions;
    const double* frequencies;
    void* q;
    void* k;
    int64_t ldq, ldk;
};
cudaError_t launch_qk_norm_rope(const QkNormRope& r, cudaStream_t stream);

struct Kv8Append {
    const void* k;
    const void* v;
    fq_dtype xt;
    int64_t tokens, ldk, ldv;
    fq_kv8_cache cache;
    const int32_t* table;
    int64_t ld_table;
    int table_width, batch;
    const int32_t* kv_len;
    const int32_t* offsets;
    int64_t max_new;
};
cudaError_t launch_kv8_append(const Kv8Append& a, cudaStream_t stream);

// What the attention kernels read, write and share.  Queries and outputs are rows of heads * head_dim; keys and values
// rows of kv_heads * head_dim, or pages of the 8-bit cache.
struct Attention {
    const void* q;
    void* y;
    fq_dtype dt;
    int64_t q_rows, ldq, ldy;
    int q_heads, kv_heads, group, head_dim, batch;
    const int32_t* q_offsets;       // [batch + 1] or null: q_rows / batch each
    const int32_t* kv_len;          // [batch] or null
    float scale_log2;               // scale * log2(e)
    int causal;
    int64_t max_q, max_kv;          // what the grid is sized by; lengths are cut at max_kv
    // keys and values as rows
    const void* k;
    const void* v;
    int64_t kv_rows, ldk, ldv;
    const int32_t* kv_offsets;      // [batch + 1] or null: kv_rows / batch each
    const uint8_t* key_mask;        // [kv_rows] or null
    // ... or in pages (cached == true)
    bool cached;
    fq_kv8_cache cache;
    const int32_t* table;
    int64_t ld_table;
    int table_width;
    // split of the keys: chunks of `chunk` keys, whose partial results meet in the workspace
    int chunk;                      // keys per chunk
    int chunks;                     // of max_kv keys
    int tile_rows;                  // (token, head of a group) rows per tile
    // (few queries: equal shares of all the work instead, `ctas` of them; tiles that lie in several are listed in `splits`)
    int ctas;
    int4* splits;
    float* part;                    // [q_rows][q_heads][chunks][head_dim], then [..][2] maxima and sums
    float* part_ml;
    // (sequence, kv head) pairs of a launch; of the cache's, the codes widened to binary16 (many queries)
    int first_unit, units;
    void* wide;
    int64_t wide_keys;              // keys of a unit, a multiple of 128
};
fq_status launch_attention(Attention& a, void* workspace, size_t ws_bytes, cudaStream_t stream);
size_t attention_workspace_bytes(const Attention& a);

#ifdef __CUDACC__
__device__ __forceinline__ int32_t ld_global_s32(const int32_t* p) {
    int32_t v;
    asm volatile("ld.global.b32 %0, [%1];" : "=r"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ long long ld_global_s64(const void* p) {
    long long v;
    asm volatile("ld.global.b64 %0, [%1];" : "=l"(v) : "l"(p));
    return v;
}
// Rows of sequence b in an array of offsets that nobody has checked: cut to [0, rows], never negative in number.
__device__ __forceinline__ void sequence_rows(const int32_t* offsets, int b, int batch, int64_t rows, int64_t* first, int64_t* count) {
    if (!offsets) {
        const int64_t n = rows / batch;
        *first = n * b;
        *count = n;
        return;
    }
    const int64_t lo = min(max((int64_t)ld_global_s32(offsets + b), (int64_t)0), rows), hi = min(max((int64_t)ld_global_s32(offsets + b + 1), lo), rows);
    *first = lo;
    *count = hi - lo;
}
#endif

}  // namespace fq
