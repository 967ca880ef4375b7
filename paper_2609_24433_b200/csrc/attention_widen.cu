// The cache's codes as binary16, exactly, for the tensor-core kernel of many queries: keys [unit][key][channel], values
// [unit][channel][key], unit a (sequence, kv head).  Keys without a page become zeros.  Bound by memory: one byte in, two out.
//
// A CTA takes 128 keys of a unit: 16 codes a thread and turn, of keys along the channels, of values along the keys, as their
// pages keep them, so that no transposition is needed anywhere.  (32 sequences of 866 keys, one head of 256: 14 us under a profiler,
// of which 7 are the 43 MB; 15.5 with one load at a time.)
#include "attention_common.cuh"

#include <cuda_fp16.h>

namespace fq {
namespace {

constexpr int kThreads = 256;
constexpr int kKeys = 128;

// Four int8 -> two pairs of binary16: byte permutes put (code + 128) under the exponent of 1024, 1152 is taken off.
__device__ __forceinline__ void widen4(uint32_t w, uint32_t* lo, uint32_t* hi) {
    const uint32_t u = w ^ 0x80808080u;
    const __half2 base = __half2half2(__ushort_as_half(0x6480));
    const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
    const __half2 x = __hsub2(*reinterpret_cast<const __half2*>(&a), base), y = __hsub2(*reinterpret_cast<const __half2*>(&b), base);
    *lo = *reinterpret_cast<const uint32_t*>(&x);
    *hi = *reinterpret_cast<const uint32_t*>(&y);
}
__device__ __forceinline__ void store16(uint16_t* to, uint4 v) {
    uint32_t h[8];
    widen4(v.x, &h[0], &h[1]);
    widen4(v.y, &h[2], &h[3]);
    widen4(v.z, &h[4], &h[5]);
    widen4(v.w, &h[6], &h[7]);
    reinterpret_cast<uint4*>(to)[0] = make_uint4(h[0], h[1], h[2], h[3]);
    reinterpret_cast<uint4*>(to)[1] = make_uint4(h[4], h[5], h[6], h[7]);
}

__global__ void __launch_bounds__(kThreads) attention_widen_kernel(const Attention a) {
    __shared__ int at[kKeys / 16];                      // (page, head) of every 16 keys, -1 where there is no page
    griddep_wait();
    const int unit = a.first_unit + blockIdx.y, b = unit / a.kv_heads, hk = unit % a.kv_heads;
    const Sequence s = sequence_of(a, b);
    const int D = a.head_dim, P = a.cache.page, shift = 31 - __clz(P);
    const int64_t L = a.wide_keys;
    uint16_t* keys = static_cast<uint16_t*>(a.wide) + (int64_t)blockIdx.y * L * D;
    uint16_t* values = keys + (int64_t)a.units * L * D;
    for (int64_t j0 = (int64_t)blockIdx.x * kKeys; j0 < s.keys; j0 += (int64_t)gridDim.x * kKeys) {
        __syncthreads();
        if (threadIdx.x < kKeys / 16) {
            const int64_t j = j0 + 16 * threadIdx.x;
            int id = -1;
            if (j < s.keys) id = (int)ld_global_u32(a.table + b * a.ld_table + (j >> shift));
            at[threadIdx.x] = id >= 0 && id < a.cache.pages ? id * a.kv_heads + hk : -1;
        }
        __syncthreads();
        const int units = kKeys * D / 16, per_key = D / 16;
        for (int e0 = threadIdx.x; e0 < units; e0 += 4 * kThreads) {    // four loads under way
            uint4 v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = e0 + i * kThreads;
                if (blockIdx.z == 0) {                                  // keys: 16 channels
                    const int key = e / per_key, c = (e - key * per_key) * 16, page = e < units ? at[key / 16] : -1;
                    v[i] = ld_global_v4(a.cache.k + (page >= 0 ? ((int64_t)page * P + (key & (P - 1))) * D + c : 0), page >= 0);
                } else {                                                // values: 16 keys of a channel
                    const int d = e / (kKeys / 16), x = e % (kKeys / 16), page = e < units ? at[x] : -1;
                    v[i] = ld_global_v4(a.cache.v + (page >= 0 ? ((int64_t)page * D + d) * P + ((16 * x) & (P - 1)) : 0), page >= 0);
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = e0 + i * kThreads;
                if (e < units) store16(blockIdx.z == 0 ? keys + j0 * D + e * 16 : values + (int64_t)(e / (kKeys / 16)) * L + j0 + 16 * (e % (kKeys / 16)), v[i]);
            }
        }
    }
}

}  // namespace

cudaError_t launch_attention_widen(const Attention& a, cudaStream_t stream) {
    int64_t tiles = a.wide_keys / kKeys;
    if (tiles < 1) return cudaSuccess;
    if (tiles > 65535) tiles = 65535;
    return launch_pdl3(attention_widen_kernel, dim3((unsigned)tiles, (unsigned)a.units, 2), kThreads, 0, stream, a);
}

}  // namespace fq
