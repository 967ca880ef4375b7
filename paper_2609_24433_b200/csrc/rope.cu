// RMS norm of each query and key head and rotary positions, in one pass over what the fused qkv projection wrote.
//
// Per token t and head h (D channels x):  n = x * rsqrt(mean(x^2) + eps) * gain  (where a gain is given), then for the
// pairs (a, b) of the first r channels -- (i, i + r/2) or (2i, 2i + 1) --
//   a' = amp (a cos w - b sin w),  b' = amp (a sin w + b cos w),   w = position_t * frequency_i.
// One rounding at the store.  The angle is the one quantity that 32 bits do not hold: at position 10^5 a binary32 product
// is off by up to 4e-3 rad, so w is formed in binary64, reduced to a fraction of a turn there and only then narrowed
// (the B200 has one binary64 unit for two binary32 ones, and there is one angle per token and pair, shared by the heads).
//
// Bound by memory: D e bytes in and out per head.  A group of lanes holds a head, eight channels a lane (one 16-byte
// load in bf16), sums its squares by shuffles and swaps halves by shuffles.
#include "fq_common.cuh"
#include "layer_common.cuh"
#include "ptx_sm100.cuh"

namespace fq {
namespace {

constexpr int kThreads = 256;
constexpr int kVec = 8;                 // channels per lane
constexpr double kInvTwoPi = 0.15915494309189533577;

enum : int { kPairs = 0, kHalvesShuffled = 1, kHalvesStaged = 2 };

struct RopeArgs {
    const void* x;
    int64_t ldx;
    void* q;
    void* k;
    int64_t ldq, ldk;
    const float* q_gain;
    const float* k_gain;
    const int32_t* positions;
    const double* frequencies;
    int64_t M;
    int q_heads, heads, head_dim, rotary;
    int tokens;                         // per CTA
    float eps, amplitude;
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
__device__ __forceinline__ void store8(float* p, const float* f) {
    reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float* f) {
    uint4 v;
    v.x = pack_bf16(f[0], f[1]); v.y = pack_bf16(f[2], f[3]); v.z = pack_bf16(f[4], f[5]); v.w = pack_bf16(f[6], f[7]);
    *reinterpret_cast<uint4*>(p) = v;
}

template <typename TX, typename TY, int MODE, int LANES>
__global__ void __launch_bounds__(kThreads) qk_norm_rope_kernel(const RopeArgs a) {
    extern __shared__ float smem[];
    const int half = a.rotary / 2;
    float* cosines = smem;                               // [tokens][half], padded to float4
    const int pitch = (half + 3) & ~3;
    float* sines = smem + a.tokens * pitch;
    float* staged = sines + a.tokens * pitch;            // [groups][head_dim], halves that no lane boundary separates
    griddep_wait();
    const int64_t t0 = (int64_t)blockIdx.x * a.tokens;
    const int tokens = (int)min((int64_t)a.tokens, a.M - t0);
    for (int i = threadIdx.x; i < tokens * half; i += kThreads) {
        const int t = i / half, p = i - t * half;
        const double f = __longlong_as_double(ld_global_s64(a.frequencies + p));
        const double turns = (double)(int32_t)ld_global_u32(a.positions + t0 + t) * (f * kInvTwoPi);
        float s, c;
        sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
        cosines[t * pitch + p] = a.amplitude * c;
        sines[t * pitch + p] = a.amplitude * s;
    }
    __syncthreads();
    constexpr int kGroups = kThreads / LANES;
    const int group = threadIdx.x / LANES, lane = threadIdx.x % LANES;
    const int c0 = lane * kVec;
    const bool active = c0 < a.head_dim;
    const int items = tokens * a.heads;
    const float inv_d = 1.0f / (float)a.head_dim;
    // (every lane of a warp runs the same number of rounds: the shuffles below name all of them)
    for (int base = 0; base < items; base += kGroups) {
        const int item = base + group;
        const bool ok = active && item < items;
        const int t = ok ? item / a.heads : 0, h = ok ? item - t * a.heads : 0;
        const bool is_q = h < a.q_heads;
        float v[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = 0.0f;
        if (ok) load8(static_cast<const TX*>(a.x) + (t0 + t) * a.ldx + (int64_t)h * a.head_dim + c0, v);
        const float* gain = is_q ? a.q_gain : a.k_gain;
        float ss = 0.0f;
#pragma unroll
        for (int i = 0; i < kVec; ++i) ss = fmaf(v[i], v[i], ss);
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        if (ok && gain) {
            const float r = rsqrtf(fmaf(ss, inv_d, a.eps));
            float g[kVec];
            load8(gain + c0, g);
#pragma unroll
            for (int i = 0; i < kVec; ++i) v[i] = v[i] * r * g[i];
        }
        const float* cs = cosines + t * pitch;
        const float* sn = sines + t * pitch;
        if (MODE == kPairs) {
#pragma unroll
            for (int i = 0; i < kVec; i += 2) {
                if (ok && c0 + i < a.rotary) {
                    const float c = cs[(c0 + i) / 2], s = sn[(c0 + i) / 2], x = v[i], y = v[i + 1];
                    v[i] = x * c - y * s;
                    v[i + 1] = x * s + y * c;
                }
            }
        } else {
            float other[kVec];
            if (MODE == kHalvesShuffled) {               // half is a multiple of kVec: the partner is another lane's same slot
                const int shift = half / kVec;
                const int from = c0 < half ? lane + shift : (c0 < a.rotary ? lane - shift : lane);
#pragma unroll
                for (int i = 0; i < kVec; ++i) other[i] = __shfl_sync(0xffffffffu, v[i], from, LANES);
            } else {
                float* mine = staged + group * a.head_dim;
                __syncwarp();
                if (ok) store8(mine + c0, v);
                __syncwarp();
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    const int c = c0 + i;
                    other[i] = ok && c < a.rotary ? mine[c < half ? c + half : c - half] : 0.0f;
                }
            }
            if (ok) {
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    const int c = c0 + i;
                    if (c < half) v[i] = v[i] * cs[c] - other[i] * sn[c];
                    else if (c < a.rotary) v[i] = other[i] * sn[c - half] + v[i] * cs[c - half];
                }
            }
        }
        if (ok) {
            TY* out = is_q ? static_cast<TY*>(a.q) + (t0 + t) * a.ldq + (int64_t)h * a.head_dim
                           : static_cast<TY*>(a.k) + (t0 + t) * a.ldk + (int64_t)(h - a.q_heads) * a.head_dim;
            store8(out + c0, v);
        }
    }
}

template <typename TX, typename TY, int MODE, int LANES>
cudaError_t launch(const RopeArgs& a, cudaStream_t stream) {
    const int pitch = (a.rotary / 2 + 3) & ~3;
    const size_t smem = sizeof(float) * ((size_t)a.tokens * pitch * 2 + (MODE == kHalvesStaged ? (size_t)(kThreads / LANES) * a.head_dim : 0));
    return launch_pdl3(qk_norm_rope_kernel<TX, TY, MODE, LANES>, dim3((unsigned)((a.M + a.tokens - 1) / a.tokens)), kThreads, smem, stream, a);
}
template <typename TX, typename TY, int MODE>
cudaError_t by_lanes(const RopeArgs& a, cudaStream_t stream) {
    if (a.head_dim <= 64) return launch<TX, TY, MODE, 8>(a, stream);
    if (a.head_dim <= 128) return launch<TX, TY, MODE, 16>(a, stream);
    return launch<TX, TY, MODE, 32>(a, stream);
}
template <typename TX, typename TY>
cudaError_t by_mode(const RopeArgs& a, bool interleaved, cudaStream_t stream) {
    if (interleaved) return by_lanes<TX, TY, kPairs>(a, stream);
    if (a.rotary / 2 % kVec == 0) return by_lanes<TX, TY, kHalvesShuffled>(a, stream);
    return by_lanes<TX, TY, kHalvesStaged>(a, stream);
}

}  // namespace

cudaError_t launch_qk_norm_rope(const QkNormRope& r, cudaStream_t stream) {
    RopeArgs a = {};
    a.x = r.x; a.ldx = r.ldx; a.q = r.q; a.k = r.k; a.ldq = r.ldq; a.ldk = r.ldk;
    a.q_gain = r.q_gain; a.k_gain = r.k_gain; a.positions = r.positions; a.frequencies = r.frequencies;
    a.M = r.M; a.q_heads = r.q_heads; a.heads = r.q_heads + r.k_heads; a.head_dim = r.head_dim; a.rotary = r.rotary;
    a.eps = r.eps; a.amplitude = r.amplitude;
    const int lanes = r.head_dim <= 64 ? 8 : r.head_dim <= 128 ? 16 : 32, groups = kThreads / lanes;
    int64_t tokens = 1;
    while (tokens < 16 && tokens * a.heads < 4 * groups && (r.M + tokens - 1) / tokens > 4 * device_sm_count()) tokens *= 2;
    a.tokens = (int)tokens;
    const bool xb = r.xt == FQ_BF16, yb = r.yt == FQ_BF16;
    if (xb) return yb ? by_mode<__nv_bfloat16, __nv_bfloat16>(a, r.interleaved, stream) : by_mode<__nv_bfloat16, float>(a, r.interleaved, stream);
    return yb ? by_mode<float, __nv_bfloat16>(a, r.interleaved, stream) : by_mode<float, float>(a, r.interleaved, stream);
}

}  // namespace fq
