// RMS norm of each query and key head and rotary positions, in one pass over what the fused qkv projection wrote.
//
// Per token t and head h (D channels x):  n = x * rsqrt(mean(x^2) + eps) * gain  (where a gain is given), then for the
// pairs (a, b) of the first r channels -- (i, i + r/2) or (2i, 2i + 1) --
//   a' = amp (a cos w - b sin w),  b' = amp (a sin w + b cos w),   w = position_t * frequency_i.
// One rounding at the store.  The angle is the one quantity that 32 bits do not hold: at position 10^5 a binary32 product
// is off by up to 4e-3 rad, so w is formed in binary64, reduced to a fraction of a turn there and only then narrowed
// (the B200 has one binary64 unit for two binary32 ones, and there is one angle per token and pair, shared by the heads).
//
// Bound by memory: D e bytes in and out per head -- once the instructions per head are few.  A group of lanes holds a head, eight
// channels a lane, and walks HEADS heads of one token with the token's cosines and sines in registers (read from shared
// memory for every head, with two-way conflicts, they bounded the kernel).  Where whole heads turn by halves a lane holds four
// channels and the four that they pair with: no exchange, half the angles.  Arithmetic goes two channels at a time.
// 13056 tokens x 9 heads of 256, bf16 (18.6 us at the measured copy rate): 78 us at first, 42 with loads ahead, 38 with angles in
// registers, 32 now (instructions: 4 TB/s; binary32, with half as many for a byte, 6.2 TB/s).
#include "act_common.cuh"
#include "fq_common.cuh"
#include "layer_common.cuh"
#include "ptx_sm100.cuh"

namespace fq {
namespace {

constexpr int kThreads = 256;
constexpr double kInvTwoPi = 0.15915494309189533577;

// Neighbours; whole heads by halves; part of a head by halves that a lane boundary separates; by any halves.
enum : int { kPairs = 0, kHalvesWhole = 1, kHalvesShuffled = 2, kHalvesStaged = 3 };

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

// Four channels as they lie in memory.
template <typename T>
struct Four;
template <>
struct Four<float> {
    float4 a;
    __device__ __forceinline__ void load(const float* p) { a = ld_global_f4(p); }
    __device__ __forceinline__ void clear() { a = make_float4(0.0f, 0.0f, 0.0f, 0.0f); }
    __device__ __forceinline__ void values(float2* f) const { f[0] = make_float2(a.x, a.y); f[1] = make_float2(a.z, a.w); }
};
template <>
struct Four<__nv_bfloat16> {
    uint32_t a, b;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { asm volatile("ld.global.v2.b32 {%0, %1}, [%2];" : "=r"(a), "=r"(b) : "l"(p)); }
    __device__ __forceinline__ void clear() { a = b = 0u; }
    __device__ __forceinline__ void values(float2* f) const {
        f[0] = make_float2(__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u));
        f[1] = make_float2(__uint_as_float(b << 16), __uint_as_float(b & 0xffff0000u));
    }
};
__device__ __forceinline__ void store4(float* p, const float2* f) { *reinterpret_cast<float4*>(p) = make_float4(f[0].x, f[0].y, f[1].x, f[1].y); }
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float2* f) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(f[0].x, f[0].y), pack_bf16(f[1].x, f[1].y));
}
__device__ __forceinline__ void lds4(const float* p, float2* f) {
    const float4 a = *reinterpret_cast<const float4*>(p);
    f[0] = make_float2(a.x, a.y);
    f[1] = make_float2(a.z, a.w);
}

template <typename TX, typename TY, int MODE, int LANES, int HEADS>
__global__ void __launch_bounds__(kThreads, 5) qk_norm_rope_kernel(const RopeArgs a) {
    extern __shared__ __align__(16) float smem[];
    constexpr int kGroups = kThreads / LANES;
    const int half = a.rotary / 2, pitch = (half + 3) & ~3;
    float* gains = smem;                                 // [2][head_dim]: of queries, of keys; ones where there is none
    float* cosines = gains + 2 * a.head_dim;             // [tokens][pitch]
    float* sines = cosines + a.tokens * pitch;
    float* staged = sines + a.tokens * pitch;            // [groups][head_dim]
    griddep_wait();
    const int64_t t0 = (int64_t)blockIdx.x * a.tokens;
    const int tokens = (int)min((int64_t)a.tokens, a.M - t0);
    const int group = threadIdx.x / LANES, lane = threadIdx.x % LANES;
    const bool active = lane * 8 < a.head_dim;
    const int c0 = MODE == kHalvesWhole ? lane * 4 : lane * 8, c1 = MODE == kHalvesWhole ? half + lane * 4 : c0 + 4;

    // A group's units: (token, HEADS heads), kGroups apart.  A head's channels are loaded when the same place of the unit ahead
    // has been taken.
    const int per_token = (a.heads + HEADS - 1) / HEADS, step_t = kGroups / per_token, step_b = kGroups - step_t * per_token;
    int t = group / per_token, block = group - t * per_token, next_t = t, next_b = block;
    Four<TX> raws[HEADS][2];
    auto load = [&](int u, const TX* from) {             // `from`: the unit's first head; null behind the last unit
        if (from && next_b * HEADS + u < a.heads) {
            raws[u][0].load(from + u * a.head_dim + c0);
            raws[u][1].load(from + u * a.head_dim + c1);
        } else {
            raws[u][0].clear();
            raws[u][1].clear();
        }
    };
    auto unit = [&]() -> const TX* {
        return active && next_t < tokens ? static_cast<const TX*>(a.x) + (t0 + next_t) * a.ldx + next_b * HEADS * a.head_dim : nullptr;
    };
    {
        const TX* from = unit();
#pragma unroll
        for (int u = 0; u < HEADS; ++u) load(u, from);
    }
    for (int i = threadIdx.x; i < 2 * a.head_dim; i += kThreads) {
        const float* from = i < a.head_dim ? a.q_gain : a.k_gain;
        gains[i] = from ? ld_global_f32(from + (i < a.head_dim ? i : i - a.head_dim)) : 1.0f;
    }
    const int angle_t = half > 0 ? kThreads / half : 0, angle_p = kThreads - angle_t * half;
    for (int tt = half > 0 ? threadIdx.x / half : tokens, p = threadIdx.x - tt * half; tt < tokens;) {
        const double f = __longlong_as_double(ld_global_s64(a.frequencies + p));
        const double turns = (double)(int32_t)ld_global_u32(a.positions + t0 + tt) * (f * kInvTwoPi);
        float s, c;
        sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
        cosines[tt * pitch + p] = a.amplitude * c;
        sines[tt * pitch + p] = a.amplitude * s;
        tt += angle_t;
        p += angle_p;
        if (p >= half) { p -= half; ++tt; }
    }
    __syncthreads();
    const float inv_d = 1.0f / (float)a.head_dim;
    const bool low = c0 < half, turns = c0 < a.rotary;   // (kHalvesShuffled: of all eight channels alike)
    // (every lane of a warp runs the same number of rounds: the shuffles below name all of them)
    const int rounds = (tokens * per_token + kGroups - 1) / kGroups;
    for (int round = 0; round < rounds; ++round) {
        next_t += step_t;
        next_b += step_b;
        if (next_b >= per_token) { next_b -= per_token; ++next_t; }
        const TX* from = unit();
        const bool there = active && t < tokens;
        float2 cs[4], sn[4];                             // kPairs, kHalvesWhole: two of each
        const float *c = cosines + (there ? t : 0) * pitch, *s = sines + (there ? t : 0) * pitch;
        if (MODE == kPairs || MODE == kHalvesWhole) {
            if (there && turns) {
                lds4(c + lane * 4, cs);
                lds4(s + lane * 4, sn);
            }
        } else if (MODE == kHalvesShuffled && there && turns) {
            const int at = low ? c0 : c0 - half;
            lds4(c + at, cs);
            lds4(c + at + 4, cs + 2);
            lds4(s + at, sn);
            lds4(s + at + 4, sn + 2);
#pragma unroll
            for (int i = 0; i < 4; ++i) sn[i] = low ? make_float2(-sn[i].x, -sn[i].y) : sn[i];
        }
        const int h0 = block * HEADS;
        TY* out_q = static_cast<TY*>(a.q) + (t0 + t) * a.ldq + h0 * a.head_dim;
        TY* out_k = static_cast<TY*>(a.k) + (t0 + t) * a.ldk + (h0 - a.q_heads) * a.head_dim;
#pragma unroll
        for (int u = 0; u < HEADS; ++u) {
            const int h = h0 + u;
            const bool ok = there && h < a.heads, is_q = h < a.q_heads;
            float2 v[4];
            raws[u][0].values(v);
            raws[u][1].values(v + 2);
            load(u, from);
            if (!__any_sync(0xffffffffu, ok)) continue;
            if (a.q_gain || a.k_gain) {
                float2 ss = f2_mul(v[0], v[0]);
#pragma unroll
                for (int i = 1; i < 4; ++i) ss = f2_fma(v[i], v[i], ss);
                float sum = ss.x + ss.y;
#pragma unroll
                for (int o = LANES / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                const float r = (is_q ? a.q_gain : a.k_gain) ? rsqrtf(fmaf(sum, inv_d, a.eps)) : 1.0f;
                if (ok) {
                    float2 g[4];
                    const float* from_g = gains + (is_q ? 0 : a.head_dim);
                    lds4(from_g + c0, g);
                    lds4(from_g + c1, g + 2);
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = f2_mul(f2_mul(v[i], make_float2(r, r)), g[i]);
                }
            }
            if (MODE == kPairs) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (ok && c0 + 2 * i < a.rotary) {
                        const float cc = i & 1 ? cs[i / 2].y : cs[i / 2].x, s1 = i & 1 ? sn[i / 2].y : sn[i / 2].x;
                        v[i] = make_float2(v[i].x * cc - v[i].y * s1, v[i].x * s1 + v[i].y * cc);
                    }
                }
            } else if (MODE == kHalvesWhole) {
                if (ok) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float2 lo = v[i], hi = v[i + 2];
                        v[i] = f2_fma(hi, make_float2(-sn[i].x, -sn[i].y), f2_mul(lo, cs[i]));
                        v[i + 2] = f2_fma(hi, cs[i], f2_mul(lo, sn[i]));
                    }
                }
            } else if (MODE == kHalvesShuffled) {        // half is a multiple of eight: the partner is another lane's same slot
                const int shift = half / 8, partner = low ? lane + shift : (turns ? lane - shift : lane);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 w = make_float2(__shfl_sync(0xffffffffu, v[i].x, partner, LANES), __shfl_sync(0xffffffffu, v[i].y, partner, LANES));
                    if (ok && turns) v[i] = f2_fma(w, sn[i], f2_mul(v[i], cs[i]));
                }
            } else {
                float* mine = staged + group * a.head_dim;
                __syncwarp();
                if (ok) { store4(mine + c0, v); store4(mine + c1, v + 2); }
                __syncwarp();
                if (ok) {
                    auto turn = [&](float x, int ch) {
                        if (ch < half) return x * c[ch] - mine[ch + half] * s[ch];
                        return ch < a.rotary ? mine[ch - half] * s[ch - half] + x * c[ch - half] : x;
                    };
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = make_float2(turn(v[i].x, c0 + 2 * i), turn(v[i].y, c0 + 2 * i + 1));
                }
            }
            if (ok) {
                TY* out = (is_q ? out_q : out_k) + u * a.head_dim;
                store4(out + c0, v);
                store4(out + c1, v + 2);
            }
        }
        t = next_t;
        block = next_b;
    }
}

template <typename TX, typename TY, int MODE, int LANES, int HEADS>
cudaError_t launch(RopeArgs a, cudaStream_t stream) {
    // Tokens of a CTA: four units for every group, fewer where the tokens are not enough for four CTAs on every SM.
    const int per_token = (a.heads + HEADS - 1) / HEADS, groups = kThreads / LANES;
    int64_t tokens = 1;
    while (tokens < 32 && tokens * per_token < 4 * groups && (a.M + tokens - 1) / tokens > 4 * device_sm_count()) tokens *= 2;
    a.tokens = (int)tokens;
    const int pitch = (a.rotary / 2 + 3) & ~3;
    const size_t smem = sizeof(float) * ((size_t)2 * a.head_dim + (size_t)a.tokens * pitch * 2 + (MODE == kHalvesStaged ? (size_t)groups * a.head_dim : 0));
    return launch_pdl3(qk_norm_rope_kernel<TX, TY, MODE, LANES, HEADS>, dim3((unsigned)((a.M + a.tokens - 1) / a.tokens)), kThreads, smem, stream, a);
}
template <typename TX, typename TY, int MODE, int LANES>
cudaError_t by_heads(const RopeArgs& a, cudaStream_t stream) {
    // Few tokens: every group a head, for the shortest way; else, in bf16, two to a load of the token's angles (16384 tokens x 20
    // heads of 128: two with five CTAs an SM 36.2 us, four with four 37.0, four with three 40.7).
    constexpr int kMost = sizeof(TX) == 4 ? 1 : 2;
    if (a.M * ((a.heads + kMost - 1) / kMost) * LANES < (int64_t)2 * kThreads * device_sm_count()) return launch<TX, TY, MODE, LANES, 1>(a, stream);
    return launch<TX, TY, MODE, LANES, kMost>(a, stream);
}
template <typename TX, typename TY, int MODE>
cudaError_t by_lanes(const RopeArgs& a, cudaStream_t stream) {
    if (a.head_dim <= 64) return by_heads<TX, TY, MODE, 8>(a, stream);
    if (a.head_dim <= 128) return by_heads<TX, TY, MODE, 16>(a, stream);
    return by_heads<TX, TY, MODE, 32>(a, stream);
}
template <typename TX, typename TY>
cudaError_t by_mode(const RopeArgs& a, bool interleaved, cudaStream_t stream) {
    if (interleaved) return by_lanes<TX, TY, kPairs>(a, stream);
    if (a.rotary == a.head_dim) return by_lanes<TX, TY, kHalvesWhole>(a, stream);
    if (a.rotary / 2 % 8 == 0) return by_lanes<TX, TY, kHalvesShuffled>(a, stream);
    return by_lanes<TX, TY, kHalvesStaged>(a, stream);
}

}  // namespace

cudaError_t launch_qk_norm_rope(const QkNormRope& r, cudaStream_t stream) {
    RopeArgs a = {};
    a.x = r.x; a.ldx = r.ldx; a.q = r.q; a.k = r.k; a.ldq = r.ldq; a.ldk = r.ldk;
    a.q_gain = r.q_gain; a.k_gain = r.k_gain; a.positions = r.positions; a.frequencies = r.frequencies;
    a.M = r.M; a.q_heads = r.q_heads; a.heads = r.q_heads + r.k_heads; a.head_dim = r.head_dim; a.rotary = r.rotary;
    a.eps = r.eps; a.amplitude = r.amplitude;
    const bool xb = r.xt == FQ_BF16, yb = r.yt == FQ_BF16;
    if (xb) return yb ? by_mode<__nv_bfloat16, __nv_bfloat16>(a, r.interleaved, stream) : by_mode<__nv_bfloat16, float>(a, r.interleaved, stream);
    return yb ? by_mode<float, __nv_bfloat16>(a, r.interleaved, stream) : by_mode<float, float>(a, r.interleaved, stream);
}

}  // namespace fq
