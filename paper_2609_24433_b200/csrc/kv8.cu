// Appends keys and values of new tokens to the paged cache of 8-bit codes with one scale for each (page, head).
//
// For one page and head, x the page's new tokens, s the scale of what it holds (nothing is read, s = 0, where the new tokens
// start the page):  a = max|x|,  c = a/127 (0 below the smallest normal number),  s' = max(s, c),
//   new codes  round(x 127 / a) where c >= s, else round(x / s);   held codes  round(code s / s') where s' > s.
// Each is the rounding of the exact quotient, ties to even, so a code does not depend on how the division was done: the
// kernel multiplies by binary32 reciprocals, rounds by adding 1.5 2^23, and looks closer only where one just above and one just
// below the quotient give two codes.
//
// Bound by memory: D (e + 1) bytes per token, head and operand.  One CTA per (page, operand, head) copies its tokens into shared
// memory (cp.async, all under way at once), where the maximum and then the codes read them: of keys eight channels a thread, of
// values, whose pages keep tokens innermost, four tokens by four channels.  The loops stay rolled: with the tokens in registers,
// eight units a thread, their code was long enough to wait for itself.  52224 tokens, one head of 256, bf16 (12.4 us at the
// measured copy rate): 60 us with two passes of loads and bytes turned one by one, 39 with the tokens in registers, 30 with
// borders looked for by their distance, 27 now (issue slots: 77 %).
#include <type_traits>

#include "act_common.cuh"
#include "fq_common.cuh"
#include "layer_common.cuh"
#include "ptx_sm100.cuh"

namespace fq {
namespace {

constexpr int kMaxThreads = 256;

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

__device__ __forceinline__ void lds8(const float* p, float* f) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
__device__ __forceinline__ void lds8(const __nv_bfloat16* p, float* f) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void lds4(const float* p, float* f) {
    const float4 a = *reinterpret_cast<const float4*>(p);
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
}
__device__ __forceinline__ void lds4(const __nv_bfloat16* p, float* f) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xffff0000u);
    f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xffff0000u);
}

// The largest magnitude of the channels in 16-byte units.
template <typename T>
struct Largest;
template <>
struct Largest<float> {
    float most = 0.0f;
    __device__ __forceinline__ void take(uint4 v) {
        most = fmaxf(fmaxf(fmaxf(most, fabsf(__uint_as_float(v.x))), fabsf(__uint_as_float(v.y))), fmaxf(fabsf(__uint_as_float(v.z)), fabsf(__uint_as_float(v.w))));
    }
    __device__ __forceinline__ float value() const { return most; }
};
template <>
struct Largest<__nv_bfloat16> {
    __nv_bfloat162 most = __nv_bfloat162(__ushort_as_bfloat16(0), __ushort_as_bfloat16(0));
    __device__ __forceinline__ void take(uint4 v) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t a = w[i] & 0x7fff7fffu;
            most = __hmax2(most, *reinterpret_cast<const __nv_bfloat162*>(&a));
        }
    }
    __device__ __forceinline__ float value() const { return fmaxf(__low2float(most), __high2float(most)); }
};
__device__ __forceinline__ uint32_t pack4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {       // their low bytes
    return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
// N codes, in the low bytes of t.  (1.5 2^23 + r ends in the two's complement of c = round(r).)  The exact quotient lies between
// the products with a factor two steps above the rounded one and with one two steps below it: where both give the same code, it
// is the code.  Half the page's largest value is a border, 63.5, so that borders are nothing rare, and none is settled by a
// division.  SHORT, bf16 values over their own maximum: r = 127 X / A 2^k with X and A of 8 bits, so r in [2^j, 2^(j+1)) that is no
// border lies 2^(j-17) from one, ten times as far as the products: two codes mean a border, and the even one is it.  Else by
// 2 |x num - c den| against den, which binary64 holds exactly (c and num take 7 bits, x and den 24).
struct Factors {
    float above, below;
};
__device__ __forceinline__ Factors around(float f) {    // (0: nothing is larger than what binary32 holds of a page's scale)
    const uint32_t w = __float_as_uint(f);
    return w < 2 ? Factors{f, f} : Factors{__uint_as_float(w + 2), __uint_as_float(w - 2)};
}
template <int N, bool SHORT>
__device__ __forceinline__ void codes(const float* f, Factors by, float num, float den, uint32_t* t) {
    constexpr float kMagic = 12582912.0f;
    const float2 above = make_float2(by.above, by.above), below = make_float2(by.below, by.below), magic = make_float2(kMagic, kMagic);
    uint32_t differ = 0, other[N];
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        const float2 x = make_float2(f[i], f[i + 1]), hi = f2_fma(x, above, magic), lo = f2_fma(x, below, magic);
        t[i] = __float_as_uint(hi.x); t[i + 1] = __float_as_uint(hi.y);
        other[i] = __float_as_uint(lo.x); other[i + 1] = __float_as_uint(lo.y);
        differ |= (t[i] ^ other[i]) | (t[i + 1] ^ other[i + 1]);
    }
    if (differ) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (SHORT) {
                if (t[i] & 1) t[i] = other[i];          // (the same, or the even one)
            } else if (t[i] != other[i]) {
                const float c = __uint_as_float(t[i]) - kMagic;
                const double exact = fma((double)f[i], (double)num, -(double)c * (double)den), twice = 2.0 * fabs(exact);
                if (twice > (double)den || (twice == (double)den && (t[i] & 1))) t[i] += exact > 0.0 ? 1u : ~0u;
            }
        }
    }
}
// Four held codes, of a scale `was`, in the scale `now`.
__device__ __forceinline__ uint32_t requantize4(uint32_t w, Factors ratio, float was, float now) {
    float f[4];
    uint32_t t[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = (float)(int8_t)(w >> (8 * i));
    codes<4, false>(f, ratio, was, now, t);
    return pack4(t[0], t[1], t[2], t[3]);
}

template <typename T>
__global__ void __launch_bounds__(kMaxThreads, 5) kv8_append_kernel(const AppendArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];     // the page's new tokens, rows of head_dim T and 16 bytes
    __shared__ float warp_max[kMaxThreads / 32];
    const int kThreads = blockDim.x;
    griddep_wait();
    const int b = blockIdx.z, which = blockIdx.y & 1, head = blockIdx.y >> 1;
    int64_t row0, n;
    sequence_rows(a.offsets, b, a.batch, a.tokens, &row0, &n);
    const int64_t held = max((int64_t)ld_global_s32(a.kv_len + b), (int64_t)0);
    const int D = a.head_dim, P = a.page, shift = 31 - __clz(P);
    const int64_t end = min(held + n, (int64_t)a.table_width * P), ld = a.ld[which];
    constexpr int kUnit = 16 / sizeof(T);               // channels of a copy
    const int pitch = D + kUnit, per_row = D / kUnit;
    const T* rows = reinterpret_cast<const T*>(smem);
    for (int64_t i = (held >> shift) + blockIdx.x; (i << shift) < end; i += gridDim.x) {
        const int first = (int)max(held - (i << shift), (int64_t)0), last = (int)min(end - (i << shift), (int64_t)P), m = last - first;
        if (m <= 0) continue;
        const T* x = static_cast<const T*>(a.x[which]) + (row0 + (i << shift) + first - held) * ld + (int64_t)head * D;
        __syncthreads();                                // (the last page's readers)
        {
            const int step_t = kThreads / per_row, step_u = kThreads - step_t * per_row;
            int t = threadIdx.x / per_row, u = threadIdx.x - t * per_row;
            while (t < m) {
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(rows + t * pitch + u * kUnit)), "l"(x + t * ld + u * kUnit) : "memory");
                t += step_t;
                u += step_u;
                if (u >= per_row) { u -= per_row; ++t; }
            }
        }
        const int64_t id = (int)ld_global_u32(a.table + b * a.ld_table + i);
        const bool there = id >= 0 && id < a.pages;
        float* scale = a.scales[which] + (there ? id * a.heads + head : 0);
        const float was = there && first > 0 ? ld_global_f32(scale) : 0.0f;
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncthreads();
        if (!there) continue;
        // ---- the largest magnitude
        float most = 0.0f;
        {
            const int step_t = kThreads / per_row, step_u = kThreads - step_t * per_row;
            int t = threadIdx.x / per_row, u = threadIdx.x - t * per_row;
            Largest<T> l;
            while (t < m) {
                l.take(*reinterpret_cast<const uint4*>(rows + t * pitch + u * kUnit));
                t += step_t;
                u += step_u;
                if (u >= per_row) { u -= per_row; ++t; }
            }
            most = l.value();
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
        if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = most;
        __syncthreads();
        for (int w = 0; w < kThreads / 32; ++w) most = fmaxf(most, warp_max[w]);
        float cand = __fdiv_rn(most, 127.0f);
        if (cand < 1.17549435e-38f) cand = 0.0f;
        const float now = fmaxf(was, cand);
        const bool sets = cand >= was, grown = first > 0 && now > was;
        const float num = sets ? 127.0f : 1.0f, den = sets ? most : was;
        const Factors inv = around(now > 0.0f ? __fdiv_rn(num, den) : 0.0f), ratio = around(grown ? __fdiv_rn(was, now) : 1.0f);
        int8_t* page = a.codes[which] + (id * a.heads + head) * (int64_t)P * D;
        // ---- the codes
        uint32_t* w = reinterpret_cast<uint32_t*>(page);
        constexpr bool kBf16 = sizeof(T) == 2;
        const bool brief = kBf16 && sets;               // (all of a page's values alike)
        auto codes_of = [&](auto n, const float* f, uint32_t* c) {
            constexpr int N = decltype(n)::value;
            if (brief) codes<N, true>(f, inv, num, den, c);
            else codes<N, false>(f, inv, num, den, c);
        };
        if (which == 0) {
            const int eights = D / 8, step_t = kThreads / eights, step_u = kThreads - step_t * eights;
            int t = threadIdx.x / eights, u = threadIdx.x - t * eights;
            while (t < m) {
                float f[8];
                uint32_t c[8];
                lds8(rows + t * pitch + u * 8, f);
                codes_of(std::integral_constant<int, 8>(), f, c);
                *reinterpret_cast<uint2*>(page + (first + t) * D + u * 8) = make_uint2(pack4(c[0], c[1], c[2], c[3]), pack4(c[4], c[5], c[6], c[7]));
                t += step_t;
                u += step_u;
                if (u >= eights) { u -= eights; ++t; }
            }
            if (grown)
                for (int e = threadIdx.x; e < first * D / 4; e += kThreads) w[e] = requantize4(w[e], ratio, was, now);
        } else {
            // Words of four tokens, from the first that changes; a warp takes eight of them (a sector; pages of 16 tokens: all four)
            // of four (eight) blocks of four channels.
            const int w0 = grown ? 0 : first / 4, words = P / 4, in_run = words < 8 ? 4 : 8, runs = 32 / in_run;
            const int groups = ((last + 3) / 4 - w0 + in_run - 1) / in_run, blocks = (D / 4 + runs - 1) / runs;
            const int lane = threadIdx.x % 32, kr = lane & (in_run - 1), cr = in_run == 4 ? lane / 4 : lane / 8;
            for (int e = threadIdx.x / 32; e < groups * blocks; e += kThreads / 32) {
                const int block = e / groups, k = w0 + (e - block * groups) * in_run + kr, t = 4 * k, c = (block * runs + cr) * 4;
                if (t >= last || c >= D) continue;
                uint32_t out[4][4];                     // [token][channel]
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float f[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                    if (t + j >= first && t + j < last) lds4(rows + (t + j - first) * pitch + c, f);
                    codes_of(std::integral_constant<int, 4>(), f, out[j]);
                }
                uint32_t* to = w + c * words + k;
                const bool partial = t < first || t + 4 > last;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t v = pack4(out[0][j], out[1][j], out[2][j], out[3][j]);
                    if (partial) {                      // bytes of tokens that are not new, and of those the held ones
                        const int before = min(max(first - t, 0), 4), until = min(last - t, 4);
                        const uint32_t held_bytes = before == 4 ? ~0u : (1u << (8 * before)) - 1u;
                        const uint32_t keep = held_bytes | (until == 4 ? 0u : ~0u << (8 * until));
                        const uint32_t old = to[j * words];
                        const uint32_t same = grown ? (requantize4(old, ratio, was, now) & held_bytes) | (old & ~held_bytes) : old;
                        v = (v & ~keep) | (same & keep);
                    }
                    to[j * words] = v;
                }
            }
        }
        if (threadIdx.x == 0) *scale = now;
    }
}

template <typename T>
cudaError_t launch(const AppendArgs& a, dim3 grid, cudaStream_t stream) {
    const size_t smem = sizeof(T) * (size_t)a.page * (a.head_dim + 16 / sizeof(T));
    auto* kern = kv8_append_kernel<T>;
    const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kern), smem);
    // (32 channels of a page a thread: small pages take small CTAs, of which an SM holds more.  Also for single tokens, whose values
    // touch a word in every row of their page: 64 threads 8.6 us, 256 4.8, 32 sequences with 4 heads of 128)
    int threads = 64;
    while (threads < kMaxThreads && threads * 32 < a.page * a.head_dim) threads *= 2;
    return e != cudaSuccess ? e : launch_pdl3(kern, grid, (unsigned)threads, smem, stream, a);
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
    return r.xt == FQ_BF16 ? launch<__nv_bfloat16>(a, grid, stream) : launch<float>(a, grid, stream);
}

}  // namespace fq
