// Attention of many queries on the tcgen05 tensor cores: bf16 keys and values as rows (cross attention) or the 8-bit cache.
//
// A CTA takes one chunk of the keys of one kv head and NT tiles of 128 rows -- (token, head of a group) pairs, so that a group
// reads its keys once.  Per tile of 128 keys: S = Q K^T into TMEM; one thread per row keeps the running maximum and sum and
// writes the probabilities, 16 bits each, over S in TMEM; O += P V takes them from there as its first operand.
//   warps 0-7   softmax, a warpgroup per row tile
//   warps 8-11  which keys of a tile there are; from the cache, its codes into 128-byte-swizzled stages of 128 keys x 64 or 128 channels
//   warp 12     issues the MMAs
//   warp 13     rows: copies keys and values into the stages by TMA (14, 15 complete the warpgroup, whose registers go to the softmax)
// With two row tiles (D <= 128) the tensor core works on one while the other's probabilities are computed; with one (D > 128,
// or few rows) S is double-buffered instead.
//
// The maximum is followed lazily: O and l are rescaled only where a row's maximum has risen by more than 2^8 over the base they
// were built with, so almost never behind the first tiles; probabilities then reach 256, which changes no relative rounding.
//
// Cache: codes are widened to binary16, exactly, on their way into the stages (values keep tokens innermost and need no turn).
// The scale of a page's keys multiplies S per 16 columns; that of its values multiplies the probabilities, over 2^e with e the
// running exponent of the largest one: P = p vs 2^(7 - e) <= 2^15.  Queries: binary16 behind a power of two per row.
// Rows: bf16 operands.  The scores of masked keys are replaced; their values are zeroed in shared memory, in the tiles that have
// any, ahead of the product: 0 times a masked NaN would reach the sums.
#include "act_common.cuh"
#include "attention_common.cuh"
#include "tc_sm100.cuh"

#include <cuda_fp16.h>
#include <float.h>

namespace fq {
namespace {

constexpr int kThreads = 16 * 32;
// Registers: a softmax thread holds a row of 128 scores.  The launch's 512 x 128 are shared out as 256 x 176 + 256 x 80.
constexpr int kRegsLaunch = 128, kRegsSoftmax = 176, kRegsOther = 80;
static_assert(256 * kRegsSoftmax + 256 * kRegsOther <= kThreads * kRegsLaunch, "");
constexpr int kKeys = 128;
constexpr int kMetas = 8;
constexpr float kSlack = 8.0f;          // log2 of how far a row's maximum may rise over its base

constexpr uint32_t kWdProducer = 0x800u, kWdMma = 0x1000u, kWdSoftmax = 0x2000u;

template <int DP, int NT>
struct Shape {
    static constexpr int kParts = DP == 256 ? 2 : 1;            // stages per key or value tile
    static constexpr int kCh = DP / kParts;                     // channels per stage
    static constexpr int kStageBytes = kKeys * kCh * 2;
    static constexpr int kStages = DP == 64 ? 8 : 5;
    static constexpr int kQTile = 128 * DP * 2;
    static constexpr int kSmem = 1024 + NT * kQTile + kStages * kStageBytes;
    static constexpr int kOCol = 256;                           // S: columns 0 .. 255
    // Two tiles of 64 channels leave TMEM for probabilities of their own (columns 384 ..): the next scores are computed as soon
    // as the last ones have been read.  Elsewhere probabilities lie over their scores.
    static constexpr bool kEarly = NT == 2 && DP == 64;
    static constexpr bool kPerTile = NT == 1 || kEarly;         // every product of a tile signals its end
};

struct __align__(16) KeyMeta {
    float ks[8];                        // per 16 keys
    float lvf[8];                       // log2 of vs 2^(7 - e)
    float inv[8];                       // 2^-lvf
    uint32_t valid[4];
    int e;
    int unused[3];
};

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void sts128(uint32_t addr, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ void widen(uint32_t w, uint32_t* lo, uint32_t* hi) {     // four int8 -> two pairs of binary16
    const uint32_t u = w ^ 0x80808080u;
    const __half2 base = __half2half2(__ushort_as_half(0x6480));                    // 1024 + 128
    const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
    const __half2 x = __hsub2(*reinterpret_cast<const __half2*>(&a), base), y = __hsub2(*reinterpret_cast<const __half2*>(&b), base);
    *lo = *reinterpret_cast<const uint32_t*>(&x);
    *hi = *reinterpret_cast<const uint32_t*>(&y);
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ int exponent_of(float x) { return (int)((__float_as_uint(x) >> 23) & 255) - 127; }
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(min(max(e, -126), 127) + 127) << 23); }
__device__ __forceinline__ float max3(float x, uint32_t y, uint32_t z) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(__uint_as_float(y)), "f"(__uint_as_float(z)));
    return r;
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 2^x of two values on the FMA pipe: 2^n by the exponent bits, 2^f on [-1/2, 1/2] by a polynomial of degree 4 (Remez, relative
// error 2.7e-6 in binary32).  The exponential unit gives 16 values per clock and SM, a tile of 128 x 128 scores needs 1024
// clocks of it; kPolynomial of eight pairs go here instead.
constexpr int kPolynomial = 2;
__device__ __forceinline__ float2 ex2_polynomial(float2 x) {
    x.x = fmaxf(x.x, -126.0f);
    x.y = fmaxf(x.y, -126.0f);
    const float2 magic = make_float2(12582912.0f, 12582912.0f);             // 1.5 2^23: the sum's low bits are round(x)
    const float2 t = f2_add(x, magic);
    const float2 n = f2_add(t, make_float2(-12582912.0f, -12582912.0f));
    const float2 f = f2_fma(n, make_float2(-1.0f, -1.0f), x);
    float2 p = make_float2(0.009570102207362652f, 0.009570102207362652f);
    p = f2_fma(p, f, make_float2(0.05591785907745361f, 0.05591785907745361f));
    p = f2_fma(p, f, make_float2(0.240247443318367f, 0.240247443318367f));
    p = f2_fma(p, f, make_float2(0.6931217908859253f, 0.6931217908859253f));
    p = f2_fma(p, f, make_float2(0.9999992847442627f, 0.9999992847442627f));
    return make_float2(__uint_as_float(__float_as_uint(p.x) + (__float_as_uint(t.x) << 23)), __uint_as_float(__float_as_uint(p.y) + (__float_as_uint(t.y) << 23)));
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
          "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void mma_f16_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void mma_f16_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}
// 16-bit operands (type 0: binary16, 1: bf16) -> binary32; A K-major, B K-major or, transposed, N-major; M = 128.
__device__ __forceinline__ uint32_t instr_desc_16(int type, bool b_transposed, int n) {
    return (1u << 4) | ((uint32_t)type << 7) | ((uint32_t)type << 10) | ((b_transposed ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | (8u << 24);
}
// N-major operand, 128-byte rows of 64 channels, 128B swizzle: 8-row groups (of keys) 1024 bytes apart, 64-channel blocks one
// 16 KB plane apart.
__device__ __forceinline__ uint64_t smem_desc_n_major(uint32_t addr) {
    uint64_t d = smem_desc_sw128(addr);
    d &= ~((uint64_t)0x3FFF << 16);
    return d | (uint64_t)(16384 >> 4) << 16;
}
template <int N>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
// mbar_wait_all with the bounded loop in line: a kernel that calls a function keeps its launch's registers in every warp.
__device__ __forceinline__ bool wait_all(uint32_t bar, uint32_t parity, volatile int* abort_flag, uint32_t* watchdog, uint32_t code) {
    bool ok = true;
    if (!mbar_try_wait(bar, parity)) {
        uint64_t t0 = 0;
        for (uint32_t spin = 1; !mbar_try_wait(bar, parity); ++spin) {
            if ((spin & 0xfff) == 0) {
                if (*abort_flag) { ok = false; break; }
                const uint64_t now = global_timer_ns();
                if (t0 == 0) t0 = now;
                if (now - t0 > kWaitLimitNs) {
                    *abort_flag = 1;
                    atomicOr(watchdog, code);
                    ok = false;
                    break;
                }
            }
        }
    }
    return __all_sync(0xffffffffu, ok);
}
__device__ __forceinline__ void mbar_inval(uint32_t bar) { asm volatile("mbarrier.inval.shared::cta.b64 [%0];" ::"r"(bar) : "memory"); }

__device__ __forceinline__ bool all_valid(const KeyMeta& m) { return (m.valid[0] & m.valid[1] & m.valid[2] & m.valid[3]) == ~0u; }

template <int DP, int NT, bool CACHED>
__global__ void __launch_bounds__(kThreads, 1) attention_tiles_kernel(const Attention a, const __grid_constant__ CUtensorMap map_k,
                                                                      const __grid_constant__ CUtensorMap map_v, uint32_t* watchdog) {
    using S = Shape<DP, NT>;
    constexpr int kCh = S::kCh, kParts = S::kParts, kStages = S::kStages, kPlanes = kCh / 64;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(16) KeyMeta metas[kMetas];
    __shared__ __align__(8) uint64_t s_full_kv[kStages], s_empty_kv[kStages], s_meta[kMetas], s_used[kMetas], s_landed, s_fixed, s_s[2], s_p[2], s_o[2], s_free[2], s_q;
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort;
    volatile int* abort_flag = &s_abort;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t q_smem = smem, ring = smem + NT * S::kQTile;
    auto full_kv = [&](int n) { return smem_u32(&s_full_kv[n % kStages]); };
    auto empty_kv = [&](int n) { return smem_u32(&s_empty_kv[n % kStages]); };
    auto stage = [&](int n) { return ring + (uint32_t)(n % kStages) * S::kStageBytes; };

    auto init_barriers = [&]() {
        for (int i = 0; i < kStages; ++i) { mbar_init(smem_u32(&s_full_kv[i]), CACHED ? 4 : 1); mbar_init(smem_u32(&s_empty_kv[i]), 1); }
        for (int i = 0; i < kMetas; ++i) { mbar_init(smem_u32(&s_meta[i]), 4); mbar_init(smem_u32(&s_used[i]), 4 * NT + (CACHED ? 0 : 1)); }
        for (int i = 0; i < 2; ++i) { mbar_init(smem_u32(&s_s[i]), 1); mbar_init(smem_u32(&s_p[i]), 4); mbar_init(smem_u32(&s_o[i]), 1); mbar_init(smem_u32(&s_free[i]), 4); }
        mbar_init(smem_u32(&s_q), 4 * NT);
        mbar_init(smem_u32(&s_landed), 1);
        mbar_init(smem_u32(&s_fixed), 4);
        fence_mbarrier_init();
    };
    if (threadIdx.x == 0) {
        s_abort = 0;
        init_barriers();
    }
    if (warp == 12) tmem_alloc<1>(smem_u32(&s_tmem), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    griddep_wait();

    const int b = blockIdx.z / a.kv_heads, hk = blockIdx.z % a.kv_heads, chunk = blockIdx.y;
    const Sequence s = sequence_of(a, b);
    const int D = a.head_dim, G = a.group;
    const int64_t rows = s.queries * G;
    constexpr int kRows = NT * 128;
    bool ok = true, again = false;

    // Every warp walks the row tiles of this CTA; the longest rows of a causal sequence, its last ones, come first.
    const int64_t tiles = (rows + kRows - 1) / kRows;
    auto for_tiles = [&](auto body) {
        for (int64_t back = blockIdx.x; back < tiles && ok; back += gridDim.x) {
            const int64_t tile = tiles - 1 - back;
            const TileKeys tk = tile_keys(a, s, tile, kRows);
            const int64_t k0 = (int64_t)chunk * a.chunk;
            if (chunk > 0 && k0 >= tk.end) continue;
            const int64_t k1 = min(tk.end, k0 + a.chunk);
            if (again) {                                        // every arrival of the last tile has been waited for
                __syncthreads();
                if (threadIdx.x == 0) {
                    for (int i = 0; i < kStages; ++i) { mbar_inval(smem_u32(&s_full_kv[i])); mbar_inval(smem_u32(&s_empty_kv[i])); }
                    for (int i = 0; i < kMetas; ++i) { mbar_inval(smem_u32(&s_meta[i])); mbar_inval(smem_u32(&s_used[i])); }
                    for (int i = 0; i < 2; ++i) { mbar_inval(smem_u32(&s_s[i])); mbar_inval(smem_u32(&s_p[i])); mbar_inval(smem_u32(&s_o[i])); mbar_inval(smem_u32(&s_free[i])); }
                    mbar_inval(smem_u32(&s_q));
                    mbar_inval(smem_u32(&s_landed));
                    mbar_inval(smem_u32(&s_fixed));
                    init_barriers();
                }
                __syncthreads();
            }
            again = true;
            body(tile, tk.chunks <= 1, k0, k1, (int)((k1 - k0 + kKeys - 1) / kKeys));
            __syncthreads();
            ok = s_abort == 0;
        }
    };

    if (warp < 8) {
        more_registers<kRegsSoftmax>();
        for_tiles([&](int64_t tile, bool direct, int64_t k0, int64_t k1, int n) {
            // ================================================================ softmax
            const int mine = NT == 2 ? warp / 4 : 0;
            const int r = threadIdx.x % 128;
            const int64_t row = tile * kRows + mine * 128 + r;
            const bool active = NT == 2 || warp < 4;
            const bool there = active && row < rows;
            const int64_t token = s.q0 + (there ? row / G : 0), head = hk * G + (there ? row % G : 0);
            float factor = a.scale_log2;
            if (active) {
                // ---- this thread's row of Q
                const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(a.q) + token * a.ldq + head * D;
                const uint32_t dst = q_smem + mine * S::kQTile + r * 128;
                float down = 1.0f;
                if (CACHED) {
                    float top = 0.0f;
                    for (int d = 0; d < D; d += 8) {
                        const uint4 v = ld_global_v4(src + d, there);
                        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) top = fmaxf(top, fmaxf(fabsf(__uint_as_float(w[i] << 16)), fabsf(__uint_as_float(w[i] & 0xffff0000u))));
                    }
                    const int e = min(max(exponent_of(top), -100), 126);
                    down = power_of_two(-e);
                    factor = a.scale_log2 * power_of_two(e);
                }
#pragma unroll 4
                for (int d = 0; d < DP; d += 8) {
                    uint4 v = ld_global_v4(src + d, there && d < D);
                    if (CACHED) {
                        uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) w[i] = pack_half(__uint_as_float(w[i] << 16) * down, __uint_as_float(w[i] & 0xffff0000u) * down);
                        v = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                    sts128(dst + (d / 64) * 16384 + ((((d % 64) / 8) ^ (r & 7)) * 16), v.x, v.y, v.z, v.w);
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&s_q));
            }
            if (active) {
                const uint32_t lanes = tmem + ((uint32_t)(warp % 4) << 21);
                const uint32_t o_addr = lanes + S::kOCol + (NT == 2 ? mine * DP : 0);
                const int64_t limit64 = row_limit(a, s, row);
                float base = -INFINITY, l = 0.0f;
                int e = -127;
                for (int j = 0; j < n && ok; ++j) {
                    const int buf = NT == 2 ? mine : j & 1;
                    const uint32_t phase = NT == 2 ? j & 1 : (j >> 1) & 1;
                    ok = wait_all(smem_u32(&s_s[buf]), phase, abort_flag, watchdog, kWdSoftmax) &&
                         wait_all(smem_u32(&s_meta[j % kMetas]), (j / kMetas) & 1, abort_flag, watchdog, kWdSoftmax);
                    if (!ok) break;
                    tc_fence_after();
                    const KeyMeta& meta = metas[j % kMetas];
                    const uint32_t s_addr = lanes + 128 * buf, p_addr = S::kEarly ? lanes + 384 + 64 * mine : s_addr;
                    const int lim = (int)min(max(limit64 - (k0 + (int64_t)j * kKeys), (int64_t)-1), (int64_t)kKeys);
                    uint32_t seen[4];
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const int x = lim - 32 * c;
                        seen[c] = meta.valid[c] & (x < 0 ? 0u : x >= 31 ? ~0u : (2u << x) - 1u);
                    }
                    const bool masked = __any_sync(0xffffffffu, (seen[0] & seen[1] & seen[2] & seen[3]) != ~0u);
                    uint32_t v[128];
#pragma unroll
                    for (int c = 0; c < 4; ++c) tmem_ld32(s_addr + 32 * c, v + 32 * c);
                    tmem_ld_wait();
                    if (S::kEarly) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&s_free[mine]));
                    }
                    // ---- the largest score
                    float top = -INFINITY;
                    if (masked) {                                // (its own code: selects on every score cost a third of the loop)
#pragma unroll
                        for (int g = 0; g < 8; ++g) {
                            float x = -INFINITY;
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                if (!((seen[g / 2] >> (16 * (g % 2) + i)) & 1)) v[16 * g + i] = 0xff800000u;
                                x = fmaxf(x, __uint_as_float(v[16 * g + i]));
                            }
                            top = fmaxf(top, CACHED ? (x == -INFINITY ? x : x * (factor * meta.ks[g])) : x);
                        }
                    } else {
#pragma unroll
                        for (int g = 0; g < 8; ++g) {
                            float x = -INFINITY, y = -INFINITY;
#pragma unroll
                            for (int i = 0; i < 16; i += 4) {
                                x = max3(x, v[16 * g + i], v[16 * g + i + 1]);
                                y = max3(y, v[16 * g + i + 2], v[16 * g + i + 3]);
                            }
                            x = fmaxf(x, y);
                            top = fmaxf(top, CACHED ? x * (factor * meta.ks[g]) : x);
                        }
                    }
                    if (!CACHED) top = top == -INFINITY ? top : top * factor;
                    if (S::kEarly && j > 0) {                    // the last product has read its probabilities
                        ok = wait_all(smem_u32(&s_o[mine]), (j - 1) & 1, abort_flag, watchdog, kWdSoftmax);
                        if (!ok) break;
                        tc_fence_after();
                    }
                    // ---- a new base
                    const int now_e = CACHED ? meta.e : e;
                    const bool rise = top > base + kSlack || (base == -INFINITY && top > base);
                    if (__any_sync(0xffffffffu, rise || now_e != e)) {
                        const float now = rise ? top : base;
                        const float keep = rise ? exp2f(base - now) : 1.0f;        // (from nothing: 0)
                        base = now;
                        l *= keep;
                        if (j > 0) {
                            if (NT == 1) {
                                ok = wait_all(smem_u32(&s_o[0]), (j - 1) & 1, abort_flag, watchdog, kWdSoftmax);
                                if (!ok) break;
                                tc_fence_after();
                            }
                            const float f = CACHED ? keep * (e <= -127 ? 0.0f : exp2f((float)(e - now_e))) : keep;
#pragma unroll
                            for (int c = 0; c < DP; c += 32) {
                                uint32_t o[32];
                                tmem_ld32(o_addr + c, o);
                                tmem_ld_wait();
#pragma unroll
                                for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                                tmem_st16(o_addr + c, o);
                                tmem_st16(o_addr + c + 16, o + 16);
                            }
                        }
                        e = now_e;
                    }
                    const float minus = base == -INFINITY ? 0.0f : -base;
                    // ---- probabilities, over the scores that they come from
                    float2 sum0 = make_float2(0.0f, 0.0f), sum1 = sum0;
                    float total = 0.0f;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t p[16];
#pragma unroll
                        for (int g = 2 * c; g < 2 * c + 2; ++g) {
                            // (a masked score, -inf, needs a factor that is not 0 to give 2^-inf)
                            const float f = fmaxf(CACHED ? factor * meta.ks[g] : factor, FLT_MIN);
                            const float z = CACHED ? minus + meta.lvf[g] : minus;
#pragma unroll
                            for (int i = 0; i < 16; i += 2) {
                                float2 x = f2_fma(make_float2(__uint_as_float(v[16 * g + i]), __uint_as_float(v[16 * g + i + 1])), make_float2(f, f), make_float2(z, z));
                                if ((i / 2) % 8 < kPolynomial) x = ex2_polynomial(x);
                                else x = make_float2(ex2(x.x), ex2(x.y));
                                if (i & 2) sum1 = f2_add(sum1, x);
                                else sum0 = f2_add(sum0, x);
                                p[8 * (g % 2) + i / 2] = CACHED ? pack_half(x.x, x.y) : pack_bf16(x.x, x.y);
                            }
                            if (CACHED) {
                                sum0 = f2_add(sum0, sum1);
                                total = fmaf(sum0.x + sum0.y, meta.inv[g], total);
                                sum0 = sum1 = make_float2(0.0f, 0.0f);
                            }
                        }
                        tmem_st16(p_addr + 16 * c, p);
                    }
                    if (!CACHED) {
                        sum0 = f2_add(sum0, sum1);
                        total = sum0.x + sum0.y;
                    }
                    l += total;
                    tmem_st_wait();
                    // Every phase of s_o is waited for, so that none can pass unseen: the next one needs this warp's arrival below.
                    if (NT == 1 && j > 0) {
                        ok = wait_all(smem_u32(&s_o[0]), (j - 1) & 1, abort_flag, watchdog, kWdSoftmax);
                        if (!ok) break;
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(smem_u32(&s_p[buf]));
                        mbar_arrive(smem_u32(&s_used[j % kMetas]));
                    }
                }
                // ---- the rows' results
                if (ok && n > 0) {
                    ok = wait_all(smem_u32(&s_o[S::kPerTile ? mine : 0]), S::kPerTile ? (n - 1) & 1 : 0, abort_flag, watchdog, kWdSoftmax);
                    tc_fence_after();
                }
                if (ok) {
                    const int64_t at = (token * a.q_heads + head) * a.chunks + chunk;
                    const float whole = CACHED ? power_of_two(e / 2) : 1.0f, rest = CACHED ? power_of_two(e - e / 2 - 7) : 1.0f;
                    const float inv = direct ? (l > 0.0f ? 1.0f / l : 0.0f) : 1.0f;
                    __nv_bfloat16* y = static_cast<__nv_bfloat16*>(a.y) + token * a.ldy + head * D;
                    float* part = direct ? nullptr : a.part + at * D;
#pragma unroll
                    for (int c = 0; c < DP; c += 32) {
                        uint32_t o[32];
                        if (n > 0) {
                            tmem_ld32(o_addr + c, o);
                            tmem_ld_wait();
                        } else {
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] = 0u;
                        }
                        float f[32];
#pragma unroll
                        for (int i = 0; i < 32; ++i) f[i] = l > 0.0f ? __uint_as_float(o[i]) * whole * rest * inv : 0.0f;
#pragma unroll
                        for (int x = 0; x < 32; x += 8) {
                            if (!there || c + x >= D) continue;
                            if (direct) {
                                *reinterpret_cast<uint4*>(y + c + x) = make_uint4(pack_bf16(f[x], f[x + 1]), pack_bf16(f[x + 2], f[x + 3]),
                                                                                  pack_bf16(f[x + 4], f[x + 5]), pack_bf16(f[x + 6], f[x + 7]));
                            } else {
                                *reinterpret_cast<float4*>(part + c + x) = make_float4(f[x], f[x + 1], f[x + 2], f[x + 3]);
                                *reinterpret_cast<float4*>(part + c + x + 4) = make_float4(f[x + 4], f[x + 5], f[x + 6], f[x + 7]);
                            }
                        }
                    }
                    if (!direct && there) *reinterpret_cast<float2*>(a.part_ml + 2 * at) = make_float2(base, l);
                    tc_fence_before();
                }
            }
        });
    } else if (warp < 12) {
        fewer_registers<kRegsOther>();
        for_tiles([&](int64_t, bool, int64_t k0, int64_t k1, int n) {
            // ================================================================ keys and values
            const int uses = n * 2 * kParts;                    // of stages: per key tile its keys, then its values
            const int w = warp - 8;
            if (!CACHED) {
                int mends = 0;
                for (int j = 0; j < n && ok; ++j) {
                    KeyMeta& meta = metas[j % kMetas];
                    if (j >= kMetas) ok = mbar_wait_all_lazy(smem_u32(&s_used[j % kMetas]), ((j / kMetas) & 1) ^ 1, abort_flag, watchdog, kWdProducer);
                    if (!ok) break;
                    const KeyPlace p = key_place<false>(a, s, b, hk, k0 + (int64_t)j * kKeys + 32 * w + lane, k1);
                    const uint32_t word = __ballot_sync(0xffffffffu, p.valid);
                    if (lane == 0) {
                        meta.valid[w] = word;
                        mbar_arrive(smem_u32(&s_meta[j % kMetas]));
                    }
                    ok = wait_all(smem_u32(&s_meta[j % kMetas]), (j / kMetas) & 1, abort_flag, watchdog, kWdProducer);
                    if (!ok) break;
                    if (all_valid(meta)) continue;
                    // Zeros for the values of masked keys, the lanes across a row: the MMA warp, which sees the same words, says when
                    // the values are there and waits for the mending.  (The stages' own barriers cannot say it to a warp that looks
                    // at some of their phases only.)
                    ok = wait_all(smem_u32(&s_landed), mends & 1, abort_flag, watchdog, kWdProducer);
                    if (!ok) break;
                    ++mends;
                    for (int part = 0; part < kParts; ++part)
                        for (uint32_t gone = ~word; gone; gone &= gone - 1) {
                            const uint32_t row = stage(2 * kParts * j + kParts + part) + (32 * w + __ffs(gone) - 1) * 128;
#pragma unroll
                            for (int plane = 0; plane < kPlanes; ++plane) sts32(row + plane * 16384 + lane * 4, 0u);
                        }
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&s_fixed));
                }
            } else {
                constexpr int kUnits = kCh / 16;                 // 16-byte units of codes per lane and stage
                const int P = a.cache.page;
                const int32_t* table = a.table + b * a.ld_table;
                auto page_of = [&](int j) -> int32_t {           // of keys 16 (lane % 8) .. of tile j
                    const int64_t key = k0 + (int64_t)j * kKeys + 16 * (lane % 8);
                    if (j >= n || key >= k1) return -1;
                    const int32_t id = (int32_t)ld_global_u32(table + key / P);
                    return id >= 0 && id < a.cache.pages ? id : -1;
                };
                // A warp fills 32 rows (tokens) of a stage of keys, kCh / 4 rows (channels) of a stage of values.  A lane's row in
                // every group of eight is lane / 4 -- eight lanes then store to two neighbouring rows, whose swizzles differ in
                // the lowest bit, and meet all banks -- and its 16 codes of a 64-wide plane are the (lane % 4)th.
                constexpr int kGroups[2] = {4, kCh / 32};        // of eight rows: keys, values
                const int r8 = lane / 4, u4 = lane % 4;
                const uint32_t lo = r8 * 128 + (((2 * u4) ^ r8) * 16), hi = r8 * 128 + (((2 * u4 + 1) ^ r8) * 16);
                // Where a lane's codes of a stage lie: [0], [1] are the two groups of 16 keys, or the two planes of keys.  Codes that
                // no product needs (no page, channels from D on) are read from where there is something, never from beyond.
                const int8_t* src[2];
                int step = 0, plane1 = 0;                        // bytes to the next group of rows; keys: to the second plane
                auto locate = [&](int u, int32_t id) {
                    const int part = u % kParts;
                    if (u < kParts) {
                        const int c = part * 128 + 16 * u4;
                        step = 8 * D;
                        plane1 = c + 64 < D ? 64 : 0;
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const int32_t page = max(__shfl_sync(0xffffffffu, id, 2 * w + x), 0);
                            src[x] = a.cache.k + (((int64_t)page * a.kv_heads + hk) * P + (16 * (2 * w + x)) % P + r8) * D + (c < D ? c : 0);
                        }
                    } else {
                        const int d = part * 128 + w * (kCh / 4) + r8;
                        step = 8 * P;
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const int32_t page = max(__shfl_sync(0xffffffffu, id, u4 + 4 * x), 0);
                            src[x] = a.cache.v + ((int64_t)page * a.kv_heads + hk) * D * P + (int64_t)d * P + (16 * (u4 + 4 * x)) % P;
                        }
                    }
                };
                auto load = [&](int u, int it) -> uint4 {
                    if (u < kParts) {
                        const int rg = it % 4, plane = it / 4;
                        return ld_global_v4(src[rg / 2] + (rg % 2) * step + plane * plane1);
                    }
                    const int rg = it % kGroups[1], plane = it / kGroups[1];
                    const int d = (u % kParts) * 128 + w * (kCh / 4) + r8 + 8 * rg;
                    return ld_global_v4(d < D ? src[plane] + rg * step : a.cache.v);
                };
                uint4 codes[kUnits];                             // of the next stage, each loaded as its forerunner is stored
                int32_t id = page_of(0), id1 = page_of(1), id2;
                float ks = 0.0f, vs = 0.0f;
                auto scales_of = [&](int32_t page, float* k, float* v) {
                    *k = page >= 0 ? ld_global_f32(a.cache.k_scale + (int64_t)page * a.kv_heads + hk) : 0.0f;
                    *v = page >= 0 ? ld_global_f32(a.cache.v_scale + (int64_t)page * a.kv_heads + hk) : 0.0f;
                };
                int e = -127, use = 0;
                if (n > 0) {
                    scales_of(id, &ks, &vs);
#pragma unroll
                    for (int it = 0; it < kUnits; ++it) {
                        if (it == 0) locate(0, id);
                        codes[it] = load(0, it);
                    }
                }
                for (int j = 0; j < n && ok; ++j) {
                    id2 = page_of(j + 2);
                    float ks1, vs1;
                    scales_of(id1, &ks1, &vs1);
#pragma unroll
                    for (int u = 0; u < 2 * kParts; ++u, ++use) {
                        if (use >= kStages) ok = mbar_wait_all_lazy(empty_kv(use), ((use / kStages) & 1) ^ 1, abort_flag, watchdog, kWdProducer);
                        if (!ok) break;
                        if (u == 0) {
                            if (j >= kMetas) ok = mbar_wait_all_lazy(smem_u32(&s_used[j % kMetas]), ((j / kMetas) & 1) ^ 1, abort_flag, watchdog, kWdProducer);
                            if (!ok) break;
                            int top = vs > 0.0f ? exponent_of(vs) + 1 : -127;
#pragma unroll
                            for (int x = 1; x < 8; x <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, x));
                            e = max(e, top);
                            KeyMeta& meta = metas[j % kMetas];
                            const int64_t key = k0 + (int64_t)j * kKeys + 32 * w + lane;
                            const int32_t page = __shfl_sync(0xffffffffu, id, 2 * w + lane / 16);
                            const uint32_t word = __ballot_sync(0xffffffffu, page >= 0 && key < k1);
                            if (lane / 2 == w) {                 // lanes 2 w, 2 w + 1: the warp's two groups of 16 keys
                                meta.ks[lane] = ks;
                                // (values of scale 0 keep a probability, which the sum gets back by `inv` and binary16 rounds to 0)
                                const float lvf = log2f(fmaxf(vs * power_of_two(-e / 2) * power_of_two(7 - e + e / 2), 0x1p-60f));
                                meta.lvf[lane] = lvf;
                                meta.inv[lane] = exp2f(-lvf);
                            }
                            if (lane == 0) {
                                meta.valid[w] = word;
                                if (w == 0) meta.e = e;
                            }
                            __syncwarp();
                            if (lane == 0) mbar_arrive(smem_u32(&s_meta[j % kMetas]));
                        }
                        const int next = u + 1 < 2 * kParts ? u + 1 : 0;
                        locate(next, next ? id : id1);
                        const uint32_t dst = stage(use) + (u < kParts ? 32 * w * 128 : w * (kCh / 4) * 128);
#pragma unroll
                        for (int it = 0; it < kUnits; ++it) {
                            const int groups = kGroups[u < kParts ? 0 : 1];
                            const uint32_t at = dst + (it / groups) * (u < kParts ? 16384 : kCh * 128) + (it % groups) * 1024;
                            const uint4 x = codes[it];
                            codes[it] = load(next, it);
                            uint32_t h[8];
                            widen(x.x, &h[0], &h[1]);
                            widen(x.y, &h[2], &h[3]);
                            widen(x.z, &h[4], &h[5]);
                            widen(x.w, &h[6], &h[7]);
                            sts128(at + lo, h[0], h[1], h[2], h[3]);
                            sts128(at + hi, h[4], h[5], h[6], h[7]);
                        }
                        fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(full_kv(use));
                    }
                    id = id1;
                    id1 = id2;
                    ks = ks1;
                    vs = vs1;
                }
            }
        });
    } else {
        fewer_registers<kRegsOther>();
        for_tiles([&](int64_t, bool, int64_t k0, int64_t, int n) {
            const int uses = n * 2 * kParts;
            if (!CACHED && warp == 13) {
                // ============================================================ TMA: keys, values, keys, ..
                for (int use = 0; use < uses && ok; ++use) {
                    if (use >= kStages) ok = mbar_wait_all_lazy(empty_kv(use), ((use / kStages) & 1) ^ 1, abort_flag, watchdog, kWdProducer);
                    if (!ok) break;
                    const int j = use / (2 * kParts), u = use % (2 * kParts), part = u % kParts;
                    const CUtensorMap* map = u < kParts ? &map_k : &map_v;
                    const int row = (int)(s.k0 + k0 + (int64_t)j * kKeys);
                    if (elect_one()) {
                        mbar_arrive_expect_tx(full_kv(use), S::kStageBytes);
#pragma unroll
                        for (int plane = 0; plane < kPlanes; ++plane)
                            tma_load_3d(stage(use) + plane * 16384, map, part * 128 + plane * 64, hk, row, full_kv(use));
                    }
                    __syncwarp();
                }
                if (!ok && lane == 0) drain_after_abort();
                return;
            }
            // ================================================================ MMA issue
            if (warp != 12 || n == 0) return;
            int mends = 0;                                      // tiles with masked keys so far
            const uint32_t idesc_s = instr_desc_16(CACHED ? 0 : 1, false, kKeys), idesc_o = instr_desc_16(CACHED ? 0 : 1, !CACHED, kCh);
            auto wait_kv = [&](int use) { return wait_all(full_kv(use), (use / kStages) & 1, abort_flag, watchdog, kWdMma); };
            auto scores = [&](int j, int i, int buf) {           // S[buf] = Q_i K_j^T
                if (elect_one()) {
#pragma unroll
                    for (int p = 0; p < kParts; ++p)
#pragma unroll
                        for (int c = 0; c < kPlanes; ++c)
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                mma_f16_ss(tmem + 128 * buf, smem_desc_sw128(q_smem + i * S::kQTile + (p * kPlanes + c) * 16384 + k * 32),
                                           smem_desc_sw128(stage(2 * kParts * j + p) + c * 16384 + k * 32), idesc_s, p + c + k > 0);
                    mma_commit(smem_u32(&s_s[buf]));
                }
                __syncwarp();
            };
            auto products = [&](int j, int i, int buf) {         // O_i += P V_j
                if (elect_one()) {
#pragma unroll
                    for (int p = 0; p < kParts; ++p)
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const uint32_t v = stage(2 * kParts * j + kParts + p);
                            const uint64_t desc = CACHED ? smem_desc_sw128(v + (k / 4) * (kCh * 128) + (k % 4) * 32) : smem_desc_n_major(v + k * 2048);
                            mma_f16_ts(tmem + S::kOCol + i * DP + p * 128, tmem + (S::kEarly ? 384 + 64 * i : 128 * buf) + 8 * k, desc, idesc_o, j > 0 || k > 0);
                        }
                }
                __syncwarp();
            };
            auto release = [&](int first) {                      // stages of a key or value tile, where they are filled again
                if (elect_one()) {
#pragma unroll
                    for (int p = 0; p < kParts; ++p)
                        if (first + p + kStages < uses) mma_commit(empty_kv(first + p));
                }
                __syncwarp();
            };
            ok = wait_all(smem_u32(&s_q), 0, abort_flag, watchdog, kWdMma);
            for (int p = 0; ok && p < kParts; ++p) ok = wait_kv(p);
            if (ok) {
                tc_fence_after();
                for (int i = 0; i < NT; ++i) scores(0, i, i);
                release(0);
            }
            for (int j = 0; j < n && ok; ++j) {
                const int vuse = 2 * kParts * j + kParts, kuse = 2 * kParts * (j + 1);
                if ((NT == 1 || S::kEarly) && j + 1 < n) {
                    for (int p = 0; ok && p < kParts; ++p) ok = wait_kv(kuse + p);
                    for (int i = 0; i < NT && ok; ++i) {
                        if (S::kEarly) ok = wait_all(smem_u32(&s_free[i]), j & 1, abort_flag, watchdog, kWdMma);
                        if (!ok) break;
                        tc_fence_after();
                        scores(j + 1, i, NT == 1 ? (j + 1) & 1 : i);
                    }
                    if (!ok) break;
                    release(kuse);
                }
                for (int i = 0; i < NT && ok; ++i) {
                    const int buf = NT == 2 ? i : j & 1;
                    ok = wait_all(smem_u32(&s_p[buf]), NT == 2 ? j & 1 : (j >> 1) & 1, abort_flag, watchdog, kWdMma);
                    for (int p = 0; ok && i == 0 && p < kParts; ++p) ok = wait_kv(vuse + p);
                    if (!CACHED && ok && i == 0) {
                        ok = wait_all(smem_u32(&s_meta[j % kMetas]), (j / kMetas) & 1, abort_flag, watchdog, kWdMma);
                        const bool clean = all_valid(metas[j % kMetas]);
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&s_used[j % kMetas]));
                        if (!clean && ok) {
                            if (lane == 0) mbar_arrive(smem_u32(&s_landed));
                            ok = wait_all(smem_u32(&s_fixed), mends & 1, abort_flag, watchdog, kWdMma);
                            ++mends;
                        }
                    }
                    if (!ok) break;
                    tc_fence_after();
                    products(j, i, buf);
                    if (S::kPerTile || (j + 1 == n && i + 1 == NT)) {
                        if (elect_one()) mma_commit(smem_u32(&s_o[S::kPerTile ? i : 0]));
                        __syncwarp();
                    }
                    if (NT == 2 && !S::kEarly && j + 1 < n) {
                        for (int p = 0; ok && i == 0 && p < kParts; ++p) ok = wait_kv(kuse + p);
                        if (!ok) break;
                        scores(j + 1, i, i);
                    }
                }
                if (!ok) break;
                release(vuse);
                if (NT == 2 && !S::kEarly && j + 1 < n) release(kuse);
            }
        });
    }
    if (!ok && warp == 12) drain_after_abort();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 12) tmem_dealloc<1>(tmem, 512);
}

template <int DP, int NT, bool CACHED>
cudaError_t launch(const Attention& a, cudaStream_t stream) {
    auto* kern = attention_tiles_kernel<DP, NT, CACHED>;
    uint32_t* watchdog = watchdog_device_ptr();
    if (!watchdog) return cudaErrorUnknown;
    // (the softmax would wait for ever for registers that the launch does not bring)
    static const bool enough = [&] {
        cudaFuncAttributes f;
        return cudaFuncGetAttributes(&f, reinterpret_cast<const void*>(kern)) == cudaSuccess && f.numRegs == kRegsLaunch;
    }();
    if (!enough) return cudaErrorUnknown;
    const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kern), Shape<DP, NT>::kSmem);
    if (e != cudaSuccess) return e;
    CUtensorMap map_k = {}, map_v = {};
    if (!CACHED && a.kv_rows > 0) {                             // channels of a head, heads, rows
        const uint64_t dims[3] = {(uint64_t)a.head_dim, (uint64_t)a.kv_heads, (uint64_t)a.kv_rows};
        const uint32_t box[3] = {64, 1, kKeys};
        const uint64_t head = (uint64_t)a.head_dim * 2, sk[2] = {head, (uint64_t)a.ldk * 2}, sv[2] = {head, (uint64_t)a.ldv * 2};
        if (!encode_tiled(&map_k, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, a.k, dims, sk, box, CU_TENSOR_MAP_SWIZZLE_128B) ||
            !encode_tiled(&map_v, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, a.v, dims, sv, box, CU_TENSOR_MAP_SWIZZLE_128B))
            return cudaErrorUnknown;
    }
    const dim3 grid((unsigned)row_tiles(a), (unsigned)a.chunks, (unsigned)(a.batch * a.kv_heads));
    return launch_pdl3(kern, grid, kThreads, Shape<DP, NT>::kSmem, stream, a, map_k, map_v, watchdog);
}
template <bool CACHED>
cudaError_t by_width(const Attention& a, cudaStream_t stream) {
    if (a.head_dim > 128) return launch<256, 1, CACHED>(a, stream);
    if (a.head_dim > 64) return a.tile_rows == 256 ? launch<128, 2, CACHED>(a, stream) : launch<128, 1, CACHED>(a, stream);
    return a.tile_rows == 256 ? launch<64, 2, CACHED>(a, stream) : launch<64, 1, CACHED>(a, stream);
}

}  // namespace

cudaError_t launch_attention_tiles(const Attention& a, cudaStream_t stream) {
    return a.cached ? by_width<true>(a, stream) : by_width<false>(a, stream);
}

}  // namespace fq
