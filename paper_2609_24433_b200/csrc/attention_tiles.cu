// Attention of many queries on the tcgen05 tensor cores: bf16 keys and values as rows (cross attention) or the 8-bit cache.
//
// A CTA takes one chunk of the keys of one kv head and NT tiles of 128 rows -- (token, head of a group) pairs, so that a group
// reads its keys once.  Per tile of 128 keys: S = Q K^T into TMEM; a thread per row (two where there is one row tile) keeps the
// running maximum and sum and writes the probabilities, 16 bits each, over S in TMEM; O += P V takes them from there as its first
// operand.
//   warps 0-7    softmax: a warpgroup per row tile, or the two halves of a row
//   warps 8-11   which keys of a tile there are, the scales of cached ones
//   warp 12      issues the MMAs (D = 64 and two row tiles: those of the first one, warp 14 those of the second)
//   warp 13      copies keys and values by TMA into 128-byte-swizzled stages of 128 keys x 64 or 128 channels (the others up to 15
//                complete the warpgroup, whose registers go to the softmax)
// With two row tiles (D <= 128) the tensor core works on one while the other's probabilities are computed; with one (D > 128,
// or few rows) S is double-buffered instead.
//
// The maximum is followed lazily: O and l are rescaled only where a row's maximum has risen by more than 2^8 over the base they
// were built with, so almost never behind the first tiles; probabilities then reach 256, which changes no relative rounding.  Maxima
// carry NaN, and a row's maximum is -inf where it sees no key and nowhere else.
//
// Cache: the codes come widened to binary16, exactly, by a kernel ahead (attention_widen.cu): as many row tiles read a key as there
// are, and widening it for each of them on its way into the stages bounded the kernel (4 warps at it: 32 x 50 queries x 8 heads of
// 256 over 866 keys 49 us, 3 x 4096 tokens x 16 heads of 128 over 6656 keys 660).  The scale of a page's keys multiplies S per 16
// columns; that of its values multiplies the probabilities, over 2^e with e the running exponent of the largest one:
// P = p vs 2^(7 - e) <= 2^15.  Queries: binary16 behind a power of two per row.
// Measured: 16 x 1023 queries x 4100 states, 16 heads of 64: 458 to 479 us = 575 to 600 TFLOP/s (the exponential unit alone: 245 us); 3 x 4096
// queries over 6656 cached keys, 16/4 heads of 128, causal, with the widening: 490 to 500 us; 8 x 1024 queries x 4096 states, 16 heads of
// 128: 298 us = 920 TFLOP/s over the 3.5 waves of its CTAs.  Bound by what each row tile does in turn -- scores, maximum, exponentials, hand-over --
// of which a scheduler has two to overlap.
// Rows: bf16 operands, the probabilities too, as an MMA takes one type and values of any size are no binary16: at most 2^-8 each, which puts
// results 2.1e-3 to 2.3e-3 from those of 64 bits where bf16 outputs alone are 1.7e-3 away.  The scores of masked keys are replaced; their values are zeroed in shared memory, in the tiles that have
// any, ahead of the product: 0 times a masked NaN would reach the sums.
#include "act_common.cuh"
#include "attention_common.cuh"
#include "tc_sm100.cuh"

#include <cuda_fp16.h>
#include <float.h>

#include <type_traits>

namespace fq {
namespace {

constexpr int kThreads = 16 * 32, kSoftmaxWarps = 8, kLoadWarp = 8, kMmaWarp = 12, kTmaWarp = 13, kSecondMmaWarp = 14;
// Registers: a softmax thread holds a row of 128 scores.  The launch's 512 x 128 are shared out as 256 x 200 + 256 x 56.
constexpr int kRegsLaunch = 128, kRegsSoftmax = 200, kRegsOther = 56;
static_assert(256 * kRegsSoftmax + 256 * kRegsOther <= kThreads * kRegsLaunch, "");
constexpr int kKeys = 128;
constexpr int kMetas = 4;
constexpr float kSlack = 8.0f;          // log2 of how far a row's maximum may rise over its base
constexpr float kHuge = 4096.0f;        // bases from here on are subtracted from rounded scores

constexpr uint32_t kWdProducer = 0x800u, kWdMma = 0x1000u, kWdSoftmax = 0x2000u;

struct __align__(16) KeyMeta {
    float ks[8];                        // per 16 keys
    float lvf[8];                       // log2 of vs 2^(7 - e)
    float inv[8];                       // 2^-lvf
    uint32_t valid[4];
    int e;
    int unused[3];
};
// What the roles share beside the tiles.
template <int STAGES>
struct __align__(16) Control {
    float rows[256];                    // maxima, sums on their way between the threads of a row
    KeyMeta metas[kMetas];
    uint64_t full_kv[STAGES], empty_kv[STAGES], meta[kMetas], used[kMetas], landed, fixed, s[2], p[2], o[2], free[2], turn[8], q;
    uint32_t tmem;
    int abort;
};

template <int DP, int NT>
struct Shape {
    static constexpr int kParts = DP == 256 ? 2 : 1;            // stages per key or value tile
    static constexpr int kCh = DP / kParts;                     // channels per stage
    static constexpr int kStageBytes = kKeys * kCh * 2;
    static constexpr int kStages = DP == 64 ? 8 : 5;
    static constexpr int kQTile = 128 * DP * 2;
    static constexpr int kTiles = NT * kQTile + kStages * kStageBytes;
    static constexpr int kSmem = kTiles + (int)sizeof(Control<kStages>);
    static constexpr int kSplit = 2 / NT;                       // threads per row
    static constexpr int kCols = 128 / kSplit;                  // ... and the columns of S of each
    static constexpr int kOCol = 256;                           // S: columns 0 .. 255
    // Two tiles of 64 channels leave TMEM for probabilities of their own (columns 384 ..): the next scores are computed as soon
    // as the last ones have been read.  Elsewhere probabilities lie over their scores.
    static constexpr bool kEarly = NT == 2 && DP == 64;
    // The two row tiles then have an issuing warp each, and the two warps of a scheduler take turns at the exponentials (`turn`):
    // left alone they meet there, wait for the unit together and leave it idle together at everything else.  (48 x 8 heads of 64,
    // 1024 queries x 1500 keys: one warp 557 us, two 533, and turns 484; turns handed over a quarter early 527.  D = 128, where
    // S cannot be freed early: turns 329 against 316.)
    static constexpr int kIssuers = kEarly ? 2 : 1;
    static constexpr bool kAhead = NT == 1 || kEarly;           // scores of tile j + 1 are issued ahead of the products of tile j
    // Stages are filled in the order in which they are needed: K0 V0 K1 V1 .., or ahead: K0 K1 V0 K2 V1 ..  First use by the keys,
    // by the values of tile j of n.
    static __device__ __forceinline__ int keys(int j) { return kParts * (kAhead && j > 0 ? 2 * j - 1 : 2 * j); }
    static __device__ __forceinline__ int values(int j, int n) { return kParts * (kAhead && j + 1 < n ? 2 * j + 2 : 2 * j + 1); }
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
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ int exponent_of(float x) { return (int)((__float_as_uint(x) >> 23) & 255) - 127; }
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(min(max(e, -126), 127) + 127) << 23); }
// Maxima that a NaN among the operands reaches.
__device__ __forceinline__ float max3(float x, uint32_t y, uint32_t z) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(__uint_as_float(y)), "f"(__uint_as_float(z)));
    return r;
}
__device__ __forceinline__ float max2(float x, float y) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
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
constexpr int kPolynomial = 1;
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
// The issuing thread is the bottleneck of a tile where it computes a descriptor for every MMA (124 cycles each were measured
// against the tensor core's 64): low words advance by constants, high words and predicates are constant.
template <bool ACCUMULATE>
__device__ __forceinline__ void mma_f16_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t high, uint32_t idesc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %5, 0;\n\t"
        "mov.b64 a, {%1, %3};\n\tmov.b64 b, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %4, p;\n\t}"
        ::"r"(d), "r"(a), "r"(b), "r"(high), "r"(idesc), "n"(ACCUMULATE ? 1 : 0)
        : "memory");
}
template <bool ACCUMULATE>
__device__ __forceinline__ void mma_f16_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t high, uint32_t idesc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 b;\n\tsetp.ne.b32 p, %5, 0;\n\t"
        "mov.b64 b, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n\t}"
        ::"r"(d), "r"(a), "r"(b), "r"(high), "r"(idesc), "n"(ACCUMULATE ? 1 : 0)
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
// mbar_wait_all for two barriers, which are looked at together, with the bounded loop in line: a kernel that calls a function keeps
// its launch's registers in every warp.
__device__ __forceinline__ bool wait_all(uint32_t first, uint32_t first_parity, uint32_t bar, uint32_t parity, volatile int* abort_flag, uint32_t* watchdog, uint32_t code) {
    bool ok = true;
    const bool one = mbar_try_wait(first, first_parity), other = bar == first || mbar_try_wait(bar, parity);
    if (!(one && other)) {
        uint64_t t0 = 0;
        for (uint32_t spin = 1; !(mbar_try_wait(first, first_parity) && (bar == first || mbar_try_wait(bar, parity))); ++spin) {
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
__device__ __forceinline__ bool wait_all(uint32_t bar, uint32_t parity, volatile int* abort_flag, uint32_t* watchdog, uint32_t code) {
    return wait_all(bar, parity, bar, parity, abort_flag, watchdog, code);
}
__device__ __forceinline__ void mbar_inval(uint32_t bar) { asm volatile("mbarrier.inval.shared::cta.b64 [%0];" ::"r"(bar) : "memory"); }

__device__ __forceinline__ bool all_valid(const KeyMeta& m) { return (m.valid[0] & m.valid[1] & m.valid[2] & m.valid[3]) == ~0u; }

template <int DP, int NT, bool CACHED>
__global__ void __launch_bounds__(kThreads, 1) attention_tiles_kernel(const Attention a, const __grid_constant__ CUtensorMap map_k,
                                                                      const __grid_constant__ CUtensorMap map_v, uint32_t* watchdog) {
    using S = Shape<DP, NT>;
    constexpr int kCh = S::kCh, kParts = S::kParts, kStages = S::kStages, kPlanes = kCh / 64;
    constexpr int kSplit = S::kSplit, kCols = S::kCols;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    Control<kStages>& ctl = *reinterpret_cast<Control<kStages>*>(smem_raw + S::kTiles);
    volatile int* abort_flag = &ctl.abort;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const bool issues = warp == kMmaWarp || (S::kIssuers == 2 && warp == kSecondMmaWarp);
    const uint32_t q_smem = smem_u32(smem_raw), ring = q_smem + NT * S::kQTile;
    if (q_smem & 1023u) {                                       // (swizzled tiles start on 1024 bytes; nothing else is in shared memory)
        if (threadIdx.x == 0) atomicOr(watchdog, kWdProducer);
        return;
    }
    auto full_kv = [&](int n) { return smem_u32(&ctl.full_kv[n % kStages]); };
    auto empty_kv = [&](int n) { return smem_u32(&ctl.empty_kv[n % kStages]); };
    auto stage = [&](int n) { return ring + (uint32_t)(n % kStages) * S::kStageBytes; };

    auto init_barriers = [&]() {
        for (int i = 0; i < kStages; ++i) { mbar_init(smem_u32(&ctl.full_kv[i]), 1); mbar_init(smem_u32(&ctl.empty_kv[i]), S::kIssuers); }
        for (int i = 0; i < kMetas; ++i) { mbar_init(smem_u32(&ctl.meta[i]), 4); mbar_init(smem_u32(&ctl.used[i]), kSoftmaxWarps + (CACHED ? 0 : S::kIssuers)); }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&ctl.s[i]), 1);
            mbar_init(smem_u32(&ctl.p[i]), 4 * kSplit);
            mbar_init(smem_u32(&ctl.o[i]), 1);
            mbar_init(smem_u32(&ctl.free[i]), 4 * kSplit);
        }
        mbar_init(smem_u32(&ctl.q), kSoftmaxWarps);
        for (int i = 0; i < 8; ++i) mbar_init(smem_u32(&ctl.turn[i]), 1);
        mbar_init(smem_u32(&ctl.landed), S::kIssuers);
        mbar_init(smem_u32(&ctl.fixed), 4);
        fence_mbarrier_init();
    };
    if (threadIdx.x == 0) {
        ctl.abort = 0;
        init_barriers();
    }
    if (warp == kMmaWarp) tmem_alloc<1>(smem_u32(&ctl.tmem), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = ctl.tmem;
    griddep_wait();

    const int unit = a.first_unit + blockIdx.z, b = unit / a.kv_heads, hk = unit % a.kv_heads, chunk = blockIdx.y;
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
                    for (uint64_t* bar = ctl.full_kv; bar <= &ctl.q; ++bar) mbar_inval(smem_u32(bar));
                    init_barriers();
                }
                __syncthreads();
            }
            again = true;
            body(tile, tk.chunks <= 1, k0, k1, (int)((k1 - k0 + kKeys - 1) / kKeys));
            __syncthreads();
            ok = ctl.abort == 0;
        }
    };

    if (warp < kSoftmaxWarps) {
        more_registers<kRegsSoftmax>();
        for_tiles([&](int64_t tile, bool direct, int64_t k0, int64_t k1, int n) {
            // ================================================================ softmax
            // Warps of equal warp % 4 see the same lanes of TMEM: row tile warp / 4 / kSplit, columns kCols split .. of it.
            const int mine = warp / (4 * kSplit), split = warp / 4 % kSplit;
            const int r = mine * 128 + (warp % 4) * 32 + lane;
            const int64_t row = tile * kRows + r;
            const bool there = row < rows;
            const int64_t token = s.q0 + (there ? row / G : 0), head = hk * G + (there ? row % G : 0);
            float* const seat = ctl.rows + r;                    // this row's, NT * 128 apart by split
            auto meet = [&]() { if (kSplit > 1) asm volatile("bar.sync %0, %1;" ::"r"(1 + mine * 4 + warp % 4), "n"(32 * kSplit) : "memory"); };
            float factor = a.scale_log2;
            {
                // ---- this thread's part of its row of Q
                const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(a.q) + token * a.ldq + head * D;
                const uint32_t dst = q_smem + mine * S::kQTile + (r % 128) * 128;
                float down = 1.0f;
                // (Factors are held at FLT_MIN or more below, where a masked -inf needs one; products of rows reach 2^128 and would show it.)
                const bool tiny = !CACHED && a.scale_log2 < FLT_MIN;
                if (tiny) {
                    down = 0x1p-64f;
                    factor = a.scale_log2 * 0x1p64f;
                }
                if (CACHED) {
                    float top = 0.0f;
#pragma unroll 8
                    for (int d = 0; d < DP; d += 8) {            // (eight loads under way; one by one, 50 queries of 16 heads of 64 over 816 keys took 13.6 us for 11.3)
                        const uint4 v = ld_global_v4(src + d, there && d < D);
                        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) top = fmaxf(top, fmaxf(fabsf(__uint_as_float(w[i] << 16)), fabsf(__uint_as_float(w[i] & 0xffff0000u))));
                    }
                    const int e = min(max(exponent_of(top), -100), 126);
                    down = power_of_two(-e);
                    factor = a.scale_log2 * power_of_two(e);
                }
#pragma unroll 8
                for (int x = 0; x < DP / kSplit; x += 8) {
                    const int d = split * (DP / kSplit) + x;
                    uint4 v = ld_global_v4(src + d, there && d < D);
                    if (CACHED) {
                        uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) w[i] = pack_half(__uint_as_float(w[i] << 16) * down, __uint_as_float(w[i] & 0xffff0000u) * down);
                        v = make_uint4(w[0], w[1], w[2], w[3]);
                    } else if (tiny) {
                        uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) w[i] = pack_bf16(__uint_as_float(w[i] << 16) * down, __uint_as_float(w[i] & 0xffff0000u) * down);
                        v = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                    sts128(dst + (d / 64) * 16384 + ((((d % 64) / 8) ^ (r & 7)) * 16), v.x, v.y, v.z, v.w);
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&ctl.q));
            }
            constexpr int kOCols = DP / kSplit;                  // columns of O that this warp rescales and stores
            const uint32_t lanes = tmem + ((uint32_t)(warp % 4) << 21);
            const uint32_t o_addr = lanes + S::kOCol + (NT == 2 ? mine * DP : 0) + split * kOCols;
            const int64_t limit64 = row_limit(a, s, row);
            float base = -INFINITY, l = 0.0f;
            int e = -127;
            // (Each warp comes to every meeting, also once a wait has run out: the others may be there already.)
            for (int j = 0; j < n; ++j) {
                const int buf = NT == 2 ? mine : j & 1;
                const uint32_t phase = NT == 2 ? j & 1 : (j >> 1) & 1;
                ok = ok && wait_all(smem_u32(&ctl.meta[j % kMetas]), (j / kMetas) & 1, smem_u32(&ctl.s[buf]), phase, abort_flag, watchdog, kWdSoftmax);
                if (!ok) {
                    meet();
                    meet();
                    continue;
                }
                tc_fence_after();
                const KeyMeta& meta = ctl.metas[j % kMetas];
                const uint32_t s_addr = lanes + 128 * buf + split * kCols;
                const uint32_t p_addr = (S::kEarly ? lanes + 384 + 64 * mine : lanes + 128 * buf) + split * (kCols / 2);
                const int lim = (int)min(max(limit64 - (k0 + (int64_t)j * kKeys), (int64_t)-1), (int64_t)kKeys) - split * kCols;
                uint32_t seen[kCols / 32];
                bool partly = false, sees = false;
#pragma unroll
                for (int c = 0; c < kCols / 32; ++c) {
                    const int x = lim - 32 * c;
                    seen[c] = meta.valid[split * (kCols / 32) + c] & (x < 0 ? 0u : x >= 31 ? ~0u : (2u << x) - 1u);
                    partly = partly || seen[c] != ~0u;
                    sees = sees || seen[c] != 0u;
                }
                const bool masked = __any_sync(0xffffffffu, partly);
                const float* const ks = meta.ks + split * (kCols / 16);
                uint32_t v[kCols];
#pragma unroll
                for (int c = 0; c < kCols / 32; ++c) tmem_ld32(s_addr + 32 * c, v + 32 * c);
                tmem_ld_wait();
                if (masked) {                                    // (a branch: selects on every score cost a third of the loop)
#pragma unroll
                    for (int i = 0; i < kCols; ++i)
                        if (!((seen[i / 32] >> (i % 32)) & 1)) v[i] = 0xff800000u;
                }
                // ---- the largest score.  (A masked one, -inf, needs a factor that is not 0 to stay it.)
                float top = -INFINITY;
#pragma unroll
                for (int g = 0; g < kCols / 16; ++g) {
                    float x = -INFINITY, y = -INFINITY;
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        x = max3(x, v[16 * g + i], v[16 * g + i + 1]);
                        y = max3(y, v[16 * g + i + 2], v[16 * g + i + 3]);
                    }
                    top = max2(top, CACHED ? max2(x, y) * fmaxf(factor * ks[g], FLT_MIN) : max2(x, y));
                }
                if (!CACHED) top *= fmaxf(factor, FLT_MIN);
                if (sees) top = max2(top, -FLT_MAX);             // (-inf stays to rows that see nothing)
                if (kSplit > 1) {
                    seat[split * NT * 128] = top;
                    meet();                                      // (and all of them have read their scores)
#pragma unroll
                    for (int i = 0; i < kSplit; ++i) top = max2(top, seat[i * NT * 128]);
                    meet();                                      // (the next maxima may come)
                }
                if (S::kEarly) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&ctl.free[mine]));
                }
                // ---- a new base
                const int now_e = CACHED ? meta.e : e;
                const bool rise = !(top <= base + kSlack) && base == base;      // (a NaN becomes the base and stays it: all of the row is NaN)
                if (__any_sync(0xffffffffu, rise || now_e != e)) {
                    const float now = rise ? top : base;
                    const float keep = rise ? exp2f(base - now) : 1.0f;                // (from nothing: 0)
                    base = now;
                    l *= keep;
                    if (j > 0) {
                        if (S::kAhead) {
                            ok = wait_all(smem_u32(&ctl.o[mine]), (j - 1) & 1, abort_flag, watchdog, kWdSoftmax);
                            if (!ok) continue;
                            tc_fence_after();
                        }
                        const float f = CACHED ? keep * (e <= -127 ? 0.0f : exp2f((float)(e - now_e))) : keep;
#pragma unroll 1
                        for (int c = 0; c < kOCols; c += 16) {
                            uint32_t o[16];
                            tmem_ld16(o_addr + c, o);
                            tmem_ld_wait();
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                            tmem_st16(o_addr + c, o);
                        }
                    }
                    e = now_e;
                }
                // score - base is one FMA, exact up to the base's own rounding: of a base of 2^27 that is up to 2^3, by which the largest
                // probability would miss 1 (and its 16 bits).  Huge scores are rounded as their base was and subtracted here.
                float minus = base == -INFINITY ? 0.0f : -base;
                const bool huge = fabsf(minus) >= kHuge;
                if (__any_sync(0xffffffffu, huge)) {
#pragma unroll
                    for (int i = 0; i < kCols; ++i) {
                        const float x = __uint_as_float(v[i]);
                        v[i] = huge ? __float_as_uint(__fadd_rn(__fmul_rn(x, fmaxf(CACHED ? factor * ks[i / 16] : factor, FLT_MIN)), minus)) : v[i];
                    }
                    minus = huge ? 0.0f : minus;
                }
                if (S::kEarly && j + mine > 0) {                 // its turn at the exponentials; the last product has read its probabilities
                    const uint32_t turn = smem_u32(&ctl.turn[warp]), turn_phase = (j - 1 + mine) & 1;
                    ok = wait_all(j > 0 ? smem_u32(&ctl.o[mine]) : turn, j > 0 ? (j - 1) & 1 : turn_phase, turn, turn_phase, abort_flag, watchdog, kWdSoftmax);
                    if (!ok) continue;
                    tc_fence_after();
                }
                // ---- probabilities, over the scores or beside them
                float2 sum0 = make_float2(0.0f, 0.0f), sum1 = sum0;
                float total = 0.0f;
#pragma unroll
                for (int c = 0; c < kCols / 32; ++c) {
                    uint32_t p[16];
#pragma unroll
                    for (int g = 2 * c; g < 2 * c + 2; ++g) {
                        const float f = huge ? 1.0f : fmaxf(CACHED ? factor * ks[g] : factor, FLT_MIN);
                        const float z = CACHED ? minus + meta.lvf[split * (kCols / 16) + g] : minus;
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
                            total = fmaf(sum0.x + sum0.y, meta.inv[split * (kCols / 16) + g], total);
                            sum0 = sum1 = make_float2(0.0f, 0.0f);
                        }
                    }
                    tmem_st16(p_addr + 16 * c, p);
                }
                if (S::kEarly && lane == 0) mbar_arrive(smem_u32(&ctl.turn[warp ^ 4]));
                if (!CACHED) {
                    sum0 = f2_add(sum0, sum1);
                    total = sum0.x + sum0.y;
                }
                l += total;
                tmem_st_wait();
                // Every phase of ctl.o is waited for, so that none can pass unseen: the next one needs this warp's arrival below.
                if (NT == 1 && j > 0) {
                    ok = wait_all(smem_u32(&ctl.o[0]), (j - 1) & 1, abort_flag, watchdog, kWdSoftmax);
                    if (!ok) continue;
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(smem_u32(&ctl.p[buf]));
                    mbar_arrive(smem_u32(&ctl.used[j % kMetas]));
                }
            }
            // ---- the rows' results
            if (ok && n > 0) {
                ok = wait_all(smem_u32(&ctl.o[mine]), S::kAhead ? (n - 1) & 1 : 0, abort_flag, watchdog, kWdSoftmax);
                tc_fence_after();
            }
            if (kSplit > 1) {
                seat[split * NT * 128] = l;
                meet();
                l = 0.0f;
#pragma unroll
                for (int i = 0; i < kSplit; ++i) l += seat[i * NT * 128];
            }
            // The key with the base has 2^0, give or take the roundings.  What is far below is no sum but the 2^-126, by `inv` up to 2^-66,
            // that ex2_polynomial gives each key at -inf, masked or not.
            if (l < 0x1p-20f) l = 0.0f;
            const bool any = base != -INFINITY;                  // the row sees a key
            if (ok) {
                const int64_t at = (token * a.q_heads + head) * a.chunks + chunk;
                const float whole = CACHED ? power_of_two(e / 2) : 1.0f, rest = CACHED ? power_of_two(e - e / 2 - 7) : 1.0f;
                const float inv = direct ? reciprocal_sum(base, l) : 1.0f;
                __nv_bfloat16* y = static_cast<__nv_bfloat16*>(a.y) + token * a.ldy + head * D + split * kOCols;
                float* part = direct ? nullptr : a.part + at * D + split * kOCols;
#pragma unroll 1
                for (int c = 0; c < kOCols; c += 16) {
                    uint32_t o[16];
                    if (n > 0) {
                        tmem_ld16(o_addr + c, o);
                        tmem_ld_wait();
                    }
                    float f[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) f[i] = any ? __uint_as_float(o[i]) * whole * rest * inv : 0.0f;
                    if (!there || split * kOCols + c >= D) continue;           // (D is a multiple of 16)
#pragma unroll
                    for (int x = 0; x < 16; x += 8) {
                        if (direct) {
                            *reinterpret_cast<uint4*>(y + c + x) = make_uint4(pack_bf16(f[x], f[x + 1]), pack_bf16(f[x + 2], f[x + 3]),
                                                                              pack_bf16(f[x + 4], f[x + 5]), pack_bf16(f[x + 6], f[x + 7]));
                        } else {
                            *reinterpret_cast<float4*>(part + c + x) = make_float4(f[x], f[x + 1], f[x + 2], f[x + 3]);
                            *reinterpret_cast<float4*>(part + c + x + 4) = make_float4(f[x + 4], f[x + 5], f[x + 6], f[x + 7]);
                        }
                    }
                }
                if (!direct && there && split == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * at) = make_float2(base, l);
                tc_fence_before();
            }
        });
    } else if (warp < kMmaWarp) {
        fewer_registers<kRegsOther>();
        for_tiles([&](int64_t, bool, int64_t k0, int64_t k1, int n) {
            // ================================================================ which keys there are
            const int w = warp - kLoadWarp;
            if (!CACHED) {
                int mends = 0;
                for (int j = 0; j < n && ok; ++j) {
                    KeyMeta& meta = ctl.metas[j % kMetas];
                    if (j >= kMetas) ok = mbar_wait_all_lazy(smem_u32(&ctl.used[j % kMetas]), ((j / kMetas) & 1) ^ 1, abort_flag, watchdog, kWdProducer);
                    if (!ok) break;
                    const KeyPlace p = key_place<false>(a, s, b, hk, k0 + (int64_t)j * kKeys + 32 * w + lane, k1);
                    const uint32_t word = __ballot_sync(0xffffffffu, p.valid);
                    if (lane == 0) {
                        meta.valid[w] = word;
                        mbar_arrive(smem_u32(&ctl.meta[j % kMetas]));
                    }
                    ok = wait_all(smem_u32(&ctl.meta[j % kMetas]), (j / kMetas) & 1, abort_flag, watchdog, kWdProducer);
                    if (!ok) break;
                    if (all_valid(meta)) continue;
                    // Zeros for the values of masked keys, the lanes across a row: the MMA warp, which sees the same words, says when
                    // the values are there and waits for the mending.  (The stages' own barriers cannot say it to a warp that looks
                    // at some of their phases only.)
                    ok = wait_all(smem_u32(&ctl.landed), mends & 1, abort_flag, watchdog, kWdProducer);
                    if (!ok) break;
                    ++mends;
                    for (int part = 0; part < kParts; ++part)
                        for (uint32_t gone = ~word; gone; gone &= gone - 1) {
                            const uint32_t row = stage(S::values(j, n) + part) + (32 * w + __ffs(gone) - 1) * 128;
#pragma unroll
                            for (int plane = 0; plane < kPlanes; ++plane) sts32(row + plane * 16384 + lane * 4, 0u);
                        }
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&ctl.fixed));
                }
            } else {
                const int32_t* table = a.table + b * a.ld_table;
                auto page_of = [&](int j) -> int32_t {           // (page, head) of keys 16 (lane % 8) .. of tile j, -1 where there is none
                    const int64_t key = k0 + (int64_t)j * kKeys + 16 * (lane % 8);
                    if (j >= n || key >= k1) return -1;
                    const int32_t id = (int32_t)ld_global_u32(table + key / a.cache.page);
                    return id >= 0 && id < a.cache.pages ? id * a.kv_heads + hk : -1;
                };
                int32_t id = page_of(0), id1 = page_of(1);
                float ks = id >= 0 ? ld_global_f32(a.cache.k_scale + id) : 0.0f, vs = id >= 0 ? ld_global_f32(a.cache.v_scale + id) : 0.0f;
                int e = -127;
                for (int j = 0; j < n && ok; ++j) {
                    if (j >= kMetas) ok = mbar_wait_all_lazy(smem_u32(&ctl.used[j % kMetas]), ((j / kMetas) & 1) ^ 1, abort_flag, watchdog, kWdProducer);
                    if (!ok) break;
                    const int32_t id2 = page_of(j + 2);
                    const float ks1 = id1 >= 0 ? ld_global_f32(a.cache.k_scale + id1) : 0.0f, vs1 = id1 >= 0 ? ld_global_f32(a.cache.v_scale + id1) : 0.0f;
                    e = max(e, __reduce_max_sync(0xffffffffu, vs > 0.0f ? exponent_of(vs) + 1 : -127));
                    KeyMeta& meta = ctl.metas[j % kMetas];
                    const int64_t key = k0 + (int64_t)j * kKeys + 32 * w + lane;
                    const uint32_t word = __ballot_sync(0xffffffffu, __shfl_sync(0xffffffffu, id, 2 * w + lane / 16) >= 0 && key < k1);
                    if (lane / 2 == w) {                         // lanes 2 w, 2 w + 1: the warp's two groups of 16 keys
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
                    if (lane == 0) mbar_arrive(smem_u32(&ctl.meta[j % kMetas]));
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
            if (warp == kTmaWarp) {
                // ============================================================ TMA
                int use = 0;
                auto copy = [&](bool keys, int j) {
                    for (int part = 0; part < kParts && ok; ++part, ++use) {
                        if (use >= kStages) ok = mbar_wait_all_lazy(empty_kv(use), ((use / kStages) & 1) ^ 1, abort_flag, watchdog, kWdProducer);
                        if (ok && elect_one()) {
                            const uint32_t bar = full_kv(use);
                            const int key = (int)(k0 + (int64_t)j * kKeys);
                            mbar_arrive_expect_tx(bar, S::kStageBytes);
                            if (CACHED && !keys) {               // two planes of 64 keys, rows are channels
#pragma unroll
                                for (int plane = 0; plane < 2; ++plane)
                                    tma_load_3d(stage(use) + plane * (kCh * 128), &map_v, key + 64 * plane, part * 128, (int)blockIdx.z, bar);
                            } else {                             // planes of 64 channels, rows are keys
#pragma unroll
                                for (int plane = 0; plane < kPlanes; ++plane) {
                                    if (CACHED) tma_load_3d(stage(use) + plane * 16384, &map_k, part * 128 + plane * 64, key, (int)blockIdx.z, bar);
                                    else tma_load_3d(stage(use) + plane * 16384, keys ? &map_k : &map_v, part * 128 + plane * 64, hk, (int)s.k0 + key, bar);
                                }
                            }
                        }
                        __syncwarp();
                    }
                };
                for (int kt = 0, vt = 0; vt < n && ok;) {        // (in the order of S::keys and S::values)
                    if (kt < n && kt <= vt + (S::kAhead ? 1 : 0)) copy(true, kt++);
                    else copy(false, vt++);
                }
                if (!ok && lane == 0) drain_after_abort();
                return;
            }
            // ================================================================ MMA issue
            // With D = 128 one warp serves both row tiles in turn, products and next scores of one back to back: they then work half a period apart,
            // one at the exponentials, one at the tensor core.  (A warp for each let the MMAs of both mix, so that both ended
            // together and met again: 1.4 times the time.)
            if (!issues || n == 0) return;
            const int lo = warp == kMmaWarp ? 0 : 1, hi = S::kIssuers == 2 ? lo + 1 : NT;         // this warp's row tiles
            int mends = 0;                                      // tiles with masked keys so far
            const uint32_t idesc_s = instr_desc_16(CACHED ? 0 : 1, false, kKeys), idesc_o = instr_desc_16(CACHED ? 0 : 1, !CACHED, kCh);
            // (the high word of all descriptors: 8-row groups 1024 bytes apart, 128-byte swizzle)
            const uint32_t high = (uint32_t)(smem_desc_sw128(0) >> 32);
            const uint32_t q_low = (uint32_t)smem_desc_sw128(q_smem);
            auto scores = [&](int j, int i) {                    // S = Q_i K_j^T
                const int buf = NT == 2 ? i : j & 1;
                if (elect_one()) {
#pragma unroll
                    for (int p = 0; p < kParts; ++p) {
                        const uint32_t k_low = (uint32_t)smem_desc_sw128(stage(S::keys(j) + p));
                        const uint32_t row = q_low + i * (S::kQTile / 16) + p * kPlanes * 1024, d = tmem + 128 * buf;
                        if (p == 0) mma_f16_ss<false>(d, row, k_low, high, idesc_s);
#pragma unroll
                        for (int k = p == 0 ? 1 : 0; k < 4 * kPlanes; ++k) {
                            const int at = (k / 4) * 1024 + (k % 4) * 2;           // 64-channel planes of 16 KB, steps of 32 bytes
                            mma_f16_ss<true>(d, row + at, k_low + at, high, idesc_s);
                        }
                    }
                    mma_commit(smem_u32(&ctl.s[buf]));
                }
                __syncwarp();
            };
            auto products = [&](int j, int i) {                  // O_i += P V_j
                const int buf = NT == 2 ? i : j & 1;
                if (elect_one()) {
                    const uint32_t from = tmem + (S::kEarly ? 384 + 64 * i : 128 * buf);
#pragma unroll
                    for (int p = 0; p < kParts; ++p) {
                        const uint32_t at = stage(S::values(j, n) + p), d = tmem + S::kOCol + i * DP + p * 128;
                        const uint32_t v_low = (uint32_t)(CACHED ? smem_desc_sw128(at) : smem_desc_n_major(at));
                        if (j > 0) mma_f16_ts<true>(d, from, v_low, high, idesc_o);
                        else mma_f16_ts<false>(d, from, v_low, high, idesc_o);
#pragma unroll
                        for (int k = 1; k < 8; ++k)
                            mma_f16_ts<true>(d, from + 8 * k, v_low + (CACHED ? (k / 4) * (kCh * 8) + (k % 4) * 2 : k * 128), high, idesc_o);
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
            auto all_there = [&](int first) {
                for (int p = 0; ok && p < kParts; ++p) ok = wait_all(full_kv(first + p), ((first + p) / kStages) & 1, abort_flag, watchdog, kWdMma);
                return ok;
            };
            ok = wait_all(smem_u32(&ctl.q), 0, abort_flag, watchdog, kWdMma);
            if (all_there(0)) {
                tc_fence_after();
                for (int i = lo; i < hi; ++i) scores(0, i);
                release(0);
            }
            for (int j = 0; j < n && ok; ++j) {
                const int vuse = S::values(j, n), kuse = S::keys(j + 1);
                if (S::kAhead && j + 1 < n) {
                    all_there(kuse);
                    for (int i = lo; i < hi && ok; ++i) {
                        if (S::kEarly) ok = wait_all(smem_u32(&ctl.free[i]), j & 1, abort_flag, watchdog, kWdMma);
                        if (!ok) break;
                        tc_fence_after();
                        scores(j + 1, i);
                    }
                    if (!ok) break;
                    release(kuse);
                }
                // What the products need beside the probabilities is waited for ahead of them.
                if (all_there(vuse) && !CACHED) {
                    ok = wait_all(smem_u32(&ctl.meta[j % kMetas]), (j / kMetas) & 1, abort_flag, watchdog, kWdMma);
                    const bool clean = all_valid(ctl.metas[j % kMetas]);
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&ctl.used[j % kMetas]));
                    if (!clean && ok) {
                        if (lane == 0) mbar_arrive(smem_u32(&ctl.landed));
                        ok = wait_all(smem_u32(&ctl.fixed), mends & 1, abort_flag, watchdog, kWdMma);
                        ++mends;
                    }
                }
                if (ok && !S::kAhead && j + 1 < n) all_there(kuse);
                for (int i = lo; i < hi && ok; ++i) {
                    ok = wait_all(smem_u32(&ctl.p[NT == 2 ? i : j & 1]), NT == 2 ? j & 1 : (j >> 1) & 1, abort_flag, watchdog, kWdMma);
                    if (!ok) break;
                    tc_fence_after();
                    products(j, i);
                    if (S::kAhead || j + 1 == n) {
                        if (elect_one()) mma_commit(smem_u32(&ctl.o[i]));
                        __syncwarp();
                    }
                    if (!S::kAhead && j + 1 < n) scores(j + 1, i);
                }
                if (!ok) break;
                release(vuse);
                if (!S::kAhead && j + 1 < n) release(kuse);
            }
        });
    }
    if (!ok && issues) drain_after_abort();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == kMmaWarp) tmem_dealloc<1>(tmem, 512);
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
    bool mapped = true;
    if (CACHED && a.wide_keys > 0) {                            // widened: keys [unit][key][channel], values [unit][channel][key]
        const uint64_t D = (uint64_t)a.head_dim, L = (uint64_t)a.wide_keys, dk[3] = {D, L, (uint64_t)a.units}, dv[3] = {L, D, (uint64_t)a.units};
        const uint64_t sk[2] = {D * 2, L * D * 2}, sv[2] = {L * 2, L * D * 2};
        const uint32_t bk[3] = {64, kKeys, 1}, bv[3] = {64, (uint32_t)Shape<DP, NT>::kCh, 1};
        mapped = encode_tiled(&map_k, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, a.wide, dk, sk, bk, CU_TENSOR_MAP_SWIZZLE_128B) &&
                 encode_tiled(&map_v, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, static_cast<const uint16_t*>(a.wide) + a.units * L * D, dv, sv, bv, CU_TENSOR_MAP_SWIZZLE_128B);
    } else if (!CACHED && a.kv_rows > 0) {                      // channels of a head, heads, rows
        const uint64_t dims[3] = {(uint64_t)a.head_dim, (uint64_t)a.kv_heads, (uint64_t)a.kv_rows};
        const uint32_t box[3] = {64, 1, kKeys};
        const uint64_t head = (uint64_t)a.head_dim * 2, sk[2] = {head, (uint64_t)a.ldk * 2}, sv[2] = {head, (uint64_t)a.ldv * 2};
        mapped = encode_tiled(&map_k, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, a.k, dims, sk, box, CU_TENSOR_MAP_SWIZZLE_128B) &&
                 encode_tiled(&map_v, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, a.v, dims, sv, box, CU_TENSOR_MAP_SWIZZLE_128B);
    }
    if (!mapped) return cudaErrorUnknown;
    const dim3 grid((unsigned)row_tiles(a), (unsigned)a.chunks, (unsigned)a.units);
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
