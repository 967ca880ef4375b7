// Product of e2m1 codes with block scales on the 5th-generation tensor cores (sm_100a):
//   acc[j][t] = sum_b Sw[j][b] Sa[t][b] sum_{c in b} qW[j][c] qA[t][c]   tcgen05.mma with block scales, binary32 in TMEM
//   y[t][j]   = (delta_t s^W_j) acc + b_j
//
// Orientation as in the integer product: the MMA's 128 rows are output channels, its columns (16..256) tokens, so one kernel
// takes a single token as well as a long batch, and at few tokens the weights go from HBM straight into the tensor cores, with
// nothing to unpack.
//
// Operands: 256 channels a stage.  Codes arrive by TMA, two to a byte, K-major rows of 128 bytes with the 128-byte swizzle; an MMA
// takes 64 channels (32 bytes).  Block scales arrive as whole tiles of 512 bytes (128 rows x 4 blocks: the order in which
// tcgen05.cp spreads them over TMEM, one lane a row of 32, four columns a tile) and are copied to TMEM by the issuing thread
// ahead of the stage's MMAs.  Their TMEM columns go by the stage, so that whoever refills a stage knows that the MMAs that
// read them have ended.
//
// Roles: warp 0 producer of weights, warp 1 MMA issuer and TMEM allocator, then eight or twelve warps epilogue and one producer of tokens.
// CTAS = 2: a pair works on 256 channels, each CTA loading its 128 weight rows and half of the tokens' codes, but the scales of
// all tokens.  SPLIT: the CTAs (or pairs) of a cluster share one tile along K and exchange binary32 sums through the cluster's
// shared memory, added in the order of the slices: the result does not depend on timing.
// Every wait on a barrier is bounded (see ptx_sm100.cuh).
#include <cuda_bf16.h>

#include "act_common.cuh"
#include "fp4_common.cuh"
#include "ptx_sm100.cuh"
#include "tc_sm100.cuh"

namespace fq {
namespace {

// Epilogue warps, from warp 2 on: twelve read a tile's sums out of TMEM faster than eight (816 x 2048 x 32768 33.7 us, else 34.5; 816 x
// 2048 x 2560 6.8, else 7.1; sixteen spill).  Eight for slices of single CTAs, which are there for little work: fewer threads are set up
// faster (one token x 2048 x 2560 4.4 us, else 4.6).
template <int CTAS, bool SPLIT>
constexpr int kEpiWarps = CTAS == 1 && SPLIT ? 8 : 12;
template <int CTAS, bool SPLIT>
constexpr int kThreads = 32 * (kEpiWarps<CTAS, SPLIT> + 3);
constexpr int kRows = 128;               // channels of a CTA's tile
constexpr int kStageK = 256;             // channels of K a stage
constexpr int kMostStages = 8;
constexpr int kScaleCols = 256;          // TMEM columns from here on hold scales, those before accumulators
constexpr size_t kSmemMost = 224 * 1024; // (and 1.3 KB of static shared memory)
constexpr uint32_t kOutBytes = 32768;    // outputs on their way out
constexpr size_t kRingMost = kSmemMost - 1024 - kOutBytes;       // stages, and what slices of K receive

struct GemmParams {
    int64_t M, N;
    int K, bt, stages, m_full, n_tiles, band;   // (m_full: token tiles of bt tokens)
    int split;                           // slices of K, each CTA (pair) of a cluster one
    int kb;                              // stages of all of K
    int units, unit_step;
    uint32_t ring;                       // bytes of the stages, a multiple of 1024
    int per;                             // SPLIT: chunks that a slice finishes
    int shared_ring;                     // SPLIT: sums are received where the stages were
    const float* delta;
    const float* w_scale;
    const float* bias;
    int bf16;
    uint32_t* watchdog;
};

enum : uint32_t { kWdProducer = 1u, kWdMmaFull = 2u, kWdMmaAcc = 4u, kWdEpilogue = 8u, kWdSums = 128u };

template <int CTAS>
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int c0, int c1, uint32_t bar) {
    if (CTAS == 1) {
        tma_load_2d(dst, map, c0, c1, bar);
    } else {                             // counted on the barrier of the pair's even CTA
        asm volatile(
            "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
            ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(bar & 0xFEFFFFFFu)
            : "memory");
    }
}
template <int CTAS>
__device__ __forceinline__ void tma_load_tiles(uint32_t dst, const CUtensorMap* map, int tile, int rows, uint32_t bar) {
    if (CTAS == 1)
        asm volatile(
            "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
            ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(tile), "r"(rows), "r"(bar)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
            ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(tile), "r"(rows), "r"(bar & 0xFEFFFFFFu)
            : "memory");
}
// Arrival at the barrier of another CTA of the cluster, which orders no memory: what it announces are loads that have returned and
// MMAs that have ended.  (With a release ahead of it, which waits for the warp's stores, the tensor cores stood still 1200 cycles longer
// between two tiles.)
__device__ __forceinline__ void mbar_arrive_cta(uint32_t bar, uint32_t rank) {
    asm volatile(
        "{\n\t.reg .b32 ra;\n\t"
        "mapa.shared::cluster.u32 ra, %0, %1;\n\t"
        "mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [ra];\n\t}"
        ::"r"(bar), "r"(rank)
        : "memory");
}
// The work of one stage as ONE block of PTX: scale tiles to TMEM (512 bytes each, 32 rows of 16 bytes, to four columns of all four
// lane quadrants), four MMAs of 64 channels, the commits.  The whole warp runs it and the lane that elect.sync picks issues: the
// operands are then computed by the warp as a whole, which is much cheaper than by one lane of a divergent warp.
//   %0 accumulator column  %1, %2 matrix descriptors (weights, tokens)  %3, %4 descriptors of their scales  %5 TMEM column of the scales
//   %6 instruction descriptor  %7 add to what the accumulator holds  %8 MMAs of the stage  %9 the stage's barrier
//   %10 the accumulator's barrier, 0: not its last stage  %11 (pairs) cluster ranks whose barriers the commits arrive at
//   %12 TMEM column of the scales of the tile's first token: a tile of 64 tokens may begin in the middle of a scale tile
#define FQ_CP(CG, SRC, OFF, COL)                                                     \
    "add.u64 t, " SRC ", " OFF ";\n\tadd.u32 c, %5, " COL ";\n\t"                     \
    "@pl tcgen05.cp.cta_group::" CG ".32x128b.warpx4 [c], t;\n\t"
#define FQ_MMA(CG, KIND, STEP, SA, SB, ID, PRED, ACC)                                                        \
    "add.u64 t, %1, " STEP ";\n\tadd.u64 u, %2, " STEP ";\n\tadd.u32 c, %5, " SA ";\n\tadd.u32 e, %12, " SB ";\n\t" \
    "or.b32 f, %6, " ID ";\n\t"                                                                               \
    "@" PRED " tcgen05.mma.cta_group::" CG "." KIND " [%0], t, u, f, [c], [e], " ACC ";\n\t"
#define FQ_HEAD                                                                                  \
    "{\n\t.reg .pred pl, p1, p2, p3, pa, pt, pc;\n\t.reg .b64 t, u;\n\t.reg .b32 c, e, f;\n\t"     \
    "elect.sync _|pl, 0xffffffff;\n\t"                                                           \
    "setp.ne.b32 pa, %7, 0;\n\tsetp.eq.b32 pt, %0, %0;\n\t"                                      \
    "setp.gt.and.s32 p1, %8, 1, pl;\n\tsetp.gt.and.s32 p2, %8, 2, pl;\n\tsetp.gt.and.s32 p3, %8, 3, pl;\n\t" \
    "setp.ne.and.b32 pc, %10, 0, pl;\n\t"
#define FQ_COMMIT_1                                                                                \
    "@pl tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%9];\n\t"          \
    "@pc tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%10];\n\t}"
#define FQ_COMMIT_2                                                                                                \
    "@pl tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%9], %11;\n\t"  \
    "@pc tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%10], %11;\n\t}"
#define FQ_KIND_NV "kind::mxf4nvf4.block_scale.scale_vec::4X"
#define FQ_KIND_MX "kind::mxf4.block_scale.scale_vec::2X"
#define FQ_ID_ODD "1073741856"           /* blocks 2 and 3 of a scale tile, both operands: 2 << 29 | 2 << 4 */
#define FQ_STAGE_NV1(CG) \
    FQ_CP(CG, "%3", "0", "0") FQ_CP(CG, "%4", "0", "16") \
    FQ_MMA(CG, FQ_KIND_NV, "0", "0", "0", "0", "pl", "pa") \
    FQ_CP(CG, "%3", "32", "4") FQ_CP(CG, "%4", "32", "20") \
    FQ_MMA(CG, FQ_KIND_NV, "2", "4", "4", "0", "p1", "pt") \
    FQ_CP(CG, "%3", "64", "8") FQ_CP(CG, "%4", "64", "24") \
    FQ_MMA(CG, FQ_KIND_NV, "4", "8", "8", "0", "p2", "pt") \
    FQ_CP(CG, "%3", "96", "12") FQ_CP(CG, "%4", "96", "28") \
    FQ_MMA(CG, FQ_KIND_NV, "6", "12", "12", "0", "p3", "pt")
#define FQ_STAGE_NV2(CG) \
    FQ_CP(CG, "%3", "0", "0") FQ_CP(CG, "%4", "0", "16") FQ_CP(CG, "%4", "128", "20") \
    FQ_MMA(CG, FQ_KIND_NV, "0", "0", "0", "0", "pl", "pa") \
    FQ_CP(CG, "%3", "32", "4") FQ_CP(CG, "%4", "32", "24") FQ_CP(CG, "%4", "160", "28") \
    FQ_MMA(CG, FQ_KIND_NV, "2", "4", "8", "0", "p1", "pt") \
    FQ_CP(CG, "%3", "64", "8") FQ_CP(CG, "%4", "64", "32") FQ_CP(CG, "%4", "192", "36") \
    FQ_MMA(CG, FQ_KIND_NV, "4", "8", "16", "0", "p2", "pt") \
    FQ_CP(CG, "%3", "96", "12") FQ_CP(CG, "%4", "96", "40") FQ_CP(CG, "%4", "224", "44") \
    FQ_MMA(CG, FQ_KIND_NV, "6", "12", "24", "0", "p3", "pt")
#define FQ_STAGE_MX1(CG) \
    FQ_CP(CG, "%3", "0", "0") FQ_CP(CG, "%4", "0", "8") \
    FQ_MMA(CG, FQ_KIND_MX, "0", "0", "0", "0", "pl", "pa") \
    FQ_MMA(CG, FQ_KIND_MX, "2", "0", "0", FQ_ID_ODD, "p1", "pt") \
    FQ_CP(CG, "%3", "32", "4") FQ_CP(CG, "%4", "32", "12") \
    FQ_MMA(CG, FQ_KIND_MX, "4", "4", "4", "0", "p2", "pt") \
    FQ_MMA(CG, FQ_KIND_MX, "6", "4", "4", FQ_ID_ODD, "p3", "pt")
#define FQ_STAGE_MX2(CG) \
    FQ_CP(CG, "%3", "0", "0") FQ_CP(CG, "%4", "0", "8") FQ_CP(CG, "%4", "64", "12") \
    FQ_MMA(CG, FQ_KIND_MX, "0", "0", "0", "0", "pl", "pa") \
    FQ_MMA(CG, FQ_KIND_MX, "2", "0", "0", FQ_ID_ODD, "p1", "pt") \
    FQ_CP(CG, "%3", "32", "4") FQ_CP(CG, "%4", "32", "16") FQ_CP(CG, "%4", "96", "20") \
    FQ_MMA(CG, FQ_KIND_MX, "4", "4", "8", "0", "p2", "pt") \
    FQ_MMA(CG, FQ_KIND_MX, "6", "4", "8", FQ_ID_ODD, "p3", "pt")
template <int CTAS, bool NV, int XA>
__device__ __forceinline__ void issue_stage(uint32_t d, uint64_t wd, uint64_t xd, uint64_t ws, uint64_t xs, uint32_t cols, uint32_t xcols, uint32_t idesc,
                                            uint32_t accumulate, int steps, uint32_t bar_stage, uint32_t bar_acc, uint16_t mask) {
#define FQ_STAGE(BODY, COMMIT)                                                                                               \
    asm volatile(FQ_HEAD BODY COMMIT ::"r"(d), "l"(wd), "l"(xd), "l"(ws), "l"(xs), "r"(cols), "r"(idesc), "r"(accumulate),   \
                 "r"(steps), "r"(bar_stage), "r"(bar_acc), "h"(mask), "r"(xcols) : "memory")
    if constexpr (CTAS == 1 && NV && XA == 1) FQ_STAGE(FQ_STAGE_NV1("1"), FQ_COMMIT_1);
    else if constexpr (CTAS == 1 && NV) FQ_STAGE(FQ_STAGE_NV2("1"), FQ_COMMIT_1);
    else if constexpr (CTAS == 1 && XA == 1) FQ_STAGE(FQ_STAGE_MX1("1"), FQ_COMMIT_1);
    else if constexpr (CTAS == 1) FQ_STAGE(FQ_STAGE_MX2("1"), FQ_COMMIT_1);
    else if constexpr (NV) FQ_STAGE(FQ_STAGE_NV2("2"), FQ_COMMIT_2);
    else FQ_STAGE(FQ_STAGE_MX2("2"), FQ_COMMIT_2);
#undef FQ_STAGE
}
// Shared-memory descriptor of a run of scale tiles (no swizzle, 8-row groups 128 bytes apart).
__device__ __forceinline__ uint64_t scale_desc(uint32_t smem) {
    return (uint64_t)((smem & 0x3FFFFu) >> 4) | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
}
// Instruction descriptor: e2m1 x e2m1, both K-major, scales e4m3 or e8m0, M = m, N = n.
__device__ __forceinline__ uint32_t instr_desc_fp4(int m, int n, bool nv) {
    return (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((nv ? 0u : 1u) << 23) | ((uint32_t)(m >> 4) << 24);
}
// 16 TMEM lanes x 16 columns as a warp-level MMA accumulator has them: thread T holds, for column groups n = 0, 1,
//   r[4n + 0], r[4n + 1] = lane T/4, columns 8n + 2(T%4) and the next;  r[4n + 2], r[4n + 3] = lane T/4 + 8, the same columns.
// With channels on the lanes and tokens on the columns such a pair, rounded to 16 bits, is what stmatrix stores transposed.
__device__ __forceinline__ void tmem_ld_16x256b_x2(uint32_t taddr, uint32_t* r) {
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr)
                 : "memory");
}
__device__ __forceinline__ void stmatrix_x4_trans(uint32_t addr, uint32_t r0, uint32_t r1, uint32_t r2, uint32_t r3) {
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};"
                 ::"r"(addr), "r"(r0), "r"(r1), "r"(r2), "r"(r3));
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, int c0, int c1, uint32_t src) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];"
                 ::"l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(src)
                 : "memory");
}
// One channel at two adjacent tokens, rounded to bf16, the earlier token in the low half.
__device__ __forceinline__ uint32_t scale_pair(uint32_t a0, uint32_t a1, float2 d, float sw, float bj) {
    const float2 v = f2_fma(make_float2(__uint_as_float(a0), __uint_as_float(a1)), f2_mul(d, make_float2(sw, sw)), make_float2(bj, bj));
    uint32_t w;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(v.y), "f"(v.x));
    return w;
}
// 16 bytes into another CTA's shared memory, counted on a barrier there.
__device__ __forceinline__ void st_async_v4(uint32_t addr, const uint32_t* r, uint32_t bar) {
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];"
                 ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(map)) : "memory");
}
// (no memory clobber, as the matrix stores: the fence behind them orders them)
__device__ __forceinline__ void sts32_loose(uint32_t addr, uint32_t v) { asm volatile("st.shared.b32 [%0], %1;" ::"r"(addr), "r"(v)); }

// XA: scale tiles across a tile's tokens (two for more than 128, and for pairs).
template <int CTAS, bool NV, bool SPLIT, int XA>
__global__ void __launch_bounds__((kThreads<CTAS, SPLIT>), 1)
gemm_fp4_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_ws, const __grid_constant__ CUtensorMap map_x,
                const __grid_constant__ CUtensorMap map_xs, const __grid_constant__ CUtensorMap map_y, const GemmParams p) {
    constexpr int kEpi = kEpiWarps<CTAS, SPLIT>, kTokenWarp = 2 + kEpi;
    constexpr int kSets = kEpi / 4, kChunks = (16 / kSets + 1) / 2 * 2;       // warps to a quadrant of lanes, chunks of 16 tokens of a warp at most
    constexpr int kBuffers = kEpi == 8 ? 4 : 2;              // of a warp for 16 bf16 tokens, 1 KB each (binary32: half as many)
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t s_full[kMostStages], s_empty[kMostStages], s_acc_full[2], s_acc_empty[2], s_ended, s_sums;
    __shared__ __align__(16) float s_steps[kEpi][32];        // of the tokens that each epilogue warp is at
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort;
    constexpr int kTiles = NV ? 4 : 2;                       // scale tiles of a stage's 256 channels
    constexpr uint32_t kWBytes = kRows * 128, kWScale = kTiles * 512;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int* abort_flag = &s_abort;
    const uint32_t rank = CTAS == 2 || SPLIT ? cluster_ctarank() : 0u;
    const uint32_t half = CTAS == 2 ? rank & 1u : 0u, pair_base = rank & ~1u;
    const bool leader = half == 0;
    const int slice = SPLIT ? (int)(rank / CTAS) : 0;
    const uint32_t x_bytes = (uint32_t)(p.bt / CTAS) * 128u, x_scale = (uint32_t)XA * kWScale;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    // [weight codes][token codes] of all stages (1024-byte aligned), then their scales
    const uint32_t s_w = base, s_x = s_w + (uint32_t)p.stages * kWBytes, s_ws = s_x + (uint32_t)p.stages * x_bytes, s_xs = s_ws + (uint32_t)p.stages * kWScale,
                   s_out = base + p.ring;

    const int accs = p.bt <= 128 ? 2 : 1, acc_cols = kScaleCols / accs;
    const int slot_cols = kTiles * 4 * (1 + XA);             // TMEM columns of a stage's scales
    const int cluster = SPLIT ? p.split * CTAS : CTAS;
    const int unit0 = (int)blockIdx.x / cluster;
    const int kb0 = SPLIT ? p.kb * slice / p.split : 0, kb1 = SPLIT ? p.kb * (slice + 1) / p.split : p.kb;
    // Token tiles in bands, within a band channel tile by channel tile: what runs at a time covers a block of the output.  A last
    // token tile that is not full comes behind all others, where its shorter units even out what the CTAs have left.
    auto tile_of = [&](int unit, int* m, int* n) {
        const int full = p.m_full * p.n_tiles;
        if (unit >= full) {
            *m = p.m_full;
            *n = unit - full;
            return;
        }
        const int b = unit / (p.band * p.n_tiles), r = unit - b * (p.band * p.n_tiles), rows = min(p.band, p.m_full - b * p.band);
        *m = b * p.band + r % rows;
        *n = r / rows;
    };
    auto columns = [&](int m) {                              // tokens of a tile, rounded up to what an MMA takes
        const int64_t left = p.M - (int64_t)m * p.bt;
        return left >= p.bt ? p.bt : ((int)left + 16 * CTAS - 1) / (16 * CTAS) * (16 * CTAS);
    };
    auto load_weights = [&](int n, int kb, int s) {
        const uint32_t bar = smem_u32(&s_full[s]);
        if (leader) mbar_arrive_expect_tx(bar, (kWBytes + kWScale) * CTAS);
        tma_load<CTAS>(s_w + s * kWBytes, &map_w, kb * 128, (n * CTAS + (int)half) * kRows, bar);
        tma_load_tiles<CTAS>(s_ws + s * kWScale, &map_ws, kb * kTiles, n * CTAS + (int)half, bar);
    };
    auto load_tokens = [&](int m, int t0, int kb, int s) {
        const uint32_t bar = smem_u32(&s_full[s]);
        if (leader) mbar_arrive_expect_tx(bar, (x_bytes + x_scale) * CTAS);
        tma_load<CTAS>(s_x + s * x_bytes, &map_x, kb * 128, t0, bar);
        tma_load_tiles<CTAS>(s_xs + s * x_scale, &map_xs, kb * kTiles, (int)((int64_t)m * p.bt >> 7), bar);
    };
    auto first_token = [&](int m) { return m * p.bt + (int)half * (columns(m) / CTAS); };      // that this CTA loads
    // A weight handle is complete before the call: its first stages come while the kernel ahead still runs, and (single CTAs, whose
    // loads concern nobody else) while this one is being set up.
    // (Two of them: a copy takes its issuer 50 cycles, and everybody waits for the set-up.)
    const int ahead = unit0 < p.units ? min(p.stages, kb1 - kb0) : 0, early = CTAS == 1 ? min(ahead, 2) : 0;
    auto first_weights = [&](int from, int to) {
        if (from < to && elect_one()) {
            int m, n;
            tile_of(unit0, &m, &n);
            for (int i = from; i < to; ++i) load_weights(n, kb0 + i, i);
        }
        __syncwarp();
    };

    if (warp == 0) {
        if (lane == 0) {
            s_abort = 0;
            for (int s = 0; s < p.stages; ++s) {
                mbar_init(smem_u32(&s_full[s]), 2);          // both producers
                mbar_init(smem_u32(&s_empty[s]), 1);
            }
            for (int a = 0; a < 2; ++a) {
                mbar_init(smem_u32(&s_acc_full[a]), 1);
                mbar_init(smem_u32(&s_acc_empty[a]), kEpi * CTAS);
            }
            mbar_init(smem_u32(&s_ended), (uint32_t)p.split);
            mbar_init(smem_u32(&s_sums), 1);
            fence_mbarrier_init();
            fence_proxy_async_smem();
        }
        __syncwarp();
        first_weights(0, early);
    } else if (warp == 1) {
        tmem_alloc<CTAS>(smem_u32(&s_tmem), 512u);
    } else if (warp == kTokenWarp && lane == 0) {
        prefetch_map(&map_x);
        prefetch_map(&map_xs);
        prefetch_map(&map_y);
    }
    tc_fence_before();
    __syncthreads();
    if (CTAS == 2) cluster_sync_all();                       // the other CTAs' barriers exist
    else if (SPLIT) cluster_arrive();                        // (awaited ahead of the first word to another CTA)
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    if (warp >= 2) griddep_wait();
    griddep_launch_dependents();

    if (warp == 0 || warp == kTokenWarp) {
        // ------------------------------------------------------------ producers: of weights, of tokens
        // (what needs no wait in one go: with a wait and an election each, the fourth stage's tokens were asked for 700 cycles after the first's)
        if (warp == 0) {
            first_weights(early, ahead);
        } else if (ahead > 0 && elect_one()) {
            int m, n;
            tile_of(unit0, &m, &n);
            const int t0 = first_token(m);
            for (int i = 0; i < ahead; ++i) load_tokens(m, t0, kb0 + i, i);
        }
        __syncwarp();
        bool ok = true;
        int stage = 0, there = ahead;
        uint32_t phase = 0;
        for (int unit = unit0; unit < p.units && ok; unit += p.unit_step) {
            int m, n;
            tile_of(unit, &m, &n);
            const int t0 = first_token(m);
            for (int kb = kb0; kb < kb1; ++kb) {
                if (there > 0) {
                    --there;
                } else {
                    ok = mbar_wait_all_lazy(smem_u32(&s_empty[stage]), phase ^ 1u, abort_flag, p.watchdog, kWdProducer);
                    if (!ok) break;
                    if (elect_one()) {
                        if (warp == 0) load_weights(n, kb, stage);
                        else load_tokens(m, t0, kb, stage);
                    }
                    __syncwarp();
                }
                if (++stage == p.stages) { stage = 0; phase ^= 1u; }
            }
        }
        if (!ok && lane == 0) drain_after_abort();
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMA issuer
        if (leader) {
            bool ok = true;
            int stage = 0, acc = 0;
            uint32_t phase = 0, acc_phase = 0;
            const uint16_t mask = (uint16_t)(3u << pair_base);
            for (int unit = unit0; unit < p.units && ok; unit += p.unit_step) {
                int m, n;
                tile_of(unit, &m, &n);
                const uint32_t idesc = instr_desc_fp4(kRows * CTAS, columns(m), NV);
                ok = mbar_wait_all(smem_u32(&s_acc_empty[acc]), acc_phase ^ 1u, abort_flag, p.watchdog, kWdMmaAcc);
                if (!ok) break;
                const uint32_t d = tmem + (uint32_t)(acc * acc_cols);
                const uint32_t first = kTiles * 4 + (uint32_t)(((int64_t)m * p.bt & 127) >> 5);       // columns ahead of the tokens' scales
                for (int kb = kb0; kb < kb1; ++kb) {
                    ok = mbar_wait_all(smem_u32(&s_full[stage]), phase, abort_flag, p.watchdog, kWdMmaFull);
                    if (!ok) break;
                    tc_fence_after();
                    // (what lies past K's last scale tile is never multiplied: zeros times whatever a scale holds)
                    issue_stage<CTAS, NV, XA>(d, smem_desc_sw128(s_w + stage * kWBytes), smem_desc_sw128(s_x + stage * x_bytes), scale_desc(s_ws + stage * kWScale),
                                              scale_desc(s_xs + stage * x_scale), tmem + kScaleCols + (uint32_t)(stage * slot_cols),
                                              tmem + kScaleCols + (uint32_t)(stage * slot_cols) + first, idesc,
                                              kb != kb0 ? 1u : 0u, (p.K - kb * kStageK + 63) / 64, smem_u32(&s_empty[stage]),
                                              kb == kb1 - 1 ? smem_u32(&s_acc_full[acc]) : 0u, mask);
                    if (++stage == p.stages) { stage = 0; phase ^= 1u; }
                }
                if (++acc == accs) { acc = 0; acc_phase ^= 1u; }
            }
        }
    } else {
        // ------------------------------------------------------------ epilogue
        // The warps of a quadrant take chunks of 16 tokens in turn: chunk i of set s begins at token (s + kSets i) * 16.
        const int quad = warp & 3, set = (warp - 2) >> 2;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        float* const steps = s_steps[warp - 2];
        auto token = [&](int i) { return (set + kSets * i) * 16; };
        bool ok = true;
        float sw4[4], bj4[4], step2[kChunks / 2];        // step2[k]: steps of chunks 2k and 2k + 1, a lane each
        auto constants = [&](int m, int n) {
            const int64_t jq = (int64_t)(n * CTAS + (int)half) * kRows + quad * 32, t0 = (int64_t)m * p.bt;
#pragma unroll
            for (int i = 0; i < kChunks / 2; ++i) {
                const int t = token(2 * i + (lane >> 4)) + (lane & 15);
                step2[i] = t < p.bt && t0 + t < p.M ? ld_global_f32(p.delta + t0 + t) : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t j = jq + (p.bf16 ? (lane >> 2) + 8 * i : lane);       // bf16: the channels of this thread's fragments
                sw4[i] = j < p.N ? __ldg(p.w_scale + j) : 0.0f;
                bj4[i] = j < p.N ? __ldg(p.bias + j) : 0.0f;
            }
        };
        // Sums of one chunk, as fragments for bf16 outputs (channels 0..15, 16..31 of the quadrant), else a thread one channel.
        auto fetch = [&](uint32_t column, uint32_t* r) {
            if (p.bf16) {
                tmem_ld_16x256b_x2(tmem + lanes + column, r);
                tmem_ld_16x256b_x2(tmem + lanes + (16u << 16) + column, r + 8);
            } else {
                tmem_ld16(tmem + lanes + column, r);
            }
        };
        // Outputs of chunk i, token-major, through one of the warp's buffers, which a bulk store reads; it clips what lies past M or N.
        int stores = 0;
        auto emit = [&](const uint32_t* r, int i, int64_t t0, int64_t jq) {
            if ((i & 1) == 0 || SPLIT) {
                float st = step2[0];
#pragma unroll
                for (int k = 1; k < kChunks / 2; ++k) st = i / 2 == k ? step2[k] : st;
                __syncwarp();
                steps[lane] = st;
            }
            const float* const st = steps + (i & 1) * 16;
            const int64_t tc = t0 + token(i);
            if (stores >= (p.bf16 ? kBuffers : kBuffers / 2)) {
                if (p.bf16) bulk_wait_read<kBuffers - 1>();
                else bulk_wait_read<kBuffers / 2 - 1>();
            }
            __syncwarp();
            const uint32_t buf = s_out + (uint32_t)((warp - 2) * kBuffers + (p.bf16 ? stores % kBuffers : stores % (kBuffers / 2) * 2)) * 1024u;
            ++stores;
            if (p.bf16) {
                // scaled in pairs, [16 tokens][32 channels] by transposing matrix stores (64-byte swizzle)
                const float2 d0 = *reinterpret_cast<const float2*>(st + 2 * (lane & 3)), d1 = *reinterpret_cast<const float2*>(st + 8 + 2 * (lane & 3));
                const uint32_t tok = (uint32_t)((lane >> 4) * 8 + (lane & 7)), ch = (uint32_t)((lane >> 3) & 1), mix = (tok >> 1) & 3u;
                const uint32_t to = buf + tok * 64u;
                stmatrix_x4_trans(to + ((ch ^ mix) << 4), scale_pair(r[0], r[1], d0, sw4[0], bj4[0]), scale_pair(r[2], r[3], d0, sw4[1], bj4[1]),
                                  scale_pair(r[4], r[5], d1, sw4[0], bj4[0]), scale_pair(r[6], r[7], d1, sw4[1], bj4[1]));
                stmatrix_x4_trans(to + (((ch + 2u) ^ mix) << 4), scale_pair(r[8], r[9], d0, sw4[2], bj4[2]), scale_pair(r[10], r[11], d0, sw4[3], bj4[3]),
                                  scale_pair(r[12], r[13], d1, sw4[2], bj4[2]), scale_pair(r[14], r[15], d1, sw4[3], bj4[3]));
            } else {
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    const float4 q = reinterpret_cast<const float4*>(st)[k / 4];
                    const float d = k % 4 == 0 ? q.x : k % 4 == 1 ? q.y : k % 4 == 2 ? q.z : q.w;
                    sts32_loose(buf + (uint32_t)(k * 128 + lane * 4), __float_as_uint(__fmaf_rn(__uint_as_float(r[k]), d * sw4[0], bj4[0])));
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (elect_one()) {                               // (a group for every buffer taken, past N an empty one: the waits count them)
                if (jq < p.N) tma_store_2d(&map_y, (int)(jq * (p.bf16 ? 2 : 4)), (int)tc, buf);
                bulk_commit();
            }
            __syncwarp();
        };
        if constexpr (!SPLIT) {
            int acc = 0;
            uint32_t phase = 0;
            for (int unit = unit0; unit < p.units; unit += p.unit_step) {
                int m, n;
                tile_of(unit, &m, &n);
                const int64_t jq = (int64_t)(n * CTAS + (int)half) * kRows + quad * 32, t0 = (int64_t)m * p.bt;
                const int cols = (int)min((int64_t)p.bt, p.M - t0);                 // tokens of the tile
                constants(m, n);
                ok = mbar_wait_all(smem_u32(&s_acc_full[acc]), phase, abort_flag, p.watchdog, kWdEpilogue);
                if (!ok) break;
                tc_fence_after();
                // all of the warp's sums into registers, so that the next tile's MMAs may have the columns
                uint32_t r[kChunks][16];
#pragma unroll
                for (int i = 0; i < kChunks; ++i)
                    if (token(i) < cols) fetch((uint32_t)(acc * acc_cols + token(i)), r[i]);
                tmem_ld_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (leader) mbar_arrive(smem_u32(&s_acc_empty[acc]));
                    else mbar_arrive_cta(smem_u32(&s_acc_empty[acc]), pair_base);
                }
#pragma unroll
                for (int i = 0; i < kChunks; ++i)
                    if (token(i) < cols) emit(r[i], i, t0, jq);
                if (++acc == accs) { acc = 0; phase ^= 1u; }
            }
        }
        if constexpr (SPLIT) {
            // Slice s finishes the tile's chunks s * per .. (s + 1) * per: the others store their sums into its shared memory, as the
            // threads hold them, counted in bytes on its barrier.  They have a place of their own there, or (p.shared_ring) the one of
            // the stages, once the MMAs of all slices have ended, which each tells the others.  Each slice adds to its own sums the
            // others' in their order.
            int m, n;
            tile_of(unit0, &m, &n);
            const int64_t jq = (int64_t)(n * CTAS + (int)half) * kRows + quad * 32, t0 = (int64_t)m * p.bt;
            const int cols = (int)min((int64_t)p.bt, p.M - t0), chunks = (cols + 15) / 16, per = p.per;
            const uint32_t received = p.shared_ring ? base : s_out + kOutBytes;
            auto place = [&](int sender, int c) { return received + (uint32_t)((sender * per + c) * 4 + quad) * 2048u + (uint32_t)lane * 16u; };
            constants(m, n);
            ok = mbar_wait_all(smem_u32(&s_acc_full[0]), 0u, abort_flag, p.watchdog, kWdEpilogue);
            tc_fence_after();
            if (CTAS == 1) cluster_wait();                   // the others are there
            if (ok) {
                const int mine = max(0, min(per, chunks - slice * per));
                if (warp == 2 && lane == 0) mbar_arrive_expect_tx(smem_u32(&s_sums), (uint32_t)((p.split - 1) * mine) * 8192u);
                if (p.shared_ring) {
                    if (warp == 2 && lane < p.split) mbar_arrive_cta(smem_u32(&s_ended), (uint32_t)(lane * CTAS) + half);
                    __syncwarp();
                    ok = mbar_wait_all(smem_u32(&s_ended), 0u, abort_flag, p.watchdog, kWdSums);
                }
                if (ok) {
                    for (int i = 0; i < kChunks; ++i) {
                        const int c = token(i) / 16, owner = c / per;
                        if (c >= chunks) break;
                        if (owner == slice) continue;
                        uint32_t r[16];
                        fetch((uint32_t)(c * 16), r);
                        tmem_ld_wait();
                        const uint32_t to = (uint32_t)(owner * CTAS) + half, bar = cluster_address(smem_u32(&s_sums), to);
                        const uint32_t at = cluster_address(place(slice - (slice > owner ? 1 : 0), c - owner * per), to);
#pragma unroll
                        for (int q = 0; q < 4; ++q) st_async_v4(at + (uint32_t)(q * 512), r + 4 * q, bar);
                    }
                    if (mine > 0) ok = mbar_wait_all(smem_u32(&s_sums), 0u, abort_flag, p.watchdog, kWdSums);
                }
            }
            if (ok) {
                for (int i = 0; i < kChunks; ++i) {
                    const int c = token(i) / 16;
                    if (c >= chunks) break;
                    if (c / per != slice) continue;
                    uint32_t r[16];
                    fetch((uint32_t)(c * 16), r);
                    tmem_ld_wait();
                    for (int s = 0; s < p.split - 1; ++s) {
                        const uint32_t from = place(s, c - slice * per);
                        uint4 o[4];
#pragma unroll
                        for (int q = 0; q < 4; ++q) o[q] = lds128(from + (uint32_t)(q * 512));
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const uint32_t w[4] = {o[q].x, o[q].y, o[q].z, o[q].w};
#pragma unroll
                            for (int k = 0; k < 4; ++k) r[4 * q + k] = __float_as_uint(__fadd_rn(__uint_as_float(r[4 * q + k]), __uint_as_float(w[k])));
                        }
                    }
                    emit(r, i, t0, jq);
                }
            }
        }
    }
    __syncwarp();
    if (warp >= 2 && warp < kTokenWarp) bulk_wait_read<0>();     // stores have read their buffers before the CTA gives them up
    if (SPLIT && CTAS == 1 && (warp < 2 || warp == kTokenWarp)) cluster_wait();
    tc_fence_before();
    __syncthreads();
    if (CTAS == 2 || SPLIT) cluster_sync_all();              // nobody leaves while another may still signal it
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc<CTAS>(tmem, 512u);
    }
}

// ---- host ----------------------------------------------------------------------------------------
bool code_map(CUtensorMap* map, const uint8_t* codes, int64_t rows, int64_t K, int box_rows) {
    const uint64_t dims[2] = {(uint64_t)K / 2, (uint64_t)rows}, strides[1] = {(uint64_t)K / 2};
    const uint32_t box[2] = {128, (uint32_t)box_rows};
    return encode_tiled(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, codes, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}
bool scale_map(CUtensorMap* map, const uint8_t* scales, int64_t rows, int64_t K, fq_fp4_format f, int box_rows) {
    const int64_t tiles = fp4_scale_tiles(K, f);
    const uint64_t dims[3] = {128, (uint64_t)tiles, (uint64_t)((rows + 127) / 128)}, strides[2] = {512, (uint64_t)tiles * 512};
    const uint32_t box[3] = {128, f == FQ_NVFP4 ? 4u : 2u, (uint32_t)box_rows};
    return encode_tiled(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, scales, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_NONE);
}

struct Plan {
    int ctas, bt, split;
};
// What a slice of K receives from the others.
size_t split_bytes(int bt, int split) { return (size_t)(split - 1) * ((bt / 16 + split - 1) / split) * 8192; }
// Tiles (single CTAs of 128 channels x 64, 128 or 256 tokens, or all of them where there are few; pairs of 256 x 256) and slices of K
// by the time that they are expected to take, in us: so many waves of (stages of a slice, epilogue), and what the slices' exchange
// adds.  The constants were fitted to the launches below, with an epilogue of eight warps everywhere; with today's, about a tenth faster, the
// order is the same.  Measured with it, the choice against the next best (M x K x N, us):
//   1 x 2048 x 2560 two slices 4.4 (four 4.7, one 4.8), 1 x 16384 x 2048 four 8.3 (two 12.8, eight 14.0), 1 x 1024 x 4096 one 3.7 (two 3.8),
//   333 x 1120 x 1000 tiles of 64 tokens 5.2 (128: 6.1), 512 x 4096 x 4096 128 tokens 9.6 (pairs 10.8), 816 x 2048 x 2560 128 tokens 6.8
//   (pairs 7.9), 816 x 16384 x 2048 pairs in two slices 18.6 (128 tokens 21.8, pairs in one 24.9), 2048 x 4096 x 4096 pairs 18.9 (single
//   CTAs of 256 tokens 21.7), 816 x 2048 x 32768 pairs 33.8 (37.2), 16384 x 8192 x 8192 pairs 422 (488).
Plan plan(int64_t M, int64_t N, int64_t K, int (*held)(int)) {
    const int sms = device_sm_count();
    const int64_t kb = (K + kStageK - 1) / kStageK;
    Plan best = {1, 256, 1};
    float least = 0.0f;
    auto offer = [&](int ctas, int bt, float stage, float epilogue) {
        const int64_t tiles = (N + 128 * ctas - 1) / (128 * ctas) * ((M + bt - 1) / bt);
        for (int split = 1; split * ctas <= 8 && split <= kb; split *= 2) {
            const int cluster = split * ctas;
            if (split > 1 && tiles * cluster > sms) break;
            const float waves = (float)((tiles * cluster + sms - 1) / sms);
            float t = waves * ((float)((kb + split - 1) / split) * stage + epilogue);
            // (clusters of four on most of the device wait for one another's places)
            if (split > 1) t += (split == 2 ? 0.75f : split == 4 ? 1.5f : 2.6f) + 0.006f * (float)bt + (ctas == 1 && split == 4 && tiles * 4 > 96 ? 1.2f : 0.0f);
            if (least == 0.0f || t < least) {
                if (cluster > 1) {                            // (asked last: it costs the host more than the rest)
                    const int most = held(cluster);
                    if (most == 0 || (split > 1 && tiles > most)) continue;
                }
                least = t;
                best = {ctas, bt, split};
            }
        }
    };
    if (M <= 128) {
        const int bt = (int)((M + 15) / 16 * 16);
        offer(1, bt, 0.29f + 0.0005f * (float)bt, 0.4f + 0.004f * (float)bt);
    }
    if (M > 64) offer(1, 64, 0.30f, 0.6f);
    if (M > 128) {
        offer(1, 128, 0.36f, 0.9f);
        offer(1, 256, 0.50f, 1.8f);
        offer(2, 256, 0.38f, 1.8f);
    }
    return best;
}
int no_clusters(int) { return 0; }

struct Maps {
    CUtensorMap x, xs, y;
};
template <int CTAS, bool NV, bool SPLIT, int XA>
cudaError_t launch(const Fp4Weights& W, const Maps& maps, const GemmParams& p, int grid, size_t smem, cudaStream_t stream) {
    auto kern = gemm_fp4_kernel<CTAS, NV, SPLIT, XA>;
    const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kern), smem);
    if (e != cudaSuccess) return e;
    return launch_pdl(kern, (unsigned)grid, (unsigned)kThreads<CTAS, SPLIT>, smem, stream, (unsigned)(CTAS * p.split), W.map_codes, W.map_scales, maps.x, maps.xs, maps.y, p);
}
template <int CTAS, int XA>
cudaError_t launch(const Fp4Weights& W, const Maps& maps, const GemmParams& p, int grid, size_t smem, cudaStream_t stream) {
    if (W.format == FQ_NVFP4) return p.split > 1 ? launch<CTAS, true, true, XA>(W, maps, p, grid, smem, stream) : launch<CTAS, true, false, XA>(W, maps, p, grid, smem, stream);
    return p.split > 1 ? launch<CTAS, false, true, XA>(W, maps, p, grid, smem, stream) : launch<CTAS, false, false, XA>(W, maps, p, grid, smem, stream);
}

}  // namespace

bool fp4_weight_maps(Fp4Weights& W) {
    return W.N == 0 || (code_map(&W.map_codes, W.codes, W.N, W.K, kRows) && scale_map(&W.map_scales, W.scales, W.N, W.K, W.format, 1));
}

namespace {
// *refused: the device did not take the launch's clusters, nothing was enqueued.
fq_status launch_planned(const uint8_t* codes, const uint8_t* scales, const float* delta, int64_t M, const Fp4Weights& W, void* y, fq_dtype yt,
                         int64_t ldy, int (*held)(int), cudaStream_t stream, bool* refused) {
    const int sms = device_sm_count();
    const Plan r = plan(M, W.N, W.K, held);
    const bool nv = W.format == FQ_NVFP4;
    GemmParams p = {};
    p.M = M; p.N = W.N; p.K = (int)W.K;
    p.bt = r.bt;
    p.split = r.split;
    p.kb = (int)((W.K + kStageK - 1) / kStageK);
    const int xa = r.ctas == 2 || r.bt > 128 ? 2 : 1;
    p.m_full = (int)(M / r.bt);
    p.n_tiles = (int)((W.N + kRows * r.ctas - 1) / (kRows * r.ctas));
    p.band = p.m_full >= 16 ? 8 : p.m_full > 0 ? p.m_full : 1;
    p.units = (p.m_full + (M % r.bt ? 1 : 0)) * p.n_tiles;
    p.delta = delta; p.w_scale = W.w_scale; p.bias = W.bias;
    p.bf16 = yt == FQ_BF16;
    p.watchdog = watchdog_device_ptr();
    if (!p.watchdog) return FQ_ERR_CUDA;
    const int tiles = nv ? 4 : 2;
    const size_t stage = (size_t)kRows * 128 + (size_t)(r.bt / r.ctas) * 128 + (size_t)tiles * 512 * (1 + xa);
    const int slots = 256 / (tiles * 4 * (1 + xa));        // TMEM columns for scales
    auto fit = [&](size_t bytes) {
        const int most = slots < kMostStages ? slots : kMostStages;
        return (int)(bytes / stage) < most ? (int)(bytes / stage) : most;
    };
    // received sums beside the stages where at least five are left, else in their place (112 KB at most, of single CTAs with 256 tokens
    // in eight slices: their three stages hold more, as do all others')
    static_assert(7 * 2 * 8192 <= 3 * (kRows * 128 + 256 * 128 + 2 * 512 * 3), "received sums fit where the stages were");
    const size_t sums = split_bytes(r.bt, r.split);
    p.stages = fit(kRingMost);
    p.per = (r.bt / 16 + r.split - 1) / r.split;
    if (r.split > 1) {
        const int beside = fit(kRingMost - sums);
        p.shared_ring = beside < 5 && beside < p.stages;
        if (!p.shared_ring) p.stages = beside;
    }
    p.ring = (uint32_t)(stage * (size_t)p.stages);
    const size_t smem = 1024 + p.ring + kOutBytes + (p.shared_ring ? 0 : sums);
    Maps maps;
    if (!code_map(&maps.x, codes, M, W.K, r.bt / r.ctas) || !scale_map(&maps.xs, scales, M, W.K, W.format, xa)) return FQ_ERR_CUDA;
    {   // outputs leave in boxes of [16 tokens][32 channels]
        const int e = p.bf16 ? 2 : 4;
        const uint64_t dims[2] = {(uint64_t)W.N * e, (uint64_t)M}, strides[1] = {(uint64_t)ldy * e};
        const uint32_t box[2] = {32u * e, 16};
        if (!encode_tiled(&maps.y, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, y, dims, strides, box, p.bf16 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_NONE))
            return FQ_ERR_CUDA;
    }
    const int units = r.split > 1 ? p.units : (p.units < sms / r.ctas ? p.units : sms / r.ctas);
    p.unit_step = units;
    const int grid = units * r.ctas * r.split;
    const cudaError_t e = r.ctas == 2 ? launch<2, 2>(W, maps, p, grid, smem, stream)
                          : xa == 2  ? launch<1, 2>(W, maps, p, grid, smem, stream)
                                     : launch<1, 1>(W, maps, p, grid, smem, stream);
    *refused = r.ctas * r.split > 1 && cluster_refused(e);
    return e == cudaSuccess ? FQ_OK : FQ_ERR_CUDA;
}
}  // namespace

fq_status launch_gemm_fp4(const uint8_t* codes, const uint8_t* scales, const float* delta, int64_t M, const Fp4Weights& W, void* y, fq_dtype yt,
                          int64_t ldy, cudaStream_t stream) {
    if (M == 0 || W.N == 0) return FQ_OK;
    bool refused = false;
    const fq_status st = launch_planned(codes, scales, delta, M, W, y, yt, ldy, cluster_capacity, stream, &refused);
    return refused ? launch_planned(codes, scales, delta, M, W, y, yt, ldy, no_clusters, stream, &refused) : st;
}

}  // namespace fq
