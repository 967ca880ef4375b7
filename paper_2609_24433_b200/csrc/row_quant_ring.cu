// Rows to codes, for batches of some length: the arithmetic of row_quantize_kernel, bit for bit, with the rows (and those of the
// residual) fetched by TMA into a ring in shared memory.
//
// What the kernel that keeps rows in registers spends its time on are shuffles (16 channels a thread: four butterfly stages of
// 256 channels go across lanes, one shuffle a value each, and an SM has one warp's shuffle a cycle) and rows that wait for
// registers.  Here a thread has E = 64 (or 32) consecutive channels, which only a copy through shared memory gives without reading
// memory in strides: strides 1 .. 32 run in registers, two values an instruction, and at most two stages across lanes; and the rows
// under way take no registers.
//   - One CTA of 16 warps an SM, in row groups of gw warps; a group works on one row at a time and has `depth` slots.
//   - A row is a box (long ones several) of 128-byte lines with the 128-byte swizzle, so that reading 64..256 bytes a thread has no
//     bank conflicts; the half line that may end a row of bf16 is a copy of its own.  The multiplier lies beside the slots in the
//     order that the packed multiply takes.
//   - The stream h = x + residual is written over x in its slot and leaves as a bulk store of the whole row.
//   - E = 64: a thread holds the four block scales of 64 channels of e2m1 with e4m3 scales: one word of its scale tile.
#include <cuda_bf16.h>
#include <string.h>

#include "act_common.cuh"
#include "fp4_common.cuh"
#include "ptx_sm100.cuh"
#include "row_quant.cuh"

namespace fq {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32, kMostSlots = 64;

struct RingArgs {
    int64_t rows, rows_pad;
    int K, block, gw, ngroups, depth;
    float eps, cnorm, clip_ratio;
    const float* mult;
    int mult_ready, residual;
    uint8_t* codes;
    uint8_t* scales;
    int scale_tiles;
    float* delta;
    uint32_t row_bytes;      // of one row in a slot, a multiple of 1024
    uint32_t slot_bytes;
    uint32_t mult_bytes;     // rounded up to 1024
    uint32_t stage_off;      // codes of a warp on their way out (8-bit codes)
    uint32_t* watchdog;
};
// Rows of several boxes, or with a half line behind them.
struct LongArgs : RingArgs {
    int boxes, box_lines, lines;             // (whole lines)
    uint32_t tail_off;       // bf16 rows of an odd number of 64-byte halves: where in a slot the last one lies, 0: none
    uint32_t tx;             // bytes of a slot's copies
    const uint8_t* x;        // (for the halves)
    const uint8_t* r;
    uint8_t* h;
    int64_t pitch_x, pitch_r, pitch_h;       // bytes
};
template <bool BOXES> struct ArgsOf { using type = RingArgs; };
template <> struct ArgsOf<true> { using type = LongArgs; };

__device__ __forceinline__ uint32_t swz128(uint32_t off) { return off ^ (((off >> 7) & 7u) << 4); }
__device__ __forceinline__ void tma_load_lines(uint32_t dst, const CUtensorMap* map, int line, int row, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(line), "r"(row), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void tma_store_lines(const CUtensorMap* map, int line, int row, uint32_t src) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];"
                 ::"l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(line), "r"(row), "r"(src)
                 : "memory");
}
__device__ __forceinline__ void bulk_store_1d(void* dst, uint32_t src, uint32_t bytes) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(src), "r"(bytes) : "memory");
}
// The same box as far as L2 only.
__device__ __forceinline__ void prefetch_lines(const CUtensorMap* map, int line, int row) {
    asm volatile("cp.async.bulk.prefetch.tensor.3d.L2.global.tile [%0, {%1, %2, %3}];"
                 ::"l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(line), "r"(row)
                 : "memory");
}
// Barrier of a row group that also ANDs a predicate.
__device__ __forceinline__ bool group_and(int id, int threads, bool pred) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 q, %3, 0;\n\t"
        "bar.red.and.pred p, %1, %2, q;\n\t"
        "selp.b32 %0, 1, 0, p;\n\t}"
        : "=r"(r)
        : "r"(id), "r"(threads), "r"((uint32_t)pred)
        : "memory");
    return r != 0;
}
__device__ __forceinline__ float max3_abs(float m, float x, float y) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(m), "f"(fabsf(x)), "f"(fabsf(y)));
    return r;
}
// (not volatile: may be batched and hoisted; their addresses are pinned behind the wait that makes the data valid)
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
    uint4 v;
    asm("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
    return v;
}
__device__ __forceinline__ float4 lds128f_ordered(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
    return v;
}
__device__ __forceinline__ uint4 lds128_ordered(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void sts128(uint32_t addr, uint4 v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void pin(uint32_t& addr) { asm volatile("" : "+r"(addr) : : "memory"); }
// 16-byte piece i of a thread's slice of a swizzled row, whose (at most two) 128-byte lines begin at line0, line1.
__device__ __forceinline__ uint32_t piece(uint32_t line0, uint32_t line1, int i) { return (i < 8 ? line0 : line1) ^ (uint32_t)((i & 7) << 4); }
__device__ __forceinline__ uint32_t add_bf16x2(uint32_t a, uint32_t b) {          // in binary32, rounded once
    const float2 s = f2_add(make_float2(__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u)),
                            make_float2(__uint_as_float(b << 16), __uint_as_float(b & 0xffff0000u)));
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(s.y), "f"(s.x));
    return r;
}
__device__ __forceinline__ uint32_t add_f32(uint32_t a, uint32_t b) { return __float_as_uint(__fadd_rn(__uint_as_float(a), __uint_as_float(b))); }

// BLOCK: channels of the rotation, 0: p.block.  (Branches between the stages cost more than the stages: 13056 x 2048 in blocks of 128,
// MXFP4, 24.9 us with and 20.8 without them.)  BOXES: rows of LongArgs; the others keep to arguments of 512 bytes, since with more
// of them the same code spills (21.7 us).
template <typename XT, int E, int FMT, bool NORM, int BLOCK, bool BOXES>
__global__ void __launch_bounds__(kThreads, 1)
row_quantize_ring_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_r, const __grid_constant__ CUtensorMap map_h,
                         const typename ArgsOf<BOXES>::type p) {
    constexpr bool kFp4 = FMT >= 3, kMx = FMT == 3;
    constexpr int H = E / 2;                               // v[i] = (channel i, channel i + H)
    const int block = BLOCK ? BLOCK : p.block;
    uint32_t tail_off = 0u, tx = (uint32_t)p.K * (uint32_t)sizeof(XT) * (NORM && p.residual != 0 ? 2u : 1u);
    if constexpr (BOXES) {
        tail_off = p.tail_off;
        tx = p.tx;
    }
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t s_full[kMostSlots];
    __shared__ float2 s_part[2][kWarps];
    __shared__ int s_abort;

    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int ngroups = p.ngroups, group = warp / p.gw, wg = warp - group * p.gw;
    const bool idle = group >= ngroups;                    // warps left over
    const int col0 = (wg * 32 + lane) * E;
    const bool col_ok = col0 < p.K && !idle;
    const bool leader = wg == 0 && lane == 0 && !idle;
    volatile int* abort_flag = &s_abort;
    const bool residual = NORM && p.residual != 0;

    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* gen = smem_raw + (base - smem_u32(smem_raw));

    if (threadIdx.x == 0) {
        s_abort = 0;
        for (int s = 0; s < ngroups * p.depth; ++s) mbar_init(smem_u32(&s_full[s]), 1);
        fence_mbarrier_init();
        fence_proxy_async_smem();
    }
    auto stage_multiplier = [&]() {
        if (!p.mult) return;
        // a thread's slice as pairs (g[q], g[q + H]), its 16-byte pieces mixed by the slice's number
#pragma unroll 4
        for (int i = threadIdx.x; i < (BOXES ? (p.K + E - 1) / E * (H / 4) : p.K / 8); i += kThreads) {
            const uint32_t slice = (uint32_t)i / (H / 4), q = (uint32_t)i % (H / 4) * 4u, key = (slice & 7u) << 4;
            const float4 lo = ld_global_f4(p.mult + slice * E + q);
            const float4 hi = ld_global_f4(p.mult + slice * E + H + q, !BOXES || slice * E + H + q < (uint32_t)p.K);       // (zeros past K)
            const uint32_t to = base + slice * (E * 4u);
            sts128(to + ((q * 8u) ^ key), make_uint4(__float_as_uint(lo.x), __float_as_uint(hi.x), __float_as_uint(lo.y), __float_as_uint(hi.y)));
            sts128(to + ((q * 8u + 16u) ^ key), make_uint4(__float_as_uint(lo.z), __float_as_uint(hi.z), __float_as_uint(lo.w), __float_as_uint(hi.w)));
        }
    };
    if (p.mult_ready) stage_multiplier();
    if (tail_off) {                                      // what follows a last half line in its thread's slice: zeros, for good
        const int pieces = ngroups * p.depth * (residual ? 2 : 1) * 4;
        for (int i = threadIdx.x; i < pieces; i += kThreads)
            sts128(base + p.mult_bytes + (uint32_t)(i >> 2) * p.row_bytes + tail_off + 64u + (uint32_t)(i & 3) * 16u, make_uint4(0u, 0u, 0u, 0u));
    }
    __syncthreads();                                       // barriers before any copy
    griddep_wait();
    griddep_launch_dependents();

    const int rows = (int)p.rows, first = group * (int)gridDim.x + (int)blockIdx.x, step = (int)gridDim.x * ngroups;
    const uint32_t slot0 = base + p.mult_bytes + (uint32_t)(group * p.depth) * p.slot_bytes;
    uint64_t* const full0 = &s_full[group * p.depth];
    // f(line, bytes from the slot's begin) for each box of a row
    auto each_box = [&](auto&& f) {
        if constexpr (BOXES)
            for (int b = 0; b < p.boxes; ++b) f(b * p.box_lines, (uint32_t)(b * p.box_lines) * 128u);
        else
            f(0, 0u);
    };
    auto request = [&](int d, int row) {
        const uint32_t bar = smem_u32(&full0[d]), slot = slot0 + (uint32_t)d * p.slot_bytes;
        mbar_arrive_expect_tx(bar, tx);
        each_box([&](int line, uint32_t at) {
            tma_load_lines(slot + at, &map_x, line, row, bar);
            if (residual) tma_load_lines(slot + p.row_bytes + at, &map_r, line, row, bar);
        });
        if constexpr (BOXES)
            if (tail_off) {
                bulk_load_1d(slot + tail_off, p.x + row * p.pitch_x + p.lines * 128, 64u, bar);
                if (residual) bulk_load_1d(slot + p.row_bytes + tail_off, p.r + row * p.pitch_r + p.lines * 128, 64u, bar);
            }
    };
    int issued = 0;
    if (leader) {
        for (int d = 0; d < p.depth; ++d) {
            const int r = first + d * step;
            if (r < rows) { request(d, r); ++issued; }
        }
    }
    if (!p.mult_ready) stage_multiplier();
    __syncthreads();

    // scale tiles of the rows that only pad the last one
    if (kFp4)
        for (int64_t row = p.rows + blockIdx.x; row < p.rows_pad; row += gridDim.x)
            for (int t = threadIdx.x; t < p.scale_tiles; t += kThreads)
                *reinterpret_cast<uint32_t*>(p.scales + ((row >> 7) * p.scale_tiles + t) * 512 + (row & 31) * 16 + ((row & 127) >> 5) * 4) = 0u;
    if (idle) return;

    const uint32_t xs0 = tail_off && col0 == p.K - 32 ? tail_off : swz128((uint32_t)col0 * (uint32_t)sizeof(XT)), xs1 = swz128((uint32_t)col0 * (uint32_t)sizeof(XT) + 128u);
    const uint32_t gkey = (uint32_t)((col0 / E) & 7) << 4;
    const uint32_t g0 = base + (((uint32_t)col0 * 4u) ^ gkey), g1 = base + (((uint32_t)col0 * 4u + 128u) ^ gkey);
    const float2 neg1 = make_float2(-1.0f, -1.0f);
    const bool warp_ok = __all_sync(0xffffffffu, col_ok);
    const uint32_t stage = base + p.stage_off + (uint32_t)(warp * 32 * E);

    int n = 0, d = 0;
    uint32_t ph = 0;
    for (int row = first; row < rows; row += step, ++n) {
        bool ok = mbar_wait_all(smem_u32(&full0[d]), ph, abort_flag, p.watchdog, 0x100u);
        const uint32_t slot = slot0 + (uint32_t)d * p.slot_bytes;
        if (leader && p.depth == 1 && row + step < rows) {     // the next row has no slot yet: to L2 meanwhile
            each_box([&](int line, uint32_t) {
                prefetch_lines(&map_x, line, row + step);
                if (residual) prefetch_lines(&map_r, line, row + step);
            });
        }
        float2 v[H];
        float ss = 0.0f;
        auto load_row = [&]() {
            uint32_t x0 = slot + xs0, x1 = slot + xs1;
            pin(x0);
            pin(x1);
            constexpr int kPieces = H * (int)sizeof(XT) / 16;      // of half a slice
            constexpr int kPer = 16 / (int)sizeof(XT);             // channels of a piece
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const uint32_t alo = piece(x0, x1, i), ahi = piece(x0, x1, i + kPieces);
                uint4 lo = lds128(alo), hi = lds128(ahi);
                if (residual) {
                    const uint4 rl = lds128(alo + p.row_bytes), rh = lds128(ahi + p.row_bytes);
                    if (sizeof(XT) == 2) {
                        lo = make_uint4(add_bf16x2(lo.x, rl.x), add_bf16x2(lo.y, rl.y), add_bf16x2(lo.z, rl.z), add_bf16x2(lo.w, rl.w));
                        hi = make_uint4(add_bf16x2(hi.x, rh.x), add_bf16x2(hi.y, rh.y), add_bf16x2(hi.z, rh.z), add_bf16x2(hi.w, rh.w));
                    } else {
                        lo = make_uint4(add_f32(lo.x, rl.x), add_f32(lo.y, rl.y), add_f32(lo.z, rl.z), add_f32(lo.w, rl.w));
                        hi = make_uint4(add_f32(hi.x, rh.x), add_f32(hi.y, rh.y), add_f32(hi.z, rh.z), add_f32(hi.w, rh.w));
                    }
                    sts128(alo, lo);
                    sts128(ahi, hi);
                }
                const uint32_t wl[4] = {lo.x, lo.y, lo.z, lo.w}, wh[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (sizeof(XT) == 2) {
                        v[kPer * i + 2 * j + 0] = make_float2(__uint_as_float(wl[j] << 16), __uint_as_float(wh[j] << 16));
                        v[kPer * i + (2 * j + 1) % kPer] = make_float2(__uint_as_float(wl[j] & 0xffff0000u), __uint_as_float(wh[j] & 0xffff0000u));
                    } else {
                        v[kPer * i + j % kPer] = make_float2(__uint_as_float(wl[j]), __uint_as_float(wh[j]));
                    }
                }
            }
            if (NORM) {
                float2 s2 = make_float2(0.0f, 0.0f), t2 = s2;
#pragma unroll
                for (int i = 0; i < H; i += 2) {
                    s2 = f2_fma(v[i], v[i], s2);
                    t2 = f2_fma(v[i + 1], v[i + 1], t2);
                }
                ss = (s2.x + s2.y) + (t2.x + t2.y);
            }
            if (p.mult) {
#pragma unroll
                for (int i = 0; i < H / 2; ++i) {
                    const float4 q = lds128f_ordered(piece(g0, g1, i));
                    v[2 * i + 0] = f2_mul(v[2 * i + 0], make_float2(q.x, q.y));
                    v[2 * i + 1] = f2_mul(v[2 * i + 1], make_float2(q.z, q.w));
                }
            } else {
#pragma unroll
                for (int i = 0; i < H; ++i) v[i] = f2_mul(v[i], make_float2(p.cnorm, p.cnorm));
            }
        };
        if (warp_ok) {                                     // (uniform: no lane of the warp is past K)
            load_row();
        } else if (col_ok) {
            load_row();
        } else {
#pragma unroll
            for (int i = 0; i < H; ++i) v[i] = make_float2(0.0f, 0.0f);
        }
#pragma unroll
        for (int s = 1; s < H; s <<= 1) {
            if (s < block) {
#pragma unroll
                for (int i = 0; i < H; ++i) {
                    if ((i & s) == 0) {
                        const float2 a = v[i], b = v[i + s];
                        v[i] = f2_add(a, b);
                        v[i + s] = f2_fma(b, neg1, a);         // a - b, exact product
                    }
                }
            }
        }
        if (H < block) {
#pragma unroll
            for (int i = 0; i < H; ++i) v[i] = make_float2(__fadd_rn(v[i].x, v[i].y), __fsub_rn(v[i].x, v[i].y));
        }
        // the lane with the bit keeps partner - own
        auto across = [&](int lm) {
            const float sgn = (lane & lm) ? -1.0f : 1.0f;
#pragma unroll
            for (int i = 0; i < H; ++i) {
                const float2 o = make_float2(__shfl_xor_sync(0xffffffffu, v[i].x, lm), __shfl_xor_sync(0xffffffffu, v[i].y, lm));
                v[i] = f2_fma(v[i], make_float2(sgn, sgn), o);
            }
        };
        if constexpr (BLOCK != 0) {
#pragma unroll
            for (int s = E; s < BLOCK; s <<= 1) across(s / E);
        } else {
            for (int s = E; s < block; s <<= 1) across(s / E);
        }
        // largest magnitudes of the thread's blocks of 16 channels (32: E = 32 has two of 16, one of 32)
        float mb[E / 16];
#pragma unroll
        for (int b = 0; b < E / 32; ++b) {
            float lo = 0.0f, hi = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                lo = max3_abs(lo, v[16 * b + i].x, v[16 * b + i + 1].x);
                hi = max3_abs(hi, v[16 * b + i].y, v[16 * b + i + 1].y);
            }
            mb[b] = lo;
            mb[b + E / 32] = hi;
        }
        float m = mb[0];
#pragma unroll
        for (int b = 1; b < E / 16; ++b) m = fmaxf(m, mb[b]);
        m = warp_max_nonneg(m);
        float total = NORM ? warp_sum(ss) : 0.0f;
        if (residual) fence_proxy_async_smem();               // the stream's row, written here, is read by the copy engine
        if (p.gw > 1) {
            if (lane == 0) s_part[n & 1][warp] = make_float2(m, total);
            ok = group_and(1 + group, p.gw * 32, ok);
            const float2 t = lane < p.gw ? s_part[n & 1][group * p.gw + lane] : make_float2(0.0f, 0.0f);
            m = warp_max_nonneg(t.x);
            if (NORM && wg == 0) total = warp_sum(t.y);
        } else {
            __syncwarp();
        }
        if (!ok) break;
        float rinv = 1.0f;                                     // (-1: the step is written already)
        if (NORM && wg == 0) {
            if (squares_leave_range(total, m, p.eps)) {
                double s = 0.0;                                // the row as it lies in its slot, in binary64
                auto square = [&](uint32_t at) {
                    const uint32_t w = *reinterpret_cast<const volatile uint32_t*>(gen + (slot - base) + at);
                    if (sizeof(XT) == 2) {
                        const double a = (double)__uint_as_float(w << 16), b = (double)__uint_as_float(w & 0xffff0000u);
                        s += a * a + b * b;
                    } else {
                        s += (double)__uint_as_float(w) * (double)__uint_as_float(w);
                    }
                };
                const uint32_t end = (uint32_t)p.K * (uint32_t)sizeof(XT) - (tail_off ? 64u : 0u);
                for (uint32_t at = (uint32_t)lane * 4u; at < end; at += 128u) square(at);
                if (tail_off) square(tail_off + (uint32_t)lane * 4u);        // (zeros behind it)
                for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
                if (lane == 0) p.delta[row] = wide_step<FMT>(m, p.clip_ratio, s, p.K, p.eps);
                rinv = -1.0f;
            } else {
                rinv = inverse_rms(total, p.K, p.eps);
            }
            __syncwarp();
        }
        // Every warp of the group has read the slot.  Without a residual it is refilled here; with one its row goes out first, and the
        // slot of the row before, whose store has had time to read it, is refilled (of a single slot: its own).
        if (leader) {
            if (residual) {
                each_box([&](int line, uint32_t at) { tma_store_lines(&map_h, line, row, slot + at); });
                if constexpr (BOXES)
                    if (tail_off) bulk_store_1d(p.h + row * p.pitch_h + p.lines * 128, slot + tail_off, 64u);
                bulk_commit();
                if (p.depth == 1) {
                    bulk_wait_read<0>();
                    if (row + step < rows) { request(0, row + step); ++issued; }
                } else if (n > 0) {
                    const int nr = row + (p.depth - 1) * step;
                    bulk_wait_read<1>();
                    if (nr < rows) { request(d == 0 ? p.depth - 1 : d - 1, nr); ++issued; }
                }
            } else if (row + p.depth * step < rows) {
                fence_proxy_async_smem();
                request(d, row + p.depth * step);
                ++issued;
            }
        }
        float dl = 1.0f;
        if (kFp4) {
            float q[E / 16];
            uint32_t word = 0u;
            if (kMx) {
#pragma unroll
                for (int b = 0; b < E / 32; ++b) {
                    // (E = 64: halves of 32 channels; E = 32: one block across both halves)
                    const float mm = E == 64 ? fmaxf(mb[(2 * b) % (E / 16)], mb[(2 * b + 1) % (E / 16)]) : fmaxf(mb[0], mb[1]);
                    float qq;
                    word |= mx_scale(mm, &qq) << (8 * b);
                    q[(2 * b) % (E / 16)] = q[(2 * b + 1) % (E / 16)] = qq;
                }
                if (!col_ok) word = 0u;
                constexpr int kShare = 128 / E;                // threads of a word
                word <<= 8 * (E / 32) * (lane % kShare);
#pragma unroll
                for (int o = 1; o < kShare; o <<= 1) word |= __shfl_xor_sync(0xffffffffu, word, o);
            } else {
                float inv;
                dl = nv_step(m, &inv);
#pragma unroll
                for (int b = 0; b < E / 16; ++b) word |= nv_scale(mb[b], inv, &q[b]) << (8 * b);
                if (!col_ok) word = 0u;
                if (E == 32) {
                    word <<= 16 * (lane & 1);
                    word |= __shfl_xor_sync(0xffffffffu, word, 1);
                }
            }
            const int tile = col0 / (kMx ? 128 : 64);
            if (tile < p.scale_tiles && lane % ((kMx ? 128 : 64) / E) == 0)
                *reinterpret_cast<uint32_t*>(p.scales + ((int64_t)(row >> 7) * p.scale_tiles + tile) * 512 + (row & 31) * 16 + ((row & 127) >> 5) * 4) = word;
            uint32_t w[E / 8];
#pragma unroll
            for (int b = 0; b < E / 32; ++b) {
                const float2 q2 = make_float2(q[b], q[b + E / 32]);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float lo[8], hi[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float2 t = f2_mul(v[16 * b + 8 * j + i], q2);
                        lo[i] = t.x;
                        hi[i] = t.y;
                    }
                    w[2 * b + j] = pack_e2m1(lo);
                    w[2 * b + j + E / 16] = pack_e2m1(hi);
                }
            }
            if (col_ok) {
                uint4* dst = reinterpret_cast<uint4*>(p.codes + (int64_t)row * (p.K / 2) + col0 / 2);
#pragma unroll
                for (int j = 0; j < E / 32; ++j)
                    if (!BOXES || j == 0 || col0 + 32 * j < p.K) dst[j] = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
            }
        } else {
            constexpr int kPer = FMT == 0 ? 8 : 4, kWords = H / kPer;      // codes of a word, words of a half
            constexpr float kMost = FMT == 0 ? 7.0f : 127.0f;
            float inv;
            dl = int_step(m, p.clip_ratio, 1.0f / kMost, &inv);
            uint32_t w[2 * kWords];
#pragma unroll
            for (int j = 0; j < kWords; ++j) {
                uint32_t bl[kPer], bh[kPer];
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    float2 t = f2_mul(v[kPer * j + i], make_float2(inv, inv));
                    if (p.clip_ratio < 1.0f) {
                        t.x = fminf(fmaxf(t.x, -kMost), kMost);
                        t.y = fminf(fmaxf(t.y, -kMost), kMost);
                    }
                    // (as a packed FMA by 1: a packed multiply ahead of a packed add may be fused, which rounds ties differently)
                    t = f2_fma(t, make_float2(1.0f, 1.0f), make_float2(12582912.0f, 12582912.0f));
                    bl[i] = __float_as_uint(t.x);
                    bh[i] = __float_as_uint(t.y);
                }
                w[j] = pack_word<FMT>(bl);
                w[kWords + j] = pack_word<FMT>(bh);
            }
            if (FMT == 1) {
                // E bytes a thread: through shared memory (pieces mixed by the lane), so that a warp's store is one run
                constexpr int kP = E / 16;
                __syncwarp();
#pragma unroll
                for (int j = 0; j < kP; ++j)
                    sts128(stage + (uint32_t)(lane * E) + (uint32_t)((j ^ ((lane * E >> 7) & (kP - 1))) << 4),
                           make_uint4(w[(4 * j) % (2 * kWords)], w[(4 * j + 1) % (2 * kWords)], w[(4 * j + 2) % (2 * kWords)], w[(4 * j + 3) % (2 * kWords)]));
                __syncwarp();
#pragma unroll
                for (int j = 0; j < kP; ++j) {
                    const int at = j * 32 + lane, owner = at / kP, pc = at % kP;           // 16-byte piece `at` of the warp's run
                    const uint4 o = lds128_ordered(stage + (uint32_t)(owner * E) + (uint32_t)((pc ^ ((owner * E >> 7) & (kP - 1))) << 4));
                    if (wg * 32 * E + at * 16 < p.K) *reinterpret_cast<uint4*>(p.codes + (int64_t)row * p.K + wg * 32 * E + at * 16) = o;
                }
            } else if (col_ok) {
                uint4* dst = reinterpret_cast<uint4*>(p.codes + (int64_t)row * (p.K / 2) + col0 / 2);
#pragma unroll
                for (int j = 0; j < E / 32; ++j)
                    if (!BOXES || j == 0 || col0 + 32 * j < p.K) dst[j] = make_uint4(w[(4 * j) % (2 * kWords)], w[(4 * j + 1) % (2 * kWords)], w[(4 * j + 2) % (2 * kWords)], w[(4 * j + 3) % (2 * kWords)]);
            }
        }
        if (leader && !(NORM && rinv < 0.0f)) p.delta[row] = NORM ? __fmul_rn(dl, rinv) : dl;
        if (++d == p.depth) { d = 0; ph ^= 1u; }
    }
    if (leader && residual) bulk_wait_read<0>();             // the last rows have left shared memory
    // winding down after an expired wait: copies under way land first
    if (leader && *abort_flag) {
        for (int k = n; k < issued; ++k) {
            const uint64_t t0 = global_timer_ns();
            while (!mbar_try_wait(smem_u32(&full0[k % p.depth]), (uint32_t)((k / p.depth) & 1)))
                if (global_timer_ns() - t0 > kWaitLimitNs) { atomicOr(p.watchdog, 0x200u); break; }
        }
    }
}

struct RowMaps {
    CUtensorMap x, r, h;
};
template <typename XT, int E, int FMT, bool NORM, int BLOCK, bool BOXES>
cudaError_t go(const RowMaps& maps, const LongArgs& p, int grid, size_t smem, cudaStream_t stream) {
    auto kern = row_quantize_ring_kernel<XT, E, FMT, NORM, BLOCK, BOXES>;
    const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kern), smem);
    if (e != cudaSuccess) return e;
    return launch_pdl(kern, (unsigned)grid, (unsigned)kThreads, smem, stream, 1u, maps.x, maps.r, maps.h, static_cast<const typename ArgsOf<BOXES>::type&>(p));
}
template <typename XT, int E, int FMT, bool NORM, bool BOXES>
cudaError_t by_block(const RowMaps& maps, const LongArgs& p, int grid, size_t smem, cudaStream_t stream) {
    if constexpr (E == 64) {
        switch (p.block) {
            case 1: return go<XT, E, FMT, NORM, 1, BOXES>(maps, p, grid, smem, stream);
            case 64: return go<XT, E, FMT, NORM, 64, BOXES>(maps, p, grid, smem, stream);
            case 128: return go<XT, E, FMT, NORM, 128, BOXES>(maps, p, grid, smem, stream);
            case 256: return go<XT, E, FMT, NORM, 256, BOXES>(maps, p, grid, smem, stream);
        }
    }
    return go<XT, E, FMT, NORM, 0, BOXES>(maps, p, grid, smem, stream);
}
template <typename XT, int E, int FMT, bool NORM>
cudaError_t by_boxes(const RowMaps& maps, const LongArgs& p, int grid, size_t smem, cudaStream_t stream) {
    return p.boxes > 1 || p.tail_off ? by_block<XT, E, FMT, NORM, true>(maps, p, grid, smem, stream)
                                     : by_block<XT, E, FMT, NORM, false>(maps, p, grid, smem, stream);
}
template <typename XT, int E>
cudaError_t by_format(const RowQuant& q, const RowMaps& maps, const LongArgs& p, int grid, size_t smem, cudaStream_t stream) {
    switch (q.fmt) {
        case RowFmt::Int4: return by_boxes<XT, E, 0, true>(maps, p, grid, smem, stream);
        case RowFmt::Int8: return by_boxes<XT, E, 1, true>(maps, p, grid, smem, stream);
        case RowFmt::Mx: return q.norm ? by_boxes<XT, E, 3, true>(maps, p, grid, smem, stream) : by_boxes<XT, E, 3, false>(maps, p, grid, smem, stream);
        case RowFmt::Nv: return q.norm ? by_boxes<XT, E, 4, true>(maps, p, grid, smem, stream) : by_boxes<XT, E, 4, false>(maps, p, grid, smem, stream);
    }
    return cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_row_quantize_ring(const RowQuant& q, cudaStream_t stream) {
    if (q.rows < 256) return cudaErrorNotSupported;
    const size_t esz = q.xt == FQ_BF16 ? 2 : 4, row = (size_t)q.K * esz;
    const int sms = device_sm_count();
    // rows enough for several a group
    if (q.rows < 2 * sms || q.rows * q.K < (int64_t)sms * 8192 || q.rows > 0x7fff0000) return cudaErrorNotSupported;
    // Rows that end in half a line: short ones leave many lanes idle here, which the other kernel spreads over more warps
    // (13000 x 2080 with norm and residual 60 us against 45; 4000 x 8224 58 against 78).
    const bool tail = row % 128 != 0;
    if (tail && q.K <= 8192) return cudaErrorNotSupported;
    LongArgs p = {};
    p.lines = (int)(row / 128);
    p.boxes = (p.lines + 255) / 256;                          // (a box has 256 lines at most; of several, each begins on 1024 bytes)
    p.box_lines = p.boxes == 1 ? p.lines : ((p.lines + p.boxes - 1) / p.boxes + 7) / 8 * 8;
    const size_t whole = (size_t)p.boxes * p.box_lines * 128;
    p.tail_off = tail ? (uint32_t)whole : 0;
    p.row_bytes = (uint32_t)align_up(whole + (tail ? 128 : 0), 1024);
    p.slot_bytes = p.row_bytes * (q.residual ? 2 : 1);
    p.tx = (uint32_t)(whole + (tail ? 64 : 0)) * (q.residual ? 2 : 1);
    p.x = static_cast<const uint8_t*>(q.x); p.r = static_cast<const uint8_t*>(q.residual); p.h = static_cast<uint8_t*>(q.h);
    p.pitch_x = q.ldx * (int64_t)esz; p.pitch_r = q.ldr * (int64_t)esz; p.pitch_h = q.ldh * (int64_t)esz;
    p.mult_bytes = q.mult ? (uint32_t)align_up(sizeof(float) * align_up((size_t)q.K, 64), 1024) : 0;
    // 64 channels a thread; 32 where rows are short, where 8-bit codes on their way out would take the room of the only slot, and
    // where the slots of binary32 rows leave half of the warps idle (4000 x 8192 with norm 78 us against 73; bf16, which would pay
    // the wider rotation more dearly, 114 against 151 at 4000 x 16384)
    auto shape = [&](int e, int* gw, int* groups, size_t* stage) {
        *gw = (int)((q.K + 32 * e - 1) / (32 * e));
        *stage = q.fmt == RowFmt::Int8 ? (size_t)kThreads * e : 0;
        const int64_t room = 220 * 1024 - (int64_t)*stage - (int64_t)p.mult_bytes;
        const int slots = room > 0 ? (int)(room / p.slot_bytes) : 0;
        *groups = *gw > kWarps ? 0 : slots < kWarps / *gw ? slots : kWarps / *gw;
        p.depth = *groups > 0 ? (slots / *groups < 4 ? slots / *groups : 4) : 0;
    };
    int e = (tail || q.K % 64 == 0) && q.K >= 1536 ? 64 : 32, gw, groups;
    size_t stage;
    shape(e, &gw, &groups, &stage);
    if (e == 64 && (groups < 1 || (esz == 4 && groups * gw <= kWarps / 2))) {
        e = 32;
        shape(e, &gw, &groups, &stage);
        if (groups < 1) {
            e = 64;
            shape(e, &gw, &groups, &stage);
        }
    }
    if (groups < 1 || p.depth < 1) return cudaErrorNotSupported;
    p.ngroups = groups;
    const bool fp4 = q.fmt == RowFmt::Mx || q.fmt == RowFmt::Nv;
    p.rows = q.rows;
    p.rows_pad = fp4 ? (q.rows + 127) / 128 * 128 : q.rows;
    p.K = (int)q.K; p.block = q.block; p.gw = gw;
    p.eps = q.eps; p.cnorm = q.cnorm; p.clip_ratio = q.clip_ratio;
    p.mult = q.mult; p.mult_ready = q.mult_ready ? 1 : 0; p.residual = q.residual ? 1 : 0;
    p.codes = q.codes; p.scales = q.scales; p.delta = q.delta;
    p.scale_tiles = fp4 ? (int)fp4_scale_tiles(q.K, q.fmt == RowFmt::Nv ? FQ_NVFP4 : FQ_MXFP4) : 0;
    p.stage_off = p.mult_bytes + p.slot_bytes * (uint32_t)(p.ngroups * p.depth);
    p.watchdog = watchdog_device_ptr();
    if (!p.watchdog) return cudaErrorUnknown;
    RowMaps maps;
    auto map = [&](CUtensorMap* m, const void* ptr, int64_t ld) {
        const uint64_t dims[3] = {128 / esz, (uint64_t)p.lines, (uint64_t)q.rows}, strides[2] = {128, (uint64_t)ld * esz};
        const uint32_t box[3] = {(uint32_t)(128 / esz), (uint32_t)p.box_lines, 1};
        return encode_tiled(m, esz == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, ptr, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
    };
    if (!map(&maps.x, q.x, q.ldx)) return cudaErrorNotSupported;
    maps.r = maps.h = maps.x;
    if (q.residual && (!map(&maps.r, q.residual, q.ldr) || !map(&maps.h, q.h, q.ldh))) return cudaErrorNotSupported;
    const size_t smem = 1024 + p.stage_off + stage;
    const int grid = (int)(q.rows < sms ? q.rows : sms);
    if (q.xt == FQ_F32) return e == 64 ? by_format<float, 64>(q, maps, p, grid, smem, stream) : by_format<float, 32>(q, maps, p, grid, smem, stream);
    return e == 64 ? by_format<__nv_bfloat16, 64>(q, maps, p, grid, smem, stream) : by_format<__nv_bfloat16, 32>(q, maps, p, grid, smem, stream);
}

}  // namespace fq
