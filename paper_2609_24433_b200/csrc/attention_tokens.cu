// Attention of a few queries -- at most 16 (token, head of a group) rows a kv head, a decoding step -- over the 8-bit cache.
//
// Bound by the cache's bytes, so everything serves the loads: no thread waits for another on the way from memory to the
// matrix instructions.  Each lane copies (cp.async, 16 bytes) exactly the bytes that it will multiply into slots of its own, in
// pieces of 64 tokens x 64 channels four ahead, and waits for nothing but its own copies: no barrier until the end of
// a share's part of a tile.
//
// The products run transposed, S^T = K Q^T and O^T = V^T P^T: the cache's operand then fills the 16 rows of a warp-level MMA
// (m16n8k16, binary16 in, binary32 out) and the few queries its 8 columns, with no row idle at one query of a group of eight.
// Codes become binary16 exactly: byte permutes put (code + 128) under the exponent of 1024, one packed subtraction takes
// 1152 off.  The order in which an MMA walks channels (of S) and tokens (of O) is free as long as both operands use it, so a
// lane's 16 contiguous bytes are four steps of it: k16 step i of a 64-wide line takes bytes 16 t + 4 i .. + 3 of thread t of
// four.  Queries are divided by the power of two below their row's largest channel and rounded to binary16 (bf16 values
// keep all their bits above 2^-14 of the row's largest channel; binary32 queries and probabilities go as a sum of two terms).
//
// Every CTA takes an equal share of the call's blocks -- 256 keys of 8 or 16 rows of a kv head -- wherever that begins and ends:
// lengths are known on the device only.  A tile of rows that several shares divide is joined by a second kernel; the others are
// written here.  (48 sequences of 1 to 16384 keys, 8 heads of 128, 127 us at the measured copy rate: chunks of 4096 keys 148 us,
// shares 142; 64 of 8192 keys, 2 heads of 256, 83 at the copy rate: 112 and 95; one of 16384: 17.4 and 15.8.  Shares end up to 12 %
// apart, by what their SMs get of the memory; smaller last ones, handed out as CTAs end, cost more than they level: 147.)
//
// With p = 2^(s - m): l = sum p, O = sum (p vs 2^(7 - e)) code, e the running exponent of the largest value scale vs.  m follows the
// maximum lazily, when it has risen by more than 2^8: probabilities stay below 2^15 and, down to 2^-21, normal in binary16.
#include "attention_common.cuh"

#include <cuda_fp16.h>
#include <float.h>

namespace fq {
namespace {

constexpr int kTile = 64;               // tokens
constexpr int kSlots = 4;
constexpr int kPiece = 4096;            // 64 tokens x 64 channels: eight 16-byte units per lane
constexpr int kWarps = 4;
constexpr float kSlack = 8.0f;

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool ok) {        // zeros where !ok
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ uint4 lds_v4(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
// Four int8 -> two pairs of binary16.
__device__ __forceinline__ void widen(uint32_t w, uint32_t* lo, uint32_t* hi) {
    const uint32_t u = w ^ 0x80808080u;
    const __half2 base = __half2half2(__ushort_as_half(0x6480));
    const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
    const __half2 x = __hsub2(*reinterpret_cast<const __half2*>(&a), base), y = __hsub2(*reinterpret_cast<const __half2*>(&b), base);
    *lo = *reinterpret_cast<const uint32_t*>(&x);
    *hi = *reinterpret_cast<const uint32_t*>(&y);
}
__device__ __forceinline__ void mma(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 unpack_half(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
__device__ __forceinline__ uint32_t transpose8(uint32_t w) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(w));
    return r;
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ int exponent_of(float x) { return (int)((__float_as_uint(x) >> 23) & 255) - 127; }
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(min(max(e, -126), 127) + 127) << 23); }

// CTAs that an SM holds at once.
constexpr int tokens_resident(bool bf16, int dp, int nq) { return nq == 1 && bf16 && dp <= 128 ? 3 : 2; }

// Where a share leaves the result of its last tile (begins: block 0 is in this share), or else of its first.
__device__ __forceinline__ int64_t tokens_seat(int cta, bool begins) { return 2 * (int64_t)cta + (begins ? 1 : 0); }

// Blocks of work: of a sequence, per tile of its rows.
struct Work {
    int64_t units;                      // (tile of rows, kv head)
    int per_unit;
};
__device__ __forceinline__ Work work_of(const Attention& a, const Sequence& s, int rows) {
    Work w;
    w.units = (s.queries * a.group + rows - 1) / rows * a.kv_heads;
    w.per_unit = max((int)((s.keys + kTokensBlock - 1) / kTokensBlock), 1);
    return w;
}
// The share of this CTA, blocks first .. last - 1 of all `total`, and the sequence with the first one.
struct Share {
    int64_t first, last, total, shares; // as many shares as CTAs, or as blocks
    int64_t within;                     // blocks of the sequence ahead of the first one
    int b;
    Sequence sequence;                  // (looked up once: a round trip to memory)
};
__device__ __forceinline__ Share share_of(const Attention& a, int rows) {
    __shared__ int64_t sums[kWarps];
    __shared__ int64_t found[5];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, each = (a.batch + kWarps * 32 - 1) / (kWarps * 32);
    const int b0 = min((int)threadIdx.x * each, a.batch), b1 = min(b0 + each, a.batch);
    Sequence s = {};
    auto blocks = [&](int b) {
        s = sequence_of(a, b);
        const Work w = work_of(a, s, rows);
        return w.units * w.per_unit;
    };
    int64_t own = 0;
    for (int b = b0; b < b1; ++b) own += blocks(b);
    int64_t upto = own;                 // this thread's last
#pragma unroll
    for (int x = 1; x < 32; x <<= 1) {
        const int64_t v = __shfl_up_sync(0xffffffffu, upto, x);
        if (lane >= x) upto += v;
    }
    if (lane == 31) sums[warp] = upto;
    __syncthreads();
    Share r;
    r.total = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) upto += sums[w];
        r.total += sums[w];
    }
    r.shares = min((int64_t)gridDim.x, r.total);                // (none empty: the join goes through them without a gap)
    r.first = r.shares > (int)blockIdx.x ? r.total * blockIdx.x / r.shares : r.total;
    r.last = r.shares > (int)blockIdx.x ? r.total * (blockIdx.x + 1) / r.shares : r.total;
    if (upto - own <= r.first && r.first < upto) {
        int64_t ahead = r.first - (upto - own);
        int b = b0;
        if (each > 1)                   // (else s is the one)
            for (int64_t n; ahead >= (n = blocks(b)); ++b) ahead -= n;
        found[0] = b;
        found[1] = ahead;
        found[2] = s.q0;
        found[3] = s.queries;
        found[4] = s.keys;
    }
    __syncthreads();
    r.b = (int)found[0];                // (only read where first < last)
    r.within = found[1];
    r.sequence.k0 = 0;
    r.sequence.q0 = found[2];
    r.sequence.queries = found[3];
    r.sequence.keys = found[4];
    return r;
}

template <typename T, int DP, int NQ, bool EXACT>
__global__ void __launch_bounds__(kWarps * 32, tokens_resident(sizeof(T) == 2, DP, NQ)) attention_tokens_kernel(const Attention a) {
    constexpr int kTerms = sizeof(T) == 4 ? 2 : 1;              // binary16 terms of a query or probability
    constexpr int kLines = DP / 64;                             // 64-channel lines of a key, and of values
    constexpr int kRows = 8 * NQ;
    extern __shared__ __align__(128) uint8_t smem[];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
    griddep_wait();
    const Share share = share_of(a, kRows);
    if (a.splits && threadIdx.x == 0) a.splits[blockIdx.x] = make_int4(0, 0, 0, 0);
    const int D = EXACT ? DP : a.head_dim, P = a.cache.page, shift = 31 - __clz(P);
    const int page_bytes = P * D, pages = (int)min(a.cache.pages, (int64_t)0x7fffffff);
    const uint32_t ring = smem_u32(smem) + warp * (kSlots * kPiece) + lane * 16;

    int b = share.b;
    int64_t within = share.within;
    for (int64_t at = share.first; at < share.last;) {
        const Sequence s = b == share.b ? share.sequence : sequence_of(a, b);
        const Work work = work_of(a, s, kRows);
        if (within >= work.units * work.per_unit) {              // on to the next sequence
            ++b;
            within = 0;
            continue;
        }
        const int64_t unit = within / work.per_unit, tile = unit / a.kv_heads;
        const int hk = (int)(unit % a.kv_heads), block = (int)(within % work.per_unit);
        const int blocks = (int)min((int64_t)(work.per_unit - block), share.last - at);
        within += blocks;
        at += blocks;
        const bool whole = blocks == work.per_unit;
        if (!whole && block == 0 && threadIdx.x == 0) {          // ends in the share that holds the tile's last block
            const int64_t end = at - blocks + work.per_unit;
            a.splits[blockIdx.x] = make_int4((int)((end * share.shares - 1) / share.total), b, hk, (int)tile);
        }
        const int32_t* table = a.table + b * a.ld_table;
        // (a sequence has fewer than 2^31 keys)
        const int k0 = block * kTokensBlock, k1 = (int)min(tile_keys(a, s, tile, kRows).end, (int64_t)k0 + (int64_t)blocks * kTokensBlock);
        const int tiles = max(k1 - k0 + kTile - 1, 0) / kTile;
        const int mine = tiles > warp ? (tiles - warp + kWarps - 1) / kWarps : 0;
        auto first_key = [&](int n) { return k0 + (warp + n * kWarps) * kTile; };

        // ---- pages: a lane looks up (page, head) of keys 16 (lane % 4) .. of a tile, -1 where there is none
        auto page_of = [&](int n) -> int {
            const int j = first_key(n) + 16 * t;
            if (n >= mine || j >= k1) return -1;
            const int id = (int)ld_global_u32(table + (j >> shift));
            return id >= 0 && id < pages ? id * a.kv_heads + hk : -1;
        };
        // Copies of piece u of tile n: lines of keys, rows 16 (g / 2) + (g & 1) + 0, 2, 4, .. 14, then 64 rows of values.
        auto copy = [&](int u, int n, int at_t, int slot) {
            const uint32_t dst = ring + slot * kPiece;
            if (u < kLines) {
                const int at = __shfl_sync(0xffffffffu, at_t, g >> 1);
                const bool ok = at >= 0 && (EXACT || 64 * u + 16 * t < D);
                const int8_t* src = a.cache.k + (int64_t)at * page_bytes + ((first_key(n) + 16 * (g >> 1)) & (P - 1)) * D + (g & 1) * D + 16 * t + 64 * u;
#pragma unroll
                for (int x = 0; x < 8; ++x) cp_async16(dst + x * 512, ok ? src + 2 * x * D : a.cache.k, ok);
            } else {
                const int d = 64 * (u - kLines) + g;
                const int8_t* src = a.cache.v + (int64_t)at_t * page_bytes + d * P + ((first_key(n) + 16 * t) & (P - 1));
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const bool ok = at_t >= 0 && (EXACT || d + 8 * x < D);
                    cp_async16(dst + x * 512, ok ? src + 8 * x * P : a.cache.v, ok);
                }
            }
            cp_commit();
        };
        // Scales of this lane's tokens, those of the 16 behind 16 (g / 2).
        auto scales_of = [&](int at_t, float* ks, float* vs) {
            const int at = __shfl_sync(0xffffffffu, at_t, g >> 1);
            *ks = at >= 0 ? ld_global_f32(a.cache.k_scale + at) : 0.0f;
            *vs = at >= 0 ? ld_global_f32(a.cache.v_scale + at) : 0.0f;
        };

        int at0 = page_of(0), at1 = page_of(1), at2 = page_of(2);
        // ---- queries: column g of the n-tiles, channels 64 j + 16 t .. + 15
        uint32_t q[NQ][kTerms][kLines * 8];
        float factor[NQ][2];                                    // of scores in columns 2 t, 2 t + 1, the scale of the keys apart
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) {
            const int64_t row = tile * kRows + 8 * nq + g;
            const bool ok = row < s.queries * a.group;
            const T* src = static_cast<const T*>(a.q) + (s.q0 + (ok ? row / a.group : 0)) * a.ldq + (int64_t)(hk * a.group + (ok ? row % a.group : 0)) * D + 16 * t;
            float f[kLines * 16], top = 0.0f;
#pragma unroll
            for (int j = 0; j < kLines; ++j)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                    if (ok && 64 * j + 16 * t < D) v = load4(src + 64 * j + 4 * x);
                    f[j * 16 + 4 * x] = v.x; f[j * 16 + 4 * x + 1] = v.y; f[j * 16 + 4 * x + 2] = v.z; f[j * 16 + 4 * x + 3] = v.w;
                }
            if (nq == 0) {                                      // (behind the first queries' loads)
#pragma unroll
                for (int u = 0; u < kSlots; ++u) copy(u % (2 * kLines), u / (2 * kLines), u < 2 * kLines ? at0 : at1, u);
            }
#pragma unroll
            for (int x = 0; x < kLines * 16; ++x) top = fmaxf(top, fabsf(f[x]));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const int e = min(max(exponent_of(top), -100), 126);
            const float down = power_of_two(-e);
#pragma unroll
            for (int x = 0; x < kLines * 8; ++x) {
                const float lo = f[2 * x] * down, hi = f[2 * x + 1] * down;
                q[nq][0][x] = pack_half(lo, hi);
                if (kTerms == 2) {
                    const float2 first = unpack_half(q[nq][0][x]);
                    q[nq][kTerms - 1][x] = pack_half(lo - first.x, hi - first.y);
                }
            }
            const float mul = a.scale_log2 * power_of_two(e);
#pragma unroll
            for (int c = 0; c < 2; ++c) factor[nq][c] = __shfl_sync(0xffffffffu, mul, (2 * t + c) * 4);
        }
        float ks, vs;
        scales_of(at0, &ks, &vs);
        int limit[NQ][2], least = k1 - 1;                       // last keys that the columns see
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                limit[nq][c] = (int)min(max(row_limit(a, s, tile * kRows + 8 * nq + 2 * t + c), (int64_t)-1), (int64_t)k1 - 1);
                least = min(least, limit[nq][c]);
            }
        least = __reduce_min_sync(0xffffffffu, least);

        float o[NQ][DP / 16][4], m[NQ][2], l[NQ][2];
        int e = -127;                                           // O carries 2^(7 - e)
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) {
#pragma unroll
            for (int c = 0; c < 2; ++c) { m[nq][c] = -INFINITY; l[nq][c] = 0.0f; }
#pragma unroll
            for (int d = 0; d < DP / 16; ++d)
#pragma unroll
                for (int x = 0; x < 4; ++x) o[nq][d][x] = 0.0f;
        }
        int piece = 0;
#pragma unroll 1
        for (int n = 0; n < mine; ++n) {
            const int at3 = page_of(n + 3);
            float ks1, vs1;
            scales_of(at1, &ks1, &vs1);
            // The slot of piece u is free: it takes the piece four behind.
            auto refill = [&](int u, int slot) {
                const int v = (u + kSlots) % (2 * kLines), ahead = (u + kSlots) / (2 * kLines);
                copy(v, n + ahead, ahead == 0 ? at0 : ahead == 1 ? at1 : at2, slot);
            };
            // ---- S^T: m-tile i holds tokens 16 (g/2) + 4 i + (g & 1), and those + 2
            float sc[NQ][4][4];
#pragma unroll
            for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int x = 0; x < 4; ++x) sc[nq][i][x] = 0.0f;
#pragma unroll
            for (int j = 0; j < kLines; ++j) {
                cp_wait<kSlots - 1>();
                const int slot = kLines == 1 ? piece & (kSlots - 1) : j % kSlots;
                const uint32_t src = ring + slot * kPiece;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint4 x = lds_v4(src + (2 * i) * 512), y = lds_v4(src + (2 * i + 1) * 512);
                    const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                    for (int st = 0; st < 4; ++st) {
                        uint32_t a0, a1, a2, a3;
                        widen(xs[st], &a0, &a2);
                        widen(ys[st], &a1, &a3);
#pragma unroll
                        for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
                            for (int term = 0; term < kTerms; ++term)
                                mma(sc[nq][i], a0, a1, a2, a3, q[nq][term][j * 8 + 2 * st], q[nq][term][j * 8 + 2 * st + 1]);
                    }
                }
                refill(j, slot);
                ++piece;
            }
            // ---- softmax: columns 2 t, 2 t + 1; tokens over i, the two halves and g
            const int j0 = first_key(n);
            const bool there = __shfl_sync(0xffffffffu, at0, g >> 1) >= 0;
            const bool clean = __all_sync(0xffffffffu, there) && j0 + kTile - 1 <= least;
            const int now_e = max(e, __reduce_max_sync(0xffffffffu, vs > 0.0f ? exponent_of(vs) + 1 : -127));
            // vs 2^(7 - e): in two steps, each a normal number
            const float vf = vs * power_of_two(-now_e / 2) * power_of_two(7 - now_e + now_e / 2);
            const float down = now_e == e ? 1.0f : (e <= -127 ? 0.0f : exp2f((float)(e - now_e)));
            const bool grown = now_e != e;
            e = now_e;
            uint32_t pb[NQ][kTerms][4][2];
#pragma unroll
            for (int nq = 0; nq < NQ; ++nq) {
                const float f[2] = {factor[nq][0] * ks, factor[nq][1] * ks};
                float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int x = 0; x < 4; ++x) sc[nq][i][x] *= f[x & 1];
                const int from = j0 + 16 * (g >> 1) + (g & 1);   // this lane's first token
                if (!clean) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int x = 0; x < 4; ++x)
                            if (!(there && from + 4 * i + (x & 2) <= limit[nq][x & 1])) sc[nq][i][x] = -INFINITY;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int x = 0; x < 4; ++x) top[x & 1] = fmaxf(top[x & 1], sc[nq][i][x]);
                float base[2], keep[2];
                bool rise = grown;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    if (there && from <= limit[nq][c]) top[c] = fmaxf(top[c], -FLT_MAX);        // (-inf stays to a row that sees nothing)
#pragma unroll
                    for (int x = 4; x < 32; x <<= 1) top[c] = fmaxf(top[c], __shfl_xor_sync(0xffffffffu, top[c], x));
                    const bool up = top[c] > m[nq][c] + kSlack || (m[nq][c] == -INFINITY && top[c] > m[nq][c]);
                    const float now = up ? top[c] : m[nq][c];
                    keep[c] = up ? ex2(m[nq][c] - now) : 1.0f;          // (from nothing: 0)
                    rise = rise || up;
                    m[nq][c] = now;
                    base[c] = now == -INFINITY ? 0.0f : now;
                }
                if (__any_sync(0xffffffffu, rise)) {
#pragma unroll
                    for (int c = 0; c < 2; ++c) { l[nq][c] *= keep[c]; keep[c] *= down; }
#pragma unroll
                    for (int d = 0; d < DP / 16; ++d)
#pragma unroll
                        for (int x = 0; x < 4; ++x) o[nq][d][x] *= keep[x & 1];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float p[4];
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        p[x] = ex2(sc[nq][i][x] - base[x & 1]);
                        l[nq][x & 1] += p[x];
                        p[x] *= vf;
                    }
                    // tokens on rows -> tokens along the step, as the second operand wants them
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t first = pack_half(p[2 * h], p[2 * h + 1]);
                        pb[nq][0][i][h] = transpose8(first);
                        if (kTerms == 2) {
                            const float2 f = unpack_half(first);
                            pb[nq][kTerms - 1][i][h] = transpose8(pack_half(p[2 * h] - f.x, p[2 * h + 1] - f.y));
                        }
                    }
                }
            }
            // ---- O^T: rows 16 d + g and + 8, step i the tokens of m-tile i
#pragma unroll
            for (int j = 0; j < kLines; ++j) {
                cp_wait<kSlots - 1>();
                const int slot = kLines == 1 ? piece & (kSlots - 1) : (kLines + j) % kSlots;
                const uint32_t src = ring + slot * kPiece;
#pragma unroll
                for (int d = 4 * j; d < 4 * j + 4; ++d) {
                    const uint4 x = lds_v4(src + (2 * (d % 4)) * 512), y = lds_v4(src + (2 * (d % 4) + 1) * 512);
                    const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t a0, a1, a2, a3;
                        widen(xs[i], &a0, &a2);
                        widen(ys[i], &a1, &a3);
#pragma unroll
                        for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
                            for (int term = 0; term < kTerms; ++term) mma(o[nq][d], a0, a1, a2, a3, pb[nq][term][i][0], pb[nq][term][i][1]);
                    }
                }
                refill(kLines + j, slot);
                ++piece;
            }
            at0 = at1;
            at1 = at2;
            at2 = at3;
            ks = ks1;
            vs = vs1;
        }
        // ---- the warps' results meet in the ring's memory: [warp][row][m, l, then O 2^(e - 7)]
        cp_wait<0>();
        __syncthreads();
        constexpr int kPitch = DP + 4;
        float* meet = reinterpret_cast<float*>(smem);
        const float up_hi = power_of_two(e / 2), up_lo = power_of_two(e - e / 2 - 7);
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) l[nq][c] += __shfl_xor_sync(0xffffffffu, l[nq][c], x);
                float* to = meet + (warp * kRows + 8 * nq + 2 * t + c) * kPitch;
                if (g == 0) { to[0] = m[nq][c]; to[1] = l[nq][c]; }
#pragma unroll
                for (int d = 0; d < DP / 16; ++d) {
                    to[4 + 16 * d + g] = o[nq][d][c] * up_hi * up_lo;
                    to[4 + 16 * d + 8 + g] = o[nq][d][2 + c] * up_hi * up_lo;
                }
            }
        __syncthreads();
        for (int e2 = threadIdx.x; e2 < kRows * (DP / 4); e2 += kWarps * 32) {
            const int r = e2 / (DP / 4), d = (e2 % (DP / 4)) * 4;
            const int64_t row = tile * kRows + r;
            if (row >= s.queries * a.group || d >= D) continue;
            float top = -INFINITY;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) top = fmaxf(top, meet[(w * kRows + r) * kPitch]);
            const float base = top == -INFINITY ? 0.0f : top;
            float sum = 0.0f;
            float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float* from = meet + (w * kRows + r) * kPitch;
                const float f = exp2f(from[0] - base);
                sum = fmaf(f, from[1], sum);
                const float4 v = *reinterpret_cast<const float4*>(from + 4 + d);
                acc.x = fmaf(f, v.x, acc.x); acc.y = fmaf(f, v.y, acc.y); acc.z = fmaf(f, v.z, acc.z); acc.w = fmaf(f, v.w, acc.w);
            }
            if (whole) {
                const int64_t token = s.q0 + row / a.group, head = hk * a.group + row % a.group;
                const float inv = reciprocal_sum(top, sum);
                store4(static_cast<T*>(a.y) + token * a.ldy + head * D + d, acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
            } else {
                const int64_t seat = tokens_seat(blockIdx.x, block == 0) * kRows + r;
                *reinterpret_cast<float4*>(a.part + seat * D + d) = acc;
                if (d == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * seat) = make_float2(top, sum);
            }
        }
        __syncthreads();
    }
}

// Joins row blockIdx.y of the tile, if there is one, that begins in share blockIdx.x and goes on behind it.
template <typename T>
__global__ void __launch_bounds__(128) attention_tokens_join_kernel(const Attention a) {
    griddep_wait();
    const uint4 split_words = ld_global_v4(a.splits + blockIdx.x);
    const int4 split = make_int4((int)split_words.x, (int)split_words.y, (int)split_words.z, (int)split_words.w);
    const int first = blockIdx.x, b = split.y, hk = split.z;
    if (split.x <= first) return;
    const Sequence s = sequence_of(a, b);
    const int64_t row = (int64_t)split.w * a.tile_rows + blockIdx.y;
    if (row >= s.queries * a.group) return;
    const int64_t token = s.q0 + row / a.group, head = hk * a.group + row % a.group;
    join_row<T, 4>(a, split.x - first + 1, [&](int c) { return tokens_seat(first + c, c == 0) * a.tile_rows + blockIdx.y; },
                   static_cast<T*>(a.y) + token * a.ldy + head * a.head_dim);
}

template <typename T, int DP, int NQ, bool EXACT>
cudaError_t launch(const Attention& a, dim3 grid, cudaStream_t stream) {
    constexpr size_t ring = kWarps * kSlots * kPiece, meet = sizeof(float) * kWarps * 8 * NQ * (DP + 4);
    constexpr size_t smem = ring > meet ? ring : meet;
    auto* kern = attention_tokens_kernel<T, DP, NQ, EXACT>;
    const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kern), smem);
    return e != cudaSuccess ? e : launch_pdl3(kern, grid, kWarps * 32, smem, stream, a);
}
template <typename T, int DP>
cudaError_t by_rows(const Attention& a, dim3 grid, cudaStream_t stream) {
    constexpr int kMost = sizeof(T) == 4 ? 1 : 2;
    if (a.head_dim == DP) return a.tile_rows <= 8 ? launch<T, DP, 1, true>(a, grid, stream) : launch<T, DP, kMost, true>(a, grid, stream);
    return a.tile_rows <= 8 ? launch<T, DP, 1, false>(a, grid, stream) : launch<T, DP, kMost, false>(a, grid, stream);
}
template <typename T>
cudaError_t by_width(const Attention& a, dim3 grid, cudaStream_t stream) {
    if (a.head_dim <= 64) return by_rows<T, 64>(a, grid, stream);
    if (a.head_dim <= 128) return by_rows<T, 128>(a, grid, stream);
    return by_rows<T, 256>(a, grid, stream);
}

}  // namespace

int tokens_ctas(const Attention& a) { return 148 * tokens_resident(a.dt == FQ_BF16, a.head_dim, a.tile_rows / 8); }

cudaError_t launch_attention_tokens(const Attention& a, cudaStream_t stream) {
    const dim3 grid((unsigned)a.ctas);
    const cudaError_t e = a.dt == FQ_BF16 ? by_width<__nv_bfloat16>(a, grid, stream) : by_width<float>(a, grid, stream);
    if (e != cudaSuccess || !a.splits) return e;
    const dim3 joins((unsigned)a.ctas, (unsigned)a.tile_rows);
    return a.dt == FQ_BF16 ? launch_pdl3(attention_tokens_join_kernel<__nv_bfloat16>, joins, 128, 0, stream, a)
                           : launch_pdl3(attention_tokens_join_kernel<float>, joins, 128, 0, stream, a);
}

}  // namespace fq
