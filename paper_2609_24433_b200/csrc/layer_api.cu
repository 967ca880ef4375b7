// C ABI of the operators between a layer's projections (see include/fq.h): argument checks on the host, dispatch.
#include <math.h>

#include "attention_common.cuh"
#include "fq_common.cuh"
#include "layer_common.cuh"

using namespace fq;

namespace fq {

namespace {
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Tile and chunk of a call.  Chunks are what fills the SMs where rows, heads and sequences are few; they are planned for the row tiles of
// the whole call, also where its widened codes take several passes (wide_bytes), each of which then has a part of them.
enum class Route { Simt, Tokens, Tiles };
// 16 rows are what the few-queries kernel takes in one pass over the cache.  That is not where the two are level: with as many passes as
// it takes, at 18 / 32 / 64 / 128 rows, 16 sequences of 8192 keys, 8 heads of 128: 115 / 119 / 208 / 390 us, on tcgen05 behind the
// widening 351 / 352 / 353 / 360; 32 of 866 keys, one head of 256: 23 / 23 / 33 / 61 and 31 / 32 / 34 / 43.
Route route_of(const Attention& a) { return a.cached && a.max_q * a.group <= 16 ? Route::Tokens : a.dt == FQ_BF16 ? Route::Tiles : Route::Simt; }
Route plan(Attention& a) {
    const Route route = route_of(a);
    int64_t wave = 2 * 148;
    if (route == Route::Tokens) {
        a.tile_rows = a.dt == FQ_F32 || a.max_q * a.group <= 8 ? 8 : 16;     // (two terms of sixteen rows pass the registers)
        const int64_t blocks = (a.max_kv > 0 ? ceil_div(a.max_kv, kTokensBlock) : 1) * row_tiles(a) * a.batch * a.kv_heads;
        a.ctas = blocks < tokens_ctas(a) ? (int)blocks : tokens_ctas(a);
        if (a.ctas < 1) a.ctas = 1;
        a.chunk = kTokensBlock;
        a.chunks = 1;
        return route;
    }
    if (route == Route::Tiles) {
        a.tile_rows = a.head_dim <= 128 && a.max_q * a.group > 128 ? 256 : 128;
        wave = 148;
    } else {
        a.tile_rows = a.max_q * a.group <= 16 ? 16 : 64;
    }
    const int64_t units = row_tiles(a) * a.batch * a.kv_heads;
    const int64_t splits = route == Route::Tiles ? (units < wave ? wave / (units > 0 ? units : 1) : 1) : ceil_div(wave, units > 0 ? units : 1);
    int64_t chunk = ceil_div(ceil_div(a.max_kv, splits), 256) * 256;
    if (chunk < 256) chunk = 256;
    if (ceil_div(a.max_kv, chunk) > 65535) chunk = ceil_div(ceil_div(a.max_kv, 65535), 256) * 256;
    a.chunk = (int)chunk;
    const int64_t chunks = ceil_div(a.max_kv, chunk);
    a.chunks = (int)(chunks < 1 ? 1 : chunks);
    return route;
}
// (few queries: the first and the last tile of every share)
size_t part_bytes(const Attention& a, Route route) {
    if (route == Route::Tokens) return a.max_kv <= kTokensBlock ? 0 : align_up(sizeof(float) * 2 * (size_t)a.ctas * a.tile_rows * a.head_dim, 256);
    return a.chunks <= 1 ? 0 : align_up(sizeof(float) * (size_t)a.q_rows * a.q_heads * a.chunks * a.head_dim, 256);
}
size_t ml_bytes(const Attention& a, Route route) {
    if (route == Route::Tokens) return a.max_kv <= kTokensBlock ? 0 : align_up(sizeof(float) * 4 * (size_t)a.ctas * a.tile_rows, 256) + align_up(sizeof(int4) * (size_t)a.ctas, 256);
    return a.chunks <= 1 ? 0 : align_up(sizeof(float) * 2 * (size_t)a.q_rows * a.q_heads * a.chunks, 256);
}
// Widened codes: so many (sequence, kv head) pairs at a time as kWideBytes hold, one at least.
constexpr size_t kWideBytes = 256ull << 20;
size_t wide_bytes(Attention& a, Route route) {
    a.first_unit = 0;
    a.wide_keys = 0;
    if (route == Route::Tokens) return 0;                        // (equal shares, whatever the pairs: there may be more than an int holds)
    a.units = a.batch * a.kv_heads;
    if (route != Route::Tiles || !a.cached) return 0;
    a.wide_keys = ceil_div(a.max_kv, 128) * 128;
    const size_t unit = (size_t)a.wide_keys * a.head_dim * 4;
    if (unit == 0) return 0;
    const int64_t fit = (int64_t)(kWideBytes / unit);
    if (fit < a.units) a.units = fit > 1 ? (int)fit : 1;
    return align_up(unit * a.units, 256);
}
}  // namespace

size_t attention_workspace_bytes(const Attention& given) {
    Attention a = given;
    const Route route = plan(a);
    return part_bytes(a, route) + ml_bytes(a, route) + wide_bytes(a, route);
}

fq_status launch_attention(Attention& a, void* workspace, size_t ws_bytes, cudaStream_t stream) {
    const Route route = plan(a);
    const size_t parts = part_bytes(a, route), mls = ml_bytes(a, route), need = parts + mls + wide_bytes(a, route);
    if (need > 0) {
        if (!workspace) return FQ_ERR_INVALID_ARG;
        if ((reinterpret_cast<uintptr_t>(workspace) & 255u) != 0) return FQ_ERR_ALIGNMENT;
        if (ws_bytes < need) return FQ_ERR_NOMEM;
        a.part = static_cast<float*>(workspace);
        a.part_ml = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + parts);
        a.wide = static_cast<uint8_t*>(workspace) + parts + mls;
        if (route == Route::Tokens) a.splits = reinterpret_cast<int4*>(static_cast<uint8_t*>(workspace) + parts + mls - align_up(sizeof(int4) * (size_t)a.ctas, 256));
    }
    if (route == Route::Tiles) {
        const int all = a.batch * a.kv_heads, step = a.units;
        for (a.first_unit = 0; a.first_unit < all; a.first_unit += step) {
            a.units = all - a.first_unit < step ? all - a.first_unit : step;
            if (a.cached && launch_attention_widen(a, stream) != cudaSuccess) return FQ_ERR_CUDA;
            if (launch_attention_tiles(a, stream) != cudaSuccess) return FQ_ERR_CUDA;
        }
    } else {
        const cudaError_t e = route == Route::Tokens ? launch_attention_tokens(a, stream) : launch_attention_simt(a, stream);
        if (e != cudaSuccess) return FQ_ERR_CUDA;
    }
    if (a.chunks > 1 && launch_attention_join(a, stream) != cudaSuccess) return FQ_ERR_CUDA;
    return FQ_OK;
}

}  // namespace fq

namespace {

bool aligned(const void* p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
bool aligned16(const void* p) { return aligned(p, 16); }
bool aligned_ld(int64_t ld, fq_dtype t) { return ld % (t == FQ_F32 ? 4 : 8) == 0; }          // rows begin on 16 bytes

fq_status check_arch() {
    const int major = device_cc_major();
    if (major < 0) return FQ_ERR_CUDA;
    return major == 10 ? FQ_OK : FQ_ERR_ARCH;
}
bool valid_dtype(fq_dtype t) { return t == FQ_F32 || t == FQ_BF16; }

constexpr int64_t kMaxRows = 1ll << 31;          // rows of one call
constexpr int kMaxGridYZ = 65535;

fq_status check_cache(const fq_kv8_cache* c) {
    if (!c || c->pages < 0 || c->heads < 1 || c->head_dim < 1 || c->page < 1) return FQ_ERR_INVALID_ARG;
    if (c->head_dim % 16 != 0 || c->head_dim > 256) return FQ_ERR_UNSUPPORTED;
    if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128) return FQ_ERR_UNSUPPORTED;
    if (c->pages > 0 && (!c->k || !c->v || !c->k_scale || !c->v_scale)) return FQ_ERR_INVALID_ARG;
    if (!aligned16(c->k) || !aligned16(c->v) || !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4)) return FQ_ERR_ALIGNMENT;
    return FQ_OK;
}
fq_status check_table(const int32_t* table, int64_t ld, int64_t width, int batch) {
    if (batch < 0 || width < 0 || width > 0x7fffffff / 128 || (width > 0 && batch > 0 && (!table || (batch > 1 && ld < width)))) return FQ_ERR_INVALID_ARG;
    return FQ_OK;
}

// Shapes of a call of either attention; a.group is set here.
fq_status check_heads(Attention& a) {
    if (a.q_heads < 1 || a.kv_heads < 1 || a.head_dim < 1 || a.batch < 0 || a.q_rows < 0 || a.max_q < 0 || a.max_kv < 0) return FQ_ERR_INVALID_ARG;
    if (!valid_dtype(a.dt)) return FQ_ERR_INVALID_ARG;
    if (a.q_heads % a.kv_heads != 0) return FQ_ERR_INVALID_ARG;
    if (a.head_dim % 16 != 0 || a.head_dim > 256) return FQ_ERR_UNSUPPORTED;
    if (a.q_rows >= kMaxRows) return FQ_ERR_UNSUPPORTED;
    if (!a.q_offsets && a.batch > 0 && a.q_rows % a.batch != 0) return FQ_ERR_INVALID_ARG;
    a.group = a.q_heads / a.kv_heads;
    if (!a.q_offsets) a.max_q = a.batch > 0 ? a.q_rows / a.batch : 0;
    else if (a.max_q == 0 || a.max_q > a.q_rows) a.max_q = a.q_rows;
    if (route_of(a) != Route::Tokens && (int64_t)a.batch * a.kv_heads > kMaxGridYZ) return FQ_ERR_UNSUPPORTED;
    return FQ_OK;
}
fq_status check_rows(const void* q, int64_t ldq, const void* y, int64_t ldy, int64_t width, fq_dtype t) {
    if (!q || !y || ldq < width || ldy < width) return FQ_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(y) || !aligned_ld(ldq, t) || !aligned_ld(ldy, t)) return FQ_ERR_ALIGNMENT;
    return FQ_OK;
}

fq_status fill_kv8(Attention& a, fq_dtype dt, int64_t q_rows, int q_heads, const fq_kv8_cache* cache, int64_t table_width, int batch,
                   const int32_t* q_offsets, int64_t max_q, int64_t max_kv) {
    const fq_status st = check_cache(cache);
    if (st != FQ_OK) return st;
    a.dt = dt; a.q_rows = q_rows; a.q_heads = q_heads; a.kv_heads = cache->heads; a.head_dim = cache->head_dim; a.batch = batch;
    a.q_offsets = q_offsets; a.max_q = max_q; a.cached = true; a.cache = *cache; a.table_width = (int)table_width;
    a.max_kv = cache->pages > 0 ? table_width * cache->page : 0;
    if (max_kv < 0) return FQ_ERR_INVALID_ARG;
    if (max_kv > 0 && max_kv < a.max_kv) a.max_kv = max_kv;
    return check_heads(a);
}
fq_status fill_cross(Attention& a, fq_dtype dt, int64_t q_rows, int q_heads, int64_t kv_rows, int kv_heads, int head_dim, int batch,
                     const int32_t* q_offsets, const int32_t* kv_offsets, int64_t max_q, int64_t max_kv) {
    a.dt = dt; a.q_rows = q_rows; a.q_heads = q_heads; a.kv_heads = kv_heads; a.head_dim = head_dim; a.batch = batch;
    a.q_offsets = q_offsets; a.max_q = max_q; a.cached = false; a.kv_rows = kv_rows; a.kv_offsets = kv_offsets; a.max_kv = max_kv;
    const fq_status st = check_heads(a);
    if (st != FQ_OK) return st;
    if (kv_rows < 0) return FQ_ERR_INVALID_ARG;
    if (kv_rows >= kMaxRows) return FQ_ERR_UNSUPPORTED;
    if (!kv_offsets && batch > 0 && kv_rows % batch != 0) return FQ_ERR_INVALID_ARG;
    const int64_t most = batch == 0 ? 0 : kv_offsets ? kv_rows : kv_rows / batch;
    if (a.max_kv == 0 || a.max_kv > most) a.max_kv = most;
    return FQ_OK;
}

}  // namespace

extern "C" {

fq_status fq_rope_frequencies(int rotary_dim, double base, fq_rope_scaling scaling, double factor, double original_length,
                              double low_turns, double high_turns, double* frequencies) {
    if (rotary_dim < 0 || rotary_dim % 2 != 0 || !(base > 0.0) || (rotary_dim > 0 && !frequencies)) return FQ_ERR_INVALID_ARG;
    if (scaling != FQ_ROPE_PLAIN && scaling != FQ_ROPE_LINEAR && scaling != FQ_ROPE_BASE && scaling != FQ_ROPE_PARTS) return FQ_ERR_INVALID_ARG;
    if (scaling != FQ_ROPE_PLAIN && !(factor >= 1.0)) return FQ_ERR_INVALID_ARG;
    if (scaling == FQ_ROPE_BASE && rotary_dim <= 2) return rotary_dim == 0 ? FQ_OK : FQ_ERR_INVALID_ARG;
    if (scaling == FQ_ROPE_PARTS && (!(original_length > 0.0) || !(low_turns >= 0.0) || !(high_turns > low_turns))) return FQ_ERR_INVALID_ARG;
    if (scaling == FQ_ROPE_BASE) base *= pow(factor, (double)rotary_dim / (rotary_dim - 2));
    for (int i = 0; i < rotary_dim / 2; ++i) {
        double f = pow(base, -2.0 * i / rotary_dim);
        if (scaling == FQ_ROPE_LINEAR) f /= factor;
        if (scaling == FQ_ROPE_PARTS) {
            const double turns = f * original_length / 6.283185307179586477;
            const double keep = fmin(fmax((turns - low_turns) / (high_turns - low_turns), 0.0), 1.0);
            f = f * keep + f / factor * (1.0 - keep);
        }
        frequencies[i] = f;
    }
    return FQ_OK;
}

fq_status fq_qk_norm_rope(const void* qkv, fq_dtype xt, int64_t M, int64_t ldx, int q_heads, int k_heads, int head_dim,
                          const float* q_gain, const float* k_gain, float eps, const int32_t* positions, const double* frequencies,
                          int rotary_dim, fq_rope_layout layout, float amplitude, void* q, int64_t ldq, void* k, int64_t ldk,
                          fq_dtype yt, void* stream) {
    if (M < 0 || q_heads < 0 || k_heads < 0 || head_dim < 1 || rotary_dim < 0 || rotary_dim % 2 != 0 || rotary_dim > head_dim) return FQ_ERR_INVALID_ARG;
    if (!valid_dtype(xt) || !valid_dtype(yt) || (layout != FQ_ROPE_HALF && layout != FQ_ROPE_INTERLEAVED) || !(eps >= 0.0f)) return FQ_ERR_INVALID_ARG;
    if (head_dim % 8 != 0 || head_dim > 256 || M >= kMaxRows || q_heads > 32767 || k_heads > 32767) return FQ_ERR_UNSUPPORTED;
    if (M == 0 || q_heads + k_heads == 0) return FQ_OK;
    const int64_t width = (int64_t)(q_heads + k_heads) * head_dim;
    if (!qkv || ldx < width || (rotary_dim > 0 && (!positions || !frequencies))) return FQ_ERR_INVALID_ARG;
    if ((q_heads > 0 && (!q || ldq < (int64_t)q_heads * head_dim)) || (k_heads > 0 && (!k || ldk < (int64_t)k_heads * head_dim))) return FQ_ERR_INVALID_ARG;
    if (!aligned16(qkv) || !aligned_ld(ldx, xt) || (q_heads > 0 && (!aligned16(q) || !aligned_ld(ldq, yt))) ||
        (k_heads > 0 && (!aligned16(k) || !aligned_ld(ldk, yt))) ||
        (q_gain && !aligned16(q_gain)) || (k_gain && !aligned16(k_gain)) || (rotary_dim > 0 && (!aligned(positions, 4) || !aligned(frequencies, 8))))
        return FQ_ERR_ALIGNMENT;
    const fq_status st = check_arch();
    if (st != FQ_OK) return st;
    QkNormRope r = {};
    r.x = qkv; r.xt = xt; r.yt = yt; r.M = M; r.ldx = ldx; r.q_heads = q_heads; r.k_heads = k_heads; r.head_dim = head_dim;
    r.rotary = rotary_dim; r.interleaved = layout == FQ_ROPE_INTERLEAVED; r.q_gain = q_gain; r.k_gain = k_gain; r.eps = eps;
    r.amplitude = amplitude; r.positions = positions; r.frequencies = frequencies; r.q = q; r.k = k; r.ldq = ldq; r.ldk = ldk;
    return launch_qk_norm_rope(r, static_cast<cudaStream_t>(stream)) == cudaSuccess ? FQ_OK : FQ_ERR_CUDA;
}

fq_status fq_kv8_append(const void* k, const void* v, fq_dtype xt, int64_t tokens, int64_t ldk, int64_t ldv, const fq_kv8_cache* cache,
                        const int32_t* table, int64_t ld_table, int64_t table_width, int batch, const int32_t* kv_len,
                        const int32_t* offsets, int64_t max_new, void* stream) {
    fq_status st = check_cache(cache);
    if (st != FQ_OK) return st;
    st = check_table(table, ld_table, table_width, batch);
    if (st != FQ_OK) return st;
    if (!valid_dtype(xt) || tokens < 0 || max_new < 0) return FQ_ERR_INVALID_ARG;
    if (tokens >= kMaxRows || batch > kMaxGridYZ || cache->heads > kMaxGridYZ / 2) return FQ_ERR_UNSUPPORTED;
    if (!offsets && batch > 0 && tokens % batch != 0) return FQ_ERR_INVALID_ARG;
    if (tokens == 0 || batch == 0 || table_width == 0 || cache->pages == 0) return FQ_OK;
    const int64_t width = (int64_t)cache->heads * cache->head_dim;
    if (!k || !v || !kv_len || ldk < width || ldv < width) return FQ_ERR_INVALID_ARG;
    if (!aligned16(k) || !aligned16(v) || !aligned_ld(ldk, xt) || !aligned_ld(ldv, xt)) return FQ_ERR_ALIGNMENT;
    if (!aligned(table, 4) || !aligned(kv_len, 4) || !aligned(offsets, 4)) return FQ_ERR_ALIGNMENT;
    st = check_arch();
    if (st != FQ_OK) return st;
    Kv8Append a = {};
    a.k = k; a.v = v; a.xt = xt; a.tokens = tokens; a.ldk = ldk; a.ldv = ldv; a.cache = *cache; a.table = table; a.ld_table = ld_table;
    a.table_width = (int)table_width; a.batch = batch; a.kv_len = kv_len; a.offsets = offsets;
    a.max_new = !offsets ? tokens / batch : max_new > 0 ? max_new : tokens;
    return launch_kv8_append(a, static_cast<cudaStream_t>(stream)) == cudaSuccess ? FQ_OK : FQ_ERR_CUDA;
}

size_t fq_attention_kv8_workspace_bytes(fq_dtype dt, int64_t q_rows, int q_heads, const fq_kv8_cache* cache, int64_t table_width,
                                        int batch, int ragged, int64_t max_q, int64_t max_kv) {
    Attention a = {};
    static const int32_t none[1] = {0};          // (only whether there are offsets counts here)
    if (fill_kv8(a, dt, q_rows, q_heads, cache, table_width, batch, ragged ? none : nullptr, max_q, max_kv) != FQ_OK) return 0;
    return q_rows == 0 || batch == 0 ? 0 : attention_workspace_bytes(a);
}

fq_status fq_attention_kv8(const void* q, fq_dtype dt, int64_t q_rows, int64_t ldq, int q_heads, const fq_kv8_cache* cache,
                           const int32_t* table, int64_t ld_table, int64_t table_width, int batch, const int32_t* kv_len,
                           const int32_t* q_offsets, int64_t max_q, int64_t max_kv, int causal, float scale, void* y, int64_t ldy,
                           void* workspace, size_t ws_bytes, void* stream) {
    fq_status st = check_table(table, ld_table, table_width, batch);
    if (st != FQ_OK) return st;
    Attention a = {};
    st = fill_kv8(a, dt, q_rows, q_heads, cache, table_width, batch, q_offsets, max_q, max_kv);
    if (st != FQ_OK) return st;
    if (!(scale >= 0.0f) || isinf(scale * 1.44269504088896341f)) return FQ_ERR_INVALID_ARG;
    if (q_rows == 0 || batch == 0) return FQ_OK;
    if (!kv_len) return FQ_ERR_INVALID_ARG;
    st = check_rows(q, ldq, y, ldy, (int64_t)q_heads * a.head_dim, dt);
    if (st != FQ_OK) return st;
    if (!aligned(table, 4) || !aligned(kv_len, 4) || !aligned(q_offsets, 4)) return FQ_ERR_ALIGNMENT;
    st = check_arch();
    if (st != FQ_OK) return st;
    a.q = q; a.y = y; a.ldq = ldq; a.ldy = ldy; a.kv_len = kv_len; a.scale_log2 = scale * 1.44269504088896341f; a.causal = causal != 0;
    a.table = table; a.ld_table = ld_table;
    return launch_attention(a, workspace, ws_bytes, static_cast<cudaStream_t>(stream));
}

size_t fq_cross_attention_workspace_bytes(fq_dtype dt, int64_t q_rows, int q_heads, int64_t kv_rows, int kv_heads, int head_dim,
                                          int batch, int ragged_q, int ragged_kv, int64_t max_q, int64_t max_kv) {
    Attention a = {};
    static const int32_t none[1] = {0};
    if (fill_cross(a, dt, q_rows, q_heads, kv_rows, kv_heads, head_dim, batch, ragged_q ? none : nullptr, ragged_kv ? none : nullptr, max_q, max_kv) != FQ_OK) return 0;
    return q_rows == 0 || batch == 0 ? 0 : attention_workspace_bytes(a);
}

fq_status fq_cross_attention(const void* q, fq_dtype dt, int64_t q_rows, int64_t ldq, int q_heads, const void* k, const void* v,
                             int64_t kv_rows, int64_t ldk, int64_t ldv, int kv_heads, int head_dim, int batch, const int32_t* q_offsets,
                             const int32_t* kv_offsets, const int32_t* kv_len, const uint8_t* key_mask, int64_t max_q, int64_t max_kv,
                             float scale, void* y, int64_t ldy, void* workspace, size_t ws_bytes, void* stream) {
    Attention a = {};
    fq_status st = fill_cross(a, dt, q_rows, q_heads, kv_rows, kv_heads, head_dim, batch, q_offsets, kv_offsets, max_q, max_kv);
    if (st != FQ_OK) return st;
    if (!(scale >= 0.0f) || isinf(scale * 1.44269504088896341f)) return FQ_ERR_INVALID_ARG;
    if (q_rows == 0 || batch == 0) return FQ_OK;
    st = check_rows(q, ldq, y, ldy, (int64_t)q_heads * head_dim, dt);
    if (st != FQ_OK) return st;
    if (kv_rows > 0) {
        st = check_rows(k, ldk, v, ldv, (int64_t)kv_heads * head_dim, dt);
        if (st != FQ_OK) return st;
    }
    if (!aligned(q_offsets, 4) || !aligned(kv_offsets, 4) || !aligned(kv_len, 4)) return FQ_ERR_ALIGNMENT;
    st = check_arch();
    if (st != FQ_OK) return st;
    a.q = q; a.y = y; a.ldq = ldq; a.ldy = ldy; a.k = k; a.v = v; a.ldk = ldk; a.ldv = ldv; a.kv_len = kv_len; a.key_mask = key_mask;
    a.scale_log2 = scale * 1.44269504088896341f; a.causal = 0;
    return launch_attention(a, workspace, ws_bytes, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
