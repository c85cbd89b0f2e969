// Entry points of the attention that stands beside the MoE layer in a decoder block: argument checks, the choice of a
// kernel and of the number of parts that the keys are cut into.
#include "attn_common.h"

namespace c2r {

// Row counts, lengths and positions stay below this, so that their sums and differences fit 32 bits.
constexpr int64_t ATTN_MOST = 1ll << 30;
constexpr int64_t ATTN_MOST_KEYS = 1ll << 28;  // of a sequence: 64 times its tiles of 16 fit, too
constexpr int ATTN_MAX_HEADS = 1024;

static int check_heads(int dt, int heads, int64_t kv_heads, int64_t D) {
    if (dt != C2R_F32 && dt != C2R_BF16) return C2R_ERR_INVALID_ARG;
    if (heads < 1 || kv_heads < 1 || D < 1) return C2R_ERR_INVALID_ARG;
    if (heads > ATTN_MAX_HEADS || kv_heads > ATTN_MAX_HEADS) return C2R_ERR_UNSUPPORTED;
    if (heads % kv_heads != 0) return C2R_ERR_INVALID_ARG;
    return D == 64 || D == 128 ? C2R_OK : C2R_ERR_UNSUPPORTED;
}

static int check_cache(const c2r_kv_cache *c, int heads) {
    if (!c) return C2R_ERR_INVALID_ARG;
    if (c->dtype != C2R_F32 && c->dtype != C2R_BF16) return C2R_ERR_INVALID_ARG;
    const int rc = check_heads((int)c->dtype, heads, c->kv_heads, c->head_dim);
    if (rc != C2R_OK) return rc;
    if (c->batch < 0 || c->n_pages < 1 || c->page_size < 1 || c->max_pages < 1) return C2R_ERR_INVALID_ARG;
    if (c->batch >= ATTN_MOST || c->n_pages >= ATTN_MOST || c->page_size >= ATTN_MOST || c->max_pages >= ATTN_MOST ||
        c->page_size * c->max_pages >= ATTN_MOST_KEYS)
        return C2R_ERR_UNSUPPORTED;
    if (!c->page_table || !c->kv_len || !c->k || !c->v) return C2R_ERR_INVALID_ARG;
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->page_table, 4) || !aligned(c->kv_len, 4)) return C2R_ERR_INVALID_ARG;
    const int size = c->dtype == C2R_BF16 ? 2 : 4;
    for (const int64_t s : {c->page_stride, c->slot_stride, c->head_stride})
        if (s < 0 || s > (1ll << 40) || s * size % 16 != 0) return C2R_ERR_INVALID_ARG;
    return C2R_OK;
}

static KvView view_of(const c2r_kv_cache &c) {
    const int64_t size = c.dtype == C2R_BF16 ? 2 : 4;
    KvView v;
    v.k = static_cast<const unsigned char *>(c.k);
    v.v = static_cast<const unsigned char *>(c.v);
    v.page_bytes = c.page_stride * size;
    v.slot_bytes = c.slot_stride * size;
    v.head_bytes = c.head_stride * size;
    v.table = c.page_table;
    v.kv_len = c.kv_len;
    v.n_pages = (int32_t)c.n_pages;
    v.page_size = (int32_t)c.page_size;
    v.max_pages = (int32_t)c.max_pages;
    v.batch = (int32_t)c.batch;
    v.capacity = (int32_t)(c.page_size * c.max_pages);
    v.kv_heads = (int32_t)c.kv_heads;
    // j / d for j < 2^31: s = ceil(log2 d), mul = floor(2^32 (2^s - d) / d) + 1
    uint32_t s = 0;
    while ((1ull << s) < (uint64_t)v.page_size) ++s;
    v.div_shift = s;
    v.div_mul = (uint32_t)((((1ull << s) - (uint64_t)v.page_size) << 32) / (uint64_t)v.page_size + 1);
    return v;
}

static int check_rope(int dt, int heads, int64_t kv_heads, int64_t D, int64_t T, const float *q_weight, const float *k_weight, float eps,
                      const float *inv_freq, int rot) {
    const int rc = check_heads(dt, heads, kv_heads, D);
    if (rc != C2R_OK) return rc;
    if (T < 0 || rot < 0 || rot > D || !(eps >= 0.0f)) return C2R_ERR_INVALID_ARG;
    if (T >= ATTN_MOST || rot % 16 != 0) return C2R_ERR_UNSUPPORTED;
    if (rot > 0 && (!inv_freq || !aligned(inv_freq, 4))) return C2R_ERR_INVALID_ARG;
    if ((q_weight && !aligned(q_weight, 16)) || (k_weight && !aligned(k_weight, 16))) return C2R_ERR_INVALID_ARG;
    return C2R_OK;
}

size_t attention_workspace_bytes(int64_t T, int D, int heads, int kv_heads, int max_q_len) {
    if (T <= 0 || D <= 0 || heads <= 0 || kv_heads <= 0) return 0;
    // the most rows x parts that attn_parts() gives where it gives more than one part: `blocks` blocks become at most
    // target + blocks, and each has at most per_block rows
    const int64_t rows = T * heads;
    auto bound = [rows](int64_t target, int64_t per_block) { return rows <= target * per_block ? target * per_block + rows : 0; };
    if (max_q_len <= 0)
        return round_up((size_t)bound(ATTN_DECODE_EVEN_BLOCKS, heads / kv_heads < 16 ? heads / kv_heads : 16) * (size_t)(D + 2) * 4, 256);
    const int64_t tile = bound(ATTN_TILE_BLOCKS, ATTN_TILE_ROWS), full = bound(ATTN_ROWS_BLOCKS, ATTN_ROWS_ROWS);
    return round_up((size_t)(tile > full ? tile : full) * (size_t)(D + 2) * 4, 256);
}

// The rows x parts of a batch behind shared prefixes: parts of the prefixes, of any of the kernels, and of what lies behind.
size_t attention_shared_workspace_bytes(int64_t T, int D, int heads, int kv_heads) {
    if (T <= 0 || D <= 0 || heads <= 0 || kv_heads <= 0) return 0;
    const int64_t rows = T * heads, prefix = (int64_t)ATTN_TILE_BLOCKS * ATTN_TILE_ROWS, cols = heads / kv_heads < 16 ? heads / kv_heads : 16;
    static_assert(ATTN_TILE_BLOCKS * ATTN_TILE_ROWS >= ATTN_DECODE_BLOCKS * 16, "either kernel's parts of a prefix");
    // (own keys: parts as in decoding, or two by waves)
    return round_up((size_t)(prefix + rows + ATTN_DECODE_EVEN_BLOCKS * cols + 2 * rows) * (size_t)(D + 2) * 4, 256);
}

}  // namespace c2r

using namespace c2r;

extern "C" int c2r_qk_norm_rope(const void *q, int64_t q_stride, const void *k, int64_t k_stride, c2r_dtype dt, int64_t T, int heads, int kv_heads,
                                int head_dim, const float *q_weight, const float *k_weight, float eps, const float *inv_freq, int rot_dim,
                                int neighbours, const int32_t *position, void *q_out, int64_t q_out_stride, void *k_out, int64_t k_out_stride,
                                void *stream) {
    drop_stale_error();
    const int rc = check_rope(dt, heads, kv_heads, head_dim, T, q_weight, k_weight, eps, inv_freq, rot_dim);
    if (rc != C2R_OK) return rc;
    if (T == 0) return C2R_OK;
    const int size = dt == C2R_BF16 ? 2 : 4;
    const int64_t wq = (int64_t)heads * head_dim, wk = (int64_t)kv_heads * head_dim;
    if (!rows_ok(q, q_stride, wq, size) || !rows_ok(k, k_stride, wk, size) || !rows_ok(q_out, q_out_stride, wq, size) ||
        !rows_ok(k_out, k_out_stride, wk, size))
        return C2R_ERR_INVALID_ARG;
    if (rot_dim > 0 && (!position || !aligned(position, 4))) return C2R_ERR_INVALID_ARG;
    RopeCall a = {};
    a.q = static_cast<const unsigned char *>(q);
    a.k = static_cast<const unsigned char *>(k);
    a.q_out = static_cast<unsigned char *>(q_out);
    a.k_out = static_cast<unsigned char *>(k_out);
    a.q_bytes = q_stride * size, a.k_bytes = k_stride * size, a.q_out_bytes = q_out_stride * size, a.k_out_bytes = k_out_stride * size;
    a.q_weight = q_weight, a.k_weight = k_weight, a.inv_freq = inv_freq, a.position = position;
    a.T = T, a.heads = heads, a.kv_heads = kv_heads, a.rot = rot_dim, a.eps = eps;
    return launch_qk_norm_rope(a, dt == C2R_BF16, head_dim, neighbours != 0, static_cast<hipStream_t>(stream));
}

extern "C" int c2r_qk_norm_rope_append(const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride, int64_t T,
                                       int heads, const float *q_weight, const float *k_weight, float eps, const float *inv_freq, int rot_dim,
                                       int neighbours, const int32_t *q_start, const int32_t *position, const c2r_kv_cache *cache, void *q_out,
                                       int64_t q_out_stride, void *stream) {
    drop_stale_error();
    int rc = check_cache(cache, heads);
    if (rc != C2R_OK) return rc;
    const int dt = (int)cache->dtype, kv_heads = (int)cache->kv_heads, D = (int)cache->head_dim;
    rc = check_rope(dt, heads, kv_heads, D, T, q_weight, k_weight, eps, inv_freq, rot_dim);
    if (rc != C2R_OK) return rc;
    if (T == 0) return C2R_OK;
    if (!q_start && T != cache->batch) return C2R_ERR_INVALID_ARG;
    // two rows of the cache in one place would be written in any order (reading them is harmless)
    if ((cache->page_size > 1 && cache->slot_stride < D) || (kv_heads > 1 && cache->head_stride < D) || (cache->n_pages > 1 && cache->page_stride < D))
        return C2R_ERR_INVALID_ARG;
    const int size = dt == C2R_BF16 ? 2 : 4;
    const int64_t wq = (int64_t)heads * D, wk = (int64_t)kv_heads * D;
    if (!rows_ok(q, q_stride, wq, size) || !rows_ok(k, k_stride, wk, size) || !rows_ok(v, v_stride, wk, size) || !rows_ok(q_out, q_out_stride, wq, size))
        return C2R_ERR_INVALID_ARG;
    if ((position && !aligned(position, 4)) || (q_start && !aligned(q_start, 4))) return C2R_ERR_INVALID_ARG;
    RopeCall a = {};
    a.q = static_cast<const unsigned char *>(q);
    a.k = static_cast<const unsigned char *>(k);
    a.v = static_cast<const unsigned char *>(v);
    a.q_out = static_cast<unsigned char *>(q_out);
    a.q_bytes = q_stride * size, a.k_bytes = k_stride * size, a.v_bytes = v_stride * size, a.q_out_bytes = q_out_stride * size;
    a.q_weight = q_weight, a.k_weight = k_weight, a.inv_freq = inv_freq, a.position = position, a.q_start = q_start;
    a.T = T, a.heads = heads, a.kv_heads = kv_heads, a.rot = rot_dim, a.eps = eps;
    a.kv = view_of(*cache);
    return launch_qk_norm_rope(a, dt == C2R_BF16, D, neighbours != 0, static_cast<hipStream_t>(stream));
}

// The checks that both forms of attention share, and the call without its split.
static int attention_call(const void *q, int64_t q_stride, int64_t T, int heads, const c2r_kv_cache *cache, float scale, int64_t window,
                          int64_t sinks, void *out, int64_t out_stride, AttnCall &a) {
    const int rc = check_cache(cache, heads);
    if (rc != C2R_OK) return rc;
    if (T < 0 || window < 0 || sinks < 0 || !(scale == scale)) return C2R_ERR_INVALID_ARG;
    if (T >= ATTN_MOST) return C2R_ERR_UNSUPPORTED;
    if (T == 0 || cache->batch == 0) return C2R_OK;
    const int size = cache->dtype == C2R_BF16 ? 2 : 4;
    const int64_t width = heads * cache->head_dim, capacity = cache->page_size * cache->max_pages;
    if (!rows_ok(q, q_stride, width, size) || !rows_ok(out, out_stride, width, size)) return C2R_ERR_INVALID_ARG;
    a = AttnCall{};
    a.kv = view_of(*cache);
    a.q = static_cast<const unsigned char *>(q);
    a.out = static_cast<unsigned char *>(out);
    a.q_bytes = q_stride * size, a.out_bytes = out_stride * size;
    a.T = T;
    a.max_q = 1;
    a.heads = heads, a.group = heads / (int)cache->kv_heads;
    // a window of as many tokens as a sequence can have is none, and more sinks than keys are all of them
    a.window = window >= ATTN_MOST ? 0 : (int)window;
    a.sinks = a.window == 0 ? 0 : sinks > capacity ? (int)capacity : (int)sinks;
    a.scale_log2 = scale * 1.4426950408889634f;
    a.scale_size = a.scale_log2 == 0.0f ? 1.0f : fabsf(a.scale_log2);
    a.splits = 1;
    return C2R_OK;
}

static int64_t longest(const c2r_kv_cache *cache, int64_t max_kv_len) {
    const int64_t capacity = cache->page_size * cache->max_pages;
    return max_kv_len > 0 && max_kv_len < capacity ? max_kv_len : capacity;
}

// Parts that the keys of a bf16 prompt are cut into: the number whose estimated time is least.  Blocks of 128 rows look at up to
// `tiles` tiles, those of a prompt's first rows at fewer; a block with more than tiles / n is cut.  The call takes as long as its
// longest part, or as the tiles over the GPU's 512 places and some of a part behind them.  A cut costs a second launch and the writing and
// reading of the cut rows' sums.  A tile (heads of 128) takes 1.6 us where a block has a CU to itself and 2.2 where two share it; the
// estimate has 1.6 for both and its other constants fitted to the calls measured.  Measured, us, 1 to 4 parts (16 heads unless said): 2000 tokens 51, 46, 42, 57; 1000 behind 16000 361, 208, 182, 160; 500
// behind 2000, 32 heads 53, 48, 46, 43; three ragged chunks of 700 behind 5000 135, 94, 77, 91; but 4 x 2048 88, 138, 141, 198 and
// 4000 tokens 96, 115, 106, 135; 256 behind 8000 in 8 parts 41 and whole 174.  Over 24 such calls the choice is 4 % over the best of
// 1, 2, 3, 4, 6 and 8 parts on average, and 19 % at most (a ragged batch, whose lengths the host does not know).
static int64_t prompt_parts(const AttnCall &a, int64_t blocks, int64_t tiles, int64_t longest, int D) {
    // (a batch's T rows may be far fewer than batch * max_q; every sequence and key head has a block that is not full)
    const double rows = (double)a.T * a.heads, real = rows / ATTN_TILE_ROWS + a.kv.batch * a.kv.kv_heads * 0.5;
    const double units = real < blocks ? real : blocks, rate = D == 128 ? 1.6 : 0.92;
    const double fewest = a.window && a.window < a.kv.capacity ? 0.9 * tiles : a.max_q < longest ? tiles * (1.0 - (double)a.max_q / longest) : 0.0;
    constexpr int SAMPLES = 8;
    int64_t best = 1;
    double least = 0.0;
    // (numbers of parts of one length are one: 8 tokens behind 200000 keys, one head: 108 estimates and 3 us of the
    // host's time for 782 and 18)
    for (int64_t n = 1, length; n == 1 || (n * units <= ATTN_TILE_BLOCKS && n <= ceil_div(tiles, ATTN_TILE_TILES)); n = ceil_div(tiles, length - 1)) {
        length = ceil_div(tiles, n);
        const double each = (double)length;
        double all = 0.0, cut = 0.0;  // a block's tiles; its parts, where it is cut
        for (int i = 0; i < SAMPLES; ++i) {
            const double c = fewest + (tiles - fewest) * (i + 0.5) / SAMPLES;
            all += c / SAMPLES;
            if (c > each) cut += (double)(int64_t)(c / each + 1.0) / SAMPLES;
        }
        const double part = each * rate, spread = 0.9 * units * all * rate / ATTN_TILE_BLOCKS + 0.4 * part;
        const double t = (part > spread ? part : spread) + (n == 1 ? 0.0 : 5.0 + rows * cut * D * 8 / 2e6);
        if (n == 1 || t < least) least = t, best = n;
        if (length <= 1) break;
    }
    return best;
}

// Partial results go to the workspace where the keys are cut.
static int place_parts(AttnCall &a, int D, void *ws, size_t ws_bytes) {
    if (a.splits == 1 && !a.shared) return C2R_OK;
    const size_t rows = (size_t)a.T * a.heads * a.splits;
    if (!ws || !aligned(ws, 256) || ws_bytes < rows * (size_t)(D + 2) * 4) return C2R_ERR_WORKSPACE;
    a.part_o = static_cast<float *>(ws);
    a.part_ml = a.part_o + rows * D;
    return C2R_OK;
}

// Few blocks: parts of 8 tiles or more (256 keys in bf16) until the GPU's 768 places are taken.  Many: long sequences in
// parts of 24 or more, so that a batch of ragged lengths ends evenly.  Microseconds, bf16, heads of 128:
//   1 x 4096 keys, 16 key heads: parts of 4, 8, 24 tiles 13.5, 13.4, 16;  1 x 32000: parts of 8, 21, 24 57, 52.5, 53
//   131 ragged sequences of up to 8000, 8 key heads, 1, 2, 3, 5 parts: 393, 420, 376, 371
//   256 ragged sequences of up to 500, 16 key heads, parts of 8 tiles and whole: 120 and 97
static int64_t decode_parts(int64_t blocks, int64_t tiles) {
    const int64_t fill = attn_parts(blocks, tiles, ATTN_DECODE_BLOCKS, ATTN_DECODE_TILES);
    const int64_t even = attn_parts(blocks, tiles, ATTN_DECODE_EVEN_BLOCKS, ATTN_DECODE_EVEN_TILES);
    return fill > even ? fill : even;
}

extern "C" int c2r_attention_decode(const void *q, int64_t q_stride, int heads, const c2r_kv_cache *cache, int64_t max_kv_len, float scale,
                                    int64_t window, int64_t sinks, void *out, int64_t out_stride, void *ws, size_t ws_bytes, void *stream) {
    drop_stale_error();
    if (!cache) return C2R_ERR_INVALID_ARG;
    AttnCall a;
    int rc = attention_call(q, q_stride, cache->batch, heads, cache, scale, window, sinks, out, out_stride, a);
    if (rc != C2R_OK || cache->batch == 0) return rc;
    const bool bf16 = cache->dtype == C2R_BF16;
    const int64_t blocks = cache->batch * cache->kv_heads * ceil_div(a.group, 16);
    const int64_t tiles = attn_max_tiles(a, bf16 ? 32 : 16, 1, longest(cache, max_kv_len));
    attn_split(a, tiles, decode_parts(blocks, tiles));
    if (blocks * a.splits >= ATTN_MOST_BLOCKS) return C2R_ERR_UNSUPPORTED;
    rc = place_parts(a, (int)cache->head_dim, ws, ws_bytes);
    return rc == C2R_OK ? launch_attn_decode(a, bf16, (int)cache->head_dim, static_cast<hipStream_t>(stream)) : rc;
}

extern "C" int c2r_attention_prefill(const void *q, int64_t q_stride, int64_t T, int heads, const int32_t *q_start, int64_t max_q_len,
                                     const c2r_kv_cache *cache, int64_t max_kv_len, float scale, int64_t window, int64_t sinks, void *out,
                                     int64_t out_stride, void *ws, size_t ws_bytes, void *stream) {
    drop_stale_error();
    AttnCall a;
    int rc = attention_call(q, q_stride, T, heads, cache, scale, window, sinks, out, out_stride, a);
    if (rc != C2R_OK) return rc;
    if (max_q_len < 0) return C2R_ERR_INVALID_ARG;
    if (T == 0 || cache->batch == 0 || max_q_len == 0) return C2R_OK;
    if (!q_start || !aligned(q_start, 4)) return C2R_ERR_INVALID_ARG;
    a.q_start = q_start;
    a.max_q = (int)(max_q_len < T ? max_q_len : T);
    const bool bf16 = cache->dtype == C2R_BF16;
    const int64_t per_block = bf16 ? ATTN_TILE_ROWS : ATTN_ROWS_ROWS;
    if (T * a.group >= (1ll << 31)) return C2R_ERR_UNSUPPORTED;
    const int64_t each = ceil_div((int64_t)a.max_q * a.group, per_block), by_rows = T * a.group / per_block + cache->batch;
    a.by_rows = each * cache->batch > ATTN_BY_ROWS * by_rows;
    const int64_t blocks = cache->kv_heads * (a.by_rows ? by_rows : each * cache->batch);
    if (blocks >= ATTN_MOST_BLOCKS) return C2R_ERR_UNSUPPORTED;
    a.row_blocks = (int)(a.by_rows ? by_rows : each);
    const int64_t tiles = attn_max_tiles(a, bf16 ? 64 : 16, ceil_div(per_block, a.group) + 1, longest(cache, max_kv_len));
    // Full precision: parts of 6 tiles (96 keys) or more until there are 1024 blocks.  us, parts of 4, 6, 8 tiles: 512 tokens, 4 heads
    // of 64 14.6, 15.5, 17.0; 2 x 64 behind 4000 21.6, 23.1, 19.8; 3 x 5 behind 3000 23.1, 19.8, 22.8.  512, 1024, 2048 blocks: 1500
    // tokens, 8 heads of 64 59, 55, 63; 8 ragged of up to 512 44, 52, 52; 2 ragged of up to 2000, 4 heads of 128 184, 191, 165; 400 behind
    // 6000, 8 heads 164, 177, 153: none is ahead everywhere.
    int64_t parts = bf16 ? prompt_parts(a, blocks, tiles, longest(cache, max_kv_len), (int)cache->head_dim) : attn_parts(blocks, tiles, ATTN_ROWS_BLOCKS, ATTN_ROWS_TILES);
    // (partial results are laid out by rows of q: rows that no sequence has, or past its max_q_len, take their room, too, and
    // more parts than the workspace query foresees are not made)
    const int64_t room = (bf16 ? ATTN_TILE_BLOCKS : ATTN_ROWS_BLOCKS) * per_block / (T * heads) + 1;
    // (the join has blocks for max_q rows of every sequence)
    if (ceil_div((int64_t)a.max_q * heads, 4) * cache->batch > ATTN_JOIN_BLOCKS) parts = 1;
    attn_split(a, tiles, parts < room ? parts : room);
    if (blocks * a.splits >= ATTN_MOST_BLOCKS) return C2R_ERR_UNSUPPORTED;
    rc = place_parts(a, (int)cache->head_dim, ws, ws_bytes);
    if (rc != C2R_OK) return rc;
    return bf16 ? launch_attn_tile(a, (int)cache->head_dim, static_cast<hipStream_t>(stream))
                : launch_attn_rows_f32(a, (int)cache->head_dim, static_cast<hipStream_t>(stream));
}

extern "C" int c2r_attention_decode_shared(const void *q, int64_t q_stride, int heads, const c2r_kv_cache *cache, const int32_t *shared_start,
                                           const int32_t *shared_len, int64_t n_shared, int64_t max_shared_len, int64_t max_own_len, float scale,
                                           int64_t window, int64_t sinks, void *out, int64_t out_stride, void *ws, size_t ws_bytes, void *stream) {
    drop_stale_error();
    if (!cache || n_shared < 0) return C2R_ERR_INVALID_ARG;
    AttnCall a;
    int rc = attention_call(q, q_stride, cache->batch, heads, cache, scale, window, sinks, out, out_stride, a);
    if (rc != C2R_OK || cache->batch == 0) return rc;
    if (n_shared >= ATTN_MOST_RUNS) return C2R_ERR_UNSUPPORTED;
    if (n_shared == 0) return c2r_attention_decode(q, q_stride, heads, cache, max_own_len, scale, window, sinks, out, out_stride, ws, ws_bytes, stream);
    if (!shared_start || !shared_len || !aligned(shared_start, 4) || !aligned(shared_len, 4)) return C2R_ERR_INVALID_ARG;
    const bool bf16 = cache->dtype == C2R_BF16;
    const int D = (int)cache->head_dim;
    if (cache->batch * a.group >= (1ll << 30)) return C2R_ERR_UNSUPPORTED;
    a.shared_start = shared_start, a.shared_len = shared_len, a.shared = (int)n_shared;
    // the prefixes
    const bool tiled = bf16 && cache->batch * a.group > ATTN_PREFIX_ROWS * n_shared;
    const int64_t per_block = tiled ? ATTN_TILE_ROWS : 16, KT = tiled ? 64 : bf16 ? 32 : 16;
    const int64_t rows = cache->batch * a.group / per_block + n_shared;
    // (of a prefix that lies before a sequence's own keys, a window leaves its own length at most)
    int64_t prefix_tiles = ceil_div(longest(cache, max_shared_len), KT);
    if (a.window) {
        const int64_t near = ceil_div(a.window, KT) + 1 + ceil_div(a.sinks, KT);
        if (near < prefix_tiles) prefix_tiles = near;
    }
    const int most = tiled ? attn_prefix_blocks(D) : ATTN_DECODE_BLOCKS;
    int64_t parts = attn_parts(rows * cache->kv_heads, prefix_tiles, most, tiled ? ATTN_TILE_TILES : ATTN_DECODE_TILES);
    // (no more blocks than that: one too many takes as long as as many again)
    static_assert(attn_prefix_blocks(64) <= ATTN_TILE_BLOCKS && attn_prefix_blocks(128) <= ATTN_TILE_BLOCKS, "the workspace query counts on it");
    if (tiled && parts > 1 && parts * rows * cache->kv_heads > most) --parts;
    a.prefix_tiles = (int)ceil_div(prefix_tiles, parts);
    a.prefix_splits = (int)ceil_div(prefix_tiles, a.prefix_tiles);
    a.prefix_blocks = (int)rows;
    // what lies behind them
    const int64_t blocks = cache->batch * cache->kv_heads * ceil_div(a.group, 16);
    const int64_t tiles = attn_max_tiles(a, bf16 ? 32 : 16, 1, longest(cache, max_own_len));
    // many sequences with few keys each: a wave for each, of 8 tiles at most
    static_assert(ATTN_WAVE_MOST <= 2 * ATTN_WAVE_TILES, "two parts at most: the workspace query counts on it");
    a.own_by_wave = blocks >= ATTN_WAVE_SETS && tiles <= ATTN_WAVE_MOST;
    attn_split(a, tiles, a.own_by_wave ? ceil_div(tiles, ATTN_WAVE_TILES) : decode_parts(blocks, tiles));
    if (rows * cache->kv_heads * a.prefix_splits + blocks * a.splits >= ATTN_MOST_BLOCKS) return C2R_ERR_UNSUPPORTED;
    a.splits += a.prefix_splits;
    rc = place_parts(a, D, ws, ws_bytes);
    if (rc != C2R_OK) return rc;
    return launch_attn_shared(a, bf16, tiled, D, static_cast<hipStream_t>(stream));
}
