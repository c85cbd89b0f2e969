// What the attention kernels share: the view of the paged cache, which keys a query sees, the tiles to visit, the exact
// row for inputs that are not finite, and the layout of partial results.
#pragma once
#include "ffn_copy.h"

namespace c2r {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// The cache as the kernels see it.  Byte strides in 64 bits: a long cache passes 4 GB.
struct KvView {
    const unsigned char *k, *v;
    int64_t page_bytes, slot_bytes, head_bytes;
    const int32_t *table, *kv_len;
    int32_t n_pages, page_size, max_pages, batch, kv_heads;
    int32_t capacity;  // keys that a sequence's row of the table can name
    uint32_t div_mul, div_shift;  // key index / page_size = (mulhi(div_mul, j) + j) >> div_shift, j < 2^31

    __device__ __forceinline__ int page_of(int j) const { return (int)((__umulhi(div_mul, (uint32_t)j) + (uint32_t)j) >> div_shift); }
    // Tokens of sequence b.  Those from place `capacity` on are in no page: positions count them, and no query sees them.
    __device__ __forceinline__ int tokens(int b) const { return min(max(kv_len[b], 0), 1 << 30); }
    // The table's entry for key j of sequence b (j below capacity), as it stands there: nothing waits for it before it is used.
    __device__ __forceinline__ int page(int b, int j) const { return table[(int64_t)b * max_pages + page_of(j)]; }
    // Where key j lies; an entry outside the cache reads as page 0.
    __device__ __forceinline__ int64_t offset(int page, int j) const {
        const int p = (uint32_t)page < (uint32_t)n_pages ? page : 0;
        return p * page_bytes + (int64_t)(j - page_of(j) * page_size) * slot_bytes;
    }
};

// How many i of 0 .. n - 1 are `below`, which are the first ones: the wave looks at 64 evenly spread ones, then at the 64 steps
// between two of them, ...
template <class F>
__device__ __forceinline__ int count_first(int n, const F &below) {
    int lo = 0;  // the count lies in lo .. lo + n
    const int lane = lane_id();
    while (n > 0) {
        const int step = (n + 63) / 64, at = lo + (lane + 1) * step - 1;  // last one of each of 64 runs
        const int runs = __popcll(__ballot(at < lo + n && below(at)));
        lo += runs * step;
        const int rest = n - runs * step;
        n = rest < step - 1 ? rest : step - 1;
        if (step == 1) break;
    }
    return lo;
}

// In the place of a part's denominator: it holds no key of this row and has written no sums; all of the row's keys were in the
// first part, which has written the result.
constexpr float PART_EMPTY = -1.0f, PART_DONE = -2.0f;

// Keys of a sequence that a block looks at, of those its queries see: all of them, a prefix, or what lies behind one.
struct KeyRange {
    int from = 0, to = 0x7fffffff;
};

// One call of attention.  New tokens of sequence b: rows q_start[b] .. of q (b .. b + 1 where q_start is null); the last of
// them stands at position kv_len[b] - 1.
struct AttnCall {
    KvView kv;
    const unsigned char *q;
    unsigned char *out;
    int64_t q_bytes, out_bytes;  // from one token to the next
    const int32_t *q_start;
    int64_t T;
    int max_q;                // new tokens of a sequence that the grid has blocks for
    int heads, group;         // query heads, and of them per key head
    int window, sinks;        // window 0: none
    float scale_log2;         // scale * log2(e): the softmax is taken in powers of two
    float scale_size;         // its absolute value, or 1 where it is 0
    int splits, split_tiles;  // the key tiles of one row of blocks, cut after every split_tiles; 1: no partial results
    // Prompts: blocks of rows for every key head and part.  by_rows: counted through all sequences, T * group / BM + batch of them;
    // else as many for each sequence as max_q needs.
    int row_blocks;
    bool by_rows;
    // Runs of sequences that begin with the same keys: run i is the sequences shared_start[i] .. shared_start[i + 1] - 1, its keys the
    // first shared_len[i] of the first of them.  The first prefix_splits of the parts are cut from these, after every
    // prefix_tiles tiles, the others from the sequences' own keys.  prefix_blocks: rows of blocks that the prefixes have.
    const int32_t *shared_start, *shared_len;
    int shared, prefix_splits, prefix_tiles, prefix_blocks;
    bool own_by_wave;  // a sequence's own keys are one wave's, for the heads of a key head, and not a block's
    float *part_o, *part_ml;  // [splits][T * heads][D] sums, [splits][T * heads][2] maximum and denominator (or PART_..)

    __device__ __forceinline__ int first_row(int b) const { return q_start ? (int)clamp_row(q_start[b]) : b; }
    __device__ __forceinline__ int new_tokens(int b) const {
        if (!q_start) return 1;
        const int64_t n = clamp_row(q_start[b + 1]) - clamp_row(q_start[b]);
        return n > 0 ? (int)n : 0;
    }
    __device__ __forceinline__ int64_t clamp_row(int32_t r) const { return r < 0 ? 0 : (int64_t)r > T ? T : r; }
    // Block x of a key head's and part's: sequence b, block rb of its rows, a sequence's last (longest) ones first.  False: there
    // is none.
    // by_rows: sequence b has the numbers from q_start[b] * group / BM + b on, which are enough: floor(x + y) + 1 >= floor(x) +
    // ceil(y).
    template <int BM>
    __device__ __forceinline__ bool block_of(int x, int &b, int &rb) const {
        if (!by_rows) {
            b = x % kv.batch, rb = row_blocks - 1 - x / kv.batch;
            return true;
        }
        auto begin = [&](int i) { return (int)(clamp_row(q_start[i]) * group / BM) + i; };
        b = count_first(kv.batch, [&](int i) { return begin(i) <= x; }) - 1;
        if (b < 0) return false;
        const int64_t rows = (int64_t)min(new_tokens(b), max_q) * group;
        rb = (int)((rows + BM - 1) / BM) - 1 - (x - begin(b));
        return rb >= 0;
    }
    __device__ __forceinline__ int shared_first(int i) const { return (int)clamp_row(shared_start[i]); }
    __device__ __forceinline__ int shared_keys(int i) const { return min(max(shared_len[i], 0), kv.capacity); }
    // A run: its sequences first .. end - 1, and its keys.  The last run that begins at or below x by begin(run, its first sequence); -1: none.
    struct Run {
        int i, first, end, keys;
    };
    template <class F>
    __device__ __forceinline__ Run run_at(int x, const F &begin) const {
        Run run;
        if (shared <= C2R_WAVE) {  // one run to a lane: all that is to be known comes with one trip to memory
            const int r = min(lane_id(), shared - 1), first = shared_first(r), end = shared_first(r + 1), keys = shared_keys(r);
            run.i = __popcll(__ballot(lane_id() < shared && begin(r, first) <= x)) - 1;
            const int at = max(run.i, 0);
            run.first = __shfl(first, at), run.end = __shfl(end, at), run.keys = __shfl(keys, at);
        } else {
            run.i = count_first(shared, [&](int r) { return begin(r, shared_first(r)) <= x; }) - 1;
            const int at = max(run.i, 0);
            run.first = shared_first(at), run.end = shared_first(at + 1), run.keys = shared_keys(at);
        }
        run.first = __builtin_amdgcn_readfirstlane(run.first), run.end = __builtin_amdgcn_readfirstlane(run.end);
        run.keys = __builtin_amdgcn_readfirstlane(run.keys);
        return run;
    }
    // The keys that sequence b has before its own ones.
    __device__ __forceinline__ int prefix_of(int b) const {
        const Run run = run_at(b, [](int, int first) { return first; });
        return run.i >= 0 && b < run.end ? run.keys : 0;
    }
    // Block x of a key head's and part's: a run and block rb of its (sequence, head of the group) rows, counted as in block_of.
    template <int BM>
    __device__ __forceinline__ bool prefix_block_of(int x, Run &run, int &rb, int &rows) const {
        auto begin = [&](int r, int first) { return (int)((int64_t)first * group / BM) + r; };
        run = run_at(x, begin);
        if (run.i < 0) return false;
        rows = (run.end - run.first) * group;
        rb = x - begin(run.i, run.first);
        return rb * BM < rows && run.keys > 0;
    }
    // The last key that is cached of those up to position p, and of those the last one of keys[.., to).
    __device__ __forceinline__ int last_key(int p) const { return min(p, kv.capacity - 1); }
    __device__ __forceinline__ int last_key(int p, KeyRange keys) const { return min(last_key(p), keys.to - 1); }
    // Whether the query at position p sees key j; whether it sees none.
    __device__ __forceinline__ bool sees(int p, int j) const { return j <= last_key(p) && (!window || j > p - window || j < sinks); }
    __device__ __forceinline__ bool sees(int p, int j, KeyRange keys) const { return j >= keys.from && j < keys.to && sees(p, j); }
    __device__ __forceinline__ bool blind(int p) const { return p < 0 || (window && !sinks && p - window >= kv.capacity - 1); }
};

// The key tiles (KT keys, aligned) that queries at positions p_min .. p_max look at: those of the first `sinks` keys that lie
// before the window, then the window's.
template <int KT>
struct KeyTiles {
    int sink_tiles, first, count, skipped;  // skipped: tiles before the range's first
    __device__ __forceinline__ KeyTiles(const AttnCall &a, int p_min, int p_max, KeyRange keys = KeyRange()) {
        skipped = keys.from / KT;
        const int last = a.last_key(p_max, keys);  // (a window that begins past the cache's end leaves the sinks)
        sink_tiles = 0, first = skipped;
        if (a.window) {
            const int lo = p_min - a.window + 1;
            first = lo > keys.from ? lo / KT : skipped;
            // (sinks past the range's end are no tiles of it)
            int s = (int)(((int64_t)a.sinks + KT - 1) / KT);
            if (keys.to != 0x7fffffff) s = min(s, last < 0 ? 0 : last / KT + 1);
            sink_tiles = max((s < first ? s : first) - skipped, 0);
        }
        count = last < keys.from ? 0 : sink_tiles + max(last / KT - first + 1, 0);
    }
    __device__ __forceinline__ int base(int x) const { return (x < sink_tiles ? skipped + x : first + x - sink_tiles) * KT; }
    __device__ __forceinline__ void part(int n, int tiles, int s, int &x0, int &x1) const {
        const int64_t lo = (int64_t)s * tiles, hi = s + 1 == n ? count : lo + tiles;
        x0 = lo < count ? (int)lo : count;
        x1 = hi < count ? (int)hi : count;
    }
    // [x0, x1): the part of split s.  The last one takes what is left, however long a sequence is.
    __device__ __forceinline__ void part(const AttnCall &a, int s, int &x0, int &x1) const {
        part(a.splits, a.split_tiles, s, x0, x1);
    }
    // Whether split 0 has all of them: it then writes the result itself and says so to the join (PART_DONE).
    __device__ __forceinline__ bool uncut(const AttnCall &a) const { return a.splits == 1 || count <= a.split_tiles; }
};

// A tile [base, base + KT) that every query of p_min .. p_max sees whole.
template <int KT>
__device__ __forceinline__ bool tile_whole(const AttnCall &a, int base, int p_min, int p_max, KeyRange keys = KeyRange()) {
    return base >= keys.from && base + KT - 1 <= a.last_key(p_min, keys) && (!a.window || base > p_max - a.window || base + KT <= a.sinks);
}

__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }
// What the scores are taken against: the running maximum, but 0 while every score was -infinity (-inf - -inf is a NaN).
__device__ __forceinline__ float reference_of(float m) { return m == -__builtin_inff() ? 0.0f : m; }

template <bool BF16>
__device__ __forceinline__ float load_element(const unsigned char *p, int i) {
    if constexpr (BF16) return bf16_bits_to_f32(reinterpret_cast<const uint16_t *>(p)[i]);
    return reinterpret_cast<const float *>(p)[i];
}

// One query's row by the definition, a key at a time: nothing that it does not see enters, not even times zero.  The tile
// kernels multiply the values of a tile's hidden keys with a weight of zero, which an infinity or a NaN there (a later token
// of the same prompt, a page that was never written) turns into a NaN; a row that comes out not finite is done again here, so
// that finite inputs pay one check per output.  The whole wave runs it: a lane holds a key's score, then D / 64 elements.
template <bool BF16, int D, int KT>
__device__ __forceinline__ void exact_row(const AttnCall &a, const KeyTiles<KT> tiles, int x0, int x1, int step, int b, int kv_head,
                                          int p, const unsigned char *q_row, float &m_out, float &l_out, float (&o)[D / 64],
                                          KeyRange keys = KeyRange()) {
    constexpr int N = D / 64;
    const int lane = lane_id();
    float m = -__builtin_inff(), l = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = 0.0f;
    for (int x = x0; x < x1; x += step) {
        const int j = tiles.base(x) + lane;
        const bool see = lane < KT && a.sees(p, j, keys);
        int64_t at = 0;
        float s = -__builtin_inff();
        if (see) {
            at = a.kv.offset(a.kv.page(b, j), j) + kv_head * a.kv.head_bytes;
            float dot = 0.0f;
            for (int i = 0; i < D; ++i) dot = __builtin_fmaf(load_element<BF16>(q_row, i), load_element<BF16>(a.kv.k + at, i), dot);
            s = dot * a.scale_log2;
        }
        float t = s;
        for (int w = 32; w; w >>= 1) t = fmaxf(t, __shfl_xor(t, w));
        const float m_new = fmaxf(m, t), ref = reference_of(m_new);
        const float alpha = __builtin_amdgcn_exp2f(m - ref), pr = see ? __builtin_amdgcn_exp2f(s - ref) : 0.0f;
        l *= alpha;
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] *= alpha;
        m = m_new;
        uint64_t left = __ballot(see);
        while (left) {
            const int src = __ffsll((unsigned long long)left) - 1;
            left &= left - 1;
            const float w = __shfl(pr, src);
            const unsigned char *row = a.kv.v + __shfl(at, src);
            l += w;
#pragma unroll
            for (int i = 0; i < N; ++i) o[i] = __builtin_fmaf(w, load_element<BF16>(row, lane * N + i), o[i]);
        }
    }
    m_out = m;
    l_out = l;
}

// One call of the norms and the rotation.
struct RopeCall {
    const unsigned char *q, *k, *v;
    unsigned char *q_out, *k_out;  // k_out null: keys and values go to the cache
    int64_t q_bytes, k_bytes, v_bytes, q_out_bytes, k_out_bytes;
    const float *q_weight, *k_weight, *inv_freq;
    const int32_t *position, *q_start;
    int64_t T, first, end;  // a launch takes the tokens first .. end
    int heads, kv_heads, rot, parts;
    float eps;
    KvView kv;
};

// qk_rope.hip
int launch_qk_norm_rope(RopeCall a, bool bf16, int D, bool neighbours, hipStream_t st);
// attn_join.hip: out = joined partial results of a call with more than one split.
int launch_attn_join(const AttnCall &a, bool bf16, int D, hipStream_t st);
// attn_decode.hip: one new token per sequence.
int launch_attn_decode(const AttnCall &a, bool bf16, int D, hipStream_t st);
// attn_shared.hip: one new token per sequence behind prefixes that runs of sequences share.
int launch_attn_shared(const AttnCall &a, bool bf16, bool tiled, int D, hipStream_t st);
// attn_rows.hip: prompts in full precision.
int launch_attn_rows_f32(const AttnCall &a, int D, hipStream_t st);
// attn_tile.hip: prompts in bf16, key tiles through LDS.
int launch_attn_tile(const AttnCall &a, int D, hipStream_t st);

// How many blocks a call is cut into at most where it has few rows, by kernel (the reasons stand beside each), and the key
// tiles of a part.
constexpr int ATTN_DECODE_BLOCKS = 768, ATTN_DECODE_TILES = 8, ATTN_DECODE_EVEN_BLOCKS = 4608, ATTN_DECODE_EVEN_TILES = 24;
constexpr int ATTN_TILE_BLOCKS = 512, ATTN_TILE_TILES = 4, ATTN_TILE_ROWS = 128;
constexpr int ATTN_ROWS_BLOCKS = 1024, ATTN_ROWS_TILES = 6, ATTN_ROWS_ROWS = 64;

// Rows are counted through all sequences where that makes less than half of the blocks: a batch of a few chunks among single
// tokens, whose other blocks would find no row.  us by rows and with as many blocks for each sequence: 32 / 8 heads, one chunk of
// 1500 and 255 single tokens behind 1000 208 and 351, the chunk last 220 and 358; 500 behind 8000 and 15 singles 101 and 135; 2 of
// 1000 and 30 of 20, 16 heads 27 and 27, but with the long ones last, whose blocks then start last, 39 and 29; not so many idle ones:
// 4 x 2048 93 and 85, five ragged chunks 83.4 and 81.3.
constexpr int ATTN_BY_ROWS = 2;
// Blocks of a join from which on keys are not cut: nearly all of them would find nothing to do.
constexpr int64_t ATTN_JOIN_BLOCKS = 1 << 17;

// Rows per run and key head, the batch's mean, above which keys of shared prefixes go through LDS (the host does not know how sequences share
// out over runs, and the sums are alike up to their last bits either way).  us in registers and through LDS, by rows: 16 heads of 128 behind 4000
// keys 12: 16.6 and 19.1, 16: 17.1 and 19.2, 17: 20.8 and 19.3, 24: 21.5 and 19.8, 64: 30.5 and 23.9, 256: 74 and 46; 16 heads of 64 behind 16000
// 16: 22.1 and 27.6, 24: 24.8 and 27.8, 40: 30.6 and 28.9, 64: 40 and 31.
// The blocks of 128 rows that its parts make at most: one to a CU, beside the sequences' own keys, with heads of 64 two.  131 sequences of 32 / 8
// heads of 128 behind 8000 keys with up to 500 each, in 3, 4, 5, 6, 7 parts: 89, 74, 66, 63, 73 us; 128 of 16 heads of 64 behind 16000 with 100 each,
// at most 256 and 512 blocks: 54 and 37.
constexpr int ATTN_PREFIX_ROWS = 16;
constexpr int attn_prefix_blocks(int D) { return D == 64 ? 512 : 256; }
// Own keys by waves (attn_shared.hip): parts of 8 tiles, where no sequence has more than two and there are enough of them.
constexpr int ATTN_WAVE_TILES = 8, ATTN_WAVE_MOST = 16, ATTN_WAVE_SETS = 768;
constexpr int64_t ATTN_MOST_RUNS = 1 << 20;

// A grid's threads are counted in 32 bits.
constexpr int64_t ATTN_MOST_BLOCKS = 1ll << 24;

static inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Parts that up to `tiles` key tiles are cut into where there are `blocks` blocks without a cut: as many as make `target`
// blocks, of `least` tiles or more.
static inline int64_t attn_parts(int64_t blocks, int64_t tiles, int target, int least) {
    int64_t n = ceil_div(target, blocks);
    if (n > ceil_div(tiles, least)) n = ceil_div(tiles, least);
    return n < 1 ? 1 : n;
}
static inline void attn_split(AttnCall &a, int64_t tiles, int64_t parts) {
    const int64_t each = ceil_div(tiles > 0 ? tiles : 1, parts);
    a.split_tiles = (int)each;
    a.splits = (int)ceil_div(tiles > 0 ? tiles : 1, each);
}

// Key tiles of KT that `rows` queries in a row can look at, of a sequence of up to max_len keys.
static inline int64_t attn_max_tiles(const AttnCall &a, int KT, int64_t rows, int64_t max_len) {
    const int64_t all = ceil_div(max_len, KT);
    if (!a.window) return all;
    const int64_t near = ceil_div((int64_t)a.window + rows - 1, KT) + 1 + ceil_div(a.sinks, KT);
    return near < all ? near : all;
}

}  // namespace c2r
