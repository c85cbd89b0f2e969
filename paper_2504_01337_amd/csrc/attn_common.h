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
    // The last key that is cached of those up to position p.
    __device__ __forceinline__ int last_key(int p) const { return min(p, kv.capacity - 1); }
    // Whether the query at position p sees key j; whether it sees none.
    __device__ __forceinline__ bool sees(int p, int j) const { return j <= last_key(p) && (!window || j > p - window || j < sinks); }
    __device__ __forceinline__ bool blind(int p) const { return p < 0 || (window && !sinks && p - window >= kv.capacity - 1); }
};

// The key tiles (KT keys, aligned) that queries at positions p_min .. p_max look at: those of the first `sinks` keys that lie
// before the window, then the window's.
template <int KT>
struct KeyTiles {
    int sink_tiles, first, count;
    __device__ __forceinline__ KeyTiles(const AttnCall &a, int p_min, int p_max) {
        sink_tiles = first = 0;
        if (a.window) {
            const int lo = p_min - a.window + 1;
            first = lo > 0 ? lo / KT : 0;
            const int s = (int)(((int64_t)a.sinks + KT - 1) / KT);
            sink_tiles = s < first ? s : first;
        }
        const int last = a.last_key(p_max);  // (a window that begins past the cache's end leaves the sinks)
        count = last < 0 ? 0 : sink_tiles + max(last / KT - first + 1, 0);
    }
    __device__ __forceinline__ int base(int x) const { return (x < sink_tiles ? x : first + x - sink_tiles) * KT; }
    // [x0, x1): the part of split s.  The last one takes what is left, however long a sequence is.
    __device__ __forceinline__ void part(const AttnCall &a, int s, int &x0, int &x1) const {
        const int64_t lo = (int64_t)s * a.split_tiles, hi = s + 1 == a.splits ? count : lo + a.split_tiles;
        x0 = lo < count ? (int)lo : count;
        x1 = hi < count ? (int)hi : count;
    }
    // Whether split 0 has all of them: it then writes the result itself and says so to the join (PART_DONE).
    __device__ __forceinline__ bool uncut(const AttnCall &a) const { return a.splits == 1 || count <= a.split_tiles; }
};

// A tile [base, base + KT) that every query of p_min .. p_max sees whole.
template <int KT>
__device__ __forceinline__ bool tile_whole(const AttnCall &a, int base, int p_min, int p_max) {
    return base + KT - 1 <= a.last_key(p_min) && (!a.window || base > p_max - a.window || base + KT <= a.sinks);
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
                                          int p, const unsigned char *q_row, float &m_out, float &l_out, float (&o)[D / 64]) {
    constexpr int N = D / 64;
    const int lane = lane_id();
    float m = -__builtin_inff(), l = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = 0.0f;
    for (int x = x0; x < x1; x += step) {
        const int j = tiles.base(x) + lane;
        const bool see = lane < KT && a.sees(p, j);
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
