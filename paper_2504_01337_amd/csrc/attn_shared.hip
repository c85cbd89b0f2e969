// Attention of one new token per sequence where runs of sequences begin with the same keys: those are read once for a run, as far as 16
// rows go, and not once for a sequence.  The rows of a block are either (sequence, query head) pairs of one run and one key head, against
// a part of the run's keys, or the query heads of one sequence that share a key head, against a part of the keys behind.  All
// results are partial, and joined.  Prefixes in bf16 that many rows look at go through LDS in blocks of 128 rows (attn_tile.h), in the same launch.
// Bound by memory: 64 sequences behind five prefixes of up to 4000 with up to 2000 keys each, 16 heads 132 us (5.4 TB/s), joined in 5; four behind 2000 9
// and 4, latency.  131 sequences of 32 / 8 heads behind 8000 keys with up to 500 each: 56 and 6; the prefix's blocks alone take 47.5, the others 37.
#include "attn_stream.h"
#include "attn_tile.h"

namespace c2r {

template <int D>
struct SharedLds {
    float o[4 * 16 * D], ml[4 * 16 * 2];
};

template <bool BF16, int D>
__device__ __forceinline__ void attn_shared_block(const AttnCall &a, uint32_t id, uint32_t prefix_grid, SharedLds<D> &lds) {
    using S = Stream<BF16, D>;
    constexpr int SZ = S::SZ, KT = S::KT;
    float *const join_o = lds.o, *const join_ml = lds.ml;
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, n = lane & 15;
    // blocks: those of the prefixes, then those of the sequences; parts of the keys fastest, then key heads, rows
    int b, kv_head, row0, left, part, splits, split_tiles;
    KeyRange keys;
    const bool prefix = id < prefix_grid;
    if (prefix) {
        splits = a.prefix_splits, split_tiles = a.prefix_tiles;
        part = (int)(id % splits);
        id /= splits;
        kv_head = (int)(id % a.kv.kv_heads);
        AttnCall::Run run;
        int rb, rows;
        if (!a.prefix_block_of<16>((int)(id / a.kv.kv_heads), run, rb, rows)) return;
        b = run.first, keys.to = run.keys;
        row0 = rb * 16, left = min(rows - row0, 16);
    } else {
        id -= prefix_grid;
        splits = a.splits - a.prefix_splits, split_tiles = a.split_tiles;
        part = (int)(id % splits);
        id /= splits;
        const int col_sets = (a.group + 15) / 16;
        row0 = (int)(id % col_sets) * 16, left = min(a.group - row0, 16);
        id /= col_sets;
        kv_head = (int)(id % a.kv.kv_heads);
        b = (int)(id / a.kv.kv_heads);
        keys.from = a.prefix_of(b);
    }
    // row r: a sequence and a head
    auto sequence = [&](int r) { return b + r / a.group; };
    auto head_of = [&](int r) { return kv_head * a.group + r % a.group; };
    auto place = [&](int r, int in) { return ((int64_t)in * a.kv.batch + sequence(r)) * a.heads + head_of(r); };
    auto put_empty = [&](int r, int in) {
        float *ml = a.part_ml + place(r, in) * 2;
        ml[0] = -__builtin_inff(), ml[1] = PART_EMPTY;
    };
    if (!prefix && part == 0 && keys.from == 0)  // (no block has a prefix of these)
        for (int i = threadIdx.x; i < left * a.prefix_splits; i += 256) put_empty(row0 + i % left, i / left);
    const int here = part + (prefix ? 0 : a.prefix_splits);
    const int row = row0 + min(n, left - 1), p = a.kv.tokens(sequence(row)) - 1;
    int p_min = p, p_max = p;
#pragma unroll
    for (int w = 8; w; w >>= 1) p_min = min(p_min, __shfl_xor(p_min, w)), p_max = max(p_max, __shfl_xor(p_max, w));
    p_min = __builtin_amdgcn_readfirstlane(p_min), p_max = __builtin_amdgcn_readfirstlane(p_max);
    const KeyTiles<KT> tiles(a, p_min, p_max, keys);
    int x0, x1;
    tiles.part(splits, split_tiles, part, x0, x1);
    if (x0 == x1) {
        if (threadIdx.x < (uint32_t)left) put_empty(row0 + threadIdx.x, here);
        return;
    }
    auto q_row = [&](int r) { return a.q + sequence(r) * a.q_bytes + (int64_t)head_of(r) * (D * SZ); };
    u32x4 q[S::KSTEPS];
    const unsigned char *mine_q = q_row(row);
#pragma unroll
    for (int c = 0; c < S::KSTEPS; ++c) q[c] = *reinterpret_cast<const u32x4 *>(mine_q + c * 64 + g * 16);
    typename S::State st;
    S::clear(st);
    S::template run<4>(a, q, st, tiles, x0 + wave, x1, b, kv_head * a.kv.head_bytes, p, p_min, p_max, keys);
    uint32_t redo = S::finish(st, left);
    float *mine = join_o + wave * 16 * D;
    if (n < left && !(redo >> n & 1)) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int e = 0; e < S::VEL; ++e) mine[n * D + (g * 4 + r) * S::VEL + e] = st.o[e][r];
        if (g == 0) join_ml[(wave * 16 + n) * 2] = st.m, join_ml[(wave * 16 + n) * 2 + 1] = st.l;
    }
    while (redo) {
        const int col = __ffs(redo) - 1;
        redo &= redo - 1;
        float m, l, o[D / 64];
        exact_row<BF16, D, KT>(a, tiles, x0 + wave, x1, 4, b, kv_head, a.kv.tokens(sequence(row0 + col)) - 1, q_row(row0 + col), m, l, o, keys);
#pragma unroll
        for (int e = 0; e < D / 64; ++e) mine[col * D + lane * (D / 64) + e] = o[e];
        if (lane == 0) join_ml[(wave * 16 + col) * 2] = m, join_ml[(wave * 16 + col) * 2 + 1] = l;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < left * (D / 4); i += 256) {
        const int col = i / (D / 4), d = i % (D / 4) * 4;
        float m4[4], M = -__builtin_inff(), l = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) m4[w] = join_ml[(w * 16 + col) * 2], M = fmaxf(M, m4[w]);
        const float ref = reference_of(M);
        f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = __builtin_amdgcn_exp2f(m4[w] - ref);
            l = __builtin_fmaf(f, join_ml[(w * 16 + col) * 2 + 1], l);
            const f32x4 o = *reinterpret_cast<const f32x4 *>(join_o + (w * 16 + col) * D + d);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] = __builtin_fmaf(f, o[e], sum[e]);
        }
        const int64_t at = place(row0 + col, here);
        *reinterpret_cast<f32x4 *>(a.part_o + at * D + d) = sum;
        if (d == 0) a.part_ml[at * 2] = M, a.part_ml[at * 2 + 1] = a.blind(a.kv.tokens(sequence(row0 + col)) - 1) ? PART_EMPTY : l;
    }
}

// The keys that one sequence has behind its prefix, by one wave for the query heads of a key head: many sequences with few keys each, where four
// waves with a few tiles each mostly wait for where their keys are.  256 sequences with up to 100 keys each behind 2000, 16 heads: a call 63 -> 50
// us; 131 with up to 500 behind 8000, 32 / 8 heads: 63 -> 62; 256 with up to 700 behind 3000: 102 -> 109, so only short ones.
template <bool BF16, int D>
__device__ __forceinline__ void attn_own_wave(const AttnCall &a, uint32_t id) {
    using S = Stream<BF16, D>;
    constexpr int SZ = S::SZ, KT = S::KT;
    const int lane = lane_id(), g = lane >> 4, n = lane & 15, splits = a.splits - a.prefix_splits, col_sets = (a.group + 15) / 16;
    const int part = (int)(id % splits);
    id /= splits;
    const int row0 = (int)(id % col_sets) * 16, left = min(a.group - row0, 16);
    id /= col_sets;
    const int kv_head = (int)(id % a.kv.kv_heads), b = (int)(id / a.kv.kv_heads);
    if (b >= a.kv.batch) return;
    const int p = a.kv.tokens(b) - 1, head0 = kv_head * a.group + row0;
    KeyRange keys;
    keys.from = a.prefix_of(b);
    auto place = [&](int col, int in) { return ((int64_t)in * a.kv.batch + b) * a.heads + head0 + col; };
    auto put_empty = [&](int col, int in) {
        float *ml = a.part_ml + place(col, in) * 2;
        ml[0] = -__builtin_inff(), ml[1] = PART_EMPTY;
    };
    if (part == 0 && keys.from == 0)  // (no block has a prefix of these)
        for (int i = lane; i < left * a.prefix_splits; i += 64) put_empty(i % left, i / left);
    const int here = part + a.prefix_splits;
    const KeyTiles<KT> tiles(a, p, p, keys);
    int x0, x1;
    tiles.part(splits, a.split_tiles, part, x0, x1);
    if (x0 == x1) {
        if (lane < left) put_empty(lane, here);
        return;
    }
    const unsigned char *q_rows = a.q + b * a.q_bytes + (int64_t)head0 * (D * SZ);
    u32x4 q[S::KSTEPS];
#pragma unroll
    for (int c = 0; c < S::KSTEPS; ++c) q[c] = *reinterpret_cast<const u32x4 *>(q_rows + min(n, left - 1) * (D * SZ) + c * 64 + g * 16);
    typename S::State st;
    S::clear(st);
    S::template run<1>(a, q, st, tiles, x0, x1, b, kv_head * a.kv.head_bytes, p, p, p, keys);
    uint32_t redo = S::finish(st, left);
    if (n < left && !(redo >> n & 1)) {
        float *o = a.part_o + place(n, here) * D + g * 4 * S::VEL;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int e = 0; e < S::VEL; e += 4) *reinterpret_cast<f32x4 *>(o + r * S::VEL + e) = f32x4{st.o[e][r], st.o[e + 1][r], st.o[e + 2][r], st.o[e + 3][r]};
        if (g == 0) a.part_ml[place(n, here) * 2] = st.m, a.part_ml[place(n, here) * 2 + 1] = a.blind(p) ? PART_EMPTY : st.l;
    }
    while (redo) {
        const int col = __ffs(redo) - 1;
        redo &= redo - 1;
        float m, l, o[D / 64];
        exact_row<BF16, D, KT>(a, tiles, x0, x1, 1, b, kv_head, p, q_rows + col * (D * SZ), m, l, o, keys);
#pragma unroll
        for (int e = 0; e < D / 64; ++e) a.part_o[place(col, here) * D + lane * (D / 64) + e] = o[e];
        if (lane == 0) a.part_ml[place(col, here) * 2] = m, a.part_ml[place(col, here) * 2 + 1] = a.blind(p) ? PART_EMPTY : l;
    }
}

template <bool BF16, int D>
__global__ __launch_bounds__(256, D == 128 ? 3 : 4) void attn_shared_kernel(AttnCall a, uint32_t prefix_grid) {
    __shared__ __align__(16) SharedLds<D> lds;
    if (a.own_by_wave && blockIdx.x >= prefix_grid) attn_own_wave<BF16, D>(a, (blockIdx.x - prefix_grid) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
    else attn_shared_block<BF16, D>(a, blockIdx.x, prefix_grid, lds);
}

// Prefixes whose keys go through LDS, and the sequences' own keys: the first are bound by the matrix pipe, the others by memory, and side by
// side on a CU they take little more than the longer of the two.  The prefixes' blocks are first, one to a CU (heads of 64: two).  Four blocks to a CU
// would be 128 registers, which heads of 64 do not fit (142; up to 20 of them through memory): 24 sequences of 16 heads behind 4000 keys 17.8 us for
// 16.8, 128 24.1 for 21.7.
template <int D, bool ALIGNED, bool ANY_SCALE>
__global__ __launch_bounds__(256, D == 128 ? 2 : 3) void attn_shared_tile_kernel(AttnCall a, uint32_t prefix_grid) {
    __shared__ __align__(1024) union {
        TileLds<D> tile;
        SharedLds<D> own;
    } lds;
    if (blockIdx.x < prefix_grid) attn_tile_block<D, ALIGNED, ANY_SCALE, true>(a, blockIdx.x, lds.tile);
    else if (a.own_by_wave) attn_own_wave<true, D>(a, (blockIdx.x - prefix_grid) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
    else attn_shared_block<true, D>(a, blockIdx.x - prefix_grid, 0, lds.own);
}

int launch_attn_shared(const AttnCall &a, bool bf16, bool tiled, int D, hipStream_t st) {
    const uint32_t prefix = (uint32_t)((int64_t)a.prefix_blocks * a.kv.kv_heads * a.prefix_splits);
    const int64_t own = (int64_t)(a.splits - a.prefix_splits) * a.kv.kv_heads * ((a.group + 15) / 16) * a.kv.batch;
    const dim3 grid(prefix + (unsigned)(a.own_by_wave ? ceil_div(own, 4) : own)), block(256);
    const bool aligned = tile_aligned(a.kv);
    if (tiled && !(a.scale_log2 > 0.0f)) {
        if (D == 128) attn_shared_tile_kernel<128, false, true><<<grid, block, 0, st>>>(a, prefix);
        else attn_shared_tile_kernel<64, false, true><<<grid, block, 0, st>>>(a, prefix);
    } else if (tiled) {
        if (D == 128) aligned ? attn_shared_tile_kernel<128, true, false><<<grid, block, 0, st>>>(a, prefix) : attn_shared_tile_kernel<128, false, false><<<grid, block, 0, st>>>(a, prefix);
        else aligned ? attn_shared_tile_kernel<64, true, false><<<grid, block, 0, st>>>(a, prefix) : attn_shared_tile_kernel<64, false, false><<<grid, block, 0, st>>>(a, prefix);
    } else if (bf16) {
        if (D == 128) attn_shared_kernel<true, 128><<<grid, block, 0, st>>>(a, prefix);
        else attn_shared_kernel<true, 64><<<grid, block, 0, st>>>(a, prefix);
    } else {
        if (D == 128) attn_shared_kernel<false, 128><<<grid, block, 0, st>>>(a, prefix);
        else attn_shared_kernel<false, 64><<<grid, block, 0, st>>>(a, prefix);
    }
    const int rc = launch_status();
    return rc == C2R_OK ? launch_attn_join(a, bf16, D, st) : rc;
}

}  // namespace c2r
