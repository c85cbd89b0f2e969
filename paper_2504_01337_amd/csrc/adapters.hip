// Low-rank adapters of many requests beside a projection that they share: for every row t with an adapter a
//     out[t] = y[t] + c_a B_a (A_a x[t])
// Rows are put in order of their adapters and cut into tiles of up to 16 MG rows of one adapter, so that an adapter's weights are
// read once per tile.  Two products on the matrix pipe: h = A_a x (contraction d_in, a block's waves share it out and add up
// through LDS, blocks share it out where there are few) and B_a h (contraction r), with y added in 32 bits and one rounding.
// h stays in 32 bits: bf16 takes it in two pieces, the rounded number and what is left of it.
// Bound by memory: x, y, out and the adapters in use.  8192 rows in e4m3, 2048 to 6144, rank 16: 55 us of a call (219 MB: 4.0 TB/s), of which the second
// product 40, the first 8.7, the order of the rows 7; 131 rows, 4096 to 6144, 20 adapters of rank 64: 15 (30 MB), of which 8.6 and 7; one row 5.7 and
// 4, a launch and a chain of dependent loads each.  fp32: 8192 rows 106 us (472 MB: 4.5 TB/s), 131 rows 23.
#include "ffn_copy.h"

namespace c2r {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int AD_MOST_ADAPTERS = 1024, AD_MOST_RANK = 128;
constexpr float BF16_MOST = 3.3895313892515355e38f;  // (2 - 2^-7) 2^127

// What x holds: the weights' type, or e4m3 with a scale for every row beside bf16 weights.
enum { AD_F32 = 0, AD_BF16 = 1, AD_E4M3 = 2 };

// Rows are in slots, tile_rows of them to a tile, so that what a block reads first follows from its number alone.
struct AdapterTile {
    int adapter, rows;  // -1: rows without one, -2: no tile
};

struct AdapterCall {
    const unsigned char *x, *A, *B, *y;
    unsigned char *out;
    const int32_t *adapter;
    const float *x_scale, *scale;
    int64_t x_bytes, y_bytes, out_bytes;
    int T, E, r, d_in, d_out, tile_rows, ranks16, parts, max_tiles;
    bool in_blocks;     // the first product's blocks work the order out
    bool copy_rest;     // rows without an adapter are copied
    AdapterTile *tiles;
    int *slots;         // the row in every slot of a tile's rows
    float *h;           // [parts][slots][16 ranks16]
};

// ---- the order of the rows ----

// One block: counts, tiles and slots of every adapter.
__global__ __launch_bounds__(1024) void adapter_order_kernel(AdapterCall a) {
    __shared__ int next[AD_MOST_ADAPTERS + 1], rows_of[AD_MOST_ADAPTERS], tiles_of[16];
    const int tid = threadIdx.x;
    // rows' ids come in batches; the first batch's stay
    constexpr int BATCH = 8;
    int held[BATCH];
    auto load = [&](int t0, int (&ids)[BATCH]) {
#pragma unroll
        for (int i = 0; i < BATCH; ++i) ids[i] = t0 + i * 1024 < a.T ? a.adapter[t0 + i * 1024] : 0;
    };
    auto group = [&](int e) { return (uint32_t)e < (uint32_t)a.E ? e : a.E; };
    load(tid, held);
    for (int i = tid; i <= a.E; i += 1024) next[i] = 0;
    __syncthreads();
    // lanes of a wave mostly have rows of one request: they are counted with one addition
    auto take = [&](int g) {
        const int first = __builtin_amdgcn_readfirstlane(g);
        if (__all(g == first)) {
            const uint64_t here = __ballot(true);
            int at = 0;
            if (lane_id() == __ffsll((unsigned long long)here) - 1) at = atomicAdd(&next[first], __popcll(here));
            return __builtin_amdgcn_readfirstlane(at) + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(here >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)here, 0));
        }
        return atomicAdd(&next[g], 1);
    };
    // (of one batch the places stay, too: counted from 0 here)
    int place[BATCH];
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
        held[i] = group(held[i]), place[i] = 0;
        if (tid + i * 1024 < a.T) place[i] = take(held[i]);
    }
    for (int t0 = tid + BATCH * 1024; t0 < a.T; t0 += BATCH * 1024) {
        int ids[BATCH];
        load(t0, ids);
#pragma unroll
        for (int i = 0; i < BATCH; ++i)
            if (t0 + i * 1024 < a.T) take(group(ids[i]));
    }
    __syncthreads();
    const int mine = tid < a.E ? next[tid] : 0, tiles = (mine + a.tile_rows - 1) / a.tile_rows, rest = a.copy_rest ? next[a.E] : 0;
    const int upto = wave_inclusive_scan(tiles);
    if (lane_id() == 63) tiles_of[tid >> 6] = upto;
    __syncthreads();
    int tile = upto - tiles, with_one = 0;
    for (int w = 0; w < 16; ++w) {
        if (w < tid >> 6) tile += tiles_of[w];
        with_one += tiles_of[w];
    }
    const int rest_tiles = (rest + a.tile_rows - 1) / a.tile_rows;
    if (tid < a.E) next[tid] = tile * a.tile_rows, rows_of[tid] = mine;
    if (tid == 1023) next[a.E] = with_one * a.tile_rows;  // (E is 1024 at most: no other thread's)
    __syncthreads();
    for (int i = tid; i < a.max_tiles; i += 1024) {
        AdapterTile t = {-2, 0};
        if (i < with_one) {
            int lo = 0, hi = a.E - 1;  // the last adapter whose slots begin at or before the tile's and that has any rows
            while (lo < hi) {
                const int mid = (lo + hi + 1) / 2;
                if (next[mid] <= i * a.tile_rows) lo = mid;
                else hi = mid - 1;
            }
            t = {lo, min(rows_of[lo] - (i * a.tile_rows - next[lo]), a.tile_rows)};
        } else if (i < with_one + rest_tiles) {
            t = {-1, min(rest - (i - with_one) * a.tile_rows, a.tile_rows)};
        }
        a.tiles[i] = t;
    }
    if (a.T <= BATCH * 1024) {
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int t = tid + i * 1024;
            if (t < a.T && (held[i] < a.E || a.copy_rest)) a.slots[next[held[i]] + place[i]] = t;
        }
        return;
    }
    __syncthreads();  // (the tiles have been described: from here on next[] moves)
    for (int t0 = tid; t0 < a.T; t0 += BATCH * 1024) {
        load(t0, held);
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int t = t0 + i * 1024, g = group(held[i]);
            if (t < a.T && (g < a.E || a.copy_rest)) a.slots[take(g)] = t;
        }
    }
}

// Every block of the first product works its tile out itself where that is less work than a launch of one block ahead of it: 131 rows 17 -> 15 us
// of a call.  A row's place among those of its adapter is that of its number.  here[]: the rows in places
// in_tile .. + slots of the tile.  lds: 1024 + 1 + 8 words.
constexpr int AD_FEW_ROWS = 256;
__device__ __forceinline__ AdapterTile few_rows_tile(const AdapterCall &a, int at, int in_tile, int slots, int *here, int *lds) {
    int *const count = lds, *const upto = lds + AD_MOST_ADAPTERS + 1, *const found = upto + 4;
    const int tid = threadIdx.x, wave = tid >> 6;
    const int e = tid < a.T ? a.adapter[tid] : 0, mine = tid >= a.T ? -1 : (uint32_t)e < (uint32_t)a.E ? e : a.E;
    for (int i = tid; i <= a.E; i += 256) count[i] = 0;
    if (tid < slots) here[tid] = -1;
    if (tid == 0) found[0] = -1;
    __syncthreads();
    if (mine >= 0) atomicAdd(&count[mine], 1);
    __syncthreads();
    // four adapters to a thread, and the rows without one behind them
    int tiles = 0;
    auto tiles_of = [&](int i) { return (count[i] + a.tile_rows - 1) / a.tile_rows; };
    for (int i = tid * 4; i < min(tid * 4 + 4, a.E); ++i) tiles += tiles_of(i);
    const int sum = wave_inclusive_scan(tiles);
    if (lane_id() == 63) upto[wave] = sum;
    __syncthreads();
    int first = sum - tiles, all = 0;
    for (int w = 0; w < 4; ++w) first += w < wave ? upto[w] : 0, all += upto[w];
    if (at >= first && at < first + tiles) {
        int i = tid * 4;
        for (; at >= first + tiles_of(i); ++i) first += tiles_of(i);
        found[0] = i, found[1] = at - first;
    } else if (tid == 0 && a.copy_rest && at >= all && at < all + tiles_of(a.E)) {
        found[0] = a.E, found[1] = at - all;
    }
    __syncthreads();
    const int group = found[0];
    if (group < 0) return AdapterTile{-2, 0};
    const uint64_t same = __ballot(mine == group);
    if (lane_id() == 0) upto[wave] = __popcll(same);
    __syncthreads();
    int rank = (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(same >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)same, 0));
    for (int w = 0; w < wave; ++w) rank += upto[w];
    rank -= found[1] * a.tile_rows + in_tile;
    if (mine == group && rank >= 0 && rank < slots) here[rank] = tid;
    const AdapterTile tile = {group < a.E ? group : -1, min(count[group] - found[1] * a.tile_rows, a.tile_rows)};
    __syncthreads();
    return tile;
}

// The same for up to eight times as many rows, of up to 255 adapters: a wave has a quarter of the rows, and counts of its own.  (8192 rows that
// way took 66 us of a call where the block ahead takes 59.)
constexpr int AD_SOME_ROWS = 2048, AD_SOME_ADAPTERS = 255;
__device__ __forceinline__ AdapterTile some_rows_tile(const AdapterCall &a, int at, int in_tile, int slots, int *here, int *lds) {
    constexpr int EACH = AD_SOME_ROWS / 256;  // rows of a thread
    int *const count = lds, *const upto = lds + 4 * (AD_SOME_ADAPTERS + 1), *const found = upto + 4;
    const int tid = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid >> 6), groups = a.E + 1;
    const int r0 = wave * (EACH * 64) + lane;
    int g[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) g[i] = r0 + i * 64 < a.T ? a.adapter[r0 + i * 64] : 0;
    for (int i = tid; i < 4 * groups; i += 256) count[i] = 0;
    if (tid < slots) here[tid] = -1;
    if (tid == 0) found[0] = -1;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        g[i] = r0 + i * 64 >= a.T ? -1 : (uint32_t)g[i] < (uint32_t)a.E ? g[i] : a.E;
        const int first = __builtin_amdgcn_readfirstlane(g[i]);
        if (__all(g[i] == first || g[i] < 0)) {  // (mostly rows of one request)
            const int n = __popcll(__ballot(g[i] >= 0));
            if (lane == 0 && n) atomicAdd(&count[wave * groups + first], n);
        } else if (g[i] >= 0) {
            atomicAdd(&count[wave * groups + g[i]], 1);
        }
    }
    __syncthreads();
    auto rows_of = [&](int g) { return count[g] + count[groups + g] + (count[2 * groups + g] + count[3 * groups + g]); };
    const int tiles = tid < a.E ? (rows_of(tid) + a.tile_rows - 1) / a.tile_rows : 0, sum = wave_inclusive_scan(tiles);
    if (lane == 63) upto[wave] = sum;
    __syncthreads();
    int first = sum - tiles, all = 0;
    for (int w = 0; w < 4; ++w) first += w < wave ? upto[w] : 0, all += upto[w];
    if (at >= first && at < first + tiles) found[0] = tid, found[1] = at - first;
    else if (tid == 255 && a.copy_rest && at >= all && at < all + (rows_of(a.E) + a.tile_rows - 1) / a.tile_rows) found[0] = a.E, found[1] = at - all;
    __syncthreads();
    const int group = found[0];
    if (group < 0) return AdapterTile{-2, 0};
    const int from = found[1] * a.tile_rows + in_tile;
    int rank = 0;
    for (int w = 0; w < wave; ++w) rank += count[w * groups + group];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const uint64_t same = __ballot(g[i] == group);
        const int mine = rank - from + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(same >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)same, 0));
        if (g[i] == group && mine >= 0 && mine < slots) here[mine] = r0 + i * 64;
        rank += __popcll(same);
    }
    const AdapterTile tile = {group < a.E ? group : -1, min(rows_of(group) - found[1] * a.tile_rows, a.tile_rows)};
    __syncthreads();
    return tile;
}
static bool rows_in_blocks(int64_t T, int E) { return T <= AD_FEW_ROWS || (T <= AD_SOME_ROWS && E <= AD_SOME_ADAPTERS); }

// ---- h = A x ----

// 16 rows x 256 bytes of the weights' type, and the 16 rows x as many elements of x: loads in which 16 (8) neighbouring lanes are in one row, which
// costs the memory pipe a quarter of what a lane for a row does (an address at a time; 8192 rows 14 us), then through LDS to where the matrix
// instructions want them.  Lane l loads row 4 i + l / 16 (e4m3: 8 i + l / 8), 16-byte piece l % 16 (l % 8); lane (g, n) gets pieces 4 j + g of row n.
// A wave's own LDS, whose accesses keep their order: nobody waits.  Piece p of row r stands at p ^ r, so that neither side meets on a bank.
template <int X>
struct Strip {
    static constexpr int PER_ROW = X == AD_E4M3 ? 8 : 16, LOADS = PER_ROW / 4, ROWS = 64 / PER_ROW, PIECE = X == AD_F32 ? 4 : X == AD_BF16 ? 8 : 16;
    u32x4 w[LOADS];
    // row(r): where row r begins; elements from `at` on, of which `left` (a multiple of 8, or none) are in the row
    template <class Rows>
    __device__ __forceinline__ void load(const Rows &row, int at, int left) {
        const int piece = lane_id() % PER_ROW * PIECE;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const unsigned char *from = row(i) + (int64_t)(at + piece) * 16 / PIECE;
            w[i] = u32x4{0, 0, 0, 0};
            if constexpr (X == AD_E4M3) {  // (rows of whole 8 bytes)
                typedef u32x4 half_aligned __attribute__((aligned(8)));
                if (left > piece + 8) {
                    w[i] = *reinterpret_cast<const half_aligned *>(from);
                } else if (left > piece) {
                    const u32x2 lo = *reinterpret_cast<const u32x2 *>(from);
                    w[i][0] = lo[0], w[i][1] = lo[1];
                }
            } else {
                if (left > piece) w[i] = *reinterpret_cast<const u32x4 *>(from);
            }
        }
    }
    __device__ __forceinline__ void hand_on(unsigned char *lds, u32x4 (&to)[4]) const {
        const int lane = lane_id(), g = lane >> 4, n = lane & 15;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int r = i * ROWS + lane / PER_ROW;
            *reinterpret_cast<u32x4 *>(lds + (r * PER_ROW + (lane % PER_ROW ^ r % PER_ROW)) * 16) = w[i];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (X == AD_E4M3) {  // 8 bytes; every e4m3 number is a bf16 one
                const u32x2 v = *reinterpret_cast<const u32x2 *>(lds + (n * PER_ROW + ((j * 2 + (g >> 1)) ^ n % PER_ROW)) * 16 + (g & 1) * 8);
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(v[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(v[i], true);
                    to[j][2 * i] = pack_bf16x2(lo[0], lo[1]), to[j][2 * i + 1] = pack_bf16x2(hi[0], hi[1]);
                }
#endif
            } else {
                to[j] = *reinterpret_cast<const u32x4 *>(lds + (n * PER_ROW + ((j * 4 + g) ^ n)) * 16);
            }
        }
    }
};

template <bool BF16>
__device__ __forceinline__ f32x4 multiply(const u32x4 &a, const u32x4 &b, f32x4 c) {
#if defined(__HIP_DEVICE_COMPILE__)
    if constexpr (BF16) {
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
    }
#endif
    return c;
}

// Blocks: parts of d_in fastest, then 16 RG ranks, then 16 rows of a tile.  A wave's step is 256 bytes of every rank's row (128 elements of d_in,
// 64 in fp32), and its products leave lane (g, n) with ranks 4 g .. of row n.  (32 or 64 rows to a block read the weights less often, and have fewer
// loads in flight: 8192 rows of rank 64 75 us of a call, 80 and 97; 4096 to 4096 of rank 128 101, 98, 119.)
template <int X, int RG>
__global__ __launch_bounds__(256) void adapter_down_kernel(AdapterCall a) {
    constexpr bool BF16 = X != AD_F32;
    constexpr int W = BF16 ? AD_BF16 : AD_F32, WS = BF16 ? 2 : 4, STEP = 256 / WS;
    __shared__ __align__(16) unsigned char strips[4][4096];
    __shared__ f32x4 sums[RG == 1 ? 5 : 4][RG][64];  // (also few_rows_tile's)
    static_assert(sizeof(sums) >= (AD_MOST_ADAPTERS + 1 + 8) * 4, "room for few_rows_tile");
    __shared__ int here[16];  // the rows of these slots
    const int chunks = (a.ranks16 + RG - 1) / RG, part = blockIdx.x % a.parts, id = blockIdx.x / a.parts, chunk = id % chunks, rows_at = id / chunks;
    const int slot0 = rows_at * 16, in_tile = slot0 % a.tile_rows;
    const int lane = lane_id(), wave = threadIdx.x >> 6;
    AdapterTile tile;
    if (a.in_blocks) {
        int *const lds = reinterpret_cast<int *>(sums);
        tile = a.T <= AD_FEW_ROWS ? few_rows_tile(a, slot0 / a.tile_rows, in_tile, 16, here, lds) : some_rows_tile(a, slot0 / a.tile_rows, in_tile, 16, here, lds);
        if (part == 0 && chunk == 0) {  // for the second product
            if (threadIdx.x < 16) a.slots[slot0 + threadIdx.x] = here[threadIdx.x];
            if (threadIdx.x == 0 && in_tile == 0) a.tiles[slot0 / a.tile_rows] = tile;
        }
    } else {
        tile = a.tiles[slot0 / a.tile_rows];
        if (threadIdx.x < 16) here[threadIdx.x] = in_tile + (int)threadIdx.x < tile.rows ? a.slots[slot0 + threadIdx.x] : -1;
        __syncthreads();
    }
    const int left = tile.rows - in_tile;
    if (tile.adapter < 0 || left <= 0) return;
    const unsigned char *x_row[Strip<X>::LOADS], *a_row[RG][4];
#pragma unroll
    for (int i = 0; i < Strip<X>::LOADS; ++i)  // (an empty slot goes along with row 0)
        x_row[i] = a.x + (int64_t)max(here[i * Strip<X>::ROWS + lane / Strip<X>::PER_ROW], 0) * a.x_bytes;
#pragma unroll
    for (int q = 0; q < RG; ++q)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            a_row[q][i] = a.A + ((int64_t)tile.adapter * a.r + min((chunk * RG + q) * 16 + i * 4 + lane / 16, a.r - 1)) * ((int64_t)a.d_in * WS);
    f32x4 acc[RG];
#pragma unroll
    for (int q = 0; q < RG; ++q) acc[q] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int steps = (a.d_in + STEP - 1) / STEP, each = (steps + a.parts - 1) / a.parts;
    const int s1 = min((part + 1) * each, steps);
    // (DEPTH steps are asked for together)
    constexpr int DEPTH = RG == 1 ? 4 : 2;
    for (int s = part * each + wave; s < s1; s += 4 * DEPTH) {
        Strip<X> xs[DEPTH];
        Strip<W> as[DEPTH][RG];
#pragma unroll
        for (int i = 0; i < DEPTH; ++i) {
            const int k = (s + 4 * i) * STEP, in = s + 4 * i < s1 ? a.d_in - k : 0;
#pragma unroll
            for (int q = 0; q < RG; ++q) as[i][q].load([&](int l) { return a_row[q][l]; }, k, chunk * RG + q < a.ranks16 ? in : 0);
            xs[i].load([&](int l) { return x_row[l]; }, k, in);
        }
#pragma unroll
        for (int i = 0; i < DEPTH; ++i) {
            u32x4 xv[4];
            xs[i].hand_on(strips[wave], xv);
#pragma unroll
            for (int q = 0; q < RG; ++q) {
                u32x4 av[4];
                as[i][q].hand_on(strips[wave], av);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[q] = multiply<BF16>(av[j], xv[j], acc[q]);
            }
        }
    }
#pragma unroll
    for (int q = 0; q < RG; ++q) sums[wave][q][lane] = acc[q];
    __syncthreads();
    // lane (g, n) of piece q: ranks 4 g .. of 16, row n of 16
    for (int i = threadIdx.x; i < RG * 64; i += 256) {
        const int l = i & 63, q = i >> 6, at = l & 15, rank = (chunk * RG + q) * 16 + (l >> 4) * 4;
        if (at >= left || rank >= a.ranks16 * 16) continue;
        f32x4 v = sums[0][q][l] + sums[1][q][l] + (sums[2][q][l] + sums[3][q][l]);
        float by = a.scale ? a.scale[tile.adapter] : 1.0f;
        if (X == AD_E4M3) by *= a.x_scale[here[at]];
        v *= by;
        if (rank >= a.r) v = f32x4{0.0f, 0.0f, 0.0f, 0.0f};  // (r is a multiple of 8)
        *reinterpret_cast<f32x4 *>(a.h + ((int64_t)part * a.max_tiles * a.tile_rows + slot0 + at) * (a.ranks16 * 16) + rank) = v;
    }
}

// ---- out = y + B h ----

// Blocks: 256 columns, 64 to a wave, then tiles.  The products leave a lane with pieces of 16 rows, and a load or store whose neighbouring lanes
// are in different rows takes an address at a time (64 cycles; 8192 x 6144 in bf16 51 us), so they go through LDS, 16 rows at a time, and y and
// out are touched in whole stretches of a row, 512 bytes by half a wave (45 us), and pass by the caches (38).  STEPS: products that r takes (32 ranks each in bf16, 16 in fp32),
// with B's rows for all of them in registers.
template <bool BF16, int MG, int STEPS, bool STREAMED>
__global__ __launch_bounds__(256, BF16 && STEPS <= 2 ? 5 : 1) void adapter_up_kernel(AdapterCall a) {
    constexpr int SZ = BF16 ? 2 : 4, KS = BF16 ? 32 : 16, E16 = 16 / SZ, PITCH = STEPS * KS + E16;  // (rows four banks apart)
    constexpr int SLOTS = MG * 16, QUADS = STEPS * KS / 4, H = (SLOTS * QUADS + 255) / 256;
    constexpr int LANES = 256 / E16, ROWS = 256 / LANES, PIECES = 16 / ROWS;  // threads to a row; rows at a time, pieces of a thread's of 16 rows
    constexpr int STAGE = 256 + 4;
    __shared__ __align__(16) unsigned char h_lds[(BF16 ? 2 : 1) * SLOTS * PITCH * SZ];
    __shared__ __align__(16) float stage[16 * STAGE];
    const int col_blocks = (a.d_out + 255) / 256, at = blockIdx.x / col_blocks, c0 = blockIdx.x % col_blocks * 256;
    const AdapterTile tile = a.tiles[at];
    const int lane = lane_id(), wave = threadIdx.x >> 6, g = lane >> 4, n = lane & 15;
    const int mine = c0 + threadIdx.x % LANES * E16, mine_row = threadIdx.x / LANES;
    int row[MG][PIECES];
#pragma unroll
    for (int m = 0; m < MG; ++m)
#pragma unroll
        for (int p = 0; p < PIECES; ++p) row[m][p] = a.slots[at * SLOTS + m * 16 + p * ROWS + mine_row];
    // h of the tile's slots; what stands in empty ones is not used
    const int width = a.ranks16 * 16;
    f32x4 h[H];
    const float *const h_tile = a.h + (int64_t)at * SLOTS * width;
#pragma unroll
    for (int i = 0; i < H; ++i) {
        const int q = threadIdx.x + i * 256, k = q % QUADS * 4;
        h[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if (q < SLOTS * QUADS && k < width) h[i] = *reinterpret_cast<const f32x4 *>(h_tile + q / QUADS * width + k);
    }
    if (tile.adapter == -2) return;
    u32x4 y[MG][PIECES];
    auto in = [&](int m, int p) { return m * 16 + p * ROWS + mine_row < tile.rows && mine < a.d_out; };
#pragma unroll
    for (int m = 0; m < MG; ++m)
#pragma unroll
        for (int p = 0; p < PIECES; ++p)
            if (in(m, p)) {
                const u32x4 *from = reinterpret_cast<const u32x4 *>(a.y + (int64_t)row[m][p] * a.y_bytes + (int64_t)mine * SZ);
                if constexpr (STREAMED) y[m][p] = __builtin_nontemporal_load(from);
                else y[m][p] = *from;
            }
    auto put = [&](int m, int p, const u32x4 &w) {
        u32x4 *to = reinterpret_cast<u32x4 *>(a.out + (int64_t)row[m][p] * a.out_bytes + (int64_t)mine * SZ);
        if constexpr (STREAMED) __builtin_nontemporal_store(w, to);
        else *to = w;
    };
    if (tile.adapter < 0) {
#pragma unroll
        for (int m = 0; m < MG; ++m)
#pragma unroll
            for (int p = 0; p < PIECES; ++p)
                if (in(m, p)) put(m, p, y[m][p]);
        return;
    }
    u32x4 b[STEPS][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int col = min(c0 + wave * 64 + i * 16 + n, a.d_out - 1);
        const unsigned char *b_row = a.B + ((int64_t)tile.adapter * a.d_out + col) * ((int64_t)a.r * SZ);
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
            const int at_k = k * KS + g * E16;
            b[k][i] = at_k < a.r ? *reinterpret_cast<const u32x4 *>(b_row + (int64_t)at_k * SZ) : u32x4{0, 0, 0, 0};
        }
    }
    // h added up over the parts, zeros in empty slots and behind its ranks
#pragma unroll
    for (int i = 0; i < H; ++i) {
        const int q = threadIdx.x + i * 256, slot = q / QUADS, k = q % QUADS * 4;
        if (q >= SLOTS * QUADS) break;
        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
        if (slot < tile.rows && k < width) {
            v = h[i];
            for (int part = 1; part < a.parts; ++part)
                v += *reinterpret_cast<const f32x4 *>(h_tile + ((int64_t)part * a.max_tiles * SLOTS + slot) * width + k);
        }
        unsigned char *to = h_lds + (slot * PITCH + k) * SZ;
        if constexpr (BF16) {
            // (what is finite stays so: above bf16's largest number the first piece is that one)
            float near[4], left[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) near[e] = fabsf(v[e]) < __builtin_inff() ? fminf(fmaxf(v[e], -BF16_MOST), BF16_MOST) : v[e];
            const u32x2 w = {pack_bf16x2(near[0], near[1]), pack_bf16x2(near[2], near[3])};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float d = v[e] - __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
                left[e] = d == d ? d : 0.0f;  // (nothing is left of an infinity)
            }
            *reinterpret_cast<u32x2 *>(to) = w;
            *reinterpret_cast<u32x2 *>(to + SLOTS * PITCH * SZ) = u32x2{pack_bf16x2(left[0], left[1]), pack_bf16x2(left[2], left[3])};
        } else {
            *reinterpret_cast<f32x4 *>(to) = v;
        }
    }
    lds_hand_over();
#pragma unroll
    for (int m = 0; m < MG; ++m) {
        if (m * 16 >= tile.rows) break;
        f32x4 acc[4] = {};
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
            const unsigned char *from = h_lds + ((m * 16 + n) * PITCH + k * KS + g * E16) * SZ;
            const u32x4 hv = *reinterpret_cast<const u32x4 *>(from);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] = multiply<BF16>(b[k][i], hv, acc[i]);
            if constexpr (BF16) {
                const u32x4 left = *reinterpret_cast<const u32x4 *>(from + SLOTS * PITCH * SZ);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[i] = multiply<BF16>(b[k][i], left, acc[i]);
            }
        }
        // (one stage and five blocks on a CU: 8192 rows of rank 64 74 us of a call, two stages and three blocks 78)
        float *const st = stage;
        if (m > 0) lds_hand_over();
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<f32x4 *>(st + n * STAGE + wave * 64 + i * 16 + g * 4) = acc[i];
        lds_hand_over();
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            if (!in(m, p)) continue;
            const float *const more = st + (p * ROWS + mine_row) * STAGE + threadIdx.x % LANES * E16;
            u32x4 w;
            const f32x4 lo = *reinterpret_cast<const f32x4 *>(more);
            if constexpr (BF16) {
                const f32x4 hi = *reinterpret_cast<const f32x4 *>(more + 4);
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    w[c] = pack_bf16x2(__uint_as_float(y[m][p][c] << 16) + (c < 2 ? lo : hi)[(c & 1) * 2],
                                       __uint_as_float(y[m][p][c] & 0xffff0000u) + (c < 2 ? lo : hi)[(c & 1) * 2 + 1]);
            } else {
#pragma unroll
                for (int c = 0; c < 4; ++c) w[c] = __float_as_uint(__uint_as_float(y[m][p][c]) + lo[c]);
            }
            put(m, p, w);
        }
    }
}

// ---- sizes ----

struct AdapterPlan {
    int tile_rows, ranks16, rank_groups, parts;
    int64_t tiles, down_blocks, h_bytes, tile_bytes, slot_bytes;
};

static AdapterPlan adapter_plan(int64_t T, int d_in, int E, int r) {
    AdapterPlan p;
    // (the host does not know how rows share out: as evenly as they might)
    // Tiles of 16 and 64 rows, us of a call, 2048 to 4096 in bf16, rows of any adapter: 8 adapters of rank 64, 216, 432, 864 rows 14.0 and 16.4, 17.2
    // and 20.9, 20.7 and 22.5; 30 of rank 16, 744, 1488, 2976 rows 16.4 and 20.0, 19.6 and 22.3, 27.6 and 26.0; of rank 64 22.0 and 25.5, 27.3 and 29.8,
    // 43.0 and 35.9; requests of 100 rows, 6200 rows of 30 of rank 64 64 and 56.  (What 64 rows save in weights pays from some 2000 rows on; below, fewer blocks
    // cost a fifth of a call at most.)
    p.tile_rows = T >= 48ll * (E + 1) ? 64 : 16;
    p.ranks16 = (r + 15) / 16;
    // 16, 32 and 64 ranks to a block of the first product, us of a call, 4096 to 4096, 8 adapters: of rank 48, 1, 131, 1000, 8192 rows 10.9, 10.7, 11.8;
    // 12.9, 11.6, 12.5; 23.7, 24.9, 27.3; 81, 73, 72; of rank 128 12.6, 12.4, 13.5; 16.2, 17.7, 18.4; 38.5, 33.3, 36.7; 139, 109, 105.  (x is read
    // once per 64 ranks, which many rows want; few would rather have more blocks.)
    p.rank_groups = p.ranks16 >= 3 ? 4 : p.ranks16;
    const int64_t groups = T < E + 1 ? T : E + 1;
    p.tiles = T / p.tile_rows + groups;
    if (p.tiles > T) p.tiles = T;
    p.down_blocks = p.tiles * (p.tile_rows / 16) * ((p.ranks16 + p.rank_groups - 1) / p.rank_groups);
    int64_t parts = (512 + p.down_blocks - 1) / p.down_blocks;
    const int64_t most = d_in / 512;
    if (parts > most) parts = most;
    p.parts = (int)(parts < 1 ? 1 : parts);
    p.tile_bytes = (int64_t)round_up((size_t)p.tiles * sizeof(AdapterTile), 256);
    p.slot_bytes = (int64_t)round_up((size_t)p.tiles * p.tile_rows * 4, 256);
    p.h_bytes = (int64_t)round_up((size_t)p.parts * p.tiles * p.tile_rows * p.ranks16 * 16 * 4, 256);
    return p;
}

size_t adapters_workspace_bytes(int64_t T, int d_in, int E, int r) {
    if (T <= 0 || d_in <= 0 || E <= 0 || r <= 0) return 0;
    const AdapterPlan p = adapter_plan(T, d_in, E, r);
    return (size_t)(p.tile_bytes + p.slot_bytes + p.h_bytes);
}

template <int X>
static void adapter_down(const AdapterCall &a, const AdapterPlan &p, hipStream_t st) {
    const dim3 grid((unsigned)(p.down_blocks * p.parts)), block(256);
    if (p.rank_groups == 1) adapter_down_kernel<X, 1><<<grid, block, 0, st>>>(a);
    else if (p.rank_groups == 2) adapter_down_kernel<X, 2><<<grid, block, 0, st>>>(a);
    else adapter_down_kernel<X, 4><<<grid, block, 0, st>>>(a);
}

template <bool BF16, int MG, bool STREAMED>
static void adapter_up(const AdapterCall &a, const AdapterPlan &p, hipStream_t st) {
    constexpr int ONE = BF16 ? 1 : 2;  // products of 32 ranks
    const dim3 grid((unsigned)(p.tiles * ((a.d_out + 255) / 256))), block(256);
    if (p.ranks16 <= 2) adapter_up_kernel<BF16, MG, ONE, STREAMED><<<grid, block, 0, st>>>(a);
    else if (p.ranks16 <= 4) adapter_up_kernel<BF16, MG, 2 * ONE, STREAMED><<<grid, block, 0, st>>>(a);
    else adapter_up_kernel<BF16, MG, 4 * ONE, STREAMED><<<grid, block, 0, st>>>(a);
}

template <int X>
static void adapter_products(const AdapterCall &a, const AdapterPlan &p, hipStream_t st) {
    adapter_down<X>(a, p, st);
    const bool streamed = (int64_t)a.T * a.d_out * (X == AD_F32 ? 4 : 2) >= STREAMED_BYTES;
    if (p.tile_rows == 64) streamed ? adapter_up<X != AD_F32, 4, true>(a, p, st) : adapter_up<X != AD_F32, 4, false>(a, p, st);
    else streamed ? adapter_up<X != AD_F32, 1, true>(a, p, st) : adapter_up<X != AD_F32, 1, false>(a, p, st);
}

}  // namespace c2r

using namespace c2r;

extern "C" int c2r_adapters(const void *x, int64_t x_stride, const float *x_scale, c2r_dtype dt, int64_t T, int d_in, int d_out,
                            const int32_t *adapter, int n_adapters, int rank, const void *A, const void *B, const float *scale, const void *y,
                            int64_t y_stride, void *out, int64_t out_stride, void *ws, size_t ws_bytes, void *stream) {
    drop_stale_error();
    if (dt != C2R_F32 && dt != C2R_BF16) return C2R_ERR_INVALID_ARG;
    if (T < 0 || d_in < 1 || d_out < 1 || n_adapters < 1 || rank < 1 || (x_scale && dt != C2R_BF16)) return C2R_ERR_INVALID_ARG;
    if (d_in % 8 != 0 || d_out % 8 != 0 || rank % 8 != 0 || rank > AD_MOST_RANK || n_adapters > AD_MOST_ADAPTERS) return C2R_ERR_UNSUPPORTED;
    if (T >= (1ll << 24) || d_in > (1 << 20) || d_out > (1 << 20)) return C2R_ERR_UNSUPPORTED;
    if (T == 0) return C2R_OK;
    const int size = dt == C2R_BF16 ? 2 : 4;
    if (x_scale ? !x || !aligned(x, 8) || x_stride < d_in || x_stride > (1ll << 40) || x_stride % 8 != 0 || !aligned(x_scale, 4)
                : !rows_ok(x, x_stride, d_in, size))
        return C2R_ERR_INVALID_ARG;
    if (!rows_ok(y, y_stride, d_out, size) || !rows_ok(out, out_stride, d_out, size)) return C2R_ERR_INVALID_ARG;
    if (!adapter || !aligned(adapter, 4) || !A || !B || !aligned(A, 16) || !aligned(B, 16) || (scale && !aligned(scale, 4))) return C2R_ERR_INVALID_ARG;
    const AdapterPlan p = adapter_plan(T, d_in, n_adapters, rank);
    if (p.tiles * ((d_out + 255) / 256) >= (1ll << 24)) return C2R_ERR_UNSUPPORTED;
    if (!ws || !aligned(ws, 256) || ws_bytes < (size_t)(p.tile_bytes + p.slot_bytes + p.h_bytes)) return C2R_ERR_WORKSPACE;
    AdapterCall a = {};
    a.x = static_cast<const unsigned char *>(x), a.A = static_cast<const unsigned char *>(A), a.B = static_cast<const unsigned char *>(B);
    a.y = static_cast<const unsigned char *>(y), a.out = static_cast<unsigned char *>(out);
    a.adapter = adapter, a.x_scale = x_scale, a.scale = scale;
    a.x_bytes = x_stride * (x_scale ? 1 : size), a.y_bytes = y_stride * size, a.out_bytes = out_stride * size;
    a.T = (int)T, a.E = n_adapters, a.r = rank, a.d_in = d_in, a.d_out = d_out;
    a.tile_rows = p.tile_rows, a.ranks16 = p.ranks16, a.parts = p.parts, a.max_tiles = (int)p.tiles;
    a.copy_rest = y != out || y_stride != out_stride;
    unsigned char *w = static_cast<unsigned char *>(ws);
    a.tiles = reinterpret_cast<AdapterTile *>(w);
    a.slots = reinterpret_cast<int *>(w + p.tile_bytes);
    a.h = reinterpret_cast<float *>(w + p.tile_bytes + p.slot_bytes);
    hipStream_t st = static_cast<hipStream_t>(stream);
    a.in_blocks = rows_in_blocks(T, n_adapters);
    if (!a.in_blocks) adapter_order_kernel<<<dim3(1), dim3(1024), 0, st>>>(a);
    if (dt == C2R_F32) adapter_products<AD_F32>(a, p, st);
    else if (x_scale) adapter_products<AD_E4M3>(a, p, st);
    else adapter_products<AD_BF16>(a, p, st);
    return launch_status();
}
