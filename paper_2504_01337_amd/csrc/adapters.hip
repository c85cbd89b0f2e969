// Low-rank adapters of many requests beside a projection that they share: for every row t with an adapter a
//     out[t] = y[t] + c_a B_a (A_a x[t])
// Rows are put in order of their adapters and cut into tiles of up to 16 MG rows of one adapter, so that an adapter's weights are
// read once per tile.  Two products on the matrix pipe: h = A_a x (contraction d_in, a block's waves share it out and add up
// through LDS, blocks share it out where there are few) and B_a h (contraction r), with y added in 32 bits and one rounding.
// h stays in 32 bits: bf16 takes it in two pieces, the rounded number and what is left of it.
// Bound by memory: x, y, out and the adapters in use.
#include "ffn_copy.h"

namespace c2r {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int AD_MOST_ADAPTERS = 1024, AD_MOST_RANK = 128, AD_STEP = 64;

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
    bool copy_rest;     // rows without an adapter are copied
    AdapterTile *tiles;
    int *slots;         // the row in every slot, -1: none
    float *h;           // [parts][slots][16 ranks16]
};

// ---- the order of the rows ----

// One block: counts, tiles and slots of every adapter.
__global__ __launch_bounds__(1024) void adapter_order_kernel(AdapterCall a) {
    __shared__ int next[AD_MOST_ADAPTERS + 1], tiles_of[16];
    const int tid = threadIdx.x;
    // a batch of rows' ids is asked for together; the first batch's stay
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
    for (int t0 = tid; t0 < a.T; t0 += BATCH * 1024) {
        int ids[BATCH];
        if (t0 == tid) {
#pragma unroll
            for (int i = 0; i < BATCH; ++i) ids[i] = held[i];
        } else {
            load(t0, ids);
        }
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
    auto describe = [&](int adapter, int first, int rows, int from, int step) {
        const int n = (rows + a.tile_rows - 1) / a.tile_rows;
        for (int i = from; i < n; i += step) a.tiles[first + i] = AdapterTile{adapter, min(rows - i * a.tile_rows, a.tile_rows)};
        for (int i = rows + from; i < n * a.tile_rows; i += step) a.slots[first * a.tile_rows + i] = -1;
    };
    if (tid < a.E) next[tid] = tile * a.tile_rows, describe(tid, tile, mine, 0, 1);
    describe(-1, with_one, rest, tid, 1024);
    for (int i = with_one + (rest + a.tile_rows - 1) / a.tile_rows + tid; i < a.max_tiles; i += 1024) a.tiles[i] = AdapterTile{-2, 0};
    if (tid == 1023) next[a.E] = with_one * a.tile_rows;  // (E is 1024 at most: no other thread's)
    __syncthreads();
    for (int t0 = tid; t0 < a.T; t0 += BATCH * 1024) {
        if (t0 != tid) load(t0, held);
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int t = t0 + i * 1024, g = group(held[i]);
            if (t < a.T && (g < a.E || a.copy_rest)) a.slots[take(g)] = t;
        }
    }
}

// ---- h = A x ----

// Sixteen elements of a row from `at` on, of which `left` (a multiple of 8, or none) are in it: as they lie there, and opened to bf16 or fp32.
template <int X>
struct Sixteen {
    static constexpr int WORDS = X == AD_F32 ? 4 : X == AD_BF16 ? 2 : 1;
    u32x4 w[WORDS];
    __device__ __forceinline__ void load(const unsigned char *row, int at, int left) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const bool in = left > half * 8;
            if constexpr (X == AD_F32) {
                const u32x4 *p = reinterpret_cast<const u32x4 *>(row + (int64_t)(at + half * 8) * 4);
                w[half * 2] = in ? p[0] : u32x4{0, 0, 0, 0};
                w[half * 2 + 1] = in ? p[1] : u32x4{0, 0, 0, 0};
            } else if constexpr (X == AD_BF16) {
                w[half] = in ? *reinterpret_cast<const u32x4 *>(row + (int64_t)(at + half * 8) * 2) : u32x4{0, 0, 0, 0};
            } else {
                const u32x2 v = in ? *reinterpret_cast<const u32x2 *>(row + at + half * 8) : u32x2{0, 0};
                w[0][half * 2] = v[0], w[0][half * 2 + 1] = v[1];
            }
        }
    }
    __device__ __forceinline__ void open(u32x4 (&to)[X == AD_F32 ? 4 : 2]) const {
        if constexpr (X == AD_E4M3) {  // (every e4m3 number is a bf16 one)
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w[0][i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w[0][i], true);
                to[i >> 1][i % 2 * 2] = pack_bf16x2(lo[0], lo[1]), to[i >> 1][i % 2 * 2 + 1] = pack_bf16x2(hi[0], hi[1]);
            }
#endif
        } else {
#pragma unroll
            for (int i = 0; i < WORDS; ++i) to[i] = w[i];
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

// Blocks: parts of d_in fastest, then 16 RG ranks, then 16 MG rows of a tile.  A wave's step is 64 elements of d_in, lane (g, n) has 16 of them of
// rank n and of row n.
template <int X, int MG, int RG>
__global__ __launch_bounds__(256) void adapter_down_kernel(AdapterCall a) {
    constexpr bool BF16 = X != AD_F32;
    constexpr int W = BF16 ? AD_BF16 : AD_F32, WS = BF16 ? 2 : 4;
    __shared__ f32x4 sums[4][MG * RG][64];
    const int chunks = (a.ranks16 + RG - 1) / RG, part = blockIdx.x % a.parts, id = blockIdx.x / a.parts, chunk = id % chunks, rows_at = id / chunks;
    const int slot0 = rows_at * (MG * 16), in_tile = slot0 % a.tile_rows;
    const AdapterTile tile = a.tiles[slot0 / a.tile_rows];
    const int lane = lane_id(), wave = threadIdx.x >> 6, g = lane >> 4, n = lane & 15;
    int row[MG];
#pragma unroll
    for (int m = 0; m < MG; ++m) row[m] = a.slots[slot0 + m * 16 + n];
    const int left = tile.rows - in_tile;
    if (tile.adapter < 0 || left <= 0) return;
    const unsigned char *x_row[MG], *a_row[RG];
#pragma unroll
    for (int m = 0; m < MG; ++m) x_row[m] = a.x + (int64_t)max(row[m], 0) * a.x_bytes;  // (an empty slot goes along with row 0)
#pragma unroll
    for (int q = 0; q < RG; ++q)
        a_row[q] = a.A + ((int64_t)tile.adapter * a.r + min((chunk * RG + q) * 16 + n, a.r - 1)) * ((int64_t)a.d_in * WS);
    f32x4 acc[MG][RG];
#pragma unroll
    for (int m = 0; m < MG; ++m)
#pragma unroll
        for (int q = 0; q < RG; ++q) acc[m][q] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int steps = (a.d_in + AD_STEP - 1) / AD_STEP, each = (steps + a.parts - 1) / a.parts;
    const int s1 = min((part + 1) * each, steps);
    // (DEPTH steps are asked for together)
    constexpr int DEPTH = MG * RG == 1 ? 8 : MG * RG <= 4 ? 4 : 2;
    for (int s = part * each + wave; s < s1; s += 4 * DEPTH) {
        Sixteen<X> xs[DEPTH][MG];
        Sixteen<W> as[DEPTH][RG];
#pragma unroll
        for (int i = 0; i < DEPTH; ++i) {
            const int k = (s + 4 * i) * AD_STEP + g * 16, in = s + 4 * i < s1 ? a.d_in - k : 0;
#pragma unroll
            for (int q = 0; q < RG; ++q) as[i][q].load(a_row[q], k, in);
#pragma unroll
            for (int m = 0; m < MG; ++m) xs[i][m].load(x_row[m], k, in);
        }
#pragma unroll
        for (int i = 0; i < DEPTH; ++i)
#pragma unroll
            for (int m = 0; m < MG; ++m) {
                u32x4 x[BF16 ? 2 : 4];
                xs[i][m].open(x);
#pragma unroll
                for (int q = 0; q < RG; ++q)
#pragma unroll
                    for (int w = 0; w < (BF16 ? 2 : 4); ++w) acc[m][q] = multiply<BF16>(as[i][q].w[w], x[w], acc[m][q]);
            }
    }
#pragma unroll
    for (int m = 0; m < MG; ++m)
#pragma unroll
        for (int q = 0; q < RG; ++q) sums[wave][m * RG + q][lane] = acc[m][q];
    __syncthreads();
    // lane (g, n) of piece (m, q): ranks 4 g .. of 16, row n of 16
    for (int i = threadIdx.x; i < MG * RG * 64; i += 256) {
        const int l = i & 63, mq = i >> 6, at = mq / RG * 16 + (l & 15), rank = (chunk * RG + mq % RG) * 16 + (l >> 4) * 4;
        if (at >= left || rank >= a.ranks16 * 16) continue;
        f32x4 v = sums[0][mq][l] + sums[1][mq][l] + (sums[2][mq][l] + sums[3][mq][l]);
        float by = a.scale ? a.scale[tile.adapter] : 1.0f;
        if (X == AD_E4M3) by *= a.x_scale[a.slots[slot0 + at]];
        v *= by;
        if (rank >= a.r) v = f32x4{0.0f, 0.0f, 0.0f, 0.0f};  // (r is a multiple of 8)
        *reinterpret_cast<f32x4 *>(a.h + ((int64_t)part * a.max_tiles * a.tile_rows + slot0 + at) * (a.ranks16 * 16) + rank) = v;
    }
}

// ---- out = y + B h ----

// Blocks: 256 columns, 64 to a wave, then tiles.  The products leave a lane with pieces of 16 rows, and a load or store whose neighbouring lanes
// are in different rows takes an address at a time (64 cycles; 8192 x 6144 in bf16 51 us), so they go through LDS, 16 rows at a time, and y and
// out are touched in whole stretches of a row, 512 bytes by half a wave (45 us), and pass by the caches (38).  STEPS: products that r takes (32 ranks each in bf16, 16 in fp32);
// B's rows for all of them, y and h are asked for together.
template <bool BF16, int MG, int STEPS>
__global__ __launch_bounds__(256) void adapter_up_kernel(AdapterCall a) {
    constexpr int SZ = BF16 ? 2 : 4, KS = BF16 ? 32 : 16, E16 = 16 / SZ, PITCH = STEPS * KS + E16;  // (rows four banks apart)
    constexpr int SLOTS = MG * 16, QUADS = STEPS * KS / 4, H = (SLOTS * QUADS + 255) / 256;
    constexpr int LANES = 256 / E16, ROWS = 256 / LANES, PIECES = 16 / ROWS;  // threads to a row; rows at a time, pieces of a thread's of 16 rows
    constexpr int STAGE = 256 + 4;
    __shared__ __align__(16) unsigned char h_lds[(BF16 ? 2 : 1) * SLOTS * PITCH * SZ];
    __shared__ __align__(16) float stage[MG > 1 ? 2 : 1][16 * STAGE];
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
            if (in(m, p)) y[m][p] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(a.y + (int64_t)row[m][p] * a.y_bytes + (int64_t)mine * SZ));
    auto put = [&](int m, int p, const u32x4 &w) { __builtin_nontemporal_store(w, reinterpret_cast<u32x4 *>(a.out + (int64_t)row[m][p] * a.out_bytes + (int64_t)mine * SZ)); };
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
            const u32x2 w = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
            float left[4];
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
        // (two stages: a wave has read one before it comes to the barrier behind which others write it again)
        float *const st = stage[MG > 1 ? m & 1 : 0];
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
    int tile_rows, down_rows, ranks16, rank_groups, parts;
    int64_t tiles, down_blocks, h_bytes, tile_bytes, slot_bytes;
};

static AdapterPlan adapter_plan(int64_t T, int d_in, int E, int r) {
    AdapterPlan p;
    // (the host does not know how rows share out: as evenly as they might)
    p.tile_rows = T >= 48ll * (E + 1) ? 64 : 16;
    p.ranks16 = (r + 15) / 16;
    p.rank_groups = p.ranks16 >= 3 ? 4 : p.ranks16;
    p.down_rows = p.tile_rows == 64 && p.ranks16 <= 2 ? 16 : p.tile_rows;
    const int64_t groups = T < E + 1 ? T : E + 1;
    p.tiles = T / p.tile_rows + groups;
    if (p.tiles > T) p.tiles = T;
    p.down_blocks = p.tiles * (p.tile_rows / p.down_rows) * ((p.ranks16 + p.rank_groups - 1) / p.rank_groups);
    int64_t parts = (256 + p.down_blocks - 1) / p.down_blocks;
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

template <int X, int MG>
static void adapter_down(const AdapterCall &a, const AdapterPlan &p, hipStream_t st) {
    const dim3 grid((unsigned)(p.down_blocks * p.parts)), block(256);
    if (p.rank_groups == 1) adapter_down_kernel<X, MG, 1><<<grid, block, 0, st>>>(a);
    else if (p.rank_groups == 2) adapter_down_kernel<X, MG, 2><<<grid, block, 0, st>>>(a);
    else adapter_down_kernel<X, MG, 4><<<grid, block, 0, st>>>(a);
}

template <int X>
static void adapter_products(const AdapterCall &a, const AdapterPlan &p, hipStream_t st) {
    if (p.down_rows == 64) adapter_down<X, 4>(a, p, st);
    else adapter_down<X, 1>(a, p, st);
    const dim3 grid((unsigned)(p.tiles * ((a.d_out + 255) / 256))), block(256);
    constexpr bool BF16 = X != AD_F32;
    constexpr int ONE = BF16 ? 1 : 2;  // products of 32 ranks
    if (p.tile_rows == 64) {
        if (p.ranks16 <= 2) adapter_up_kernel<BF16, 4, ONE><<<grid, block, 0, st>>>(a);
        else if (p.ranks16 <= 4) adapter_up_kernel<BF16, 4, 2 * ONE><<<grid, block, 0, st>>>(a);
        else adapter_up_kernel<BF16, 4, 4 * ONE><<<grid, block, 0, st>>>(a);
    } else {
        if (p.ranks16 <= 2) adapter_up_kernel<BF16, 1, ONE><<<grid, block, 0, st>>>(a);
        else if (p.ranks16 <= 4) adapter_up_kernel<BF16, 1, 2 * ONE><<<grid, block, 0, st>>>(a);
        else adapter_up_kernel<BF16, 1, 4 * ONE><<<grid, block, 0, st>>>(a);
    }
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
    adapter_order_kernel<<<dim3(1), dim3(1024), 0, st>>>(a);
    if (dt == C2R_F32) adapter_products<AD_F32>(a, p, st);
    else if (x_scale) adapter_products<AD_E4M3>(a, p, st);
    else adapter_products<AD_BF16>(a, p, st);
    return launch_status();
}
