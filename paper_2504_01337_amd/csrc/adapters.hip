// Low-rank adapters of many requests beside a projection that they share: for every row t with an adapter a
//     out[t] = y[t] + c_a B_a (A_a x[t])
// Rows are put in order of their adapters and cut into tiles of up to 16 MG rows of one adapter, so that an adapter's weights are
// read once per tile.  Two products on the matrix pipe: h = A_a x (contraction d_in, a block's waves share it out and add up
// through LDS, blocks share it out where there are few) and B_a h (contraction r), with y added in 32 bits and one rounding.
// h stays in 32 bits: bf16 takes it in two pieces, the rounded number and what is left of it.
// Bound by memory: x, y, out and the adapters in use.
#include "c2r_internal.h"

namespace c2r {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int AD_MOST_ADAPTERS = 1024, AD_MOST_RANK = 128, AD_STEP = 64;

// What x holds: the weights' type, or e4m3 with a scale for every row beside bf16 weights.
enum { AD_F32 = 0, AD_BF16 = 1, AD_E4M3 = 2 };

struct AdapterTile {
    int adapter, first, rows, pad;  // -1: rows without one; rows at order[first ..]
};

struct AdapterCall {
    const unsigned char *x, *A, *B, *y;
    unsigned char *out;
    const int32_t *adapter;
    const float *x_scale, *scale;
    int64_t x_bytes, y_bytes, out_bytes;
    int T, E, r, d_in, d_out, tile_rows, ranks16, parts;
    bool copy_rest;     // rows without an adapter are copied
    AdapterTile *tiles;
    int *order, *n_tiles;
    float *h;           // [parts][T][16 ranks16], rows in their order
};

// ---- the order of the rows ----

// One block: counts, places and tiles of every adapter.
__global__ __launch_bounds__(1024) void adapter_order_kernel(AdapterCall a) {
    __shared__ int next[AD_MOST_ADAPTERS + 1], rows_of[16], tiles_of[16];
    const int tid = threadIdx.x;
    for (int i = tid; i <= a.E; i += 1024) next[i] = 0;
    __syncthreads();
    auto group = [&](int t) {
        const int e = a.adapter[t];
        return (uint32_t)e < (uint32_t)a.E ? e : a.E;
    };
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
    for (int t = tid; t < a.T; t += 1024) take(group(t));
    __syncthreads();
    // exclusive sums over the groups, E + 1 of them: thread i has group i, thread 0 of the last wave's end the last one as well
    const int mine = tid < a.E ? next[tid] : 0, tiles = (mine + a.tile_rows - 1) / a.tile_rows;
    const int rows_to = wave_inclusive_scan(mine), tiles_to = wave_inclusive_scan(tiles);
    if (lane_id() == 63) rows_of[tid >> 6] = rows_to, tiles_of[tid >> 6] = tiles_to;
    __syncthreads();
    int row = rows_to - mine, tile = tiles_to - tiles, all_rows = 0, all_tiles = 0;
    for (int w = 0; w < 16; ++w) {
        if (w < tid >> 6) row += rows_of[w], tile += tiles_of[w];
        all_rows += rows_of[w], all_tiles += tiles_of[w];
    }
    if (tid < a.E) {
        next[tid] = row;
        for (int i = 0; i < tiles; ++i) a.tiles[tile + i] = AdapterTile{tid, row + i * a.tile_rows, min(mine - i * a.tile_rows, a.tile_rows), 0};
    }
    const int rest = next[a.E], rest_tiles = a.copy_rest ? (rest + a.tile_rows - 1) / a.tile_rows : 0;
    for (int i = tid; i < rest_tiles; i += 1024)
        a.tiles[all_tiles + i] = AdapterTile{-1, all_rows + i * a.tile_rows, min(rest - i * a.tile_rows, a.tile_rows), 0};
    __syncthreads();
    if (tid == 0) next[a.E] = all_rows, *a.n_tiles = all_tiles + rest_tiles;
    __syncthreads();
    for (int t = tid; t < a.T; t += 1024) a.order[take(group(t))] = t;
}

// ---- h = A x ----

// Sixteen elements of a row from `at` on, of which `left` (a multiple of 8, or none) are in it: as bf16, or fp32.
template <int X>
struct Sixteen {
    u32x4 w[X == AD_F32 ? 4 : 2];
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
#if defined(__HIP_DEVICE_COMPILE__)
                const u32x2 v = in ? *reinterpret_cast<const u32x2 *>(row + at + half * 8) : u32x2{0, 0};
#pragma unroll
                for (int i = 0; i < 2; ++i) {  // (every e4m3 number is a bf16 one)
                    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(v[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(v[i], true);
                    w[half][2 * i] = pack_bf16x2(lo[0], lo[1]), w[half][2 * i + 1] = pack_bf16x2(hi[0], hi[1]);
                }
#endif
            }
        }
    }
};

template <bool BF16, int WORDS>
__device__ __forceinline__ f32x4 multiply(const u32x4 (&a)[WORDS], const u32x4 (&b)[WORDS], f32x4 c) {
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
        if constexpr (BF16) {
            c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[i]), __builtin_bit_cast(bf16x8, b[i]), c, 0, 0, 0);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[i][e]), __uint_as_float(b[i][e]), c, 0, 0, 0);
        }
    }
#endif
    return c;
}

// Blocks: parts of d_in fastest, then 16 RG ranks, then tiles.  A wave's step is 64 elements of d_in, lane (g, n) has 16 of them of
// rank n and of row n.
template <int X, int MG, int RG>
__global__ __launch_bounds__(256) void adapter_down_kernel(AdapterCall a) {
    constexpr bool BF16 = X != AD_F32;
    constexpr int W = BF16 ? AD_BF16 : AD_F32, WS = BF16 ? 2 : 4;
    __shared__ f32x4 sums[4][MG * RG][64];
    const int chunks = (a.ranks16 + RG - 1) / RG, part = blockIdx.x % a.parts, id = blockIdx.x / a.parts, chunk = id % chunks, at = id / chunks;
    if (at >= *a.n_tiles) return;
    const AdapterTile tile = a.tiles[at];
    if (tile.adapter < 0) return;
    const int lane = lane_id(), wave = threadIdx.x >> 6, g = lane >> 4, n = lane & 15;
    const unsigned char *x_row[MG], *a_row[RG];
#pragma unroll
    for (int m = 0; m < MG; ++m) x_row[m] = a.x + (int64_t)a.order[tile.first + min(m * 16 + n, tile.rows - 1)] * a.x_bytes;
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
    for (int s = part * each + wave; s < s1; s += 4) {
        const int k = s * AD_STEP + g * 16, left = a.d_in - k;
        Sixteen<X> xv[MG];
        Sixteen<W> av[RG];
#pragma unroll
        for (int q = 0; q < RG; ++q) av[q].load(a_row[q], k, left);
#pragma unroll
        for (int m = 0; m < MG; ++m) xv[m].load(x_row[m], k, left);
#pragma unroll
        for (int m = 0; m < MG; ++m)
#pragma unroll
            for (int q = 0; q < RG; ++q) acc[m][q] = multiply<BF16>(av[q].w, xv[m].w, acc[m][q]);
    }
#pragma unroll
    for (int m = 0; m < MG; ++m)
#pragma unroll
        for (int q = 0; q < RG; ++q) sums[wave][m * RG + q][lane] = acc[m][q];
    __syncthreads();
    // lane (g, n) of piece (m, q): ranks 4 g .. of 16, row n of 16
    for (int i = threadIdx.x; i < MG * RG * 64; i += 256) {
        const int l = i & 63, mq = i >> 6, row = mq / RG * 16 + (l & 15), rank = (chunk * RG + mq % RG) * 16 + (l >> 4) * 4;
        if (row >= tile.rows || rank >= a.ranks16 * 16) continue;
        f32x4 v = sums[0][mq][l] + sums[1][mq][l] + (sums[2][mq][l] + sums[3][mq][l]);
        float by = a.scale ? a.scale[tile.adapter] : 1.0f;
        if (X == AD_E4M3) by *= a.x_scale[a.order[tile.first + row]];
        v *= by;
        if (rank >= a.r) v = f32x4{0.0f, 0.0f, 0.0f, 0.0f};  // (r is a multiple of 8)
        *reinterpret_cast<f32x4 *>(a.h + ((int64_t)part * a.T + tile.first + row) * (a.ranks16 * 16) + rank) = v;
    }
}

// ---- out = y + B h ----

// Blocks: 256 columns, 64 to a wave, then tiles.  Column 16 g + 4 i + e of a wave's 64 is word e of lane g's i-th product, so that a
// lane ends with 16 columns of its rows side by side.
template <bool BF16, int MG>
__global__ __launch_bounds__(256) void adapter_up_kernel(AdapterCall a) {
    constexpr int SZ = BF16 ? 2 : 4, KS = BF16 ? 32 : 16, E16 = 16 / SZ, MOST = AD_MOST_RANK, PITCH = MOST + E16;  // (rows a bank apart)
    constexpr int PIECES = 16 * SZ / 16;  // 16-byte pieces of a lane's 16 columns
    __shared__ __align__(16) unsigned char h_lds[(BF16 ? 2 : 1) * MG * 16 * PITCH * SZ];
    const int col_blocks = (a.d_out + 255) / 256, at = blockIdx.x / col_blocks, cb = blockIdx.x % col_blocks;
    if (at >= *a.n_tiles) return;
    const AdapterTile tile = a.tiles[at];
    const int lane = lane_id(), wave = threadIdx.x >> 6, g = lane >> 4, n = lane & 15;
    const int c0 = cb * 256 + wave * 64, mine = c0 + g * 16;  // this lane's columns
    int64_t row[MG];
    u32x4 y[MG][PIECES];
#pragma unroll
    for (int m = 0; m < MG; ++m) {
        row[m] = a.order[tile.first + min(m * 16 + n, tile.rows - 1)];
#pragma unroll
        for (int p = 0; p < PIECES; ++p)
            if (mine + p / (PIECES / 2) * 8 < a.d_out) y[m][p] = *reinterpret_cast<const u32x4 *>(a.y + row[m] * a.y_bytes + (int64_t)mine * SZ + p * 16);
    }
    if (tile.adapter < 0) {
#pragma unroll
        for (int m = 0; m < MG; ++m)
#pragma unroll
            for (int p = 0; p < PIECES; ++p)
                if (m * 16 + n < tile.rows && mine + p / (PIECES / 2) * 8 < a.d_out)
                    *reinterpret_cast<u32x4 *>(a.out + row[m] * a.out_bytes + (int64_t)mine * SZ + p * 16) = y[m][p];
        return;
    }
    // h of the tile's rows: added up over the parts, zeros behind its ranks and rows
    const int width = a.ranks16 * 16, padded = (width + KS - 1) / KS * KS, quads = padded / 4;
    for (int i = threadIdx.x; i < MG * 16 * quads; i += 256) {
        const int hr = i / quads, k = (i - hr * quads) * 4;
        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
        if (hr < tile.rows && k < width)
            for (int part = 0; part < a.parts; ++part)
                v += *reinterpret_cast<const f32x4 *>(a.h + ((int64_t)part * a.T + tile.first + hr) * width + k);
        unsigned char *to = h_lds + (hr * PITCH + k) * SZ;
        if constexpr (BF16) {
            const u32x2 w = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
            float left[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float d = v[e] - __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
                left[e] = d == d ? d : 0.0f;  // (nothing is left of an infinity)
            }
            *reinterpret_cast<u32x2 *>(to) = w;
            *reinterpret_cast<u32x2 *>(to + MG * 16 * PITCH * SZ) = u32x2{pack_bf16x2(left[0], left[1]), pack_bf16x2(left[2], left[3])};
        } else {
            *reinterpret_cast<f32x4 *>(to) = v;
        }
    }
    __syncthreads();
    f32x4 acc[MG][4];
#pragma unroll
    for (int m = 0; m < MG; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[m][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const unsigned char *b_row[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int col = min(c0 + (n >> 2) * 16 + i * 4 + (n & 3), a.d_out - 1);
        b_row[i] = a.B + ((int64_t)tile.adapter * a.d_out + col) * ((int64_t)a.r * SZ);
    }
    for (int k = 0; k < padded; k += KS) {
        const int mine_k = k + g * E16;
        u32x4 b[4][1];
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i][0] = mine_k < a.r ? *reinterpret_cast<const u32x4 *>(b_row[i] + (int64_t)mine_k * SZ) : u32x4{0, 0, 0, 0};
#pragma unroll
        for (int m = 0; m < MG; ++m) {
            const unsigned char *from = h_lds + ((m * 16 + n) * PITCH + mine_k) * SZ;
            const u32x4 h[1] = {*reinterpret_cast<const u32x4 *>(from)};
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[m][i] = multiply<BF16>(b[i], h, acc[m][i]);
            if constexpr (BF16) {
                const u32x4 left[1] = {*reinterpret_cast<const u32x4 *>(from + MG * 16 * PITCH * SZ)};
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[m][i] = multiply<BF16>(b[i], left, acc[m][i]);
            }
        }
    }
#pragma unroll
    for (int m = 0; m < MG; ++m) {
        if (m * 16 + n >= tile.rows) continue;
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            if (mine + p / (PIECES / 2) * 8 >= a.d_out) continue;
            u32x4 w;
            if constexpr (BF16) {
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    w[c] = pack_bf16x2(__uint_as_float(y[m][p][c] << 16) + acc[m][p * 2 + (c >> 1)][(c & 1) * 2],
                                       __uint_as_float(y[m][p][c] & 0xffff0000u) + acc[m][p * 2 + (c >> 1)][(c & 1) * 2 + 1]);
            } else {
#pragma unroll
                for (int c = 0; c < 4; ++c) w[c] = __float_as_uint(__uint_as_float(y[m][p][c]) + acc[m][p][c]);
            }
            *reinterpret_cast<u32x4 *>(a.out + row[m] * a.out_bytes + (int64_t)mine * SZ + p * 16) = w;
        }
    }
}

// ---- sizes ----

struct AdapterPlan {
    int tile_rows, ranks16, rank_groups, parts;
    int64_t tiles, h_bytes, tile_bytes, order_bytes;
};

static AdapterPlan adapter_plan(int64_t T, int d_in, int E, int r) {
    AdapterPlan p;
    // (the host does not know how rows share out: as evenly as they might)
    p.tile_rows = T >= 48ll * (E + 1) ? 64 : 16;
    p.ranks16 = (r + 15) / 16;
    p.rank_groups = p.ranks16 >= 3 ? 4 : p.ranks16;
    const int64_t groups = T < E + 1 ? T : E + 1;
    p.tiles = T / p.tile_rows + groups;
    if (p.tiles > T) p.tiles = T;
    const int64_t blocks = p.tiles * ((p.ranks16 + p.rank_groups - 1) / p.rank_groups);
    int64_t parts = (512 + blocks - 1) / blocks;
    const int64_t most = d_in / 512;
    if (parts > most) parts = most;
    p.parts = (int)(parts < 1 ? 1 : parts);
    p.tile_bytes = (int64_t)round_up((size_t)p.tiles * sizeof(AdapterTile) + 16, 256);
    p.order_bytes = (int64_t)round_up((size_t)T * 4, 256);
    p.h_bytes = (int64_t)round_up((size_t)p.parts * T * p.ranks16 * 16 * 4, 256);
    return p;
}

size_t adapters_workspace_bytes(int64_t T, int d_in, int E, int r) {
    if (T <= 0 || d_in <= 0 || E <= 0 || r <= 0) return 0;
    const AdapterPlan p = adapter_plan(T, d_in, E, r);
    return (size_t)(p.tile_bytes + p.order_bytes + p.h_bytes);
}

template <int X, int MG>
static void adapter_down(const AdapterCall &a, const AdapterPlan &p, hipStream_t st) {
    const dim3 grid((unsigned)(p.tiles * ((p.ranks16 + p.rank_groups - 1) / p.rank_groups) * p.parts)), block(256);
    if (p.rank_groups == 1) adapter_down_kernel<X, MG, 1><<<grid, block, 0, st>>>(a);
    else if (p.rank_groups == 2) adapter_down_kernel<X, MG, 2><<<grid, block, 0, st>>>(a);
    else adapter_down_kernel<X, MG, 4><<<grid, block, 0, st>>>(a);
}

template <int MG>
static void adapter_products(const AdapterCall &a, const AdapterPlan &p, int kind, hipStream_t st) {
    if (kind == AD_F32) adapter_down<AD_F32, MG>(a, p, st);
    else if (kind == AD_BF16) adapter_down<AD_BF16, MG>(a, p, st);
    else adapter_down<AD_E4M3, MG>(a, p, st);
    const dim3 grid((unsigned)(p.tiles * ((a.d_out + 255) / 256))), block(256);
    if (kind == AD_F32) adapter_up_kernel<false, MG><<<grid, block, 0, st>>>(a);
    else adapter_up_kernel<true, MG><<<grid, block, 0, st>>>(a);
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
    if (!ws || !aligned(ws, 256) || ws_bytes < (size_t)(p.tile_bytes + p.order_bytes + p.h_bytes)) return C2R_ERR_WORKSPACE;
    AdapterCall a = {};
    a.x = static_cast<const unsigned char *>(x), a.A = static_cast<const unsigned char *>(A), a.B = static_cast<const unsigned char *>(B);
    a.y = static_cast<const unsigned char *>(y), a.out = static_cast<unsigned char *>(out);
    a.adapter = adapter, a.x_scale = x_scale, a.scale = scale;
    a.x_bytes = x_stride * (x_scale ? 1 : size), a.y_bytes = y_stride * size, a.out_bytes = out_stride * size;
    a.T = (int)T, a.E = n_adapters, a.r = rank, a.d_in = d_in, a.d_out = d_out;
    a.tile_rows = p.tile_rows, a.ranks16 = p.ranks16, a.parts = p.parts;
    a.copy_rest = y != out || y_stride != out_stride;
    unsigned char *w = static_cast<unsigned char *>(ws);
    a.n_tiles = reinterpret_cast<int *>(w), a.tiles = reinterpret_cast<AdapterTile *>(w + 16);
    a.order = reinterpret_cast<int *>(w + p.tile_bytes);
    a.h = reinterpret_cast<float *>(w + p.tile_bytes + p.order_bytes);
    hipStream_t st = static_cast<hipStream_t>(stream);
    adapter_order_kernel<<<dim3(1), dim3(1024), 0, st>>>(a);
    const int kind = dt == C2R_F32 ? AD_F32 : x_scale ? AD_E4M3 : AD_BF16;
    if (p.tile_rows == 64) adapter_products<4>(a, p, kind, st);
    else adapter_products<1>(a, p, kind, st);
    return launch_status();
}
