// Attention whose keys and values go straight from memory into the matrix instructions' operand registers.
//
// Sixteen query rows are the columns of every product: S^T = K q^T with v_mfma_f32_16x16x32_bf16 (16x16x4_f32), rows = keys.
// Its result leaves lane (g = lane / 16, n = lane % 16) with keys 4g .. 4g + 3 of row n, which is how the second product
// o^T = V^T p wants its weights if the keys of a step are counted in that order: no lane hands p to another.  A sum over
// keys may take them in any order, so V is simply loaded in the same one.  Elements of D are permuted likewise: a lane loads
// whole 16-byte pieces of K and V rows, and in bf16 turns its 8 keys x 8 elements of V in registers (v_perm_b32).
//
// decode: the rows are the query heads that share a key head (a group of 1 leaves 15 columns idle: the matrix pipe has the
//   time).  Every key is used by these rows alone, so nothing is shared over waves and LDS holds only the join of a block's
//   four waves, which take the block's tiles in turn.  Bound by memory: K and V of the visible keys once.  The next tile's
//   16 KB per wave are in flight while one is worked on.
// rows (full precision prompts): a wave has 16 (token, head) rows, the four waves of a block neighbouring ones, so that a
//   tile that one wave loads is in the CU's cache for the others.  Bound by the fp32 matrix pipe.
#include <type_traits>

#include "attn_common.h"

namespace c2r {

template <bool BF16, int D, bool ROWS>
struct Stream {
    static constexpr int SZ = BF16 ? 2 : 4;
    static constexpr int SUB = BF16 ? 2 : 1;       // 16-key pieces of a tile
    static constexpr int KT = 16 * SUB;            // keys per tile
    static constexpr int EPL = 16 / SZ;            // elements of a 16-byte piece
    static constexpr int KSTEPS = D / (4 * EPL);   // pieces of a K row per lane
    static constexpr int VKEYS = 4 * SUB;          // keys of V per lane
    static constexpr int VEL = D / 16;             // elements of each
    static constexpr int VDW = VEL * SZ / 4;       // the same in 32-bit words

    // A tile's operands: K row (lane % 16) of each piece, V rows 4 * (lane / 16) + 0..3 of each piece.
    struct Tile {
        u32x4 k[SUB][KSTEPS];
        uint32_t v[VKEYS][VDW];
    };

    __device__ static __forceinline__ void load(const AttnCall &a, Tile &t, int b, int64_t head_off, int base, int last) {
        const int lane = lane_id(), g = lane >> 4, n = lane & 15;
        // keys past the last visible one are loaded as that one and masked
        const int jl = min(base + (lane & (KT - 1)), last);
        const int page = a.kv.page(b, jl);
#pragma unroll
        for (int s = 0; s < SUB; ++s) {
            const int src = s * 16 + n, j = min(base + src, last);
            const unsigned char *row = a.kv.k + (a.kv.offset(__shfl(page, src), j) + head_off) + g * 16;
#pragma unroll
            for (int i = 0; i < KSTEPS; ++i) t.k[s][i] = *reinterpret_cast<const u32x4 *>(row + i * 64);
        }
#pragma unroll
        for (int r = 0; r < VKEYS; ++r) {
            const int src = (r >> 2) * 16 + g * 4 + (r & 3), j = min(base + src, last);
            const unsigned char *row = a.kv.v + (a.kv.offset(__shfl(page, src), j) + head_off) + n * (VEL * SZ);
            if constexpr (VDW == 2) {
                const u32x2 w = *reinterpret_cast<const u32x2 *>(row);
                t.v[r][0] = w[0], t.v[r][1] = w[1];
            } else {
#pragma unroll
                for (int i = 0; i < VDW / 4; ++i) {
                    const u32x4 w = *reinterpret_cast<const u32x4 *>(row + i * 16);
#pragma unroll
                    for (int c = 0; c < 4; ++c) t.v[r][i * 4 + c] = w[c];
                }
            }
        }
    }

    struct State {
        f32x4 o[VEL];   // o^T: lane (g, n), word r of o[i]: element (4g + r) * VEL + i of row n
        float m, l;     // maximum of row n in powers of two; denominator over this lane's keys
    };

    __device__ static __forceinline__ void step(const AttnCall &a, const Tile &t, const u32x4 (&q)[KSTEPS], State &st, int base, int p,
                                                bool whole) {
        const int lane = lane_id(), g = lane >> 4;
        f32x4 s[SUB];
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            s[u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < KSTEPS; ++i) {
#if defined(__HIP_DEVICE_COMPILE__)
                if constexpr (BF16) {
                    s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, t.k[u][i]), __builtin_bit_cast(bf16x8, q[i]),
                                                                   s[u], 0, 0, 0);
                } else {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        s[u] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(t.k[u][i][c]), __uint_as_float(q[i][c]), s[u], 0, 0, 0);
                }
#endif
            }
        }
        float x[VKEYS];
#pragma unroll
        for (int r = 0; r < VKEYS; ++r) x[r] = s[r >> 2][r & 3] * a.scale_log2;
        if (!whole) {
#pragma unroll
            for (int r = 0; r < VKEYS; ++r)
                if (!a.sees(p, base + (r >> 2) * 16 + g * 4 + (r & 3))) x[r] = -__builtin_inff();
        }
        float top = x[0];
#pragma unroll
        for (int r = 1; r < VKEYS; ++r) top = fmaxf(top, x[r]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        // The sums are rescaled only where the maximum has grown by more than 2^8: weights up to 256 lose nothing in a
        // 32-bit sum, and most tiles go without the multiplications.
        const bool grow = top > st.m + 8.0f || (st.m == -__builtin_inff() && top > st.m);
        if (__any(grow)) {
            const float alpha = grow ? __builtin_amdgcn_exp2f(st.m - top) : 1.0f;
            if (grow) st.m = top;
            st.l *= alpha;
#pragma unroll
            for (int i = 0; i < VEL; ++i) st.o[i] *= alpha;
        }
        const float ref = reference_of(st.m);
        float w[VKEYS];
#pragma unroll
        for (int r = 0; r < VKEYS; ++r) w[r] = __builtin_amdgcn_exp2f(x[r] - ref);
#pragma unroll
        for (int r = 0; r < VKEYS; ++r) st.l += w[r];
#if defined(__HIP_DEVICE_COMPILE__)
        if constexpr (BF16) {
            // the weights are rounded to bf16 for the matrix pipe (the denominator adds them unrounded): a relative 2^-8
            // at most each, at random, against the 2^-8 of the output's own rounding
            const u32x4 pw = {pack_bf16x2(w[0], w[1]), pack_bf16x2(w[2], w[3]), pack_bf16x2(w[4], w[5]), pack_bf16x2(w[6], w[7])};
#pragma unroll
            for (int i = 0; i < VEL; ++i) {
                const uint32_t sel = i & 1 ? 0x07060302u : 0x05040100u;
                u32x4 vt;
#pragma unroll
                for (int c = 0; c < 4; ++c) vt[c] = __builtin_amdgcn_perm(t.v[2 * c + 1][i >> 1], t.v[2 * c][i >> 1], sel);
                st.o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vt), __builtin_bit_cast(bf16x8, pw), st.o[i], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int r = 0; r < VKEYS; ++r)
#pragma unroll
                for (int i = 0; i < VEL; ++i)
                    st.o[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(t.v[r][i]), w[r], st.o[i], 0, 0, 0);
        }
#endif
    }
};

// One row's result: to `out` where the keys were not split, else the partial sums.
template <bool BF16, int N>
__device__ __forceinline__ void store_elements(unsigned char *p, const float *v) {
    if constexpr (BF16) {
        uint32_t w[N / 2];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) reinterpret_cast<uint32_t *>(p)[i] = w[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) reinterpret_cast<float *>(p)[i] = v[i];
    }
}

template <bool BF16, int D, bool ROWS>
__global__ __launch_bounds__(256, 2) void attn_stream_kernel(AttnCall a, int row_blocks) {
    using S = Stream<BF16, D, ROWS>;
    constexpr int SZ = S::SZ, KT = S::KT;
    __shared__ float join_o[ROWS ? 1 : 4 * 16 * D], join_ml[ROWS ? 1 : 4 * 16 * 2];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, n = lane & 15;
    // blocks: split fastest, then key heads, row blocks, sequences
    int64_t id = blockIdx.x;
    const int split = (int)(id % a.splits);
    id /= a.splits;
    const int kv_head = (int)(id % a.kv.kv_heads);
    id /= a.kv.kv_heads;
    const int rb = (int)(id % row_blocks), b = (int)(id / row_blocks);
    const int len = a.kv.length(b), tokens = ROWS ? min(a.new_tokens(b), a.max_q) : 1, rows = tokens * a.group;
    const int row0 = ROWS ? (rb * 4 + wave) * 16 : rb * 16, left = min(rows - row0, 16);
    if (left <= 0) return;  // (all four waves alike where they meet at a barrier)
    // the lane's column: query token i, head hh of the group; columns past the end repeat the last one
    const int row = row0 + min(n, left - 1), i = row / a.group, hh = row - i * a.group;
    const int before = len - (ROWS ? a.new_tokens(b) : 1), p = before + i;
    const int p_min = before + row0 / a.group, p_max = before + (row0 + left - 1) / a.group;
    const int64_t token = a.first_row(b) + i;
    const int head = kv_head * a.group + hh;
    const unsigned char *q_row = a.q + token * a.q_bytes + (int64_t)head * (D * SZ);
    u32x4 q[S::KSTEPS];
#pragma unroll
    for (int c = 0; c < S::KSTEPS; ++c) q[c] = *reinterpret_cast<const u32x4 *>(q_row + c * 64 + g * 16);

    const KeyTiles<KT> tiles(a, p_min, p_max);
    int x0, x1;
    tiles.part(a, split, x0, x1);
    constexpr int STEP = ROWS ? 1 : 4;
    const int first = ROWS ? x0 : x0 + wave;
    const int64_t head_off = kv_head * a.kv.head_bytes;

    typename S::State st;
#pragma unroll
    for (int e = 0; e < S::VEL; ++e) st.o[e] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    st.m = -__builtin_inff();
    st.l = 0.0f;
    typename S::Tile t0, t1;
    const int last = p_max;  // no tile is visited where this is negative
    if (first < x1) S::load(a, t0, b, head_off, tiles.base(first), last);
    for (int x = first; x < x1; x += 2 * STEP) {
        if (x + STEP < x1) S::load(a, t1, b, head_off, tiles.base(x + STEP), last);
        S::step(a, t0, q, st, tiles.base(x), p, tile_whole<KT>(a, tiles.base(x), p_min, p_max));
        if (x + STEP >= x1) break;
        if (x + 2 * STEP < x1) S::load(a, t0, b, head_off, tiles.base(x + 2 * STEP), last);
        S::step(a, t1, q, st, tiles.base(x + STEP), p, tile_whole<KT>(a, tiles.base(x + STEP), p_min, p_max));
    }
    st.l += __shfl_xor(st.l, 16);
    st.l += __shfl_xor(st.l, 32);
    bool bad = not_finite(st.l);
#pragma unroll
    for (int e = 0; e < S::VEL; ++e)
#pragma unroll
        for (int r = 0; r < 4; ++r) bad |= not_finite(st.o[e][r]);
    bad = bad && n < left;
    uint64_t redo = __ballot(bad);
    redo = (redo | redo >> 16 | redo >> 32 | redo >> 48) & 0xffff;

    const int64_t part_rows = a.T * a.heads;
    if constexpr (ROWS) {
        const int64_t prow = (int64_t)split * part_rows + token * a.heads + head;
        auto put = [&](int64_t pr, unsigned char *out, int at, const float *v, auto count, float m, float l, int pos, bool ml) {
            constexpr int N = decltype(count)::value;
            if (a.splits == 1) {
                float s[N];
                const float inv = 1.0f / l;
#pragma unroll
                for (int e = 0; e < N; ++e) s[e] = pos < 0 ? 0.0f : v[e] * inv;
                store_elements<BF16, N>(out + (int64_t)at * SZ, s);
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) a.part_o[pr * D + at + e] = v[e];
                if (ml) a.part_ml[pr * 2] = m, a.part_ml[pr * 2 + 1] = pos < 0 || x0 == x1 ? -1.0f : l;
            }
        };
        unsigned char *out = a.out + token * a.out_bytes + (int64_t)head * (D * SZ);
        if (n < left) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float v[S::VEL];
#pragma unroll
                for (int e = 0; e < S::VEL; ++e) v[e] = st.o[e][r];
                put(prow, out, (g * 4 + r) * S::VEL, v, std::integral_constant<int, S::VEL>{}, st.m, st.l, p, r == 0 && g == 0);
            }
        }
        while (redo) {
            const int c = __ffsll((unsigned long long)redo) - 1;
            redo &= redo - 1;
            const int rc = row0 + c, ic = rc / a.group, hc = kv_head * a.group + rc - ic * a.group;
            const int64_t tc = a.first_row(b) + ic;
            float m, l, o[D / 64];
            exact_row<BF16, D, KT>(a, tiles, x0, x1, 1, b, kv_head, before + ic, a.q + tc * a.q_bytes + (int64_t)hc * (D * SZ), m, l, o);
            put((int64_t)split * part_rows + tc * a.heads + hc, a.out + tc * a.out_bytes + (int64_t)hc * (D * SZ), lane * (D / 64), o,
                std::integral_constant<int, D / 64>{}, m, l, before + ic, lane == 0);
        }
    } else {
        // the four waves' sums side by side in LDS, then joined
        float *mine = join_o + wave * 16 * D;
        if (n < left) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int e = 0; e < S::VEL; ++e) mine[n * D + (g * 4 + r) * S::VEL + e] = st.o[e][r];
            if (g == 0) join_ml[(wave * 16 + n) * 2] = st.m, join_ml[(wave * 16 + n) * 2 + 1] = st.l;
        }
        while (redo) {
            const int c = __ffsll((unsigned long long)redo) - 1;
            redo &= redo - 1;
            float m, l, o[D / 64];
            exact_row<BF16, D, KT>(a, tiles, first, x1, STEP, b, kv_head, p_max, a.q + a.first_row(b) * a.q_bytes + (int64_t)(kv_head * a.group + row0 + c) * (D * SZ),
                                   m, l, o);
#pragma unroll
            for (int e = 0; e < D / 64; ++e) mine[c * D + lane * (D / 64) + e] = o[e];
            if (lane == 0) join_ml[(wave * 16 + c) * 2] = m, join_ml[(wave * 16 + c) * 2 + 1] = l;
        }
        __syncthreads();
        for (int at = threadIdx.x; at < left * (D / 4); at += 256) {
            const int c = at / (D / 4), d = at % (D / 4) * 4;
            float m4[4], M = -__builtin_inff(), l = 0.0f;
#pragma unroll
            for (int w = 0; w < 4; ++w) m4[w] = join_ml[(w * 16 + c) * 2], M = fmaxf(M, m4[w]);
            const float ref = reference_of(M);
            f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float f = __builtin_amdgcn_exp2f(m4[w] - ref);
                l = __builtin_fmaf(f, join_ml[(w * 16 + c) * 2 + 1], l);
                const f32x4 o = *reinterpret_cast<const f32x4 *>(join_o + (w * 16 + c) * D + d);
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] = __builtin_fmaf(f, o[e], sum[e]);
            }
            const int hc = kv_head * a.group + row0 + c;
            const int64_t t = a.first_row(b);
            if (a.splits == 1) {
                const float inv = 1.0f / l;
                const float v[4] = {p_max < 0 ? 0.0f : sum[0] * inv, p_max < 0 ? 0.0f : sum[1] * inv, p_max < 0 ? 0.0f : sum[2] * inv,
                                    p_max < 0 ? 0.0f : sum[3] * inv};
                store_elements<BF16, 4>(a.out + t * a.out_bytes + ((int64_t)hc * D + d) * SZ, v);
            } else {
                const int64_t prow = (int64_t)split * part_rows + t * a.heads + hc;
                if (x0 < x1) *reinterpret_cast<f32x4 *>(a.part_o + prow * D + d) = sum;
                if (d == 0) a.part_ml[prow * 2] = M, a.part_ml[prow * 2 + 1] = x0 < x1 ? l : -1.0f;
            }
        }
    }
}

int launch_attn_decode(const AttnCall &a, bool bf16, int D, hipStream_t st) {
    const int row_blocks = (a.group + 15) / 16;
    const dim3 grid((unsigned)((int64_t)a.splits * a.kv.kv_heads * row_blocks * a.kv.batch)), block(256);
    if (bf16 && D == 128) attn_stream_kernel<true, 128, false><<<grid, block, 0, st>>>(a, row_blocks);
    else if (bf16) attn_stream_kernel<true, 64, false><<<grid, block, 0, st>>>(a, row_blocks);
    else if (D == 128) attn_stream_kernel<false, 128, false><<<grid, block, 0, st>>>(a, row_blocks);
    else attn_stream_kernel<false, 64, false><<<grid, block, 0, st>>>(a, row_blocks);
    const int rc = launch_status();
    return rc == C2R_OK && a.splits > 1 ? launch_attn_join(a, bf16, D, st) : rc;
}

int launch_attn_rows_f32(const AttnCall &a, int D, hipStream_t st) {
    const int row_blocks = (int)ceil_div((int64_t)a.max_q * a.group, ATTN_ROWS_ROWS);
    const dim3 grid((unsigned)((int64_t)a.splits * a.kv.kv_heads * row_blocks * a.kv.batch)), block(256);
    if (D == 128) attn_stream_kernel<false, 128, true><<<grid, block, 0, st>>>(a, row_blocks);
    else attn_stream_kernel<false, 64, true><<<grid, block, 0, st>>>(a, row_blocks);
    const int rc = launch_status();
    return rc == C2R_OK && a.splits > 1 ? launch_attn_join(a, false, D, st) : rc;
}

}  // namespace c2r
