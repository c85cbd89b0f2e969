// Attention of one new token per sequence.  The rows of a block are the query heads of one sequence that share a key head (16
// columns of a product at most; a group of 1 leaves 15 idle, the matrix pipe has the time).  Bound by memory: K and V of the
// visible keys are read once, and nothing is shared but by these rows.  A block's four waves take the tiles of its part of the
// keys in turn and add their sums up through LDS.  Heads of 128, bf16: 131 ragged sequences of up to 8000 keys, 32 / 8 heads 374 us with
// the join (5.5 TB/s; a plain read reaches 6.25); 16 of up to 1500, 32 heads 46 us (4.5); one of 4096, 16 heads 13 us, of which 10 here.
// Three blocks on a CU: with two, or with K and V through LDS, fewer loads are in flight.
#include "attn_stream.h"

namespace c2r {

template <bool BF16, int D>
__global__ __launch_bounds__(256, D == 128 ? 3 : 4) void attn_decode_kernel(AttnCall a) {
    using S = Stream<BF16, D>;
    constexpr int SZ = S::SZ, KT = S::KT;
    __shared__ __align__(16) float join_o[4 * 16 * D], join_ml[4 * 16 * 2];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, n = lane & 15;
    // blocks: parts of the keys fastest, then row blocks of a key head, key heads, sequences
    const uint32_t col_sets = (a.group + 15) / 16, sets = a.kv.kv_heads * col_sets;
    const uint32_t id = blockIdx.x / a.splits, split = blockIdx.x - id * a.splits, b = id / sets, set = id - b * sets;
    const int kv_head = (int)(set / col_sets), col0 = (int)(set - kv_head * col_sets) * 16, left = min(a.group - col0, 16);
    const int p = a.kv.tokens(b) - 1, head0 = kv_head * a.group + col0;
    const KeyTiles<KT> tiles(a, p, p);
    int x0, x1;
    tiles.part(a, split, x0, x1);
    const bool uncut = tiles.uncut(a);
    const int64_t part_row = ((int64_t)split * a.kv.batch + b) * a.heads + head0;
    if (uncut && split > 0) return;
    if (threadIdx.x < (uint32_t)left && a.splits > 1 && (uncut || x0 == x1)) {
        a.part_ml[(part_row + threadIdx.x) * 2] = -__builtin_inff();
        a.part_ml[(part_row + threadIdx.x) * 2 + 1] = uncut ? PART_DONE : PART_EMPTY;
    }
    if (!uncut && x0 == x1) return;
    const unsigned char *q_rows = a.q + b * a.q_bytes + (int64_t)head0 * (D * SZ);
    u32x4 q[S::KSTEPS];
#pragma unroll
    for (int c = 0; c < S::KSTEPS; ++c) q[c] = *reinterpret_cast<const u32x4 *>(q_rows + min(n, left - 1) * (D * SZ) + c * 64 + g * 16);
    typename S::State st;
    S::clear(st);
    S::template run<4>(a, q, st, tiles, x0 + wave, x1, b, kv_head * a.kv.head_bytes, p, p, p);
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
        exact_row<BF16, D, KT>(a, tiles, x0 + wave, x1, 4, b, kv_head, p, q_rows + col * (D * SZ), m, l, o);
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
        if (uncut) {
            const float inv = a.blind(p) ? 0.0f : 1.0f / l, v[4] = {sum[0] * inv, sum[1] * inv, sum[2] * inv, sum[3] * inv};
            store_elements<BF16, 4>(a.out + b * a.out_bytes + ((int64_t)(head0 + col) * D + d) * SZ, v);
        } else {
            *reinterpret_cast<f32x4 *>(a.part_o + (part_row + col) * D + d) = sum;
            if (d == 0) a.part_ml[(part_row + col) * 2] = M, a.part_ml[(part_row + col) * 2 + 1] = l;
        }
    }
}

int launch_attn_decode(const AttnCall &a, bool bf16, int D, hipStream_t st) {
    const dim3 grid((unsigned)((int64_t)a.splits * a.kv.kv_heads * ((a.group + 15) / 16) * a.kv.batch)), block(256);
    if (bf16 && D == 128) attn_decode_kernel<true, 128><<<grid, block, 0, st>>>(a);
    else if (bf16) attn_decode_kernel<true, 64><<<grid, block, 0, st>>>(a);
    else if (D == 128) attn_decode_kernel<false, 128><<<grid, block, 0, st>>>(a);
    else attn_decode_kernel<false, 64><<<grid, block, 0, st>>>(a);
    const int rc = launch_status();
    return rc == C2R_OK && a.splits > 1 ? launch_attn_join(a, bf16, D, st) : rc;
}

}  // namespace c2r
