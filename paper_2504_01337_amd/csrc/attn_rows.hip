// Attention of prompts in full precision: a wave has 16 (token, head of the group) rows, token slowest, the four waves of a
// block neighbouring ones, so that a tile that one wave loads is in the CU's cache for the others.  Bound by the fp32 matrix
// pipe (v_mfma_f32_16x16x4_f32) in principle; what it reaches is a fifth of it: every wave loads its tiles itself, 16 rows to 16 keys.
// 2 x 2000 ragged tokens, 4 heads of 128 191 us (29 TFLOP/s of 154); 512 tokens, 4 heads of 64 15.5 us with the join.
#include <type_traits>

#include "attn_stream.h"

namespace c2r {

template <int D>
__global__ __launch_bounds__(256, 3) void attn_rows_kernel(AttnCall a) {
    using S = Stream<false, D>;
    constexpr int KT = S::KT;
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, n = lane & 15;
    // blocks: split fastest, then key heads, rows
    int64_t id = blockIdx.x;
    const int split = (int)(id % a.splits);
    id /= a.splits;
    const int kv_head = (int)(id % a.kv.kv_heads);
    id /= a.kv.kv_heads;
    int b, rb;
    if (!a.block_of<ATTN_ROWS_ROWS>((int)id, b, rb)) return;
    const int fresh = a.new_tokens(b), before = a.kv.tokens(b) - fresh, rows = min(fresh, a.max_q) * a.group;
    const int row0 = (rb * 4 + wave) * 16, left = min(rows - row0, 16);
    if (left <= 0) return;
    // the lane's column: query token ti, head hh of the group; columns past the end repeat the last one
    const int row = row0 + min(n, left - 1), ti = row / a.group, hh = row - ti * a.group, p = before + ti;
    const int p_min = before + row0 / a.group, p_max = before + (row0 + left - 1) / a.group;
    const int64_t token = a.first_row(b) + ti;
    const int head = kv_head * a.group + hh;
    const unsigned char *q_row = a.q + token * a.q_bytes + (int64_t)head * (D * 4);
    u32x4 q[S::KSTEPS];
#pragma unroll
    for (int c = 0; c < S::KSTEPS; ++c) q[c] = *reinterpret_cast<const u32x4 *>(q_row + c * 64 + g * 16);

    const KeyTiles<KT> tiles(a, p_min, p_max);
    int x0, x1;
    tiles.part(a, split, x0, x1);
    const bool uncut = tiles.uncut(a);
    if (uncut && split > 0) return;
    typename S::State st;
    S::clear(st);
    S::template run<1>(a, q, st, tiles, x0, x1, b, kv_head * a.kv.head_bytes, p, p_min, p_max);
    uint32_t redo = S::finish(st, left);

    const int64_t part_rows = a.T * a.heads;
    // N elements from `at` on of one row: to `out` where this wave had all keys, else the partial sums
    auto put = [&](int64_t tok, int hd, int at, const float *v, auto count, float m, float l, int pos, bool ml) {
        constexpr int N = decltype(count)::value;
        if (uncut) {
            if (ml && a.splits > 1) a.part_ml[(tok * a.heads + hd) * 2] = -__builtin_inff(), a.part_ml[(tok * a.heads + hd) * 2 + 1] = PART_DONE;
            const float inv = 1.0f / l;
            float *out = reinterpret_cast<float *>(a.out + tok * a.out_bytes + (int64_t)hd * (D * 4)) + at;
#pragma unroll
            for (int e = 0; e < N; ++e) out[e] = a.blind(pos) ? 0.0f : v[e] * inv;
        } else {
            const int64_t pr = (int64_t)split * part_rows + tok * a.heads + hd;
#pragma unroll
            for (int e = 0; e < N; ++e) a.part_o[pr * D + at + e] = v[e];
            if (ml) a.part_ml[pr * 2] = m, a.part_ml[pr * 2 + 1] = a.blind(pos) || x0 == x1 ? PART_EMPTY : l;
        }
    };
    if (n < left && !(redo >> n & 1)) {  // (a row is written once: `out` may be q, which the exact row reads)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float v[S::VEL];
#pragma unroll
            for (int e = 0; e < S::VEL; ++e) v[e] = st.o[e][r];
            put(token, head, (g * 4 + r) * S::VEL, v, std::integral_constant<int, S::VEL>{}, st.m, st.l, p, r == 0 && g == 0);
        }
    }
    while (redo) {
        const int c = __ffs(redo) - 1;
        redo &= redo - 1;
        const int rc = row0 + c, ic = rc / a.group, hc = kv_head * a.group + rc - ic * a.group;
        const int64_t tc = a.first_row(b) + ic;
        float m, l, o[D / 64];
        exact_row<false, D, KT>(a, tiles, x0, x1, 1, b, kv_head, before + ic, a.q + tc * a.q_bytes + (int64_t)hc * (D * 4), m, l, o);
        put(tc, hc, lane * (D / 64), o, std::integral_constant<int, D / 64>{}, m, l, before + ic, lane == 0);
    }
}

int launch_attn_rows_f32(const AttnCall &a, int D, hipStream_t st) {
    const dim3 grid((unsigned)((int64_t)a.splits * a.kv.kv_heads * a.row_blocks * (a.by_rows ? 1 : a.kv.batch))), block(256);
    if (D == 128) attn_rows_kernel<128><<<grid, block, 0, st>>>(a);
    else attn_rows_kernel<64><<<grid, block, 0, st>>>(a);
    const int rc = launch_status();
    return rc == C2R_OK && a.splits > 1 ? launch_attn_join(a, false, D, st) : rc;
}

}  // namespace c2r
