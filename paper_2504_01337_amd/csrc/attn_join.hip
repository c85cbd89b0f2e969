// Joins the partial results of attention whose keys were split over blocks:
//     M = max_s m_s,   out = sum_s 2^(m_s - M) o_s / sum_s 2^(m_s - M) l_s
// in 32 bits, rounded once.  A query before its sequence's first key sees nothing: zeros.
#include "attn_common.h"

namespace c2r {

// D / 4 lanes per row, four elements each.
template <bool BF16, int D>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnCall a) {
    constexpr int LANES = D / 4;
    // a sequence's rows (token, head) over `blocks` blocks
    const int64_t blocks = ((int64_t)a.max_q * a.heads * LANES + 255) / 256, seq = blockIdx.x / blocks;
    const int b = (int)seq, c = threadIdx.x % LANES;
    const int64_t r = ((blockIdx.x - seq * blocks) * 256 + threadIdx.x) / LANES;
    const int n = a.new_tokens(b);
    if (r >= (int64_t)(n < a.max_q ? n : a.max_q) * a.heads) return;
    const int64_t rows = a.T * a.heads, t = a.first_row(b) + r / a.heads, row = (int64_t)a.first_row(b) * a.heads + r;
    const int h = (int)(r % a.heads);
    const f32x2 *ml = reinterpret_cast<const f32x2 *>(a.part_ml) + row;
    const f32x4 *po = reinterpret_cast<const f32x4 *>(a.part_o) + row * LANES + c;
    float M = -__builtin_inff();
    for (int s = 0; s < a.splits; ++s) M = fmaxf(M, ml[s * rows].x);
    const float ref = reference_of(M);
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    float l = 0.0f;
    bool any = false;
    for (int s = 0; s < a.splits; ++s) {
        const f32x2 v = ml[s * rows];
        if (v.y < 0.0f) continue;  // a part with no key of this row: its sums were not written
        any = true;
        const float w = __builtin_amdgcn_exp2f(v.x - ref);
        const f32x4 o = po[s * rows * LANES];
        l = __builtin_fmaf(w, v.y, l);
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] = __builtin_fmaf(w, o[i], sum[i]);
    }
    const float inv = any ? 1.0f / l : 0.0f;
    unsigned char *out = a.out + t * a.out_bytes + ((int64_t)h * D + c * 4) * (BF16 ? 2 : 4);
    if constexpr (BF16) {
        const u32x2 w = {pack_bf16x2(sum[0] * inv, sum[1] * inv), pack_bf16x2(sum[2] * inv, sum[3] * inv)};
        *reinterpret_cast<u32x2 *>(out) = w;
    } else {
        const f32x4 w = {sum[0] * inv, sum[1] * inv, sum[2] * inv, sum[3] * inv};
        *reinterpret_cast<f32x4 *>(out) = w;
    }
}

int launch_attn_join(const AttnCall &a, bool bf16, int D, hipStream_t st) {
    const dim3 grid((unsigned)(a.kv.batch * ceil_div((int64_t)a.max_q * a.heads * (D / 4), 256))), block(256);
    if (bf16 && D == 128) attn_join_kernel<true, 128><<<grid, block, 0, st>>>(a);
    else if (bf16) attn_join_kernel<true, 64><<<grid, block, 0, st>>>(a);
    else if (D == 128) attn_join_kernel<false, 128><<<grid, block, 0, st>>>(a);
    else attn_join_kernel<false, 64><<<grid, block, 0, st>>>(a);
    return launch_status();
}

}  // namespace c2r
