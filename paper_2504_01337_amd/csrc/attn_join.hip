// Joins the partial results of attention whose keys were split over blocks:
//     M = max_s m_s,   out = sum_s 2^(m_s - M) o_s / sum_s 2^(m_s - M) l_s
// in 32 bits, rounded once.  A query before its sequence's first key sees nothing: zeros.
#include "attn_common.h"

namespace c2r {

// A block per 256 / LANES / PARTS rows: D / 4 lanes hold four elements each, PARTS groups of them take the parts in turn (all
// of a group's loads in flight together) and are added up through LDS, in one order on every run.
template <bool BF16, int D, int PARTS>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnCall a) {
    constexpr int LANES = D / 4, ROWS = 256 / LANES / PARTS, AHEAD = 4;
    __shared__ f32x4 sums[256];
    __shared__ float dens[256];
    // a sequence's rows (token, head) over `blocks` blocks
    const int64_t blocks = ((int64_t)a.max_q * a.heads + ROWS - 1) / ROWS, seq = blockIdx.x / blocks;
    const int b = (int)seq, c = threadIdx.x % LANES, g = threadIdx.x / LANES % PARTS, rl = threadIdx.x / (LANES * PARTS);
    const int n = a.new_tokens(b);
    const int64_t here = (int64_t)(n < a.max_q ? n : a.max_q) * a.heads, r0 = (blockIdx.x - seq * blocks) * ROWS;
    if (r0 >= here) return;
    const int64_t r = r0 + rl < here ? r0 + rl : here - 1;
    const int64_t rows = a.T * a.heads, t = a.first_row(b) + r / a.heads, row = (int64_t)a.first_row(b) * a.heads + r;
    const int h = (int)(r % a.heads);
    const f32x2 *ml = reinterpret_cast<const f32x2 *>(a.part_ml) + row;
    const f32x4 *po = reinterpret_cast<const f32x4 *>(a.part_o) + row * LANES + c;
    float M = -__builtin_inff();
    bool any = false;
    for (int s0 = 0; s0 < a.splits; s0 += LANES) {  // a lane per part
        const f32x2 v = s0 + c < a.splits ? ml[(s0 + c) * rows] : f32x2{-__builtin_inff(), -1.0f};
        float top = v.x;
#pragma unroll
        for (int w = LANES / 2; w; w >>= 1) top = fmaxf(top, __shfl_xor(top, w));
        M = fmaxf(M, top);
        any |= (__ballot(!(v.y < 0.0f)) >> (lane_id() / LANES * LANES) & (LANES == 32 ? 0xffffffffu : 0xffffu)) != 0;
    }
    const float ref = reference_of(M);
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    float l = 0.0f;
    for (int s0 = g; s0 < a.splits; s0 += PARTS * AHEAD) {
        f32x2 v[AHEAD];
        f32x4 o[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int s = s0 + u * PARTS;
            v[u] = s < a.splits ? ml[s * rows] : f32x2{0.0f, -1.0f};
            o[u] = po[(s < a.splits ? s : s0) * rows * LANES];
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (v[u].y < 0.0f) continue;  // a part with no key of this row: its sums were not written
            const float w = __builtin_amdgcn_exp2f(v[u].x - ref);
            l = __builtin_fmaf(w, v[u].y, l);
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] = __builtin_fmaf(w, o[u][i], sum[i]);
        }
    }
    sums[threadIdx.x] = sum;
    dens[threadIdx.x] = l;
    __syncthreads();
    if (g != 0 || r0 + rl >= here) return;
#pragma unroll
    for (int u = 1; u < PARTS; ++u) {
        const f32x4 o = sums[threadIdx.x + u * LANES];
        l += dens[threadIdx.x + u * LANES];
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] += o[i];
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

template <bool BF16, int D, int PARTS>
static void join(const AttnCall &a, hipStream_t st) {
    constexpr int rows = 256 / (D / 4) / PARTS;
    attn_join_kernel<BF16, D, PARTS><<<dim3((unsigned)(a.kv.batch * ceil_div((int64_t)a.max_q * a.heads, rows))), dim3(256), 0, st>>>(a);
}

int launch_attn_join(const AttnCall &a, bool bf16, int D, hipStream_t st) {
    // few parts: two groups of lanes per row, else eight
    const bool few = a.splits <= 8;
    if (bf16 && D == 128) few ? join<true, 128, 2>(a, st) : join<true, 128, 8>(a, st);
    else if (bf16) few ? join<true, 64, 2>(a, st) : join<true, 64, 8>(a, st);
    else if (D == 128) few ? join<false, 128, 2>(a, st) : join<false, 128, 8>(a, st);
    else few ? join<false, 64, 2>(a, st) : join<false, 64, 8>(a, st);
    return launch_status();
}

}  // namespace c2r
