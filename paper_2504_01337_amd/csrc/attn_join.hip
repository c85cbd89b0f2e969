// Joins the partial results of attention whose keys were split over blocks:
//     M = max_s m_s,   out = sum_s 2^(m_s - M) o_s / sum_s 2^(m_s - M) l_s
// in 32 bits, rounded once.  A query before its sequence's first key sees nothing: zeros.  Rows whose keys were all in one part
// are there already.  Bound by memory: 4 D bytes read per row and part.
#include "attn_common.h"

namespace c2r {

// Rows from which on lanes go through several rows' parts; fewer rows have their parts spread over lanes.  us, the kernel alone, 2
// parts: 65536 rows of 128, half of them cut, 11.9 and 23.2 the other way (42 MB: 3.5 TB/s); 32096 rows 6.8 and 16.7.  The
// call for 2000 tokens of 16 heads: 47.2 with 2 rows at a time, 48.0 with 4, 51.5 with 8, 54.0 the other way.
constexpr int JOIN_AHEAD = 2;
constexpr int64_t JOIN_ROWS = 16384;

template <bool BF16>
__device__ __forceinline__ void put(unsigned char *out, const f32x4 &sum, float inv) {
    if constexpr (BF16) {
        *reinterpret_cast<u32x2 *>(out) = u32x2{pack_bf16x2(sum[0] * inv, sum[1] * inv), pack_bf16x2(sum[2] * inv, sum[3] * inv)};
    } else {
        *reinterpret_cast<f32x4 *>(out) = f32x4{sum[0] * inv, sum[1] * inv, sum[2] * inv, sum[3] * inv};
    }
}

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
    const int splits = ml->y == PART_DONE ? 0 : a.splits;
    for (int s0 = 0; s0 < splits; s0 += LANES) {  // a lane per part
        const f32x2 v = s0 + c < splits ? ml[(s0 + c) * rows] : f32x2{-__builtin_inff(), PART_EMPTY};
        float top = v.x;
#pragma unroll
        for (int w = LANES / 2; w; w >>= 1) top = fmaxf(top, __shfl_xor(top, w));
        M = fmaxf(M, top);
        any |= (__ballot(!(v.y < 0.0f)) >> (lane_id() / LANES * LANES) & (LANES == 32 ? 0xffffffffu : 0xffffu)) != 0;
    }
    const float ref = reference_of(M);
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    float l = 0.0f;
    for (int s0 = g; s0 < splits; s0 += PARTS * AHEAD) {
        f32x2 v[AHEAD];
        f32x4 o[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int s = s0 + u * PARTS;
            v[u] = s < splits ? ml[s * rows] : f32x2{0.0f, PART_EMPTY};
            o[u] = po[(s < splits ? s : s0) * rows * LANES];
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
    if (g != 0 || r0 + rl >= here || splits == 0) return;
#pragma unroll
    for (int u = 1; u < PARTS; ++u) {
        const f32x4 o = sums[threadIdx.x + u * LANES];
        l += dens[threadIdx.x + u * LANES];
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] += o[i];
    }
    const float inv = any ? 1.0f / l : 0.0f;
    put<BF16>(a.out + t * a.out_bytes + ((int64_t)h * D + c * 4) * (BF16 ? 2 : 4), sum, inv);
}

// Many rows: D / 4 lanes go through the parts of AHEAD rows side by side, each with a maximum that grows as they come.  Loads
// of several rows in flight where the kernel above has a few parts of one, and nothing passes through LDS.
template <bool BF16, int D>
__global__ __launch_bounds__(256) void attn_join_rows_kernel(AttnCall a) {
    constexpr int LANES = D / 4, GROUPS = 256 / LANES, AHEAD = JOIN_AHEAD;
    const int64_t blocks = ((int64_t)a.max_q * a.heads + GROUPS * AHEAD - 1) / (GROUPS * AHEAD), seq = blockIdx.x / blocks;
    const int b = (int)seq, c = threadIdx.x % LANES, g = threadIdx.x / LANES, n = a.new_tokens(b);
    const int64_t here = (int64_t)(n < a.max_q ? n : a.max_q) * a.heads, r0 = (blockIdx.x - seq * blocks) * (GROUPS * AHEAD) + g;
    if (r0 >= here) return;
    const int64_t rows = a.T * a.heads, first = (int64_t)a.first_row(b) * a.heads;
    const f32x2 *ml[AHEAD];
    const f32x4 *po[AHEAD];
    bool live[AHEAD];
    float M[AHEAD], l[AHEAD];
    f32x4 sum[AHEAD];
    f32x2 v[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
        const int64_t r = r0 + u * GROUPS, row = first + (r < here ? r : here - 1);
        live[u] = r < here;
        ml[u] = reinterpret_cast<const f32x2 *>(a.part_ml) + row;
        po[u] = reinterpret_cast<const f32x4 *>(a.part_o) + row * LANES + c;
        v[u] = ml[u][0];
        M[u] = -__builtin_inff(), l[u] = 0.0f, sum[u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    bool any[AHEAD] = {};
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) live[u] = live[u] && v[u].y != PART_DONE;
    for (int s = 0; s < a.splits; ++s) {
        f32x4 o[AHEAD];
        f32x2 next[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (live[u] && !(v[u].y < 0.0f)) o[u] = po[u][s * rows * LANES];
            next[u] = s + 1 < a.splits ? ml[u][(s + 1) * rows] : v[u];
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (live[u] && !(v[u].y < 0.0f)) {  // (else a part with no key of this row: its sums were not written)
                const float m = fmaxf(M[u], v[u].x), ref = reference_of(m);
                const float old = __builtin_amdgcn_exp2f(M[u] - ref), w = __builtin_amdgcn_exp2f(v[u].x - ref);
                l[u] = __builtin_fmaf(w, v[u].y, l[u] * old);
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[u][i] = __builtin_fmaf(w, o[u][i], sum[u][i] * old);
                M[u] = m, any[u] = true;
            }
            v[u] = next[u];
        }
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
        if (!live[u]) continue;
        const int64_t r = r0 + u * GROUPS, t = a.first_row(b) + r / a.heads;
        const int h = (int)(r % a.heads);
        const float inv = any[u] ? 1.0f / l[u] : 0.0f;
        put<BF16>(a.out + t * a.out_bytes + ((int64_t)h * D + c * 4) * (BF16 ? 2 : 4), sum[u], inv);
    }
}

template <bool BF16, int D, int PARTS>
static void join(const AttnCall &a, hipStream_t st) {
    constexpr int rows = 256 / (D / 4) / PARTS;
    attn_join_kernel<BF16, D, PARTS><<<dim3((unsigned)(a.kv.batch * ceil_div((int64_t)a.max_q * a.heads, rows))), dim3(256), 0, st>>>(a);
}

// Up to 8 parts two groups of lanes per row, else eight.  Calls, us, two and eight: 4096 keys of 16 heads in 16 parts 17.1, 15.9,
// 32000 in 48 parts 56.3, 52.9; 64 x 2047 keys, 8 parts 64.3, 65.5; 256 rows behind 8000 keys, 8 parts 41.1, 44.1.
template <bool BF16, int D>
static void join(const AttnCall &a, hipStream_t st) {
    constexpr int rows = 256 / (D / 4) * JOIN_AHEAD;
    if ((int64_t)a.max_q * a.heads * a.kv.batch >= JOIN_ROWS)
        attn_join_rows_kernel<BF16, D><<<dim3((unsigned)(a.kv.batch * ceil_div((int64_t)a.max_q * a.heads, rows))), dim3(256), 0, st>>>(a);
    else if (a.splits <= 8) join<BF16, D, 2>(a, st);
    else join<BF16, D, 8>(a, st);
}

int launch_attn_join(const AttnCall &a, bool bf16, int D, hipStream_t st) {
    if (D == 128) bf16 ? join<true, 128>(a, st) : join<false, 128>(a, st);
    else bf16 ? join<true, 64>(a, st) : join<false, 64>(a, st);
    return launch_status();
}

}  // namespace c2r
