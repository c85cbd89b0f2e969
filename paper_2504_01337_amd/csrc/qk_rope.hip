// Norms of queries and keys for each head, the position rotation, and the new rows of the key-value cache, in one pass.
//
//     y = x * rsqrt(mean(x^2) + eps) * w          (no norm without weights)
//     the first R elements in pairs (i, j): y_i cos - y_j sin, y_j cos + y_i sin at the angle position * inv_freq[i]
//
// A lane holds 16 bytes of a head's row, a whole pair or several, D * size / 16 lanes a head; a wave takes head groups of one token in
// turn, four of them in flight, so the angles of its elements are worked out once.  The angle is a product in 64 bits, in turns,
// less its whole turns: at position 100000 a 32-bit product would be off by 4e-3 radians, more than bf16 resolves.  Everything else is
// 32 bits wide up to the one rounding.
// Memory bound for many tokens: every row is read and written once.  8192 tokens, 16 query and 16 key heads of 128, bf16, 201 MB
// with the appended values: 42 us, 4.8 TB/s (a large copy runs at 4.9); without a cache, 134 MB, 26.5 us, 5.1 TB/s.  Few tokens: a
// chain of loads (sequence, length, page) behind a launch, 3.7 us for 1 token, 4.1 for 64 (in a graph).
#include <type_traits>

#include "attn_common.h"

namespace c2r {

// Waves of a token: enough that the call has ROPE_WAVES of them, and one for every ROPE_GROUPS head groups.  us, 1, 2, 3, 4, 6, 12
// waves a token (bf16, heads of 128, in a stream of calls, its host time of 10.5 in the smallest): 1000 tokens of 16/16 heads (12 groups)
// 11.4, 10.5, 10.5, 10.5, 10.7, 13.3; 2731 16.4, 17.0, 18.1, 19.7, 21.0, 27.3; 8192 43.1, 44.8, 49.1, 52.7, 58.4, 85.7; 1400 of 64/32 (32
// groups) 24.4, 19.9, 19.8, 19.1, 21.9, 25.2; 8192 110, 107, 104, 104, 110, 129.  In a graph, 300 of 16/16 9.6, 6.9, 5.8, 5.9, 5.3, 5.9.
// (Two tokens in a row to a wave, whose places are looked up side by side: 8192 of 16/16 42.1, but 2731 20.9, 12000 60.4 where one token
// takes 55.4.)
constexpr int ROPE_WAVES = 2600, ROPE_GROUPS = 12;

// The sequence that row t belongs to, or -1 past the last one: how many of q_start[0 .. batch] are at most t.
__device__ __forceinline__ int sequence_of(const int32_t *q_start, int batch, int64_t t) {
    const int n = count_first(batch + 1, [&](int i) { return q_start[i] <= t; });
    return n > batch ? -1 : n - 1;
}

// The sum over the LH neighbouring lanes of a head, in each of them.
template <int LH>
__device__ __forceinline__ float head_sum(float v) {
#if defined(__HIP_DEVICE_COMPILE__)
    auto dpp = [](float x, auto ctrl) {
        return __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(x), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    v += dpp(v, std::integral_constant<int, 0xB1>{});   // quad_perm 1 0 3 2
    v += dpp(v, std::integral_constant<int, 0x4E>{});   // quad_perm 2 3 0 1
    v += dpp(v, std::integral_constant<int, 0x141>{});  // row_half_mirror
    if constexpr (LH >= 16) v += dpp(v, std::integral_constant<int, 0x140>{});  // row_mirror
    if constexpr (LH >= 32) v += __shfl_xor(v, 16);
#endif
    return v;
}

// Cosine and sine of r turns, |r| <= 1/2.
// bf16: v_cos_f32 and v_sin_f32, which take turns; with r's rounding 2.3e-7 off at most.  Full precision: the angle to the nearest
// quarter turn, pi/4 at most, in 64 bits, and the Taylor series there, whose next terms are 2e-9 and 2e-10: 9e-8 off at most.  A pass
// over many tokens takes no longer: 8192 tokens of 16 + 16 heads of 64 without a cache 22.3 us, 22.2 with the instructions.
template <bool BF16>
__device__ __forceinline__ void direction(double r, float &c, float &s) {
    if constexpr (BF16) {
        c = 1.0f, s = 0.0f;
#if defined(__HIP_DEVICE_COMPILE__)
        c = __builtin_amdgcn_cosf((float)r);
        s = __builtin_amdgcn_sinf((float)r);
#endif
    } else {
        const double quarters = __builtin_rint(4.0 * r);
        const float x = (float)((r - 0.25 * quarters) * 6.283185307179586477), xx = x * x;
        float sx = __builtin_fmaf(xx, 1.0f / 362880.0f, -1.0f / 5040.0f), cx = __builtin_fmaf(xx, -1.0f / 3628800.0f, 1.0f / 40320.0f);
        sx = __builtin_fmaf(xx, sx, 1.0f / 120.0f), cx = __builtin_fmaf(xx, cx, -1.0f / 720.0f);
        sx = __builtin_fmaf(xx, sx, -1.0f / 6.0f), cx = __builtin_fmaf(xx, cx, 1.0f / 24.0f);
        sx = __builtin_fmaf(x * xx, sx, x), cx = __builtin_fmaf(xx, cx, -0.5f);
        cx = __builtin_fmaf(xx, cx, 1.0f);
        const int q = (int)quarters & 3;
        const float a = q & 1 ? sx : cx, b = q & 1 ? cx : sx;
        c = q == 1 || q == 2 ? -a : a;
        s = q >= 2 ? -b : b;
    }
}

// Both elements of a pair are in one lane: neighbours stand in its 16 bytes; of halves, a lane of the turned part takes 8 bytes
// of each.  (16 bytes in a row of either and the partners' by an exchange, normed and turned twice: 52.3 us for the 8192 tokens with
// their append, where this took 43.0; 1301 tokens, half of a head turned 18.6, 14.1.)
template <bool BF16, int D, bool CACHE, bool NEIGHBOURS>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(RopeCall a) {
    constexpr int SZ = BF16 ? 2 : 4, EPL = 16 / SZ, LH = D / EPL, HW = 64 / LH, BATCH = 4;
    const int lane = lane_id(), sub = lane / LH, c = lane % LH;
    const bool turned = c * EPL < a.rot;
    // this lane's two 8-byte pieces of a row: bytes
    const int low = !NEIGHBOURS && turned ? c * 8 : c * 16, high = !NEIGHBOURS && turned ? a.rot * SZ / 2 + c * 8 : low + 8;
    const int64_t w = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t run = w / a.parts, t = a.first + run;
    const int part = (int)(w - run * a.parts);
    if (t >= a.end) return;
    const int total = a.heads + (CACHE ? 2 : 1) * a.kv_heads, groups = (total + HW - 1) / HW;
    u32x4 x[BATCH] = {};
    // the rows of head groups first, first + parts, ...
    auto fetch = [&](int first) {
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            const int h = (first + u * a.parts) * HW + sub;
            if (h >= total) continue;
            const unsigned char *row = h < a.heads ? a.q + t * a.q_bytes + (int64_t)h * (D * SZ)
                                       : h < a.heads + a.kv_heads ? a.k + t * a.k_bytes + (int64_t)(h - a.heads) * (D * SZ)
                                                                  : a.v + t * a.v_bytes + (int64_t)(h - a.heads - a.kv_heads) * (D * SZ);
            if constexpr (!NEIGHBOURS) {
                const u32x2 a0 = *reinterpret_cast<const u32x2 *>(row + low), a1 = *reinterpret_cast<const u32x2 *>(row + high);
                x[u] = u32x4{a0[0], a0[1], a1[0], a1[1]};
            } else {
                x[u] = *reinterpret_cast<const u32x4 *>(row + low);
            }
        }
    };
    auto store = [&](unsigned char *row, const u32x4 &v) {
        if constexpr (!NEIGHBOURS) {
            *reinterpret_cast<u32x2 *>(row + low) = u32x2{v[0], v[1]};
            *reinterpret_cast<u32x2 *>(row + high) = u32x2{v[2], v[3]};
        } else {
            *reinterpret_cast<u32x4 *>(row + low) = v;
        }
    };
    fetch(part);  // on its way while the token's place is looked up

    // ---- the token's position, and its row's bytes from the cache's start (-1: no such place) ----
    int pos = 0;
    int64_t place = -1;
    if constexpr (CACHE) {
        const int b = a.q_start ? sequence_of(a.q_start, a.kv.batch, t) : (int)t;
        if (b < 0) return;  // a row of no sequence
        int64_t end = t + 1;
        if (a.q_start) end = a.q_start[b + 1] < a.T ? a.q_start[b + 1] : a.T;
        pos = max(a.kv.kv_len[b], 0) - (int)(end - t);
        if (pos >= 0 && pos < a.kv.capacity) {  // (past the end there is no place, and the tokens before it stay)
            const int page = a.kv.page(b, pos);
            if ((uint32_t)page < (uint32_t)a.kv.n_pages) place = a.kv.offset(page, pos);
        }
    }
    if (a.position) pos = a.position[t];

    // weights of this lane's elements
    float wq[EPL], wk[EPL];
    auto weights = [&](const float *src, int first, int second, float (&f)[EPL]) {
#pragma unroll
        for (int i = 0; i < EPL; i += EPL / 2)
#pragma unroll
            for (int j = 0; j < EPL / 2; j += 2) {
                const f32x2 v = src ? *reinterpret_cast<const f32x2 *>(src + (i ? second : first) + j) : f32x2{1.0f, 1.0f};
                f[i + j] = v[0], f[i + j + 1] = v[1];
            }
    };
    weights(a.q_weight, low / SZ, high / SZ, wq);
    weights(a.k_weight, low / SZ, high / SZ, wk);
    // frequencies of this lane's pairs
    constexpr int NA = EPL / 2;
    float freq[NA];
#pragma unroll
    for (int i = 0; i < NA; ++i) freq[i] = turned ? a.inv_freq[c * NA + i] : 0.0f;
    auto unpack = [](const u32x4 &v, float (&f)[EPL]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (BF16) {
                f[2 * i] = __uint_as_float(v[i] << 16);
                f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
            } else {
                f[i] = __uint_as_float(v[i]);
            }
        }
    };

    // the angles of this lane's elements
    float cs[NA], sn[NA];
#pragma unroll
    for (int k = 0; k < NA; ++k) {
        const double turns = (double)pos * ((double)freq[k] * 0.15915494309189533577);
        direction<BF16>(turns - __builtin_rint(turns), cs[k], sn[k]);
    }
    for (int first = part; first < groups; first += BATCH * a.parts) {
        u32x4 now[BATCH];
#pragma unroll
        for (int u = 0; u < BATCH; ++u) now[u] = x[u];
        if (first + BATCH * a.parts < groups) fetch(first + BATCH * a.parts);
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            const int hg = first + u * a.parts;
            if (hg >= groups) break;
            const int h = hg * HW + sub;
            const bool is_q = h < a.heads, is_v = h >= a.heads + a.kv_heads, real = h < total;
            float y[EPL];
            unpack(now[u], y);
            float sq = 0.0f;
#pragma unroll
            for (int k = 0; k < EPL; ++k) sq = __builtin_fmaf(y[k], y[k], sq);
            sq = head_sum<LH>(sq);
            float rs = 1.0f;
#if defined(__HIP_DEVICE_COMPILE__)
            if (is_q ? a.q_weight != nullptr : a.k_weight != nullptr) rs = __builtin_amdgcn_rsqf(__builtin_fmaf(sq, 1.0f / D, a.eps));
#endif
#pragma unroll
            for (int k = 0; k < EPL; ++k) y[k] = y[k] * rs * (is_q ? wq[k] : wk[k]);
            float out[EPL];
#pragma unroll
            for (int k = 0; k < NA; ++k) {
                const int i = NEIGHBOURS ? 2 * k : k, j = NEIGHBOURS ? 2 * k + 1 : k + NA;
                out[i] = turned ? y[i] * cs[k] - y[j] * sn[k] : y[i];
                out[j] = turned ? y[j] * cs[k] + y[i] * sn[k] : y[j];
            }
            u32x4 r;
#pragma unroll
            for (int k = 0; k < 4; ++k) r[k] = BF16 ? pack_bf16x2(out[(2 * k) % EPL], out[(2 * k + 1) % EPL]) : __float_as_uint(out[k]);
            if (!real) continue;
            if (is_q) {
                store(a.q_out + t * a.q_out_bytes + (int64_t)h * (D * SZ), r);
            } else if constexpr (!CACHE) {
                store(a.k_out + t * a.k_out_bytes + (int64_t)(h - a.heads) * (D * SZ), r);
            } else if (place >= 0) {
                const int kh = h - a.heads - (is_v ? a.kv_heads : 0);
                unsigned char *base = const_cast<unsigned char *>(is_v ? a.kv.v : a.kv.k);
                store(base + place + kh * a.kv.head_bytes, is_v ? now[u] : r);
            }
        }
    }
}

template <bool BF16, int D, bool CACHE, bool NEIGHBOURS>
static void start(RopeCall a, hipStream_t st) {
    // (a grid has room for so many tokens)
    const int64_t most = (ATTN_MOST_BLOCKS - 1) * 4 / a.parts;
    for (a.first = 0; a.first < a.T; a.first += most) {
        a.end = a.T - a.first < most ? a.T : a.first + most;
        qk_norm_rope_kernel<BF16, D, CACHE, NEIGHBOURS><<<dim3((unsigned)ceil_div((a.end - a.first) * a.parts, 4)), dim3(256), 0, st>>>(a);
    }
}

template <bool BF16, int D>
static void start(const RopeCall &a, bool cache, bool neighbours, hipStream_t st) {
    if (cache) neighbours ? start<BF16, D, true, true>(a, st) : start<BF16, D, true, false>(a, st);
    else neighbours ? start<BF16, D, false, true>(a, st) : start<BF16, D, false, false>(a, st);
}

int launch_qk_norm_rope(RopeCall a, bool bf16, int D, bool neighbours, hipStream_t st) {
    const bool cache = a.k_out == nullptr;
    const int lanes = D * (bf16 ? 2 : 4) / 16;
    const int64_t groups = ceil_div(a.heads + (cache ? 2 : 1) * a.kv_heads, 64 / lanes);
    const int64_t fill = ceil_div(ROPE_WAVES, a.T), share = ceil_div(groups, ROPE_GROUPS), parts = fill > share ? fill : share;
    a.parts = (int)(parts < groups ? parts : groups);
    if (bf16) D == 128 ? start<true, 128>(a, cache, neighbours, st) : start<true, 64>(a, cache, neighbours, st);
    else D == 128 ? start<false, 128>(a, cache, neighbours, st) : start<false, 64>(a, cache, neighbours, st);
    return launch_status();
}

}  // namespace c2r
