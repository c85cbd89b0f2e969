// Norms of queries and keys for each head, the position rotation, and the new rows of the key-value cache, in one pass.
//
//     y = x * rsqrt(mean(x^2) + eps) * w          (no norm without weights)
//     the first R elements in pairs (i, j): y_i cos - y_j sin, y_j cos + y_i sin at the angle position * inv_freq[i]
//
// A lane holds 16 bytes of a head's row, D * size / 16 lanes a head; a wave takes several heads of ONE token in turn, so the
// angles of its elements are worked out once.  The angle is a product in 64 bits, in turns, less its whole turns: at position
// 100000 a 32-bit product would be off by 4e-3 radians, more than bf16 resolves.  v_sin_f32 and v_cos_f32 take turns and are
// within 1.3e-7 of sin and cos over one turn (2^20 arguments tried).  Everything is 32 bits wide up to the one rounding.
// Memory bound: every row read and written once.
#include <type_traits>

#include "attn_common.h"

namespace c2r {

// The sequence that row t belongs to, or -1 past the last one: how many of q_start[0 .. batch] are at most t, 64 at a time.
__device__ __forceinline__ int sequence_of(const int32_t *q_start, int batch, int64_t t) {
    // (non-decreasing: the wave looks at 64 evenly spread entries, then at the 64 steps between two of them, ...)
    int lo = 0, n = batch + 1;  // the answer's count lies in lo .. lo + n
    const int lane = lane_id();
    while (n > 0) {
        const int step = (n + 63) / 64, at = lo + (lane + 1) * step - 1;  // last entry of each of 64 runs
        const bool below = at < lo + n && q_start[at] <= t;
        const int runs = __popcll(__ballot(below));
        lo += runs * step;
        const int rest = n - runs * step;
        n = rest < step - 1 ? rest : step - 1;
        if (step == 1) break;
    }
    return lo > batch ? -1 : lo - 1;
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

template <bool BF16, int D, bool CACHE, bool NEIGHBOURS>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(RopeCall a) {
    constexpr int SZ = BF16 ? 2 : 4, EPL = 16 / SZ, LH = D / EPL, HW = 64 / LH, BATCH = 4;
    const int lane = lane_id(), sub = lane / LH, c = lane % LH, e0 = c * EPL;
    const int64_t w = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t t = w / a.parts;
    const int part = (int)(w - t * a.parts);
    if (t >= a.T) return;
    const int total = a.heads + (CACHE ? 2 : 1) * a.kv_heads;
    // the first rows are on their way while the position is looked up
    u32x4 x[BATCH] = {};
    auto fetch = [&](int first) {
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            const int h = (first + u * a.parts) * HW + sub;
            if (h >= total) continue;
            const unsigned char *row = h < a.heads ? a.q + t * a.q_bytes + (int64_t)h * (D * SZ)
                                       : h < a.heads + a.kv_heads ? a.k + t * a.k_bytes + (int64_t)(h - a.heads) * (D * SZ)
                                                                  : a.v + t * a.v_bytes + (int64_t)(h - a.heads - a.kv_heads) * (D * SZ);
            x[u] = *reinterpret_cast<const u32x4 *>(row + c * 16);
        }
    };
    fetch(part);

    int index = 0;           // place in the sequence's cache
    int64_t cache_off = -1;  // bytes from the cache's start, -1: no such place
    if constexpr (CACHE) {
        const int b = a.q_start ? sequence_of(a.q_start, a.kv.batch, t) : (int)t;
        if (b < 0) return;  // rows of no sequence
        const int len = a.kv.length(b);
        if (a.q_start) {
            const int64_t end = a.q_start[b + 1];
            index = len - (int)((end < a.T ? end : a.T) - t);
        } else {
            index = len - 1;
        }
        if (index >= 0) {
            const int page = a.kv.table[(int64_t)b * a.kv.max_pages + a.kv.page_of(index)];
            if ((uint32_t)page < (uint32_t)a.kv.n_pages) cache_off = a.kv.offset(page, index);
        }
    }
    const int pos = a.position ? a.position[t] : index;
    // partner of this lane's elements, their angles
    const int half = a.rot / 2, hl = half / EPL;
    const bool turned = e0 < a.rot;
    const int partner = NEIGHBOURS || !turned ? c : c < hl ? c + hl : c - hl;
    constexpr int NA = NEIGHBOURS ? EPL / 2 : EPL;
    float cs[NA], sn[NA];
#pragma unroll
    for (int i = 0; i < NA; ++i) {
        cs[i] = 1.0f, sn[i] = 0.0f;
        if (turned) {
            const int f = NEIGHBOURS ? e0 / 2 + i : (c < hl ? e0 : e0 - half) + i;
            const double turns = (double)pos * (double)a.inv_freq[f] * 0.15915494309189533577;
            const float r = (float)(turns - __builtin_rint(turns));
#if defined(__HIP_DEVICE_COMPILE__)
            cs[i] = __builtin_amdgcn_cosf(r);
            sn[i] = __builtin_amdgcn_sinf(r);
#endif
            if (!NEIGHBOURS && c < hl) sn[i] = -sn[i];  // y_i cos - y_j sin; y_j cos + y_i sin
        }
    }
    // weights of this lane's elements and of their partners
    float wq[EPL], wk[EPL], wq_other[EPL], wk_other[EPL];
    auto weights = [&](const float *src, int at, float (&f)[EPL]) {
#pragma unroll
        for (int i = 0; i < EPL; i += 4) {
            const f32x4 v = src ? *reinterpret_cast<const f32x4 *>(src + at + i) : f32x4{1.0f, 1.0f, 1.0f, 1.0f};
#pragma unroll
            for (int j = 0; j < 4; ++j) f[i + j] = v[j];
        }
    };
    weights(a.q_weight, e0, wq);
    weights(a.k_weight, e0, wk);
    if constexpr (!NEIGHBOURS) {
        weights(a.q_weight, partner * EPL, wq_other);
        weights(a.k_weight, partner * EPL, wk_other);
    }
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
    const int groups = (total + HW - 1) / HW;
    for (int first = part; first < groups; first += BATCH * a.parts) {
        if (first != part) fetch(first);
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            const int hg = first + u * a.parts;
            if (hg >= groups) break;
            const int h = hg * HW + sub;
            const bool is_q = h < a.heads, is_v = h >= a.heads + a.kv_heads, mine = h < total;
            float y[EPL], other[EPL];
            unpack(x[u], y);
            if constexpr (!NEIGHBOURS) {
                u32x4 px;
#pragma unroll
                for (int i = 0; i < 4; ++i) px[i] = __shfl(x[u][i], sub * LH + partner);
                unpack(px, other);
            }
            float sq = 0.0f;
#pragma unroll
            for (int i = 0; i < EPL; ++i) sq = __builtin_fmaf(y[i], y[i], sq);
            sq = head_sum<LH>(sq);
            const bool norm = is_q ? a.q_weight != nullptr : a.k_weight != nullptr;
            float rs = 1.0f;
#if defined(__HIP_DEVICE_COMPILE__)
            if (norm) rs = __builtin_amdgcn_rsqf(__builtin_fmaf(sq, 1.0f / D, a.eps));
#endif
#pragma unroll
            for (int i = 0; i < EPL; ++i) {
                y[i] = y[i] * rs * (is_q ? wq[i] : wk[i]);
                if constexpr (!NEIGHBOURS) other[i] = other[i] * rs * (is_q ? wq_other[i] : wk_other[i]);
            }
            float out[EPL];
            if constexpr (NEIGHBOURS) {
#pragma unroll
                for (int i = 0; i < EPL / 2; ++i) {
                    out[2 * i] = y[2 * i] * cs[i] - y[2 * i + 1] * sn[i];
                    out[2 * i + 1] = y[2 * i + 1] * cs[i] + y[2 * i] * sn[i];
                }
            } else {
#pragma unroll
                for (int i = 0; i < EPL; ++i) out[i] = turned ? y[i] * cs[i] + other[i] * sn[i] : y[i];
            }
            u32x4 r;
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] = BF16 ? pack_bf16x2(out[(2 * i) % EPL], out[(2 * i + 1) % EPL]) : __float_as_uint(out[i]);
            if (!mine) continue;
            if (is_q) {
                *reinterpret_cast<u32x4 *>(a.q_out + t * a.q_out_bytes + (int64_t)h * (D * SZ) + c * 16) = r;
            } else if constexpr (!CACHE) {
                *reinterpret_cast<u32x4 *>(a.k_out + t * a.k_out_bytes + (int64_t)(h - a.heads) * (D * SZ) + c * 16) = r;
            } else if (cache_off >= 0) {
                const int kh = h - a.heads - (is_v ? a.kv_heads : 0);
                unsigned char *base = const_cast<unsigned char *>(is_v ? a.kv.v : a.kv.k);
                *reinterpret_cast<u32x4 *>(base + cache_off + kh * a.kv.head_bytes + c * 16) = is_v ? x[u] : r;
            }
        }
    }
}

template <bool BF16, int D, bool CACHE>
static void start(const RopeCall &a, bool neighbours, unsigned blocks, hipStream_t st) {
    if (neighbours) qk_norm_rope_kernel<BF16, D, CACHE, true><<<dim3(blocks), dim3(256), 0, st>>>(a);
    else qk_norm_rope_kernel<BF16, D, CACHE, false><<<dim3(blocks), dim3(256), 0, st>>>(a);
}

int launch_qk_norm_rope(RopeCall a, bool bf16, int D, bool neighbours, hipStream_t st) {
    const bool cache = a.k_out == nullptr;
    const int lanes = D * (bf16 ? 2 : 4) / 16, groups = (int)ceil_div(a.heads + (cache ? 2 : 1) * a.kv_heads, 64 / lanes);
    // Waves per token: one per head group while they all fit the chip at once, then four groups a wave.
    int64_t parts = ceil_div(8192, a.T);
    if (parts < ceil_div(groups, 4)) parts = ceil_div(groups, 4);
    a.parts = (int)(parts < groups ? parts : groups);
    const int64_t blocks = ceil_div(a.T * a.parts, 4);
    if (blocks >= ATTN_MOST_BLOCKS) return C2R_ERR_UNSUPPORTED;
    const unsigned n = (unsigned)blocks;
    if (bf16) {
        if (D == 128) cache ? start<true, 128, true>(a, neighbours, n, st) : start<true, 128, false>(a, neighbours, n, st);
        else cache ? start<true, 64, true>(a, neighbours, n, st) : start<true, 64, false>(a, neighbours, n, st);
    } else {
        if (D == 128) cache ? start<false, 128, true>(a, neighbours, n, st) : start<false, 128, false>(a, neighbours, n, st);
        else cache ? start<false, 64, true>(a, neighbours, n, st) : start<false, 64, false>(a, neighbours, n, st);
    }
    return launch_status();
}

}  // namespace c2r
