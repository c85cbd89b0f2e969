// Attention of prompts and of chunks of prompts, bf16: key tiles through LDS, four waves of 32 query rows each.
//
// The rows of a block are (token, head of the group) pairs of one sequence and one key head, token slowest, so grouped heads
// fill a tile like tokens do.  Per tile of 64 keys a wave computes S^T = K q^T (v_mfma_f32_32x32x16_bf16, rows = keys, columns
// = its query rows): lane (h = lane / 32, n = lane % 32) holds 32 of row n's 64 scores, so the maximum and the sum of a row
// are the lane's own and one exchange with lane n + 32.  The second product o^T = V^T p takes the weights where they are:
// within 16 keys, lane half h holds keys 4h..4h+3 and 8+4h..8+4h+3, and V's rows are counted in that order by reading them
// from LDS transposed (ds_read_b64_tr_b16: 4 keys of one element per lane).  Scores and weights never pass through LDS.
// K and V tiles are copied straight into LDS, the next pair in flight while one is worked on, one barrier per tile; a row's
// 16-byte pieces are stored at piece ^ row so that neither read meets on a bank.
#include "attn_common.h"

namespace c2r {

template <int D>
struct TileShape {
    static constexpr int KT = 64, WAVES = 4, BM = 32 * WAVES;
    static constexpr int CH = D / 8;                     // 16-byte pieces of a row
    static constexpr int RPC = 64 / CH;                  // rows per copy instruction of a wave
    static constexpr int COPIES = KT / RPC / WAVES;      // copies per wave, tile and operand
    static constexpr int BYTES = KT * D * 2;             // one operand's tile
    // where piece c of row r is kept (D = 64: two rows span the banks, so pairs of rows share a key)
    __device__ static __forceinline__ int place(int r, int c) { return (r * CH + (c ^ ((CH == 16 ? r : r >> 1) & (CH - 1)))) * 16; }
};

__device__ __forceinline__ void copy16_far(const unsigned char *src, unsigned char *lds) {
#if defined(__HIP_DEVICE_COMPILE__)
    const uint32_t lds_addr = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)lds);
    asm volatile(
        "s_mov_b32 m0, %1\n\t"
        "s_nop 0\n\t"
        "global_load_lds_dwordx4 %0, off"
        :
        : "v"(src), "s"(lds_addr)
        : "memory", "m0");
#endif
}

__device__ __forceinline__ u32x2 read_transposed(const unsigned char *lds) {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)lds));
#else
    return u32x2{};
#endif
}

// max / sum with the lane 32 away
__device__ __forceinline__ float max_halves(float v) {
#if defined(__HIP_DEVICE_COMPILE__)
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
#endif
    return v;
}
__device__ __forceinline__ float add_halves(float v) {
#if defined(__HIP_DEVICE_COMPILE__)
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
#endif
    return v;
}

template <int D>
__global__ __launch_bounds__(256, 2) void attn_tile_kernel(AttnCall a, int row_blocks) {
    using T = TileShape<D>;
    constexpr int KT = T::KT, KSTEPS = D / 16, DT = D / 32;
    __shared__ __align__(1024) unsigned char lds[2][2][T::BYTES];  // [buffer][K, V]
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, n = lane & 31;
    int64_t id = blockIdx.x;
    const int split = (int)(id % a.splits);
    id /= a.splits;
    const int kv_head = (int)(id % a.kv.kv_heads);
    id /= a.kv.kv_heads;
    const int b = (int)(id % a.kv.batch), rb = row_blocks - 1 - (int)(id / a.kv.batch);  // the longest rows first
    const int len = a.kv.length(b), fresh = a.new_tokens(b), rows = min(fresh, a.max_q) * a.group;
    const int block0 = rb * T::BM;
    if (block0 >= rows) return;
    const int before = len - fresh;
    const int block_rows = min(rows - block0, T::BM);
    // the block's range of positions, and this wave's
    const int bp_min = before + block0 / a.group, bp_max = before + (block0 + block_rows - 1) / a.group;
    const int row0 = block0 + wave * 32, left = min(rows - row0, 32);
    const int wr0 = min(row0, rows - 1), wr1 = min(row0 + 31, rows - 1);
    const int p_min = before + wr0 / a.group, p_max = before + wr1 / a.group;
    const int row = min(row0 + n, rows - 1), i = row / a.group, p = before + i;
    const int64_t token = a.first_row(b) + i;
    const int head = kv_head * a.group + row - i * a.group;
    const unsigned char *q_row = a.q + token * a.q_bytes + (int64_t)head * (D * 2);
    bf16x8 q[KSTEPS];
#pragma unroll
    for (int s = 0; s < KSTEPS; ++s) q[s] = *reinterpret_cast<const bf16x8 *>(q_row + s * 32 + h * 16);

    const KeyTiles<KT> tiles(a, bp_min, bp_max);
    int x0, x1;
    tiles.part(a, split, x0, x1);

    // ---- copies: rows (wave * COPIES + u) * RPC + lane / CH of a tile; pieces in the order the LDS image wants ----
    const int64_t head_off = kv_head * a.kv.head_bytes;
    int pages[T::COPIES];
    auto copy_row = [&](int u) { return (wave * T::COPIES + u) * T::RPC + lane / T::CH; };
    auto look_up = [&](int x) {
#pragma unroll
        for (int u = 0; u < T::COPIES; ++u) pages[u] = a.kv.page(b, min(tiles.base(x) + copy_row(u), bp_max));
    };
    auto copy = [&](int x, int buf) {
#pragma unroll
        for (int u = 0; u < T::COPIES; ++u) {
            const int r = copy_row(u), j = min(tiles.base(x) + r, bp_max);
            const int c = (lane % T::CH) ^ ((T::CH == 16 ? r : r >> 1) & (T::CH - 1));
            const int64_t at = a.kv.offset(pages[u], j) + head_off + c * 16;
            copy16_far(a.kv.k + at, &lds[buf][0][(wave * T::COPIES + u) * 1024]);
            copy16_far(a.kv.v + at, &lds[buf][1][(wave * T::COPIES + u) * 1024]);
        }
    };

    f32x16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] = 0.0f;
    float m = -__builtin_inff(), l = 0.0f;
    if (x0 < x1) {
        look_up(x0);
        copy(x0, 0);
        if (x0 + 1 < x1) look_up(x0 + 1);
    }
    for (int x = x0; x < x1; ++x) {
        const int buf = (x - x0) & 1, base = tiles.base(x);
        wait_copies_but<0>();
        lds_barrier();
        if (x + 1 < x1) {
            copy(x + 1, buf ^ 1);
            if (x + 2 < x1) look_up(x + 2);
        }
        if (left <= 0 || !tile_seen<KT>(a, base, p_min, p_max)) continue;
        f32x16 s[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[u][e] = 0.0f;
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
        for (int k = 0; k < KSTEPS; ++k)
#pragma unroll
            for (int u = 0; u < 2; ++u)
                s[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8 *>(lds[buf][0] + T::place(u * 32 + n, k * 2 + h)), q[k], s[u],
                                                               0, 0, 0);
#endif
        if (!tile_whole<KT>(a, base, p_min, p_max)) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (!a.sees(p, base + u * 32 + (e >> 2) * 8 + h * 4 + (e & 3))) s[u][e] = -__builtin_inff();
        }
        float top = s[0][0];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, s[u][e]);
        top = max_halves(top) * a.scale_log2;
        // rescaled only where the maximum has grown by more than 2^8 (see attn_stream.h)
        const bool grow = top > m + 8.0f || (m == -__builtin_inff() && top > m);
        if (__any(grow)) {
            const float alpha = grow ? __builtin_amdgcn_exp2f(m - top) : 1.0f;
            if (grow) m = top;
            l *= alpha;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] *= alpha;
        }
        const float ref = reference_of(m);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[u][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][e], a.scale_log2, -ref));
                l += s[u][e];
            }
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            // 16 keys: weights rounded to bf16 for the matrix pipe, added unrounded above
            u32x4 w;
#pragma unroll
            for (int c = 0; c < 4; ++c) w[c] = pack_bf16x2(s[k >> 1][(k & 1) * 8 + 2 * c], s[k >> 1][(k & 1) * 8 + 2 * c + 1]);
            const int r = k * 16 + h * 4 + ((lane >> 2) & 3), cb = ((lane >> 4) & 1) * 2 + ((lane >> 1) & 1), off = (lane & 1) * 8;
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const u32x2 lo = read_transposed(lds[buf][1] + T::place(r, d * 4 + cb) + off), hi = read_transposed(lds[buf][1] + T::place(r + 8, d * 4 + cb) + off);
                const u32x4 v = {lo[0], lo[1], hi[0], hi[1]};
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, w), o[d], 0, 0, 0);
            }
        }
#endif
    }
    if (left <= 0) return;
    l = add_halves(l);
    bool bad = not_finite(l);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) bad |= not_finite(o[d][e]);
    uint64_t redo = __ballot(bad && n < left);
    redo = (redo | redo >> 32) & 0xffffffffu;

    // ---- results: lane (h, n), word e of o[d]: element 32 d + 8 (e / 4) + 4 h + e % 4 of row n ----
    const int64_t part_rows = a.T * a.heads;
    if (n < left) {
        if (a.splits == 1) {
            const float inv = p < 0 ? 0.0f : 1.0f / l;
            unsigned char *out = a.out + token * a.out_bytes + (int64_t)head * (D * 2);
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int e = 0; e < 16; e += 8) {
                    // the halves of a 16-byte piece are in lanes n and n + 32: each ends with one piece of two
                    u32x4 w;
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const auto r = __builtin_amdgcn_permlane32_swap(pack_bf16x2(o[d][e + 2 * c] * inv, o[d][e + 2 * c + 1] * inv),
                                                                        pack_bf16x2(o[d][e + 4 + 2 * c] * inv, o[d][e + 5 + 2 * c] * inv), false, false);
                        w[c] = r[0], w[2 + c] = r[1];
                    }
                    *reinterpret_cast<u32x4 *>(out + (d * 32 + (e >> 2) * 8 + h * 8) * 2) = w;
                }
#endif
        } else {
            const int64_t prow = (int64_t)split * part_rows + token * a.heads + head;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int e = 0; e < 16; e += 4)
                    *reinterpret_cast<f32x4 *>(a.part_o + prow * D + d * 32 + e * 2 + h * 4) = f32x4{o[d][e], o[d][e + 1], o[d][e + 2], o[d][e + 3]};
            if (h == 0) a.part_ml[prow * 2] = m, a.part_ml[prow * 2 + 1] = p < 0 || x0 == x1 ? -1.0f : l;
        }
    }
    while (redo) {
        const int c = __ffsll((unsigned long long)redo) - 1;
        redo &= redo - 1;
        const int rc = row0 + c, ic = rc / a.group, hc = kv_head * a.group + rc - ic * a.group;
        const int64_t tc = a.first_row(b) + ic;
        float me, le, v[D / 64];
        exact_row<true, D, KT>(a, tiles, x0, x1, 1, b, kv_head, before + ic, a.q + tc * a.q_bytes + (int64_t)hc * (D * 2), me, le, v);
        if (a.splits == 1) {
            const float inv = before + ic < 0 ? 0.0f : 1.0f / le;
            uint16_t *out = reinterpret_cast<uint16_t *>(a.out + tc * a.out_bytes + (int64_t)hc * (D * 2)) + lane * (D / 64);
#pragma unroll
            for (int e = 0; e < D / 64; ++e) out[e] = (uint16_t)f32_to_bf16_bits(v[e] * inv);
        } else {
            const int64_t prow = (int64_t)split * part_rows + tc * a.heads + hc;
#pragma unroll
            for (int e = 0; e < D / 64; ++e) a.part_o[prow * D + lane * (D / 64) + e] = v[e];
            if (lane == 0) a.part_ml[prow * 2] = me, a.part_ml[prow * 2 + 1] = before + ic < 0 ? -1.0f : le;
        }
    }
}

int launch_attn_tile(const AttnCall &a, int D, hipStream_t st) {
    const int row_blocks = (int)ceil_div((int64_t)a.max_q * a.group, ATTN_TILE_ROWS);
    const dim3 grid((unsigned)((int64_t)a.splits * a.kv.kv_heads * row_blocks * a.kv.batch)), block(256);
    if (D == 128) attn_tile_kernel<128><<<grid, block, 0, st>>>(a, row_blocks);
    else attn_tile_kernel<64><<<grid, block, 0, st>>>(a, row_blocks);
    const int rc = launch_status();
    return rc == C2R_OK && a.splits > 1 ? launch_attn_join(a, true, D, st) : rc;
}

}  // namespace c2r
