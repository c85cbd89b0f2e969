// Attention of prompts and of chunks of prompts, bf16: key tiles through LDS, four waves of 32 query rows each.
//
// The rows of a block are (token, head of the group) pairs of one sequence and one key head, token slowest, so grouped heads
// fill a tile like tokens do.  Per tile of 64 keys a wave computes S^T = K q^T (v_mfma_f32_32x32x16_bf16, rows = keys, columns
// = its query rows): lane (h = lane / 32, n = lane % 32) holds 32 of row n's 64 scores, so the maximum and the sum of a row
// are the lane's own and one exchange with lane n + 32.  The second product o^T = V^T p takes the weights where they are:
// within 16 keys, lane half h holds keys 4h..4h+3 and 8+4h..8+4h+3, and V's rows are counted in that order by reading them
// from LDS transposed (ds_read_b64_tr_b16: 4 keys of one element per lane).  Scores and weights never pass through LDS.
// K and V tiles are copied straight into LDS, the next pair in flight while one is worked on, one barrier per tile; a row's
// 16-byte pieces are stored at piece ^ key(row) so that neither read meets on a bank.
//
// Bound by issue: a tile of 128 rows is 32 products a wave and some 210 vector instructions, and the chip is power limited under
// both (1.9 GHz).  Heads of 128: one prompt of 8192 tokens, 16 heads 288 us (950 TFLOP/s of visible pairs; the library's product
// of 8192^3 reaches 1143); 4 prompts of 2048 86 us (800); 16000 tokens through a window of 2048 with 16 sinks 292 to 314 (800 to 870);
// heads of 64, 4 x 2048 51 us (670).  128 rows to a block: K and V are read from LDS by four waves, and 64 rows to a wave, with half
// those reads, need more registers than stay out of the accumulation half (slower).
#pragma once
#include "attn_common.h"

namespace c2r {

template <int D>
struct TileShape {
    static constexpr int KT = 64, WAVES = 4, BM = 32 * WAVES;
    static constexpr int CH = D / 8;                     // 16-byte pieces of a row
    static constexpr int RPC = 64 / CH;                  // rows per copy instruction of a wave
    static constexpr int COPIES = KT / RPC / WAVES;      // copies per wave, tile and operand
    static constexpr int BYTES = KT * D * 2;             // one operand's tile
    // Piece c of row r is kept at piece c ^ key(r) of it.  The keys of 256 bytes' worth of rows (16, or 8 pairs) differ, for
    // the reads of K, which touch one piece of each; and those of four rows in a row differ in the bits that count 64 bytes,
    // for the transposed reads of V, which touch 64 bytes of each.
    __device__ static __forceinline__ int key(int r) { return CH == 16 ? (r & 3) << 2 | (r >> 2 & 3) : (r >> 1 & 1) << 2 | (r >> 2 & 3); }
    __device__ static __forceinline__ int place(int r, int c) { return (r * CH + (c ^ key(r))) * 16; }
};

template <int D>
using TileLds = unsigned char[2][2][TileShape<D>::BYTES];  // [buffer][K, V], 1024-byte aligned

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

// Reads at an LDS address: 16 bytes, and 4 keys of one element (see above).
__device__ __forceinline__ bf16x8 read16(uint32_t at) {
#if defined(__HIP_DEVICE_COMPILE__)
    return *(const __attribute__((address_space(3))) bf16x8 *)at;
#else
    return bf16x8{};
#endif
}
__device__ __forceinline__ u32x2 read_transposed(uint32_t at) {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)at));
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

// v + both of a pair of bf16 numbers
__device__ __forceinline__ float add_pair(float v, uint32_t pair) {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    v = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), bf16x2{(__bf16)1.0f, (__bf16)1.0f}, v, false);
#endif
    return v;
}

// ALIGNED: pages of whole groups of 16 keys, and of less than 4 GB, so that the 16 rows which a wave copies of a tile lie in
// one page: one look-up and one scalar address.  Working out every lane's page takes as many vector instructions per tile as
// the softmax.
// ANY_SCALE: the loop takes maxima of scores before their scale and hides keys by scores of -infinity, so the scale there is positive.
// A negative one becomes the queries' sign, and with 0 the queries are 0 (or NaN, where the definition gives one).  A form of its own,
// as this costs every block some 0.2 us: 32 prompts of 300 43.4 us for 42.7.
// SHARED: the rows are (sequence, head of the group) pairs of a run of sequences, one token each at its own position, and the keys those
// that the run's sequences begin with: partial results only.
template <int D, bool ALIGNED, bool ANY_SCALE, bool SHARED>
__device__ __forceinline__ void attn_tile_block(const AttnCall &a, int64_t id, TileLds<D> &lds) {
    using T = TileShape<D>;
    constexpr int KT = T::KT, KSTEPS = D / 16, DT = D / 32, VALU = 0x2, MFMA = 0x8, DS_READ = 0x100;
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, n = lane & 31;
    const int splits = SHARED ? a.prefix_splits : a.splits;
    const int split = (int)(id % splits);
    id /= splits;
    const int kv_head = (int)(id % a.kv.kv_heads);
    id /= a.kv.kv_heads;
    int b, rb, rows, before = 0;  // before: the position of row 0's token
    KeyRange keys;
    if constexpr (SHARED) {
        AttnCall::Run run;
        if (!a.prefix_block_of<T::BM>((int)id, run, rb, rows)) return;
        b = run.first, keys.to = run.keys;
    } else {
        if (!a.block_of<T::BM>((int)id, b, rb)) return;
        const int len = a.kv.tokens(b), fresh = a.new_tokens(b);
        rows = min(fresh, a.max_q) * a.group;
        before = len - fresh;
    }
    const int block0 = rb * T::BM;
    if (block0 >= rows) return;
    const int block_rows = min(rows - block0, T::BM);
    auto position = [&](int i) { return SHARED ? a.kv.tokens(b + i) - 1 : before + i; };
    const int row0 = block0 + wave * 32, left = min(rows - row0, 32);
    const int row = min(row0 + n, rows - 1), i = row / a.group, p = position(i);
    // the block's range of positions, and this wave's
    int bp_min, bp_max, p_min, p_max;
    if constexpr (SHARED) {
        auto range = [&](int p0, int p1, int &lo, int &hi) {
            lo = min(p0, p1), hi = max(p0, p1);
#pragma unroll
            for (int w = 32; w; w >>= 1) lo = min(lo, __shfl_xor(lo, w)), hi = max(hi, __shfl_xor(hi, w));
            lo = __builtin_amdgcn_readfirstlane(lo), hi = __builtin_amdgcn_readfirstlane(hi);
        };
        range(p, p, p_min, p_max);
        range(position((block0 + min(lane, block_rows - 1)) / a.group), position((block0 + min(lane + 64, block_rows - 1)) / a.group), bp_min, bp_max);
    } else {
        const int wr0 = min(row0, rows - 1), wr1 = min(row0 + 31, rows - 1);
        bp_min = before + block0 / a.group, bp_max = before + (block0 + block_rows - 1) / a.group;
        p_min = before + wr0 / a.group, p_max = before + wr1 / a.group;
    }
    const int last = a.last_key(bp_max, keys);
    const int64_t token = (SHARED ? b : a.first_row(b)) + i;
    const int head = kv_head * a.group + row - i * a.group;
    const unsigned char *q_row = a.q + token * a.q_bytes + (int64_t)head * (D * 2);
    bf16x8 q[KSTEPS];
#pragma unroll
    for (int s = 0; s < KSTEPS; ++s) q[s] = *reinterpret_cast<const bf16x8 *>(q_row + s * 32 + h * 16);
    if constexpr (ANY_SCALE) {
        const float sign = a.scale_log2 < 0.0f ? -1.0f : a.scale_log2 > 0.0f ? 1.0f : 0.0f;
#pragma unroll
        for (int s = 0; s < KSTEPS; ++s) {
            u32x4 w = __builtin_bit_cast(u32x4, q[s]);
#pragma unroll
            for (int c = 0; c < 4; ++c) w[c] = pack_bf16x2(__uint_as_float(w[c] << 16) * sign, __uint_as_float(w[c] & 0xffff0000u) * sign);
            q[s] = __builtin_bit_cast(bf16x8, w);
        }
    }
    const float scale = ANY_SCALE ? a.scale_size : a.scale_log2;

    const KeyTiles<KT> tiles(a, bp_min, bp_max, keys);
    int x0, x1;
    if constexpr (SHARED) tiles.part(splits, a.prefix_tiles, split, x0, x1);
    else tiles.part(a, split, x0, x1);
    const bool uncut = !SHARED && tiles.uncut(a);
    const int64_t part_rows = a.T * a.heads;
    if (uncut && split > 0) return;
    if ((SHARED || a.splits > 1) && (uncut || x0 == x1)) {
        for (int r = threadIdx.x; r < block_rows; r += 256) {
            const int rr = block0 + r, ir = rr / a.group;
            float *ml = a.part_ml + ((int64_t)split * part_rows + ((SHARED ? b : a.first_row(b)) + ir) * a.heads + kv_head * a.group + rr - ir * a.group) * 2;
            ml[0] = -__builtin_inff(), ml[1] = uncut ? PART_DONE : PART_EMPTY;
        }
        if (!uncut) return;
    }

    // ---- copies: rows first_row(u) + lane / CH of a tile; pieces in the order the LDS image wants ----
    const int64_t head_off = kv_head * a.kv.head_bytes;
    constexpr int WAVE_ROWS = KT / T::WAVES;
    int pages[ALIGNED ? 1 : T::COPIES];
    const int lane_row = lane / T::CH;
    auto first_row = [&](int u) { return (wave * T::COPIES + u) * T::RPC; };
    auto piece = [&](int u) { return (lane % T::CH) ^ T::key(first_row(u) + lane_row); };
    uint32_t in_group[T::COPIES];  // ALIGNED: this lane's bytes from the wave's first row on
    if constexpr (ALIGNED) {
#pragma unroll
        for (int u = 0; u < T::COPIES; ++u) in_group[u] = (u * T::RPC + lane_row) * (uint32_t)a.kv.slot_bytes + piece(u) * 16;
    }
    // keys past the block's last visible one stand for that one, and are masked
    auto look_up = [&](int x) {
        const int base = tiles.base(x);
        if constexpr (ALIGNED) {
            pages[0] = a.kv.page(b, min(base + wave * WAVE_ROWS, last));
        } else {
#pragma unroll
            for (int u = 0; u < T::COPIES; ++u) pages[u] = a.kv.page(b, min(base + first_row(u) + lane_row, last));
        }
    };
    const unsigned char *const k_head = a.kv.k + head_off, *const v_head = a.kv.v + head_off;
    // copies [from, to) of a tile
    auto copy = [&](int x, int buf, int from, int to) {
        const int base = tiles.base(x);
        if constexpr (ALIGNED) {
            const uint32_t named = __builtin_amdgcn_readfirstlane(pages[0]), page = named < (uint32_t)a.kv.n_pages ? named : 0;
            const int j0 = min(base + wave * WAVE_ROWS, last & ~(WAVE_ROWS - 1)), over = last - j0;
            const uint32_t slot = j0 - a.kv.page_of(j0) * a.kv.page_size;
            const uint64_t at = (uint64_t)page * (uint32_t)a.kv.page_bytes + slot * (uint32_t)a.kv.slot_bytes;
            uint32_t off[T::COPIES];
#pragma unroll
            for (int u = 0; u < T::COPIES; ++u) off[u] = in_group[u];
            if (over < WAVE_ROWS - 1) {
#pragma unroll
                for (int u = 0; u < T::COPIES; ++u) off[u] = min(u * T::RPC + lane_row, over) * (uint32_t)a.kv.slot_bytes + piece(u) * 16;
            }
#pragma unroll
            for (int u = from; u < to; ++u) {
                copy16_to_lds(k_head + at, off[u], &lds[buf][0][first_row(u) * (D * 2)]);
                copy16_to_lds(v_head + at, off[u], &lds[buf][1][first_row(u) * (D * 2)]);
            }
        } else {
#pragma unroll
            for (int u = from; u < to; ++u) {
                const int64_t at = a.kv.offset(pages[u], min(base + first_row(u) + lane_row, last)) + piece(u) * 16;
                copy16_far(k_head + at, &lds[buf][0][first_row(u) * (D * 2)]);
                copy16_far(v_head + at, &lds[buf][1][first_row(u) * (D * 2)]);
            }
        }
    };

    // ---- reads.  Piece 2k + h of K row n lies at keys_at ^ 32k.  V rows 4h + (lane / 4) % 4 and 8 more, elements 16 of half
    //      a piece row from 32d on: values_at ^ 64d, and ^ 32 for the row 8 further, whose key differs in that bit ----
#if defined(__HIP_DEVICE_COMPILE__)
    const uint32_t lds_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)&lds[0][0][0];
#else
    const uint32_t lds_at = 0;
#endif
    const uint32_t keys_at = lds_at + T::place(n, h);
    const uint32_t values_at = lds_at + T::BYTES + T::place(h * 4 + (lane >> 2 & 3), (lane >> 4 & 1) * 2 + (lane >> 1 & 1)) + (lane & 1) * 8;

    f32x16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] = 0.0f;
    float m = 0.0f, l = 0.0f;  // what scores are taken against (see below); denominator over this lane's keys
    bool bare = true;               // no score above -infinity yet
    float top = -__builtin_inff();  // the last tile's largest score
    // by a whole number of powers of two, so exact; by 2^126 at most, as 2^-127 is no normal number and would come out as zero
    auto move = [&] {
        const bool far = top > m + 30.0f;
        if (!__any(far)) return;
        const float to = fminf(__builtin_ceilf(top), m + 126.0f);
#if defined(__HIP_DEVICE_COMPILE__)
        const float alpha = far ? __builtin_amdgcn_exp2f(m - to) : 1.0f;
        if (far) m = to;
        l *= alpha;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] *= alpha;
#endif
    };
    if (x0 < x1) {
        look_up(x0);
        copy(x0, 0, 0, T::COPIES);
        look_up(x0 + 1 < x1 ? x0 + 1 : x0);
    }
    for (int x = x0; x < x1; ++x) {
        const int buf = (x - x0) & 1, base = tiles.base(x);
        wait_copies_but<0>();
        lds_barrier();
        // (a wave that sees nothing of a tile that others of its block see goes along: every weight comes out as zero)
        const bool whole = tile_whole<KT>(a, base, p_min, p_max, keys);
        f32x16 s[2];
        bf16x8 kf[2][KSTEPS];
        u32x4 vf[2][2][DT], w[2][2];  // V and weights of 32 keys: two products of 16 keys
        u32x4 rest[2][2];             // SHARED: what the weights' rounding leaves
        // (the addresses are worked out where they are used: held over the loop, they would not fit the registers)
        uint32_t ka = keys_at + buf * (2 * T::BYTES), va = values_at + buf * (2 * T::BYTES);
        asm volatile("" : "+v"(ka), "+v"(va));
        auto read_keys = [&](int u, int k) { kf[u][k] = read16((ka ^ (k * 32)) + u * (32 * D * 2)); };
        auto read_values = [&](int u, int k, int d) {
            const u32x2 lo = read_transposed((va ^ (d * 64)) + (u * 32 + k * 16) * (D * 2));
            const u32x2 hi = read_transposed((va ^ (d * 64 + 32)) + (u * 32 + k * 16 + 8) * (D * 2));
            vf[u][k][d] = u32x4{lo[0], lo[1], hi[0], hi[1]};
        };
        // (weights stay where they are worked out, among the products beside them)
        auto pin = [&](int u) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                asm volatile("" : "+v"(w[u][k]));
                if constexpr (SHARED) asm volatile("" : "+v"(rest[u][k]));
            }
        };
        auto mask = [&](int u) {
            // in keys from this lane's first one on; worked out here and nowhere before (few tiles need it)
            int first = base + u * 32;
            asm volatile("" : "+s"(first));
            const int at = first + h * 4, to = a.last_key(p, keys) - at, from = a.window ? p - a.window - at : -1, sinks = a.window ? a.sinks - at : 0;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int c = (e >> 2) * 8 + (e & 3);
                s[u][e] = (c <= to) & ((c > from) | (c < sinks)) ? s[u][e] : -__builtin_inff();
            }
        };
        auto largest = [&](int u) {
            float top = s[u][0];
#pragma unroll
            for (int e = 1; e < 16; ++e) top = fmaxf(top, s[u][e]);
            return top;
        };
        // Weights are rounded to bf16 for the matrix pipe, 2^-8 of each, and added up as rounded (v_dot2c_f32_bf16, both of a pair in one
        // instruction): a row that sees one key is its value exactly.  A second product with what the rounding leaves would give the
        // 32-bit weights' result and costs a quarter to a third: 4 x 2048 tokens 85 us and 109, one prompt of 8192 288 and 383, root mean
        // square error 2.2e-3 and 1.6e-3, of which the result's own rounding is 1.6e-3.
        // SHARED: both pieces, as single tokens have them everywhere else (attn_stream.h), so that what a sequence gets does not hang on
        // how many others there are.
        auto weigh = [&](int u) {
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
                const float lo = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][e], scale, -m));
                const float hi = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][e + 1], scale, -m));
                const uint32_t pair = pack_bf16x2(lo, hi);
                w[u][e >> 3][(e >> 1) & 3] = pair;
                l = add_pair(l, pair);
                if constexpr (SHARED) {
                    const uint32_t left = pack_bf16x2(lo - __uint_as_float(pair << 16), hi - __uint_as_float(pair & 0xffff0000u));
                    rest[u][e >> 3][(e >> 1) & 3] = left;
                    l = add_pair(l, left);
                }
            }
        };
#if defined(__HIP_DEVICE_COMPILE__)
        auto score = [&](int u, int k) { s[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[u][k], q[k], s[u], 0, 0, 0); };
        auto add = [&](int u, int k, int d) {
            o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[u][k][d]), __builtin_bit_cast(bf16x8, w[u][k]), o[d], 0, 0, 0);
            if constexpr (SHARED)
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[u][k][d]), __builtin_bit_cast(bf16x8, rest[u][k]), o[d], 0, 0, 0);
        };
        // A wave issues in order, and a product holds the matrix pipe for 32 cycles: in between there is time for some eight
        // vector instructions.  So the softmax of the first 32 keys stands among the scores of the second 32, and theirs among
        // the first 32's values; operands are read from LDS half a stretch ahead of their products.
        constexpr int HK = KSTEPS / 2, HV = DT;  // half of 32 keys' products
        constexpr int EACH = SHARED ? 2 : 1, WEIGH = SHARED ? 48 : 0;  // products of a step of values; what both pieces of the weights take more
#define STRETCH(N, READS, OTHERS)                                       \
    _Pragma("unroll") for (int i_ = 0; i_ < (N); ++i_) {                \
        __builtin_amdgcn_sched_group_barrier(MFMA, 1, 0);               \
        if (READS) __builtin_amdgcn_sched_group_barrier(DS_READ, READS, 0); \
        if (OTHERS) __builtin_amdgcn_sched_group_barrier(VALU, OTHERS, 0);  \
    }
        // (Copies of the next tile go out in halves after the first two stretches: all at once, right behind the barrier, the
        // waves wait for each other's.  With the maximum moved behind the products, 4 x 2048 tokens 101 -> 94 us.)
        // Scores are taken against m, a whole number near the largest score of a row's first tile that has any, and moved on
        // where a later score is over 2^30 above it: bf16 has the exponents of fp32, so weights of 2^30 are as good as weights
        // of 1, and nothing waits for a maximum.  (A score 2^127 above the ones before it overflows, which the check of the
        // results finds.)
        if (__any(bare)) {
            float here = -__builtin_inff();
#pragma unroll
            for (int u = 0; u < 2; ++u) {
#pragma unroll
                for (int e = 0; e < 16; ++e) s[u][e] = 0.0f;
#pragma unroll
                for (int k = 0; k < KSTEPS; ++k) {
                    read_keys(u, k);
                    score(u, k);
                }
                if (!whole) mask(u);
                here = fmaxf(here, largest(u));
            }
            top = fmaxf(top, max_halves(here) * scale);
            if (bare && top != -__builtin_inff()) m = __builtin_ceilf(top), bare = false;
            __builtin_amdgcn_sched_barrier(0);
        }
        float part;  // of the largest score
        move();
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[u][e] = 0.0f;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < HK; ++k) read_keys(0, k);
#pragma unroll
        for (int k = 0; k < KSTEPS; ++k) {
            score(0, k);
            if (k < HK) read_keys(0, k + HK);
            else read_keys(1, k - HK);
        }
        __builtin_amdgcn_sched_group_barrier(DS_READ, HK, 0);
        STRETCH(KSTEPS, 1, 0)
        __builtin_amdgcn_sched_barrier(0);
        if (x + 1 < x1) copy(x + 1, buf ^ 1, 0, T::COPIES / 2);
        if (!whole) mask(0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < KSTEPS; ++k) {
            score(1, k);
            if (k < HK) read_keys(1, k + HK);
        }
#pragma unroll
        for (int d = 0; d < DT; ++d) read_values(0, 0, d);
        weigh(0);
        part = largest(0);
        STRETCH(HK, 1, (64 + WEIGH) / KSTEPS)
        STRETCH(HK, 2 * HV / HK, (64 + WEIGH) / KSTEPS)
        pin(0);
        asm volatile("" : "+v"(part), "+v"(l));
        __builtin_amdgcn_sched_barrier(0);
        if (x + 1 < x1) {
            copy(x + 1, buf ^ 1, T::COPIES / 2, T::COPIES);
            look_up(x + 2 < x1 ? x + 2 : x + 1);
        }
        if (!whole) mask(1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int d = 0; d < 2 * DT; ++d) {
            add(0, d / DT, d % DT);
            if (d < DT) read_values(0, 1, d);
            else read_values(1, 0, d - DT);
        }
        weigh(1);
        STRETCH(2 * DT * EACH, 2 / EACH, (56 + WEIGH) / (2 * DT * EACH))
        pin(1);
        asm volatile("" : "+v"(l));
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int d = 0; d < 2 * DT; ++d) {
            add(1, d / DT, d % DT);
            if (d < DT) read_values(1, 1, d);
        }
        top = max_halves(fmaxf(part, largest(1))) * scale;
        STRETCH(DT * EACH, 2 / EACH, 2 / EACH)
        STRETCH(DT * EACH, 0, 2 / EACH)
        asm volatile("" : "+v"(top));
        __builtin_amdgcn_sched_barrier(0);
#undef STRETCH
        __builtin_amdgcn_sched_barrier(0);
#endif
    }
    if (left <= 0) return;
    move();  // (sums of 2^100 and more would not join with those of other blocks)
    l = add_halves(l);
    if (bare) m = -__builtin_inff();
    bool bad = not_finite(l);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) bad |= not_finite(o[d][e]);
    uint64_t redo = __ballot(bad && n < left);
    redo = (redo | redo >> 32) & 0xffffffffu;

    // ---- results: lane (h, n), word e of o[d]: element 32 d + 8 (e / 4) + 4 h + e % 4 of row n ----
    if (n < left && !(redo >> n & 1)) {  // (a row is written once: `out` may be q, which the exact row reads)
        if (uncut) {
            const float inv = a.blind(p) ? 0.0f : 1.0f / l;
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
            if (h == 0) a.part_ml[prow * 2] = m, a.part_ml[prow * 2 + 1] = a.blind(p) ? PART_EMPTY : l;
        }
    }
    while (redo) {
        const int c = __ffsll((unsigned long long)redo) - 1;
        redo &= redo - 1;
        const int rc = row0 + c, ic = rc / a.group, hc = kv_head * a.group + rc - ic * a.group;
        const int64_t tc = (SHARED ? b : a.first_row(b)) + ic;
        const int pc = position(ic);
        float me, le, v[D / 64];
        exact_row<true, D, KT>(a, tiles, x0, x1, 1, b, kv_head, pc, a.q + tc * a.q_bytes + (int64_t)hc * (D * 2), me, le, v, keys);
        if (uncut) {
            const float inv = a.blind(pc) ? 0.0f : 1.0f / le;
            uint16_t *out = reinterpret_cast<uint16_t *>(a.out + tc * a.out_bytes + (int64_t)hc * (D * 2)) + lane * (D / 64);
#pragma unroll
            for (int e = 0; e < D / 64; ++e) out[e] = (uint16_t)f32_to_bf16_bits(v[e] * inv);
        } else {
            const int64_t prow = (int64_t)split * part_rows + tc * a.heads + hc;
#pragma unroll
            for (int e = 0; e < D / 64; ++e) a.part_o[prow * D + lane * (D / 64) + e] = v[e];
            if (lane == 0) a.part_ml[prow * 2] = me, a.part_ml[prow * 2 + 1] = a.blind(pc) ? PART_EMPTY : le;
        }
    }
}

static inline bool tile_aligned(const KvView &kv) {
    return kv.page_size % 16 == 0 && kv.page_bytes < (1ll << 32) && kv.page_size * kv.slot_bytes < (1ll << 32);
}

}  // namespace c2r
