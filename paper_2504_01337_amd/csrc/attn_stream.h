// Attention whose keys and values go straight from memory into the matrix instructions' operand registers.
//
// Sixteen query rows are the columns of every product: S^T = K q^T with v_mfma_f32_16x16x32_bf16 (16x16x4_f32), rows = keys.
// Its result leaves lane (g = lane / 16, n = lane % 16) with keys 4g .. 4g + 3 of row n, which is how the second product
// o^T = V^T p wants its weights if the keys of a step are counted in that order: no lane hands p to another.  A sum over
// keys may take them in any order, so V is simply loaded in the same one.  Elements of D are permuted likewise: a lane loads
// whole 16-byte pieces of K and V rows, and in bf16 turns its 8 keys x 8 elements of V in registers (v_perm_b32).
//
// A tile is 16 KB of loads per wave (D = 128); the next one's are in flight while one is worked on.
#pragma once
#include "attn_common.h"

namespace c2r {

template <bool BF16, int D>
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

    // Lane l looks after key l % KT of a tile: its entry of the page table, then where its row lies.  Keys past the last visible
    // one stand for that one, and are masked.
    __device__ static __forceinline__ int look_up(const AttnCall &a, int b, int base, int last) {
        return a.kv.page(b, min(base + (lane_id() & (KT - 1)), last));
    }
    __device__ static __forceinline__ int64_t place(const AttnCall &a, int page, int64_t head_off, int base, int last) {
        return a.kv.offset(page, min(base + (lane_id() & (KT - 1)), last)) + head_off;
    }
    // The row of key `from` (in units of 4: lane numbers as the exchange counts them).
    __device__ static __forceinline__ int64_t of_lane(int64_t at, int from) {
#if defined(__HIP_DEVICE_COMPILE__)
        const uint32_t lo = __builtin_amdgcn_ds_bpermute(from, (int)at), hi = __builtin_amdgcn_ds_bpermute(from, (int)(at >> 32));
        return (int64_t)((uint64_t)hi << 32 | lo);
#else
        return at + from;
#endif
    }

    __device__ static __forceinline__ void load_keys(const AttnCall &a, Tile &t, int64_t at) {
        const int g = lane_id() >> 4, n = lane_id() & 15;
#pragma unroll
        for (int s = 0; s < SUB; ++s) {
            const unsigned char *row = a.kv.k + of_lane(at, 4 * n + 64 * s) + g * 16;
#pragma unroll
            for (int i = 0; i < KSTEPS; ++i) t.k[s][i] = *reinterpret_cast<const u32x4 *>(row + i * 64);
        }
    }

    __device__ static __forceinline__ void load_values(const AttnCall &a, Tile &t, int64_t at) {
        const int g = lane_id() >> 4, n = lane_id() & 15;
#pragma unroll
        for (int r = 0; r < VKEYS; ++r) {
            const unsigned char *row = a.kv.v + of_lane(at, 16 * g + 64 * (r >> 2) + 4 * (r & 3)) + n * (VEL * SZ);
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

    __device__ static __forceinline__ void scores(const Tile &t, const u32x4 (&q)[KSTEPS], f32x4 (&s)[SUB]) {
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
    }

    // Scores to weights w; the sums so far are rescaled to the new maximum.
    __device__ static __forceinline__ void weights(const AttnCall &a, const f32x4 (&s)[SUB], State &st, int base, int p, bool whole,
                                                   float (&w)[VKEYS]) {
        const int g = lane_id() >> 4;
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
#pragma unroll
        for (int r = 0; r < VKEYS; ++r) w[r] = __builtin_amdgcn_exp2f(x[r] - ref);
#pragma unroll
        for (int r = 0; r < VKEYS; ++r) st.l += w[r];
    }

    __device__ static __forceinline__ void add_values(const Tile &t, const float (&w)[VKEYS], State &st) {
#if defined(__HIP_DEVICE_COMPILE__)
        if constexpr (BF16) {
            // the matrix pipe takes the weights in two bf16 pieces, the rounded weight and what is left of it: 2^-16 of each at most is
            // lost, far below the output's own rounding (2^-8), and this kernel's memory-bound loop has the time for both products
            u32x4 pw, rest;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                pw[c] = pack_bf16x2(w[2 * c], w[2 * c + 1]);
                rest[c] = pack_bf16x2(w[2 * c] - __uint_as_float(pw[c] << 16), w[2 * c + 1] - __uint_as_float(pw[c] & 0xffff0000u));
            }
#pragma unroll
            for (int i = 0; i < VEL; ++i) {
                const uint32_t sel = i & 1 ? 0x07060302u : 0x05040100u;
                u32x4 vt;
#pragma unroll
                for (int c = 0; c < 4; ++c) vt[c] = __builtin_amdgcn_perm(t.v[2 * c + 1][i >> 1], t.v[2 * c][i >> 1], sel);
                st.o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vt), __builtin_bit_cast(bf16x8, pw), st.o[i], 0, 0, 0);
                st.o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vt), __builtin_bit_cast(bf16x8, rest), st.o[i], 0, 0, 0);
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

    // The tiles [x0, x1) of a row of blocks, tiles apart by STEP.
    template <int STEP>
    __device__ static __forceinline__ void run(const AttnCall &a, const u32x4 (&q)[KSTEPS], State &st, const KeyTiles<KT> &tiles, int x0, int x1,
                                               int b, int64_t head_off, int p, int p_min, int p_max) {
        const int last = a.last_key(p_max);
        // A tile's key registers are free once its scores are there, its value registers once they are added: the next
        // tile's rows are asked for at these two places, so one tile's registers keep a tile's loads in flight all the time.
        // Loads come back in the order they were sent; page numbers are asked for two tiles ahead, for when their rows are
        // wanted they would wait for everything in flight.  No load of the loop is conditional, so that the counts of loads in
        // flight, by which the compiler waits, are known.
        const int count = x0 < x1 ? (x1 - x0 + STEP - 1) / STEP : 0;
        if (count == 0) return;
        auto base = [&](int i) { return tiles.base(x0 + min(i, count - 1) * STEP); };
        auto pages = [&](int i) { return look_up(a, b, base(i), last); };
        Tile t;
        f32x4 s[SUB];
        float w[VKEYS];
        const int page = pages(0);
        int next = pages(1);
        const int64_t first = place(a, page, head_off, base(0), last);
        load_keys(a, t, first);
        load_values(a, t, first);
        for (int i = 0; i + 1 < count; ++i) {
            const int after = pages(i + 2);
            scores(t, q, s);
            const int64_t at = place(a, next, head_off, base(i + 1), last);
            load_keys(a, t, at);
            weights(a, s, st, base(i), p, tile_whole<KT>(a, base(i), p_min, p_max), w);
            add_values(t, w, st);
            load_values(a, t, at);
            next = after;
        }
        scores(t, q, s);
        weights(a, s, st, base(count - 1), p, tile_whole<KT>(a, base(count - 1), p_min, p_max), w);
        add_values(t, w, st);
    }

    __device__ static __forceinline__ void clear(State &st) {
#pragma unroll
        for (int e = 0; e < VEL; ++e) st.o[e] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        st.m = -__builtin_inff();
        st.l = 0.0f;
    }

    // After the last tile: the denominators over all keys; which of the first `left` rows did not come out finite, a bit each.
    __device__ static __forceinline__ uint32_t finish(State &st, int left) {
        st.l += __shfl_xor(st.l, 16);
        st.l += __shfl_xor(st.l, 32);
        bool bad = not_finite(st.l);
#pragma unroll
        for (int e = 0; e < VEL; ++e)
#pragma unroll
            for (int r = 0; r < 4; ++r) bad |= not_finite(st.o[e][r]);
        uint64_t redo = __ballot(bad && (lane_id() & 15) < left);
        redo |= redo >> 32;
        return (uint32_t)(redo | redo >> 16) & 0xffffu;
    }
};

// N elements of a row.
template <bool BF16, int N>
__device__ __forceinline__ void store_elements(unsigned char *p, const float *v) {
    if constexpr (BF16 && N == 1) {
        *reinterpret_cast<uint16_t *>(p) = (uint16_t)f32_to_bf16_bits(v[0]);
    } else if constexpr (BF16) {
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

}  // namespace c2r
