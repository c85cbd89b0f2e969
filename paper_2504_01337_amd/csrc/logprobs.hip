// Log probabilities of given tokens, the entropy and the n largest, from rows of logits, in one pass over them:
//     M = max l,  s = sum e^(l - M),  u = sum e^(l - M) (l - M),   log p = l - M - ln s,   H = ln s - u / s
// A lane keeps sums of its own, in powers of two, against a reference of its own: the largest of its first logits, moved on only where a
// later one is far above it (2^16 in a 32-bit sum lose nothing), so that no logit waits for a maximum.  The lanes' largest logits, which the
// sums want anyway, bound the n-th largest of the row from below: only lanes whose largest is not under the n-th largest of these are
// looked through again, some n of 256.  Rows are cut into parts where there are few; a second launch joins them.
// Bound by memory for many rows: 4096 rows of 128200 in bf16 171 us (6.1 TB/s).  251 rows of 50257 in fp32, five alternatives: 14.4 us and 4 for the
// join (50 MB); one row of 151936 in bf16, twenty: 7.4 and 3.9, latency.
#include "c2r_internal.h"

namespace c2r {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int LP_THREADS = 256, LP_MOST_TOP = 64, LP_MOST_PARTS = 64, LP_CANDIDATES = 1024;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

typedef unsigned long long Key;  // a logit and its token, see key_of

struct LogitsCall {
    const unsigned char *logits;
    int64_t row_bytes, T;
    const int32_t *tokens;
    float *logprob, *entropy, *top_logprob;
    int32_t *top_token;
    int V, given, n, parts;
    // of every row and part: {M, s, u, -}, and its n largest
    f32x4 *stats;
    Key *part_keys;
};

// A logit and its token as one number, larger for what comes first: the larger logit, the lower index of equal ones (zeros of either
// sign are equal).  0: none.
__device__ __forceinline__ uint32_t in_order(float v) {
    const uint32_t b = __float_as_uint(v + 0.0f);  // (-0 + 0 = 0)
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_order(uint32_t b) { return __uint_as_float(b ^ ((uint32_t)((int32_t)~b >> 31) | 0x80000000u)); }
constexpr uint32_t LOWEST = 0x007fffffu;  // of -infinity
__device__ __forceinline__ Key key_of(float v, int token) { return (Key)in_order(v) << 32 | (uint32_t)~token; }
__device__ __forceinline__ int token_of(Key k) { return (int)~(uint32_t)k; }
__device__ __forceinline__ float logit_of(Key k) { return from_order((uint32_t)(k >> 32)); }

// Over the 64 lanes, in every lane: the largest, the sum (in one order).
template <bool MAX>
__device__ __forceinline__ float wave_all(float v) {
#if defined(__HIP_DEVICE_COMPILE__)
    auto step = [&](auto moved) {
        const float o = __uint_as_float((uint32_t)moved);
        v = MAX ? fmaxf(v, o) : v + o;
    };
    const int none = MAX ? (int)0xff800000u : 0;
    step(__builtin_amdgcn_update_dpp(none, (int)__float_as_uint(v), 0x111, 0xf, 0xf, false));  // row_shr:1, 2, 4, 8
    step(__builtin_amdgcn_update_dpp(none, (int)__float_as_uint(v), 0x112, 0xf, 0xf, false));
    step(__builtin_amdgcn_update_dpp(none, (int)__float_as_uint(v), 0x114, 0xf, 0xf, false));
    step(__builtin_amdgcn_update_dpp(none, (int)__float_as_uint(v), 0x118, 0xf, 0xf, false));
    step(__builtin_amdgcn_update_dpp(none, (int)__float_as_uint(v), 0x142, 0xa, 0xf, false));  // row_bcast:15 into rows 1, 3
    step(__builtin_amdgcn_update_dpp(none, (int)__float_as_uint(v), 0x143, 0xc, 0xf, false));  // row_bcast:31 into rows 2, 3
    v = __uint_as_float(__builtin_amdgcn_readlane((int)__float_as_uint(v), 63));
#endif
    return v;
}

// A lower bound of the n-th largest of 64 lanes' numbers (EACH of a lane's), in their order: its first 16 bits in bf16, 24 in fp32, one after another.
// In bf16 these are all that a number has (behind them stand ones if it is negative), so that is the n-th largest itself.  Every lane must be active.
template <bool BF16, int EACH>
__device__ __forceinline__ uint32_t wave_nth(const uint32_t (&mine)[EACH], int n) {
    uint32_t at = 0;
#pragma unroll
    for (int bit = 31; bit >= (BF16 ? 16 : 8); --bit) {
        const uint32_t next = at | 1u << bit;
        int reach = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) reach += __popcll(__ballot(mine[i] >= next));
        if (reach >= n) at = next;
    }
    return BF16 && !(at >> 31) ? at | 0xffffu : at;
}

// The same, and one of the numbers: many that are equal are then equal to it.
template <bool BF16, int EACH>
__device__ __forceinline__ float wave_nth_of(const uint32_t (&mine)[EACH], int n) {
    const uint32_t at = wave_nth<BF16>(mine, n);
    if (at <= LOWEST) return -__builtin_inff();
    if constexpr (BF16) return from_order(at);
    float least = __builtin_inff();
#pragma unroll
    for (int i = 0; i < EACH; ++i) least = mine[i] >= at ? fminf(least, from_order(mine[i])) : least;
    return -wave_all<true>(-least);
}

// STREAMED: each logit is wanted once and there are many: they pass by the caches (4096 rows of 128200 in bf16: 171 us, and 194 the other way).
template <bool BF16, bool STREAMED = false>
struct Row {
    static constexpr int SZ = BF16 ? 2 : 4, N = 16 / SZ;  // elements of a 16-byte piece
    const unsigned char *at;
    int V, head, pieces;  // elements before the first whole piece, and the pieces
    __device__ Row(const LogitsCall &a, int64_t t) : at(a.logits + t * a.row_bytes), V(a.V) {
        head = min((int)((0 - (uintptr_t)at) & 15) / SZ, V);
        pieces = (V - head) / N;
    }
    __device__ int tail() const { return V - head - pieces * N; }
    __device__ float element(int i) const {
        if constexpr (BF16) return bf16_bits_to_f32(reinterpret_cast<const uint16_t *>(at)[i]);
        return reinterpret_cast<const float *>(at)[i];
    }
    __device__ u32x4 piece(int p) const {
        const u32x4 *from = reinterpret_cast<const u32x4 *>(at + ((int64_t)head + (int64_t)p * N) * SZ);
        if constexpr (STREAMED) return __builtin_nontemporal_load(from);
        return *from;
    }
    __device__ static void open(const u32x4 &w, float (&v)[N]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (BF16) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            else v[i] = __uint_as_float(w[i]);
        }
    }
};

// A lane's sums, in powers of two against `ref`.
struct Sums {
    float top, limit, ref, s, u;
    __device__ __forceinline__ void clear() { top = limit = -__builtin_inff(), ref = s = u = 0.0f; }
    template <int N>
    __device__ __forceinline__ void add(const float (&v)[N]) {
        float here = v[0];
#pragma unroll
        for (int i = 1; i < N; ++i) here = fmaxf(here, v[i]);
        top = fmaxf(top, here);
        if (__any(here > limit)) {
            if (here > limit) {
                // (a masked logit, the type's lowest, has no power of two: sums are against 0 until another comes)
                const float to = fmaxf(here * LOG2E, -1e30f), d = ref - to;
                const float f = s == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(d);
                u = __builtin_fmaf(s, d, u) * f;
                s *= f;
                ref = to, limit = here + 11.0f;
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float t = __builtin_fmaf(v[i], LOG2E, -ref), e = __builtin_amdgcn_exp2f(t);
            s += e;
            u = __builtin_fmaf(e, fmaxf(t, -200.0f), u);  // (e is 0 long before; 0 times -infinity is no number)
        }
    }
};

// The sums of a block's lanes, against its largest logit M: {M, s, u, -} in every thread.  from: what a lane's own sums are against less the
// given M, in powers of two.
template <class From>
__device__ __forceinline__ f32x4 block_sums(float top, float s, float u, const From &from, f32x4 *lds) {
    // (nothing to move where there is no sum, or where nothing is left of it: 0 times an infinity is no number)
    auto against = [](float d, float &s, float &u) {
        const float f = s == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(d);
        u = f == 0.0f ? 0.0f : __builtin_fmaf(s, d, u) * f;
        s *= f;
    };
    const float wave_top = wave_all<true>(top);
    against(from(wave_top), s, u);
    s = wave_all<false>(s), u = wave_all<false>(u);
    if (lane_id() == 0) lds[threadIdx.x >> 6] = f32x4{wave_top, s, u, 0.0f};
    __syncthreads();
    f32x4 all = {-__builtin_inff(), 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < 4; ++w) all[0] = fmaxf(all[0], lds[w][0]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        f32x4 v = lds[w];
        float vs = v[1], vu = v[2];
        against((v[0] - all[0]) * LOG2E, vs, vu);
        all[1] += vs, all[2] += vu;
    }
    return all;
}
__device__ __forceinline__ float block_sum(float v, float *lds) {
    v = wave_all<false>(v);
    __syncthreads();
    if (lane_id() == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return lds[0] + lds[1] + (lds[2] + lds[3]);
}

// The candidates' n first in order, written by put(place, key); places that no candidate fills get key 0.
template <class Put>
__device__ __forceinline__ void put_in_order(const Key *keys, int count, int n, const Put &put) {
    for (int i = threadIdx.x; i < count; i += LP_THREADS) {
        const Key k = keys[i];
        int rank = 0;
        for (int j = 0; j < count; ++j) rank += keys[j] > k;
        if (rank < n) put(rank, k);
    }
    for (int i = count + threadIdx.x; i < n; i += LP_THREADS) put(i, 0);
}

// A place among the candidates for every lane that has one.
__device__ __forceinline__ int take_place(bool wants, int *count) {
    const uint64_t here = __ballot(wants);
    int at = 0;
    if (wants && lane_id() == __ffsll((unsigned long long)here) - 1) at = atomicAdd(count, __popcll(here));
    if (!wants) return 0;
    return __builtin_amdgcn_readfirstlane(at) + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(here >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)here, 0));
}

// What the sums say of a row: the entropy, and lane by lane the given tokens (first: the lane's first one's logit).
template <class R>
__device__ __forceinline__ float given_logit(const LogitsCall &a, int64_t t, const R &row, int g) {
    const int tok = a.tokens[t * a.given + g];
    return (uint32_t)tok < (uint32_t)a.V ? row.element(tok) : -__builtin_inff();
}
template <class R>
__device__ __forceinline__ void put_row(const LogitsCall &a, int64_t t, const R &row, float first, float M, float s, float u, float ln_s) {
    if (threadIdx.x == 0 && a.entropy) a.entropy[t] = ln_s - u / s * LN2;
    for (int g = threadIdx.x; g < a.given; g += LP_THREADS) {
        const float l = g == (int)threadIdx.x ? first : given_logit(a, t, row, g);
        a.logprob[t * a.given + g] = (uint32_t)a.tokens[t * a.given + g] < (uint32_t)a.V ? l - M - ln_s : -__builtin_inff();
    }
}

template <bool BF16, bool STREAMED>
__global__ __launch_bounds__(LP_THREADS) void logprobs_kernel(LogitsCall a) {
    using R = Row<BF16, STREAMED>;
    constexpr int N = R::N, AHEAD = STREAMED ? 8 : 4;
    __shared__ f32x4 wave_sums[4];
    __shared__ float tops[LP_THREADS], wave_lds[4];
    __shared__ Key cand[LP_CANDIDATES], wave_keys[4];
    __shared__ int list[LP_THREADS], counts[2], wave_counts[4];
    const int64_t t = blockIdx.x / a.parts;
    const int part = (int)(blockIdx.x - t * a.parts), tid = threadIdx.x;
    const R row(a, t);
    const bool whole = a.parts == 1;
    // this part's pieces; the first part has the elements before them, the last one those behind
    const int each = (row.pieces + a.parts - 1) / a.parts, p0 = min(part * each, row.pieces), p1 = min(p0 + each, row.pieces);
    const int head = part == 0 ? row.head : 0, tail = part == a.parts - 1 ? row.tail() : 0;
    const int extra = tid < head ? tid : tid >= 128 && tid < 128 + tail ? row.V - tail + tid - 128 : -1;
    float first = 0.0f;
    if (whole && tid < a.given) first = given_logit(a, t, row, tid);
    Sums sums;
    sums.clear();
    int p = p0 + tid;
    for (; p + (AHEAD - 1) * LP_THREADS < p1; p += AHEAD * LP_THREADS) {
        u32x4 w[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) w[i] = row.piece(p + i * LP_THREADS);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            float v[N];
            R::open(w[i], v);
            sums.add(v);
        }
    }
    if (p < p1) {  // what is left: AHEAD - 1 pieces at most, asked for together
        u32x4 w[AHEAD - 1];
#pragma unroll
        for (int i = 0; i < AHEAD - 1; ++i) w[i] = row.piece(min(p + i * LP_THREADS, p1 - 1));
#pragma unroll
        for (int i = 0; i < AHEAD - 1; ++i) {
            if (p + i * LP_THREADS >= p1) break;
            float v[N];
            R::open(w[i], v);
            sums.add(v);
        }
    }
    if (extra >= 0) {
        const float v[1] = {row.element(extra)};
        sums.add(v);
    }
    tops[tid] = sums.top;
    if (tid < 2) counts[tid] = 0;
    const f32x4 all = block_sums(sums.top, sums.s, sums.u, [&](float M) { return __builtin_fmaf(-M, LOG2E, sums.ref); }, wave_sums);
    const float M = all[0];
    float s = all[1], u = all[2];
    if (M != -__builtin_inff() ? !(s > 0.0f && s < __builtin_inff() && fabsf(u) < __builtin_inff()) : s != 0.0f) {
        // powers of two of these logits are out of range (all of them the type's lowest, say), or there is an infinity or a NaN: by the
        // definition, which gives a NaN for those
        s = u = 0.0f;
        auto add = [&](float x) {
            const float t2 = (x - M) * LOG2E, e = x == -__builtin_inff() && M != x ? 0.0f : __builtin_amdgcn_exp2f(t2);
            s += e;
            u = __builtin_fmaf(e, fmaxf(t2, -200.0f), u);
        };
        for (p = p0 + tid; p < p1; p += LP_THREADS) {
            float v[N];
            R::open(row.piece(p), v);
            for (int i = 0; i < N; ++i) add(v[i]);
        }
        if (extra >= 0) add(row.element(extra));
        s = block_sum(s, wave_lds), u = block_sum(u, wave_lds);
    }
    const float ln_s = logf(s);
    if (whole) put_row(a, t, row, first, M, s, u, ln_s);
    else if (tid == 0) a.stats[t * a.parts + part] = f32x4{M, s, u, 0.0f};
    if (a.n == 0) return;

    // ---- the n largest ----
    // a number that n logits at least reach: of every four lanes' largest the n-th, which few others reach while n is small beside 64, or of every lane's
    // (109 rows of 63989 in bf16, 64 alternatives: 22.5 us, and 52 the other way)
    float limit = M;
    if (a.n > 1) {
        const int lane = lane_id();
        if (a.n <= 16) {
            const uint32_t four[1] = {in_order(fmaxf(fmaxf(tops[lane], tops[lane + 64]), fmaxf(tops[lane + 128], tops[lane + 192])))};
            limit = wave_nth_of<BF16>(four, a.n);
        } else {
            const uint32_t each[4] = {in_order(tops[lane]), in_order(tops[lane + 64]), in_order(tops[lane + 128]), in_order(tops[lane + 192])};
            limit = wave_nth_of<BF16>(each, a.n);
        }
    }
    const bool listed = (p0 + tid < p1 || extra >= 0) && sums.top >= limit;
    const int place = take_place(listed, &counts[0]);
    if (listed) list[place] = tid;
    __syncthreads();
    const int lanes = counts[0], rounds = p1 > p0 ? (p1 - p0 + LP_THREADS - 1) / LP_THREADS : 0;
    // candidates: the listed lanes' logits from the limit on, or above it
    auto collect = [&](bool above) {
        auto take = [&](float v, int tok) {
            if (above ? v > limit : v >= limit) {
                const int to = atomicAdd(&counts[1], 1);
                if (to < LP_CANDIDATES) cand[to] = key_of(v, tok);
            }
        };
        const int all = lanes * rounds;
        for (int j0 = tid; j0 < all; j0 += AHEAD * LP_THREADS) {
            u32x4 w[AHEAD];
            int at[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int j = j0 + i * LP_THREADS, q = j / lanes;
                at[i] = j < all ? p0 + q * LP_THREADS + list[j - q * lanes] : p1;
                w[i] = row.piece(min(at[i], p1 - 1));
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                if (at[i] >= p1) continue;
                float v[N], top;
                R::open(w[i], v);
                top = v[0];
#pragma unroll
                for (int e = 1; e < N; ++e) top = fmaxf(top, v[e]);
                if (top < limit) continue;
#pragma unroll 1
                for (int e = 0; e < N; ++e) {
                    float x = v[0];
#pragma unroll
                    for (int k = 1; k < N; ++k) x = e == k ? v[k] : x;
                    take(x, row.head + at[i] * N + e);
                }
            }
        }
        if (extra >= 0) take(row.element(extra), extra);
        __syncthreads();
        return counts[1];
    };
    int count = limit == -__builtin_inff() ? LP_CANDIDATES + 1 : collect(false);
    if (count > LP_CANDIDATES) {
        // many equal ones at the limit: what is above it, then as many of them as are wanted, in order
        __syncthreads();
        if (tid == 0) counts[1] = 0;
        __syncthreads();
        count = collect(true);
        if (count <= LP_CANDIDATES) {
            int want = a.n - count;
            auto next = [&](bool here, const float *v, int tokens, int first) {  // each thread's `tokens` logits from `first` on, threads in order
                int mine = 0;
                if (here)
                    for (int e = 0; e < tokens; ++e) mine += v[e] == limit;
                const int upto = wave_inclusive_scan(mine);
                __syncthreads();
                if (lane_id() == 63) wave_counts[tid >> 6] = upto;
                __syncthreads();
                int place = upto - mine, total = 0;
                for (int w = 0; w < 4; ++w) place += w < tid >> 6 ? wave_counts[w] : 0, total += wave_counts[w];
                if (here)
                    for (int e = 0; e < tokens; ++e)
                        if (v[e] == limit) {
                            if (place < want) cand[count + place] = key_of(limit, first + e);
                            ++place;
                        }
                const int taken = min(max(want, 0), total);
                count += taken, want -= taken;
            };
            float one = 0.0f;
            if (extra >= 0) one = row.element(extra);
            next(tid < head, &one, 1, extra);
            for (int q = p0; q < p1 && want > 0; q += LP_THREADS) {
                float v[N] = {};
                if (q + tid < p1) R::open(row.piece(q + tid), v);
                next(q + tid < p1, v, N, row.head + (q + tid) * N);
            }
            next(extra >= 0 && tid >= head, &one, 1, extra);
        } else {
            // more above it than there is room for (large logits side by side in one lane's pieces): one token after another
            Key last = ~0ull;
            count = 0;
            for (int k = 0; k < a.n; ++k) {
                Key best = 0;
                auto look = [&](float v, int tok) {
                    const Key here = key_of(v, tok);
                    if (v == v && here < last && here > best) best = here;
                };
                for (int q = p0 + tid; q < p1; q += LP_THREADS) {
                    float v[N];
                    R::open(row.piece(q), v);
                    for (int e = 0; e < N; ++e) look(v[e], row.head + q * N + e);
                }
                if (extra >= 0) look(row.element(extra), extra);
                for (int w = 32; w; w >>= 1) {
                    const Key o = __shfl_xor(best, w);
                    if (o > best) best = o;
                }
                __syncthreads();
                if (lane_id() == 0) wave_keys[tid >> 6] = best;
                __syncthreads();
                for (int w = 0; w < 4; ++w)
                    if (wave_keys[w] > best) best = wave_keys[w];
                if (best == 0) break;
                if (tid == 0) cand[k] = best;
                last = best, count = k + 1;
            }
        }
        __syncthreads();
    }
    const int64_t out = (whole ? t : t * a.parts + part) * a.n;
    put_in_order(cand, count, a.n, [&](int place, Key k) {
        if (whole) a.top_token[out + place] = k ? token_of(k) : -1, a.top_logprob[out + place] = k ? logit_of(k) - M - ln_s : __builtin_nanf("");
        else a.part_keys[out + place] = k;
    });
}

// The parts of a row.  What it reads from memory is asked for at its start.
template <bool BF16>
__global__ __launch_bounds__(LP_THREADS) void logprobs_join_kernel(LogitsCall a) {
    constexpr int HELD = 4;
    __shared__ f32x4 wave_sums[4];
    __shared__ Key cand[LP_MOST_PARTS * LP_MOST_TOP];
    __shared__ int count;
    const int64_t t = blockIdx.x;
    const int tid = threadIdx.x, lane = lane_id(), entries = a.parts * a.n;
    const Row<BF16> row(a, t);
    const Key *keys = a.part_keys + t * entries;
    const f32x4 mine = tid < a.parts ? a.stats[t * a.parts + tid] : f32x4{-__builtin_inff(), 0.0f, 0.0f, 0.0f};
    // of every part the entry up to which all parts together have n
    const int firsts = (a.n + a.parts - 1) / a.parts;
    const Key bound = a.n > 0 && lane < a.parts ? keys[lane * a.n + firsts - 1] : 0;
    Key held[HELD];
#pragma unroll
    for (int i = 0; i < HELD; ++i) held[i] = tid + i * LP_THREADS < entries ? keys[tid + i * LP_THREADS] : 0;
    float first = 0.0f;
    if (tid < a.given) first = given_logit(a, t, row, tid);
    if (tid == 0) count = 0;
    const f32x4 all = block_sums(mine[0], mine[1], mine[2], [&](float M) { return (mine[0] - M) * LOG2E; }, wave_sums);
    const float M = all[0], s = all[1], u = all[2], ln_s = logf(s);
    put_row(a, t, row, first, M, s, u, ln_s);
    if (a.n == 0) return;
    uint32_t limit = (uint32_t)(bound >> 32);
    if (firsts == 1) {
        const uint32_t one[1] = {limit};
        limit = wave_nth<BF16>(one, a.n);
    } else {
        if (lane >= a.parts) limit = ~0u;
        for (int w = 32; w; w >>= 1) limit = min(limit, (uint32_t)__shfl_xor((int)limit, w));
    }
    auto take = [&](Key k) {
        const bool wants = k != 0 && (uint32_t)(k >> 32) >= limit;
        const int to = take_place(wants, &count);
        if (wants) cand[to] = k;
    };
#pragma unroll
    for (int i = 0; i < HELD; ++i) take(held[i]);
    for (int i = HELD * LP_THREADS + tid; i < entries; i += LP_THREADS) take(keys[i]);
    __syncthreads();
    put_in_order(cand, count, a.n, [&](int place, Key k) {
        a.top_token[t * a.n + place] = k ? token_of(k) : -1, a.top_logprob[t * a.n + place] = k ? logit_of(k) - M - ln_s : __builtin_nanf("");
    });
}

// Parts of a row: as many as make 1024 blocks, of some 4096 logits at least (of 2049 where V is 4097).  us with 1024, 2048 and 4096 blocks: 251 rows of 50257 in fp32 18.5, 19.7, 21.6; 1100 rows of
// 50257 in bf16 28.7, 35.1, 36.8; 1900 of 32000 30.9, 40.7, 40.9; one row of 151936 in parts of 4096, 8192: 11.2, 13.0.
static int logprobs_parts(int64_t T, int V) {
    int64_t n = T < 1 ? 1 : (1024 + T - 1) / T;
    const int64_t most = (V + 4095) / 4096;
    if (n > most) n = most;
    return (int)(n < 1 ? 1 : n > LP_MOST_PARTS ? LP_MOST_PARTS : n);
}

size_t logprobs_workspace_bytes(int64_t T, int V, int n) {
    if (T <= 0 || V <= 0) return 0;
    const int parts = logprobs_parts(T, V);
    return parts == 1 ? 0 : round_up((size_t)T * parts * (16 + 8 * (size_t)(n > 0 ? n : 0)), 256);
}

}  // namespace c2r

using namespace c2r;

extern "C" int c2r_token_logprobs(const void *logits, c2r_dtype dt, int64_t stride, int64_t T, int V, const int32_t *tokens, int n_given, int n_top,
                                  float *logprob, float *entropy, int32_t *top_token, float *top_logprob, void *ws, size_t ws_bytes, void *stream) {
    drop_stale_error();
    if (dt != C2R_F32 && dt != C2R_BF16) return C2R_ERR_INVALID_ARG;
    if (T < 0 || V < 1 || n_given < 0 || n_top < 0 || n_top > V) return C2R_ERR_INVALID_ARG;
    if (T >= (1ll << 24) || V > (1 << 24) || n_top > LP_MOST_TOP || n_given > 1024) return C2R_ERR_UNSUPPORTED;
    if (T == 0) return C2R_OK;  // (arrays of no rows may have no address)
    if (n_given == 0 && n_top == 0 && !entropy) return C2R_ERR_INVALID_ARG;
    const int size = dt == C2R_BF16 ? 2 : 4;
    if (!logits || !aligned(logits, size) || stride < V || stride > (1ll << 40)) return C2R_ERR_INVALID_ARG;
    if (n_given > 0 && (!tokens || !logprob || !aligned(tokens, 4) || !aligned(logprob, 4))) return C2R_ERR_INVALID_ARG;
    if (n_top > 0 && (!top_token || !top_logprob || !aligned(top_token, 4) || !aligned(top_logprob, 4))) return C2R_ERR_INVALID_ARG;
    if (entropy && !aligned(entropy, 4)) return C2R_ERR_INVALID_ARG;
    LogitsCall a = {};
    a.logits = static_cast<const unsigned char *>(logits);
    a.row_bytes = stride * size, a.T = T;
    a.tokens = tokens, a.logprob = logprob, a.entropy = entropy, a.top_token = top_token, a.top_logprob = top_logprob;
    a.V = V, a.given = n_given, a.n = n_top, a.parts = logprobs_parts(T, V);
    if (a.parts > 1) {
        if (!ws || !aligned(ws, 256) || ws_bytes < (size_t)T * a.parts * (16 + 8 * (size_t)n_top)) return C2R_ERR_WORKSPACE;
        a.stats = static_cast<f32x4 *>(ws);
        a.part_keys = reinterpret_cast<Key *>(a.stats + T * a.parts);
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)(T * a.parts)), rows((unsigned)T), block(LP_THREADS);
    const bool streamed = T * V * size >= 4 * STREAMED_BYTES;
    if (dt == C2R_BF16) streamed ? logprobs_kernel<true, true><<<grid, block, 0, st>>>(a) : logprobs_kernel<true, false><<<grid, block, 0, st>>>(a);
    else streamed ? logprobs_kernel<false, true><<<grid, block, 0, st>>>(a) : logprobs_kernel<false, false><<<grid, block, 0, st>>>(a);
    const int rc = launch_status();
    if (rc != C2R_OK || a.parts == 1) return rc;
    if (dt == C2R_BF16) logprobs_join_kernel<true><<<rows, block, 0, st>>>(a);
    else logprobs_join_kernel<false><<<rows, block, 0, st>>>(a);
    return launch_status();
}
