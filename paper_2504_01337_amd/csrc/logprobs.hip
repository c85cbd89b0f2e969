// Log probabilities of given tokens, the entropy and the n largest, from rows of logits, in one pass over them:
//     M = max l,  s = sum e^(l - M),  u = sum e^(l - M) (l - M),   log p = l - M - ln s,   H = ln s - u / s
// A lane keeps sums of its own, in powers of two, against a reference of its own: the largest of its first logits, moved on only where a
// later one is far above it (2^16 in a 32-bit sum lose nothing), so that no logit waits for a maximum.  The lanes' largest logits, which the
// sums want anyway, bound the n-th largest of the row from below: only lanes whose largest is not under the n-th largest of these are
// looked through again, some n of 256.  Rows are cut into parts where there are few; a second launch joins them.
#include "c2r_internal.h"

namespace c2r {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int LP_THREADS = 256, LP_MOST_TOP = 64, LP_MOST_PARTS = 64, LP_CANDIDATES = 1024;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct LogitsCall {
    const unsigned char *logits;
    int64_t row_bytes, T;
    const int32_t *tokens;
    float *logprob, *entropy, *top_logprob;
    int32_t *top_token;
    int V, given, n, parts;
    // of every row and part: {M, s, u, -}, and its n largest
    f32x4 *stats;
    float *part_value;
    int32_t *part_token;
};

// One token before another: the larger logit, the lower index of equal ones.
__device__ __forceinline__ bool before(float va, int ia, float vb, int ib) { return va > vb || (va == vb && ia < ib); }

template <bool BF16>
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
    __device__ u32x4 piece(int p) const { return *reinterpret_cast<const u32x4 *>(at + ((int64_t)head + (int64_t)p * N) * SZ); }
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

__device__ __forceinline__ float block_max(float v, float *lds) {
#pragma unroll
    for (int w = 32; w; w >>= 1) v = fmaxf(v, __shfl_xor(v, w));
    __syncthreads();
    if (lane_id() == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return fmaxf(fmaxf(lds[0], lds[1]), fmaxf(lds[2], lds[3]));
}
__device__ __forceinline__ float block_sum(float v, float *lds) {
#pragma unroll
    for (int w = 32; w; w >>= 1) v += __shfl_xor(v, w);
    __syncthreads();
    if (lane_id() == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return lds[0] + lds[1] + (lds[2] + lds[3]);
}

// The candidates' n first in order, written by put(place, value, token); places that no candidate fills get token -1.
template <class Put>
__device__ __forceinline__ void put_in_order(const float *value, const int *token, int count, int n, const Put &put) {
    for (int i = threadIdx.x; i < count; i += LP_THREADS) {
        const float v = value[i];
        const int tok = token[i];
        int rank = 0;
        for (int j = 0; j < count; ++j) rank += before(value[j], token[j], v, tok);
        if (rank < n) put(rank, v, tok);
    }
    for (int i = count + threadIdx.x; i < n; i += LP_THREADS) put(i, -__builtin_inff(), -1);
}

// What the sums say of a row: lane by lane the given tokens, and the entropy.
template <bool BF16>
__device__ __forceinline__ void put_row(const LogitsCall &a, int64_t t, const Row<BF16> &row, float M, float s, float u, float ln_s) {
    if (threadIdx.x == 0 && a.entropy) a.entropy[t] = ln_s - u / s * LN2;
    for (int g = threadIdx.x; g < a.given; g += LP_THREADS) {
        const int tok = a.tokens[t * a.given + g];
        a.logprob[t * a.given + g] = (uint32_t)tok < (uint32_t)a.V ? row.element(tok) - M - ln_s : -__builtin_inff();
    }
}

template <bool BF16>
__global__ __launch_bounds__(LP_THREADS) void logprobs_kernel(LogitsCall a) {
    using R = Row<BF16>;
    constexpr int N = R::N, AHEAD = 4;
    __shared__ float wave_lds[4], tops[LP_THREADS], cand_value[LP_CANDIDATES], shared_limit;
    __shared__ int list[LP_THREADS], cand_token[LP_CANDIDATES], counts[2], wave_counts[4];
    const int64_t t = blockIdx.x / a.parts;
    const int part = (int)(blockIdx.x - t * a.parts), tid = threadIdx.x;
    const R row(a, t);
    // this part's pieces; the first part has the elements before them, the last one those behind
    const int each = (row.pieces + a.parts - 1) / a.parts, p0 = min(part * each, row.pieces), p1 = min(p0 + each, row.pieces);
    const int head = part == 0 ? row.head : 0, tail = part == a.parts - 1 ? row.tail() : 0;
    const int extra = tid < head ? tid : tid >= 128 && tid < 128 + tail ? row.V - tail + tid - 128 : -1;
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
    for (; p < p1; p += LP_THREADS) {
        float v[N];
        R::open(row.piece(p), v);
        sums.add(v);
    }
    if (extra >= 0) {
        const float v[1] = {row.element(extra)};
        sums.add(v);
    }
    const float M = block_max(sums.top, wave_lds);
    float d = __builtin_fmaf(-M, LOG2E, sums.ref), f = sums.s == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(d);
    float u = block_sum(sums.s == 0.0f ? 0.0f : __builtin_fmaf(sums.s, d, sums.u) * f, wave_lds), s = block_sum(sums.s * f, wave_lds);
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
    const bool whole = a.parts == 1;
    const float ln_s = logf(s);
    if (whole) put_row<BF16>(a, t, row, M, s, u, ln_s);
    else if (tid == 0) a.stats[t * a.parts + part] = f32x4{M, s, u, 0.0f};
    if (a.n == 0) return;

    // ---- the n largest ----
    const bool holds = p0 + tid < p1 || extra >= 0;
    float limit = M;
    if (a.n > 1) {
        tops[tid] = sums.top;
        __syncthreads();
        int rank = 0;
        for (int j = 0; j < LP_THREADS; ++j) rank += before(tops[j], j, sums.top, tid);
        if (rank == a.n - 1) shared_limit = sums.top;
        __syncthreads();
        limit = shared_limit;
    }
    if (tid == 0) counts[0] = 0;
    __syncthreads();
    if (holds && sums.top >= limit) list[atomicAdd(&counts[0], 1)] = tid;
    __syncthreads();
    const int lanes = counts[0], rounds = p1 > p0 ? (p1 - p0 + LP_THREADS - 1) / LP_THREADS : 0;
    // candidates: the listed lanes' logits from the limit on, or above it
    auto collect = [&](bool above) {
        __syncthreads();
        if (tid == 0) counts[1] = 0;
        __syncthreads();
        auto take = [&](float v, int tok) {
            if (above ? v > limit : v >= limit) {
                const int to = atomicAdd(&counts[1], 1);
                if (to < LP_CANDIDATES) cand_value[to] = v, cand_token[to] = tok;
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
                float v[N];
                R::open(w[i], v);
#pragma unroll
                for (int e = 0; e < N; ++e) take(v[e], row.head + at[i] * N + e);
            }
        }
        if (extra >= 0) take(row.element(extra), extra);
        __syncthreads();
        return counts[1];
    };
    int count = limit == -__builtin_inff() ? LP_CANDIDATES + 1 : collect(false);
    if (count > LP_CANDIDATES) {
        // many equal ones at the limit: what is above it, then as many of them as are wanted, in order
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
                            if (place < want) cand_value[count + place] = limit, cand_token[count + place] = first + e;
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
            float last = __builtin_inff();
            int last_token = -1;
            count = 0;
            for (int k = 0; k < a.n; ++k) {
                float best = -__builtin_inff();
                int token = row.V;
                auto look = [&](float v, int tok) {
                    if (before(last, last_token, v, tok) && (token == row.V ? v == v : before(v, tok, best, token))) best = v, token = tok;
                };
                for (int q = p0 + tid; q < p1; q += LP_THREADS) {
                    float v[N];
                    R::open(row.piece(q), v);
                    for (int e = 0; e < N; ++e) look(v[e], row.head + q * N + e);
                }
                if (extra >= 0) look(row.element(extra), extra);
                for (int w = 32; w; w >>= 1) {
                    const float v = __shfl_xor(best, w);
                    const int tok = __shfl_xor(token, w);
                    if (before(v, tok, best, token)) best = v, token = tok;
                }
                __syncthreads();
                if (lane_id() == 0) wave_lds[tid >> 6] = best, wave_counts[tid >> 6] = token;
                __syncthreads();
                for (int w = 0; w < 4; ++w)
                    if (before(wave_lds[w], wave_counts[w], best, token)) best = wave_lds[w], token = wave_counts[w];
                if (token == row.V) break;
                if (tid == 0) cand_value[k] = best, cand_token[k] = token;
                last = best, last_token = token, count = k + 1;
            }
        }
        __syncthreads();
    }
    const int64_t out = (whole ? t : t * a.parts + part) * a.n;
    put_in_order(cand_value, cand_token, count, a.n, [&](int place, float v, int tok) {
        if (whole) a.top_token[out + place] = tok, a.top_logprob[out + place] = tok < 0 ? __builtin_nanf("") : v - M - ln_s;
        else a.part_value[out + place] = v, a.part_token[out + place] = tok;
    });
}

// The parts of a row.
template <bool BF16>
__global__ __launch_bounds__(LP_THREADS) void logprobs_join_kernel(LogitsCall a) {
    __shared__ float wave_lds[4], value[LP_MOST_PARTS * LP_MOST_TOP], some_value[2 * LP_MOST_TOP + LP_MOST_PARTS];
    __shared__ int token[LP_MOST_PARTS * LP_MOST_TOP], some_token[2 * LP_MOST_TOP + LP_MOST_PARTS], count, limit_token;
    __shared__ float limit_value;
    const int64_t t = blockIdx.x;
    const int tid = threadIdx.x;
    const Row<BF16> row(a, t);
    const f32x4 mine = tid < a.parts ? a.stats[t * a.parts + tid] : f32x4{-__builtin_inff(), 0.0f, 0.0f, 0.0f};
    const float M = block_max(mine[0], wave_lds);
    const float d = (mine[0] - M) * LOG2E, f = mine[1] == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(d);
    const float s = block_sum(mine[1] * f, wave_lds), u = block_sum(f == 0.0f ? 0.0f : __builtin_fmaf(mine[1], d, mine[2]) * f, wave_lds);
    const float ln_s = logf(s);
    put_row<BF16>(a, t, row, M, s, u, ln_s);
    if (a.n == 0) return;
    // the n-th of the first ones of every part bounds the row's n-th from below
    const int64_t from = t * a.parts * a.n;
    const int firsts = (a.n + a.parts - 1) / a.parts, some = firsts * a.parts;
    if (tid < some) {
        const int64_t at = from + tid / firsts * a.n + tid % firsts;
        some_value[tid] = a.part_value[at], some_token[tid] = a.part_token[at];
    }
    if (tid == 0) count = 0;
    __syncthreads();
    // (places without a token, -infinity and -1, come behind every token here)
    auto key = [&](int tok) { return tok < 0 ? 0x7fffffff : tok; };
    if (tid < some) {
        int rank = 0;
        for (int j = 0; j < some; ++j) rank += j != tid && (before(some_value[j], key(some_token[j]), some_value[tid], key(some_token[tid])) ||
                                                              (some_token[j] < 0 && some_token[tid] < 0 && j < tid));
        if (rank == a.n - 1) limit_value = some_value[tid], limit_token = key(some_token[tid]);
    }
    __syncthreads();
    for (int i = tid; i < a.parts * a.n; i += LP_THREADS) {
        const float v = a.part_value[from + i];
        const int tok = a.part_token[from + i];
        if (tok >= 0 && !before(limit_value, limit_token, v, tok)) {
            const int to = atomicAdd(&count, 1);
            value[to] = v, token[to] = tok;
        }
    }
    __syncthreads();
    put_in_order(value, token, count, a.n, [&](int place, float v, int tok) {
        a.top_token[t * a.n + place] = tok, a.top_logprob[t * a.n + place] = tok < 0 ? __builtin_nanf("") : v - M - ln_s;
    });
}

// Parts of a row: as many as fill the GPU with blocks, of 4096 logits or more.
static int logprobs_parts(int64_t T, int V) {
    int64_t n = T < 1 ? 1 : (2048 + T - 1) / T;
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
    if (n_given == 0 && n_top == 0 && !entropy) return C2R_ERR_INVALID_ARG;
    if (T == 0) return C2R_OK;
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
        a.part_value = reinterpret_cast<float *>(a.stats + T * a.parts);
        a.part_token = reinterpret_cast<int32_t *>(a.part_value + T * a.parts * n_top);
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)(T * a.parts)), rows((unsigned)T), block(LP_THREADS);
    if (dt == C2R_BF16) logprobs_kernel<true><<<grid, block, 0, st>>>(a);
    else logprobs_kernel<false><<<grid, block, 0, st>>>(a);
    const int rc = launch_status();
    if (rc != C2R_OK || a.parts == 1) return rc;
    if (dt == C2R_BF16) logprobs_join_kernel<true><<<rows, block, 0, st>>>(a);
    else logprobs_join_kernel<false><<<rows, block, 0, st>>>(a);
    return launch_status();
}
