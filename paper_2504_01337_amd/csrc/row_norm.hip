// The residual's sum and the root-mean-square norm of whole rows, with the rows in bf16 or fp32, in 8 bits with a scale each, or both:
//     s = x + r (rounded as it is kept),  y = s * rsqrt(mean(s^2) + eps) * weight,  c = max |y| / 448,  y8 = y / c
// A row is read once: its elements stay in the registers of the lanes that loaded them, 8 at a time, while the two numbers that
// a whole row has to give (the sum of squares, then the largest |y|) go round: within a wave up to rows of 4096, and within a block for longer rows or
// few of them (one row of 2048: 2.4 us with a block, of which 2 are a launch's).  Bound by memory: 8192 rows of 2048 in bf16, with the sum
// and 8 bits, 24 us (6.2 TB/s; the library's copy reaches 5.05); 517 rows of 256 in fp32 3.0.
#include "c2r_internal.h"

namespace c2r {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct NormCall {
    const unsigned char *x, *r;  // r null: s = x
    const float *weight;
    unsigned char *sum, *y, *y8;  // each may be null
    float *scale;
    int64_t x_bytes, r_bytes, sum_bytes, y_bytes, y8_bytes;  // from one row to the next
    int64_t T;
    int d;
    float eps;
};

constexpr float E4M3_MOST = 448.0f;
constexpr float LEAST_SCALE = 1.1754943508222875e-38f;  // 2^-126: its reciprocal is finite

template <bool BF16>
__device__ __forceinline__ void load8(const unsigned char *p, float (&v)[8]) {
    if constexpr (BF16) {
        const u32x4 w = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    } else {
        const f32x4 a = reinterpret_cast<const f32x4 *>(p)[0], b = reinterpret_cast<const f32x4 *>(p)[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
    }
}

// STREAMED: 8192 rows of 2048 in bf16, with the sum and 8 bits, 151 MB: 26.3 us and 30.2 the other way; with a product of the rows behind it, 83.7 and
// 85.0 for both, with a sum of both outputs 40.8 and 40.1; 8192 of 4096 44 and 59, 264 and 265, 94 and 90.
template <bool STREAMED, class T>
__device__ __forceinline__ void put(unsigned char *p, const T &v) {
    if constexpr (STREAMED) __builtin_nontemporal_store(v, reinterpret_cast<T *>(p));
    else *reinterpret_cast<T *>(p) = v;
}
template <bool BF16, bool STREAMED>
__device__ __forceinline__ void store8(unsigned char *p, const float (&v)[8]) {
    if constexpr (BF16) {
        put<STREAMED>(p, u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])});
    } else {
        put<STREAMED>(p, f32x4{v[0], v[1], v[2], v[3]});
        put<STREAMED>(p + 16, f32x4{v[4], v[5], v[6], v[7]});
    }
}

// What THREADS threads of a block have, added up (or the largest), in all of them.
template <int THREADS, bool MAX>
__device__ __forceinline__ float row_total(float v, float *lds) {
    auto both = [](float a, float b) { return MAX ? fmaxf(a, b) : a + b; };
#pragma unroll
    for (int w = 32; w; w >>= 1) v = both(v, __shfl_xor(v, w));
    if constexpr (THREADS > 64) {
        const int wave = threadIdx.x >> 6;
        if (lane_id() == 0) lds[wave] = v;
        __syncthreads();
        v = lds[0];
#pragma unroll
        for (int w = 1; w < THREADS / 64; ++w) v = both(v, lds[w]);
    }
    return v;
}

// THREADS threads to a row, PIECES pieces of 8 elements to a thread.
template <bool BF16, int THREADS, int PIECES, bool STREAMED>
__global__ __launch_bounds__(THREADS > 256 ? THREADS : 256) void row_norm_kernel(NormCall a) {
    constexpr int BLOCK = THREADS > 256 ? THREADS : 256, SZ = BF16 ? 2 : 4;
    __shared__ float sums[BLOCK / 64], tops[BLOCK / 64];
    const int64_t t = (int64_t)blockIdx.x * (BLOCK / THREADS) + threadIdx.x / THREADS;
    if (t >= a.T) return;  // (a whole wave, or with more threads than a wave to a row, the whole block)
    const int lane = threadIdx.x % THREADS, pieces = a.d / 8;
    const unsigned char *x = a.x + t * a.x_bytes, *r = a.r + t * a.r_bytes;
    float s[PIECES][8];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int p = i * THREADS + lane;
#pragma unroll
        for (int e = 0; e < 8; ++e) s[i][e] = 0.0f;
        if (p < pieces) load8<BF16>(x + (int64_t)p * (8 * SZ), s[i]);
    }
    if (a.r) {
        float more[PIECES][8];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int p = i * THREADS + lane;
#pragma unroll
            for (int e = 0; e < 8; ++e) more[i][e] = 0.0f;
            if (p < pieces) load8<BF16>(r + (int64_t)p * (8 * SZ), more[i]);
        }
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                s[i][e] += more[i][e], s[i][e + 1] += more[i][e + 1];
                if constexpr (BF16) {  // the norm is that of the sum as it is kept, whether this call writes it or not
                    const uint32_t w = pack_bf16x2(s[i][e], s[i][e + 1]);
                    s[i][e] = __uint_as_float(w << 16), s[i][e + 1] = __uint_as_float(w & 0xffff0000u);
                }
            }
    }
    float squares = 0.0f;
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) squares = __builtin_fmaf(s[i][e], s[i][e], squares);
    squares = row_total<THREADS, false>(squares, sums);
    const float by = 1.0f / sqrtf(squares / (float)a.d + a.eps);
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int p = i * THREADS + lane;
        if (p >= pieces) continue;
        if (a.sum) store8<BF16, STREAMED>(a.sum + t * a.sum_bytes + (int64_t)p * (8 * SZ), s[i]);
        float w[8] = {1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f};
        if (a.weight) load8<false>(reinterpret_cast<const unsigned char *>(a.weight + (int64_t)p * 8), w);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[i][e] = s[i][e] * by * w[e], top = fmaxf(top, fabsf(s[i][e]));
        if (a.y) store8<BF16, STREAMED>(a.y + t * a.y_bytes + (int64_t)p * (8 * SZ), s[i]);
    }
    if (!a.y8) return;
    top = row_total<THREADS, true>(top, tops);
    const float c = fmaxf(top / E4M3_MOST, LEAST_SCALE), inv = 1.0f / c;
    if (lane == 0) a.scale[t] = c;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int p = i * THREADS + lane;
        if (p >= pieces) continue;
        u32x2 w = {0, 0};
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float *v = &s[i][4 * e];
            const int low = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inv, v[1] * inv, 0, false);
            w[e] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inv, v[3] * inv, low, true);
        }
#endif
        put<STREAMED>(a.y8 + t * a.y8_bytes + (int64_t)p * 8, w);
    }
}

// A grid's threads are counted in 32 bits: more rows take several launches.
template <bool BF16, int THREADS, int PIECES>
static void norm(NormCall a, hipStream_t st) {
    constexpr int BLOCK = THREADS > 256 ? THREADS : 256, ROWS = BLOCK / THREADS;
    constexpr int64_t MOST = ROWS * (1ll << 21);
    const bool streamed = a.T * a.d * (BF16 ? 2 : 4) >= STREAMED_BYTES;
    for (int64_t rest = a.T; rest > 0; rest -= MOST) {
        a.T = rest < MOST ? rest : MOST;
        const dim3 grid((unsigned)((a.T + ROWS - 1) / ROWS)), block(BLOCK);
        if (streamed) row_norm_kernel<BF16, THREADS, PIECES, true><<<grid, block, 0, st>>>(a);
        else row_norm_kernel<BF16, THREADS, PIECES, false><<<grid, block, 0, st>>>(a);
        auto on = [&](auto *&p, int64_t bytes) {
            if (p) p += a.T * bytes;
        };
        on(a.x, a.x_bytes), on(a.r, a.r_bytes), on(a.sum, a.sum_bytes), on(a.y, a.y_bytes), on(a.y8, a.y8_bytes), on(a.scale, 1);
    }
}

template <bool BF16, int THREADS>
static void norm_by_pieces(const NormCall &a, hipStream_t st) {
    const int pieces = (a.d / 8 + THREADS - 1) / THREADS;
    if (pieces <= 1) norm<BF16, THREADS, 1>(a, st);
    else if (pieces <= 2) norm<BF16, THREADS, 2>(a, st);
    else if (pieces <= 4) norm<BF16, THREADS, 4>(a, st);
    else norm<BF16, THREADS, 8>(a, st);
}

// A block or a wave to a row, us of a call in a graph, bf16 with a residual: 1 x 512 3.4 and 3.5, 517 x 512 3.8 and 3.8, 8192 x 512 11.2 and 9.1; 131 x 768 3.8
// and 4.6, 2048 x 768 5.5 and 6.0, 8192 x 768 12.5 and 11.5; 131 x 2048 3.9 and 6.0, 517 x 2048 4.7 and 6.3, 8192 x 2048 22.2 and 23.9; 131 x 4096
// 4.9 and 8.6, 517 x 4096 6.4 and 12.3, 8192 x 4096 50 and 61.  (Rows wider than 512 would have blocks up to some thousand of them, and from 2048
// on always.)  Rows of more than 4096 do not fit a wave's registers.
template <bool BF16>
static void norm_by_rows(const NormCall &a, hipStream_t st) {
    if (a.d > 16384) norm<BF16, 1024, 4>(a, st);
    else if (a.d > 4096 || (a.T < 512 && a.d > 512)) norm_by_pieces<BF16, 256>(a, st);
    else norm_by_pieces<BF16, 64>(a, st);
}

constexpr int NORM_MOST = 32768;

}  // namespace c2r

using namespace c2r;

extern "C" int c2r_add_rms_norm(const void *x, int64_t x_stride, const void *residual, int64_t residual_stride, c2r_dtype dt, int64_t T, int d,
                                const float *weight, float eps, void *sum, int64_t sum_stride, void *y, int64_t y_stride, void *y8,
                                int64_t y8_stride, float *scale, void *stream) {
    drop_stale_error();
    if (dt != C2R_F32 && dt != C2R_BF16) return C2R_ERR_INVALID_ARG;
    if (T < 0 || d < 1 || !(eps >= 0.0f)) return C2R_ERR_INVALID_ARG;
    if (d % 8 != 0 || d > NORM_MOST || T >= (1ll << 30)) return C2R_ERR_UNSUPPORTED;
    if (T == 0) return C2R_OK;  // (rows that are none may have no address)
    if ((sum && !residual) || !y8 != !scale || (!sum && !y && !y8)) return C2R_ERR_INVALID_ARG;
    const int size = dt == C2R_BF16 ? 2 : 4;
    if (!rows_ok(x, x_stride, d, size) || (residual && !rows_ok(residual, residual_stride, d, size))) return C2R_ERR_INVALID_ARG;
    if ((sum && !rows_ok(sum, sum_stride, d, size)) || (y && !rows_ok(y, y_stride, d, size))) return C2R_ERR_INVALID_ARG;
    if (y8 && (!aligned(y8, 8) || y8_stride < d || y8_stride > (1ll << 40) || y8_stride % 8 != 0 || !aligned(scale, 4))) return C2R_ERR_INVALID_ARG;
    if (weight && !aligned(weight, 16)) return C2R_ERR_INVALID_ARG;
    NormCall a = {};
    a.x = static_cast<const unsigned char *>(x), a.r = static_cast<const unsigned char *>(residual);
    a.weight = weight, a.scale = scale;
    a.sum = static_cast<unsigned char *>(sum), a.y = static_cast<unsigned char *>(y), a.y8 = static_cast<unsigned char *>(y8);
    a.x_bytes = x_stride * size, a.r_bytes = residual_stride * size, a.sum_bytes = sum_stride * size, a.y_bytes = y_stride * size;
    a.y8_bytes = y8_stride;
    a.T = T, a.d = d, a.eps = eps;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dt == C2R_BF16) norm_by_rows<true>(a, st);
    else norm_by_rows<false>(a, st);
    return launch_status();
}
