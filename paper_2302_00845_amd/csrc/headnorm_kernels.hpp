// Norms of queries and keys with the position rotation, for each head of a row: forward, and backward with the gains' gradient of
// every example.
//
//   r = 1 / sqrt(mean(x^2) + eps), h = x r, u = gain h, and pairs (u_i, u_{i + dim/2}) turned by the angle pos base^(-2 i / dim):
//   y_i = u_i cos - u_{i + dim/2} sin,  y_{i + dim/2} = u_{i + dim/2} cos + u_i sin
//   back: u = dy turned by the negative angle, g = gain u, dx = r (g - h mean(g h)), dgain = sum over rows and heads of u h
//
// Bound by bytes: x in and y out; x and dy in, dx out.  A head's features lie in the registers of LANES threads, each with the same
// places of both halves, so that a pair is in one thread.  The angles' cosines and sines are the same for all heads: a workgroup
// computes those of its rows once, into LDS.  Sums in fp32, results are rounded once.  Queries' heads first and then the keys': one kind's
// gains and their sums are in registers at a time (backward 145 -> 121 of them, 141 -> 131 us for the case below).  65 536 rows of 24 heads
// of 64, bf16: 102 us, 4.0 TB/s, and back 138 us, 4.4 TB/s.  Heads whose half is no power of two of pieces leave threads idle: back, 25 700 rows
// of 10 heads of 80, fp16 54 us, 2.3 TB/s, VALU 90 % of the cycles.
#pragma once
#include "norm_kernels.hpp"

namespace cdgrab {

constexpr int kHeadMaxDim = 512, kHeadThreads = 256;
constexpr int kHeadTable = 2048;  // angles of a workgroup's rows at a time

// Turns per position, as fractions of 2^64: position * turn modulo 2^64 is the angle exactly up to the rounding of `turn`, also
// where an fp32 angle of a far position would have no digits left.
struct HeadTurns { uint64_t turn[kHeadMaxDim / 2]; };

// cos and sin of a fraction of a turn: the nearest quarter turn is taken off in whole numbers, the rest (up to an eighth) goes into
// the series of both functions, the first terms left out below 3e-9.
__device__ __forceinline__ float2 cos_sin_turns(uint64_t turns) {
    const uint32_t quarter = (uint32_t)((turns + ((uint64_t)1 << 61)) >> 62);
    const int32_t rest = (int32_t)((turns - ((uint64_t)quarter << 62)) >> 32);
    const float x = (float)rest * 1.46291807926715968e-9f, x2 = x * x;  // 2 pi / 2^32
    float s = fmaf(x2, 1.f / 362880.f, -1.f / 5040.f);
    s = fmaf(x2, s, 1.f / 120.f);
    s = fmaf(x2, s, -1.f / 6.f);
    s = fmaf(x * x2, s, x);
    float c = fmaf(x2, -1.f / 3628800.f, 1.f / 40320.f);
    c = fmaf(x2, c, -1.f / 720.f);
    c = fmaf(x2, c, 1.f / 24.f);
    c = fmaf(x2, c, -0.5f);
    c = fmaf(x2, c, 1.f);
    const float a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
    return make_float2((quarter + 1) & 2 ? -a : a, quarter & 2 ? -b : b);
}

// Without eps, or with next to none, a head of small elements is as long as any other, but their squares are below fp32's numbers: where
// a head's sum is below kHeadSmall its elements are taken kHeadUp times as large, and eps by the square of that.  (From kHeadTiny on eps
// is what counts beside such a sum, and fp16 has no elements as small: kernels of their own, RAISE, so that the others keep their
// registers; with a branch in one kernel 121 of them became 132, three wavefronts per SIMD instead of four.)
constexpr float kHeadTiny = 0x1p-80f, kHeadSmall = 0x1p-90f, kHeadUp = 0x1p100f;

struct HeadShape {
    int q_heads, heads, half;  // queries' heads, queries' and keys', half of a head's features
    int rows;                  // rows at a time
    float eps;
};

// Cosines and sines of `rows` positions from `at` on.
__device__ __forceinline__ void head_angles(float2 *table, const HeadTurns &turns, int64_t at, int rows, int half) {
    for (int q = threadIdx.x; q < rows * half; q += kHeadThreads) {
        const uint32_t r = (uint32_t)q / (uint32_t)half, i = q - r * half;
        table[q] = cos_sin_turns((uint64_t)(at + r) * turns.turn[i]);
    }
}

// Sum over the lanes of a wavefront that hold the same place of their heads: every LANES-th.
template <int LANES>
__device__ __forceinline__ float heads_sum(float x) {
    if constexpr (LANES <= 8) x = dpp_add_f32<0x128>(x);  // row_ror 8, 4, 2, 1
    if constexpr (LANES <= 4) x = dpp_add_f32<0x124>(x);
    if constexpr (LANES <= 2) x = dpp_add_f32<0x122>(x);
    if constexpr (LANES <= 1) x = dpp_add_f32<0x121>(x);
    if constexpr (LANES <= 16) {
        const auto p = __builtin_amdgcn_permlane16_swap(__float_as_int(x), __float_as_int(x), false, false);
        x = __int_as_float((int)p[0]) + __int_as_float((int)p[1]);
    }
    if constexpr (LANES <= 32) {
        const auto p = __builtin_amdgcn_permlane32_swap(__float_as_int(x), __float_as_int(x), false, false);
        x = __int_as_float((int)p[0]) + __int_as_float((int)p[1]);
    }
    return x;
}

// Workgroup b takes chunk b % chunks of the rows of example b / chunks, the queries' heads and then the keys', `rows` rows at a time;
// LANES threads a head.  BACKWARD: DY and DX in the place of Y; the gains' gradients [2][dim] to G or to `partial` [examples][chunks][2 dim].
// ONCE: rows that the caches do not hold anyway are read past them, and DX is written past them (20 000 rows of 40 heads of 128, bf16 148 -> 143
// us; Y, which is read next, is not: 65 536 rows of 24 of 64 102 -> 106).
template <typename T, int VEC, int LANES, bool BACKWARD, bool ONCE, bool RAISE>
__global__ __launch_bounds__(kHeadThreads) void head_norm(
    TokenRows tok, int chunks, HeadShape sh, HeadTurns turns, const T *__restrict__ X, int64_t x_stride, const T *__restrict__ DY,
    int64_t dy_stride, const float *__restrict__ gain_q, const float *__restrict__ gain_k, T *__restrict__ Y, int64_t y_stride,
    float *__restrict__ G, int64_t g_stride, float *__restrict__ partial)
{
    constexpr int GROUPS = kHeadThreads / LANES, WAVES = kHeadThreads / 64;
    __shared__ float2 table[kHeadTable];
    static_assert(sizeof(table) >= WAVES * kHeadMaxDim * sizeof(float), "the wavefronts' sums take its place");
    const int t = threadIdx.x % LANES, mine = threadIdx.x / LANES, half = sh.half;
    const NormSlice<VEC, LANES, 1> sl(t, half);
    const int pos = sl.pos[0];
    const int64_t e = tok.base + blockIdx.x / chunks;
    const int c = (int)(blockIdx.x % chunks);
    const RowSpan span = rows_of(tok, e);
    const int64_t per = (span.count + chunks - 1) / chunks;
    const int64_t t0 = c * per < span.count ? c * per : span.count, t1 = t0 + per < span.count ? t0 + per : span.count;
    const float inv = 0.5f / (float)half;
    for (int keys = 0; keys < 2; ++keys) {
        const int heads = keys ? sh.heads - sh.q_heads : sh.q_heads;
        const float *gain = keys ? gain_k : gain_q;
        float w[2][VEC], dw[2][VEC];
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                w[p][j] = gain ? gain[p * half + pos + j] : 1.f;
                dw[p][j] = 0.f;
            }
        for (int64_t at = t0; at < t1; at += sh.rows) {
            const int rows = (int)(t1 - at < sh.rows ? t1 - at : sh.rows), items = rows * heads;
            if (!keys || at > t0 || rows < t1 - t0 || BACKWARD) {  // (else the table is there)
                __syncthreads();  // (the last rows' angles have been read)
                head_angles(table, turns, at, rows, half);
                __syncthreads();
            }
            for (int base = 0; base < items; base += GROUPS) {  // (uniform: what is beyond the last is not written)
                const bool live = base + mine < items;
                const uint32_t item = (uint32_t)(live ? base + mine : items - 1), r = item / (uint32_t)heads;
                const int64_t row = span.first + at + r, off = (int64_t)(item - r * heads + (keys ? sh.q_heads : 0)) * 2 * half + pos;
                T x[2][VEC], dy[2][VEC];
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    load_any<T, VEC, ONCE>(X + row * x_stride + off + p * half, x[p]);
                    if constexpr (BACKWARD) load_any<T, VEC, ONCE>(DY + row * dy_stride + off + p * half, dy[p]);
                }
                const float2 *turn = table + r * half + pos;
                T y[2][VEC];
                float eps = sh.eps, up = 1.f;
                if constexpr (RAISE) {
                    float ss = 0.f;
#pragma unroll
                    for (int p = 0; p < 2; ++p)
#pragma unroll
                        for (int j = 0; j < VEC; ++j) ss = sl.own(0, j) ? fmaf((float)x[p][j], (float)x[p][j], ss) : ss;
                    if (lanes_sum<LANES>(ss) < kHeadSmall) {
                        up = kHeadUp;
                        eps = eps * kHeadUp * kHeadUp;
                    }
#pragma unroll
                    for (int p = 0; p < 2; ++p)
#pragma unroll
                        for (int j = 0; j < VEC; ++j) x[p][j] = (T)((float)x[p][j] * up);
                }
                if constexpr (!BACKWARD) {
                    float ss = 0.f;
#pragma unroll
                    for (int p = 0; p < 2; ++p)
#pragma unroll
                        for (int j = 0; j < VEC; ++j) ss = sl.own(0, j) ? fmaf((float)x[p][j], (float)x[p][j], ss) : ss;
                    ss = lanes_sum<LANES>(ss);
                    const float rs = 1.f / sqrtf(fmaf(ss, inv, eps)) + (ss - ss);  // (NaN of a sum that is not finite)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const float2 cs = turn[j];
                        const float a = (float)x[0][j] * rs * w[0][j], b = (float)x[1][j] * rs * w[1][j];
                        y[0][j] = (T)fmaf(a, cs.x, -(b * cs.y));
                        y[1][j] = (T)fmaf(b, cs.x, a * cs.y);
                    }
                } else {
                    float u[2][VEC], s[2] = {0.f, 0.f};  // sums of x^2, g x
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const float2 cs = turn[j];
                        const float a = (float)dy[0][j], b = (float)dy[1][j];
                        u[0][j] = fmaf(a, cs.x, b * cs.y);
                        u[1][j] = fmaf(b, cs.x, -(a * cs.y));
#pragma unroll
                        for (int p = 0; p < 2; ++p) {
                            const float v = sl.own(0, j) ? (float)x[p][j] : 0.f;
                            s[0] = fmaf(v, v, s[0]);
                            s[1] = fmaf(u[p][j] * w[p][j], v, s[1]);
                        }
                    }
                    s[0] = lanes_sum<LANES>(s[0]);
                    s[1] = lanes_sum<LANES>(s[1]);
                    const float rs = 1.f / sqrtf(fmaf(s[0], inv, eps)) + (s[0] - s[0]);
                    const float mean = s[1] * rs * inv;
#pragma unroll
                    for (int p = 0; p < 2; ++p)
#pragma unroll
                        for (int j = 0; j < VEC; ++j) {
                            const float hat = (float)x[p][j] * rs;
                            float d = rs * fmaf(u[p][j], w[p][j], -(hat * mean));
                            if constexpr (RAISE) d *= up;
                            y[p][j] = (T)d;
                            if (live) dw[p][j] = fmaf(u[p][j], hat, dw[p][j]);
                        }
                }
                if ((!BACKWARD || Y) && live && sl.any(0))
#pragma unroll
                    for (int p = 0; p < 2; ++p) store_any<T, VEC, BACKWARD && ONCE>(Y + row * y_stride + off + p * half, y[p]);
            }
        }
        if constexpr (BACKWARD) {
            if (!G && !partial) continue;
            float *part = reinterpret_cast<float *>(table);  // [WAVES][2 half]
            __syncthreads();
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float sum = heads_sum<LANES>(dw[p][j]);
                    if ((threadIdx.x & 63) < LANES && sl.own(0, j)) part[(threadIdx.x >> 6) * 2 * half + p * half + pos + j] = sum;
                }
            __syncthreads();
            float *to = (chunks > 1 ? partial + (e * chunks + c) * 4 * half : G + e * g_stride) + keys * 2 * half;
            for (int col = threadIdx.x; col < 2 * half; col += kHeadThreads) {
                float sum = 0.f;
#pragma unroll
                for (int q = 0; q < WAVES; ++q) sum += part[q * 2 * half + col];
                to[col] = sum;
            }
        }
    }
}

}  // namespace cdgrab
