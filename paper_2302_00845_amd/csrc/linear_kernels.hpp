// Gradient of a linear layer's weights for every example: G_e[r][c] = sum_t x_t[r] delta_t[c], and, for a bias, a last row
// sum_t delta_t[c] (the layout of softmax_pergrad, which is the case of one row per example).
//
// Per example a product of (in) x (tokens) by (tokens) x (out).  Few tokens: bound by writing G; many: by the products.
// A workgroup takes a BM x BN tile of an example's G.  Rows of x and delta arrive with their features side by side while an
// MFMA operand wants the tokens side by side: tiles go to LDS as they come, [token][feature], and ds_read_tr16 turns them
// on the way to the registers.
#pragma once
#include "mfma_tiles.hpp"

namespace cdgrab {

constexpr int kLinearThreads = 256;
constexpr int kLinearPad = 16;  // elements behind each LDS row: sixteen lanes of a transposing read then hit distinct banks

// What multiplies: fp16 and bf16 as they are; an fp32 element as the sum of three bf16, of whose nine products the six
// largest are taken (the rest is below 2^-24 of the product: as good as an fp32 product, at 2.6 times the rate of the
// fp32 MFMA).  Above 3.38e38, bf16's largest number, the first part is infinite and the second NaN.  (Held back by a v_med3
// per element the largest numbers would be whole: 64 x 128 rows, 128 -> 384 13.15 -> 13.55 us.  Left out.)  Below 2^-110 the third
// part is below bf16's smallest number.
template <typename T> struct LinearPlanes { static constexpr int N = 1, KC = 32; typedef T elem; };
template <> struct LinearPlanes<float> { static constexpr int N = 3, KC = 16; typedef bf16_t elem; };

// Operand of a 32 x 32 x 16 MFMA from LDS [token][feature]: lane l holds feature l % 32 of tokens 8 (l / 32) .. + 7.
// (A transposing read: sixteen lanes give four tokens' addresses, four lanes a token, and each receives one feature's four.)
template <typename E, int STRIDE>
__device__ __forceinline__ auto turned(const E *lds, int lane) {
    typedef __attribute__((address_space(3))) s16x4 *Ptr;
    const int token = (lane >> 5) * 8 + ((lane & 15) >> 2), feature = (lane & 16) + (lane & 3) * 4;
    const E *p = lds + token * STRIDE + feature;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(p));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(p + 4 * STRIDE));
    const s16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    typedef E vec __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(vec, both);
}

// One operand's tile of KC tokens x W features on its way from memory to LDS.
template <typename T, int W>
struct LinearStage {
    typedef LinearPlanes<T> P;
    static constexpr int GROUPS = W / 8, TOTAL = GROUPS * P::KC, PER = (TOTAL + kLinearThreads - 1) / kLinearThreads;
    static constexpr int STRIDE = W + kLinearPad, PLANE = P::KC * STRIDE;
    T v[PER][8];

    // features col0 .. col0 + W - 1 of `width`, tokens from `tok` on; what lies beyond `width` or `end` becomes zero unread
    __device__ __forceinline__ void load(const T *base, int64_t stride, int64_t tok, int64_t end, int col0, int width) {
#pragma unroll
        for (int q = 0; q < PER; ++q) {
            const int at = threadIdx.x + q * kLinearThreads;
            const int col = col0 + (at % GROUPS) * 8;
            const int64_t row = tok + at / GROUPS;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[q][j] = (T)0.f;
            if ((TOTAL % kLinearThreads == 0 || at < TOTAL) && row < end) {
                const T *p = base + row * stride + col;
                if (col + 8 <= width) load_any<T, 8>(p, v[q]);
                else
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (col + j < width) v[q][j] = p[j];
            }
        }
    }
    __device__ __forceinline__ void store(typename P::elem *lds) const {
#pragma unroll
        for (int q = 0; q < PER; ++q) {
            const int at = threadIdx.x + q * kLinearThreads;
            if (TOTAL % kLinearThreads != 0 && at >= TOTAL) break;
            typename P::elem *p = lds + (at / GROUPS) * STRIDE + (at % GROUPS) * 8;
            typedef typename P::elem vec __attribute__((ext_vector_type(8)));
            if constexpr (P::N == 1) {
                vec x;
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = v[q][j];
                *reinterpret_cast<vec *>(p) = x;
            } else {
                float left[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) left[j] = v[q][j];
#pragma unroll
                for (int pl = 0; pl < P::N; ++pl) {
                    vec x;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        x[j] = (bf16_t)left[j];
                        left[j] = left[j] - (float)x[j];
                    }
                    *reinterpret_cast<vec *>(p + pl * PLANE) = x;
                }
            }
        }
    }
    __device__ __forceinline__ void add_to(float (&sum)[PER][8]) const {
#pragma unroll
        for (int q = 0; q < PER; ++q)
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[q][j] += (float)v[q][j];
    }
};

// WAVES_M x WAVES_N wavefronts share the tile.  grid: (example, share of its tokens, tile), neighbours down G's columns or along
// its rows; `shares` > 1: the sums of a share
// go to `to` + share * share_stride, which linear_grad_finish adds up in order.
template <typename T, int BM, int BN, int WAVES_M, int WAVES_N>
__global__ __launch_bounds__(kLinearThreads) void linear_grad(TokenRows tok, int shares, const T *__restrict__ X, int64_t x_stride,
                                                              const T *__restrict__ D, int64_t d_stride, int in_dim, int out_dim,
                                                              int with_bias, int down, float *__restrict__ to, int64_t to_stride,
                                                              int64_t share_stride)
{
    typedef LinearPlanes<T> P;
    typedef typename P::elem E;
    typedef LinearStage<T, BM> SX;
    typedef LinearStage<T, BN> SD;
    static_assert(WAVES_M * WAVES_N * 64 == kLinearThreads, "");
    constexpr int MB = BM / WAVES_M / 32, NB = BN / WAVES_N / 32, STAGE = P::N * (SX::PLANE + SD::PLANE);
    static_assert(2 * STAGE * sizeof(E) >= kLinearThreads * 8 * sizeof(float), "the bias's sums take the stages' place");
    __shared__ __align__(16) E lds[2][STAGE];
    float *bias_part = reinterpret_cast<float *>(lds);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / WAVES_N, wn = wave % WAVES_N;
    const int mt = (in_dim + BM - 1) / BM, nt = (out_dim + BN - 1) / BN;
    const uint32_t b = xcd_neighbours(blockIdx.x, gridDim.x), tiles = (uint32_t)(mt * nt), rest = b / tiles, tile = b - rest * tiles;
    const int share = (int)(rest % (uint32_t)shares);
    const int64_t e = tok.base + rest / (uint32_t)shares;
    const int m0 = (int)(down ? tile % mt : tile / nt) * BM, n0 = (int)(down ? tile / mt : tile % nt) * BN;
    const RowSpan span = rows_of(tok, e);
    int64_t per = (span.count + shares - 1) / shares;
    const int64_t begin = span.first + (share * per < span.count ? share * per : span.count);
    const int64_t end = begin + per < span.first + span.count ? begin + per : span.first + span.count;
    const bool sums = with_bias && m0 == 0;

    f32x16 acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.f;
    float bias[SD::PER][8];
#pragma unroll
    for (int q = 0; q < SD::PER; ++q)
#pragma unroll
        for (int j = 0; j < 8; ++j) bias[q][j] = 0.f;

    SX sx;
    SD sd;
    int buf = 0;
    if (begin < end) {  // uniform
        sx.load(X, x_stride, begin, end, m0, in_dim);
        sd.load(D, d_stride, begin, end, n0, out_dim);
    }
    for (int64_t t = begin; t < end; t += P::KC, buf ^= 1) {
        E *lx = lds[buf], *ld = lds[buf] + P::N * SX::PLANE;
        sx.store(lx);
        sd.store(ld);
        if (sums) sd.add_to(bias);
        __syncthreads();  // (the other buffer's readers are past it as well: they come here after reading)
        if (t + P::KC < end) {
            sx.load(X, x_stride, t + P::KC, end, m0, in_dim);
            sd.load(D, d_stride, t + P::KC, end, n0, out_dim);
        }
#pragma unroll
        for (int k = 0; k < P::KC; k += 16) {
            typedef E vec __attribute__((ext_vector_type(8)));
            vec a[P::N][MB], d[P::N][NB];
#pragma unroll
            for (int p = 0; p < P::N; ++p) {
#pragma unroll
                for (int i = 0; i < MB; ++i)
                    a[p][i] = turned<E, SX::STRIDE>(lx + p * SX::PLANE + k * SX::STRIDE + (wm * MB + i) * 32, lane);
#pragma unroll
                for (int j = 0; j < NB; ++j)
                    d[p][j] = turned<E, SD::STRIDE>(ld + p * SD::PLANE + k * SD::STRIDE + (wn * NB + j) * 32, lane);
            }
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    // (smallest products first)
#pragma unroll
                    for (int s = P::N - 1; s >= 0; --s)
#pragma unroll
                        for (int p = 0; p <= s; ++p) acc[i][j] = mfma32(a[p][i], d[s - p][j], acc[i][j]);
                }
        }
    }

    float *out = to + e * to_stride + share * share_stride;
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int c = n0 + (wn * NB + j) * 32 + (lane & 31);
            const int r0 = m0 + (wm * MB + i) * 32 + 4 * (lane >> 5);
            if (c < out_dim)
#pragma unroll
                for (int q = 0; q < 16; ++q) {
                    const int r = r0 + 8 * (q >> 2) + (q & 3);
                    if (r < in_dim) out[(int64_t)r * out_dim + c] = acc[i][j][q];
                }
        }
    if (sums) {  // uniform: column sums of the delta tile, over the threads that staged the same columns
        constexpr int ROWS = kLinearThreads / SD::GROUPS;
        float mine[8];
        __syncthreads();  // (the last stage has been read)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            mine[j] = 0.f;
#pragma unroll
            for (int q = 0; q < SD::PER; ++q) mine[j] += bias[q][j];
            bias_part[threadIdx.x * 8 + j] = mine[j];
        }
        __syncthreads();
        if (threadIdx.x < BN && n0 + (int)threadIdx.x < out_dim) {
            const int g = threadIdx.x >> 3, j = threadIdx.x & 7;
            float sum = 0.f;
            for (int r = 0; r < ROWS; ++r) sum += bias_part[(r * SD::GROUPS + g) * 8 + j];
            out[(int64_t)in_dim * out_dim + n0 + threadIdx.x] = sum;
        }
    }
}

// Few rows per example (TOK at most): G is the sum of as many outer products, and writing it is all that costs.  A workgroup
// writes a stretch of kFlatElems consecutive elements of an example's G, whatever rows they belong to, with aligned 16-byte
// stores; the features and deltas that they need lie in LDS.  60 000 rows of 784 -> 10: 0.45 ms, 4.6 TB/s, two thirds of
// what a large fill reaches, nine tenths of what these stores reach by themselves.  (By tiles of MFMAs 60 000 rows of 784 -> 10 took 2.68 ms: 10 of
// 32 columns used, stores of 40 bytes, and a chain of loads, barriers and products for a few KB.)
constexpr int kFlatElems = 8192;
constexpr int kFlatLds = 16000;  // floats of features and deltas at most

// A thread's stores are a whole number of G's rows apart, so that its four columns stay the same: their deltas are in registers, and
// a store costs two features per token (the four columns lie in two rows at most; SHORT: rows of fewer than four).
// (All positions are 32-bit: 64-bit divisions alone were half of the time of a short stretch.)
template <typename T, int TOK, int THREADS, bool SHORT>
__global__ __launch_bounds__(THREADS) void linear_flat(TokenRows tok, uint32_t units, const T *__restrict__ X, int64_t x_stride,
                                                       const T *__restrict__ D, int64_t d_stride, int in_dim, int out_dim,
                                                       int with_bias, int active, float *__restrict__ G, int64_t g_stride)
{
    extern __shared__ float dyn[];
    const uint32_t local = blockIdx.x / units;
    const int64_t e = tok.base + local;
    const RowSpan span = rows_of(tok, e);
    const int count = (int)span.count;
    float *g = G + e * g_stride;
    const int shift = (int)((reinterpret_cast<uintptr_t>(g) >> 2) & 3);  // elements from a 16-byte boundary to the row's start
    const int d = (in_dim + with_bias) * out_dim;
    const int p0 = (int)(blockIdx.x - local * units) * kFlatElems - shift, lo = p0 > 0 ? p0 : 0, hi = d - p0 > kFlatElems ? p0 + kFlatElems : d;
    if (lo >= hi) return;  // uniform
    const int row0 = (int)((uint32_t)lo / (uint32_t)out_dim), rows = (int)((uint32_t)(hi - 1) / (uint32_t)out_dim) - row0 + 1;
    float *xl = dyn, *dl = dyn + TOK * (rows + 1);
    const T *x_rows = X + span.first * x_stride + row0, *d_rows = D + span.first * d_stride;
    const int have = in_dim - row0;  // features from row0 on; the row behind them is the bias's
#pragma unroll
    for (int t = 0; t < TOK; ++t) {  // (one more row than there are: read, and not used)
        if (t < count) {  // uniform
#pragma unroll 4
            for (int q = threadIdx.x; q <= rows; q += THREADS) xl[t * (rows + 1) + q] = q < have ? (float)x_rows[t * x_stride + q] : 1.f;
            for (int q = threadIdx.x; q < out_dim; q += THREADS) dl[t * out_dim + q] = (float)d_rows[t * d_stride + q];
        } else {
            for (int q = threadIdx.x; q <= rows; q += THREADS) xl[t * (rows + 1) + q] = 0.f;
            for (int q = threadIdx.x; q < out_dim; q += THREADS) dl[t * out_dim + q] = 0.f;
        }
    }
    __syncthreads();
    if ((int)threadIdx.x >= active) return;
    const int first = lo - row0 * out_dim, last = hi - row0 * out_dim;
    const int step = 4 * active, down = step / out_dim;  // elements and rows from store to store
    int at = p0 - row0 * out_dim + 4 * (int)threadIdx.x;  // (from row0's first element; above -4)
    int row[4], col[4];
    float dv[TOK][4];
    row[0] = (int)((uint32_t)(at + step) / (uint32_t)out_dim);
    col[0] = at + step - row[0] * out_dim;
    row[0] -= down;
#pragma unroll
    for (int j = 1; j < 4; ++j) {
        const bool wrap = col[j - 1] + 1 == out_dim;
        col[j] = wrap ? 0 : col[j - 1] + 1;
        row[j] = row[j - 1] + (wrap ? 1 : 0);
    }
#pragma unroll
    for (int t = 0; t < TOK; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) dv[t][j] = dl[t * out_dim + col[j]];
    float *to = g + row0 * (int64_t)out_dim;
    const auto ends = [&](int r) {  // of the stretch
        for (int j = 0; j < 4; ++j)
            if (at + j >= first && at + j < last) {
                float v = 0.f;
#pragma unroll
                for (int t = 0; t < TOK; ++t) v = fmaf(xl[t * (rows + 1) + r + row[j] - row[0]], dv[t][j], v);
                to[at + j] = v;
            }
    };
    int r = row[0];
    if (at < first) {
        ends(r);
        at += step;
        r += down;
    }
#pragma unroll 2
    for (; at + 4 <= last; at += step, r += down) {
        float o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t = 0; t < TOK; ++t) {
            const float *x = xl + t * (rows + 1) + r;
            if constexpr (SHORT) {
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] = fmaf(x[row[j] - row[0]], dv[t][j], o[j]);
            } else {
                const float here = x[0], next = x[1];
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] = fmaf(row[j] == row[0] ? here : next, dv[t][j], o[j]);
            }
        }
        *reinterpret_cast<float4 *>(to + at) = make_float4(o[0], o[1], o[2], o[3]);
    }
    if (at < last) ends(r);
}

// G[e][p] = sum over the shares, in order.
__global__ __launch_bounds__(256) void linear_grad_finish(const float *__restrict__ parts, int shares, int64_t share_stride,
                                                          int64_t examples, int64_t d, float *__restrict__ G, int64_t g_stride)
{
    const int64_t p = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (p >= d) return;
    for (int64_t e = blockIdx.y; e < examples; e += gridDim.y) {
        float sum = 0.f;
#pragma unroll 8
        for (int s = 0; s < shares; ++s) sum += parts[s * share_stride + e * d + p];
        G[e * g_stride + p] = sum;
    }
}

}  // namespace cdgrab
