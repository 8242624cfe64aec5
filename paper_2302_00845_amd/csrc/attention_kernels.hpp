// Causal attention of grouped heads within each example: forward, and backward.
//
//   s_ij = scale q_i k_j (j <= i), L_i = ln sum_j exp(s_ij), p_ij = exp(s_ij - L_i), o_i = sum_j p_ij v_j
//   backward, with D_i = do_i o_i: ds_ij = p_ij (do_i v_j - D_i),
//   dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij do_i   (over the heads that share k, v)
//
// Bound by products, 4 dim flops a pair forward and 10 back, and by the exponentials beside them.  No matrix of scores is kept: a wavefront
// holds 32 queries (forward, dq) or 32 keys (dk, dv) as the columns of its products in registers and goes over the other rows,
// which a workgroup stages in LDS.  With one column per lane a softmax's maximum and sum are a lane's own (two lanes share
// a column), and the products' results have their rows in the order in which the next product takes them: 32 x 32 x 16 MFMAs give
// lane l rows 8 i + 4 (l / 32) + 0 .. 3, and as an operand eight rows of a lane are those of two such runs if the other operand, read from
// LDS by transposing reads, takes its rows in the same order.  So probabilities never pass through LDS.
//
// Products of 16-bit elements are exact, sums are fp32; p and ds are rounded to the elements' type where they are multiplied (half a step
// relative, as much as the rounding of the outputs), statistics and the sum of p are not.  fp32 elements are three bf16, six products each
// (LinearPlanes), p and ds too.  A backward pass in two kernels, dq by queries and dk, dv by keys, takes seven products
// instead of five but adds everything up in registers in a fixed order.
#pragma once
#include "linear_kernels.hpp"

namespace cdgrab {

constexpr int kAttThreads = 256;
constexpr int kAttRows = 128;  // queries (keys) of a workgroup, 32 a wavefront
constexpr int kAttMaxDim = 128;

struct AttHeads {
    int64_t pairs;      // examples of the launch * kv_heads
    int kv_heads, group;  // queries' heads that share keys and values
    int dim;
    float scale;
};

// D features in rows of PIECES pieces of eight elements.  The pieces of a row are swapped by its number so that both kinds of reads hit
// distinct banks: sixteen rows at one piece, and four neighbouring rows at four neighbouring pieces.
template <int D>
struct AttLayout {
    static_assert(D == 32 || D == 64 || D == 96 || D == 128, "");
    static constexpr int LD = D == 96 ? 128 : D, PIECES = LD / 8;
    static __device__ __forceinline__ int swap(int r) {
        return PIECES == 4 ? (r >> 2) & 3 : PIECES == 8 ? (r & 2) << 1 | ((r >> 2) & 3) : (r & 3) << 2 | ((r >> 2) & 3);
    }
};

// Eight elements of a row from `col` on, zero beyond `dim`.
template <typename T>
__device__ __forceinline__ void att_piece(const T *row, int col, int dim, bool there, T (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (T)0.f;
    if (there) {
        if (col + 8 <= dim) load_any<T, 8>(row + col, v);
        else
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (col + j < dim) v[j] = row[col + j];
    }
}

// Eight values as the operands of all planes.
template <typename T>
struct AttFrag {
    typedef LinearPlanes<T> P;
    typedef typename P::elem E;
    typedef E vec __attribute__((ext_vector_type(8)));
    vec v[P::N];
    template <typename S>
    __device__ __forceinline__ void set(const S (&x)[8]) {
        if constexpr (P::N == 1) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[0][j] = (E)x[j];
        } else {
            float left[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) left[j] = (float)x[j];
#pragma unroll
            for (int p = 0; p < P::N; ++p)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    v[p][j] = (E)left[j];
                    left[j] -= (float)v[p][j];
                }
        }
    }
};
template <typename T>
__device__ __forceinline__ f32x16 att_mfma(const AttFrag<T> &a, const AttFrag<T> &b, f32x16 c) {
    constexpr int N = AttFrag<T>::P::N;
#pragma unroll
    for (int s = N - 1; s >= 0; --s)  // (smallest products first)
#pragma unroll
        for (int p = 0; p <= s; ++p) c = mfma32(a.v[p], b.v[s - p], c);
    return c;
}

// A wavefront's 32 columns: lane l holds features 16 k + 8 (l / 32) .. + 7 of row `row` + l % 32 for the k-th product.
template <typename T, int D>
struct AttColumns {
    AttFrag<T> k[D / 16];
    __device__ __forceinline__ void load(const T *row, int lane, int dim, bool there) {
#pragma unroll
        for (int q = 0; q < D / 16; ++q) {
            T v[8];
            att_piece<T>(row, q * 16 + (lane >> 5) * 8, dim, there, v);
            k[q].set(v);
        }
    }
};

// ROWS rows on their way from memory to LDS, all planes.
template <typename T, int D, int ROWS>
struct AttStage {
    typedef LinearPlanes<T> P;
    typedef typename P::elem E;
    typedef AttLayout<D> L;
    static constexpr int USED = D / 8, TOTAL = ROWS * USED, PER = (TOTAL + kAttThreads - 1) / kAttThreads, PLANE = ROWS * L::LD;
    static constexpr int LEN = P::N * PLANE;
    T v[PER][8];
    // rows `at` .. of `base`, those from `end` on are zero and not read
    __device__ __forceinline__ void load(const T *base, int64_t stride, int64_t at, int64_t end, int dim) {
#pragma unroll
        for (int q = 0; q < PER; ++q) {
            const int i = threadIdx.x + q * kAttThreads, r = i / USED, piece = i % USED;
            att_piece<T>(base + (at + r) * stride, piece * 8, dim, (TOTAL % kAttThreads == 0 || i < TOTAL) && at + r < end, v[q]);
        }
    }
    __device__ __forceinline__ void store(E *lds) const {
#pragma unroll
        for (int q = 0; q < PER; ++q) {
            const int i = threadIdx.x + q * kAttThreads, r = i / USED, piece = i % USED;
            if (TOTAL % kAttThreads != 0 && i >= TOTAL) break;
            AttFrag<T> f;
            f.set(v[q]);
#pragma unroll
            for (int p = 0; p < P::N; ++p)
                *reinterpret_cast<typename AttFrag<T>::vec *>(lds + p * PLANE + r * L::LD + (piece ^ L::swap(r)) * 8) = f.v[p];
        }
    }
};

// A lane's operands from a staged tile: rows along the result's rows (`along`, features are summed over), or features along the
// result's rows (`across`, rows are summed over in the order of a result's registers).
template <typename T, int D, int ROWS>
struct AttRead {
    typedef LinearPlanes<T> P;
    typedef typename P::elem E;
    typedef AttLayout<D> L;
    static constexpr int PLANE = ROWS * L::LD;
    int row, piece, token, lo, hi;
    __device__ __forceinline__ explicit AttRead(int lane) {
        row = (lane & 31) * L::LD;
        piece = ((lane >> 5) ^ L::swap(lane & 31)) * 8;
        const int r = 4 * (lane >> 5) + ((lane & 15) >> 2), x = (lane & 16) >> 3 | (lane & 3) >> 1;
        token = r * L::LD + (lane & 1) * 4;
        lo = (x ^ L::swap(r)) * 8;
        hi = (x ^ L::swap(r + 8)) * 8;
    }
    // rows first .. first + 31, features 16 k ..
    __device__ __forceinline__ AttFrag<T> along(const E *tile, int first, int k) const {
        AttFrag<T> f;
#pragma unroll
        for (int p = 0; p < P::N; ++p)
            f.v[p] = *reinterpret_cast<const typename AttFrag<T>::vec *>(tile + p * PLANE + first * L::LD + row + (piece ^ (k * 16)));
        return f;
    }
    // features 32 d .., rows first .. first + 15
    __device__ __forceinline__ AttFrag<T> across(const E *tile, int first, int d) const {
        typedef __attribute__((address_space(3))) s16x4 *Ptr;
        AttFrag<T> f;
#pragma unroll
        for (int p = 0; p < P::N; ++p) {
            const E *at = tile + p * PLANE + first * L::LD + token;
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(at + (lo ^ (d * 32))));
            const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(at + 8 * L::LD + (hi ^ (d * 32))));
            f.v[p] = __builtin_bit_cast(typename AttFrag<T>::vec, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        }
        return f;
    }
};

// Sum and maximum over the two lanes of a column.
__device__ __forceinline__ float both_sum(float x) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_int(x), __float_as_int(x), false, false);
    return __int_as_float((int)p[0]) + __int_as_float((int)p[1]);
}
__device__ __forceinline__ float both_max(float x) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_int(x), __float_as_int(x), false, false);
    return fmaxf(__int_as_float((int)p[0]), __int_as_float((int)p[1]));
}

__device__ __forceinline__ f32x16 zero16() {
    f32x16 z;
#pragma unroll
    for (int q = 0; q < 16; ++q) z[q] = 0.f;
    return z;
}

// Row of a result's register q, of its first 32 rows.
__device__ __forceinline__ int att_row(int q, int lane) { return 8 * (q >> 2) + 4 * (lane >> 5) + (q & 3); }

// Results with features along the rows, one output row per lane.
template <typename T, int D>
__device__ __forceinline__ void att_write(T *to, const f32x16 (&acc)[D / 32], float times, int dim, int lane) {
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int q = 0; q < 16; q += 4) {
            const int col = d * 32 + att_row(q, lane);
            T y[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = (T)(acc[d][q + j] * times);
            if (col + 4 <= dim) store_any<T, 4>(to + col, y);
            else
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (col + j < dim) to[col + j] = y[j];
        }
}

// What a workgroup works on: workgroups of one pair (example, key head) are a multiple of eight apart, that is on one XCD, whose L2
// then holds its keys and values; the longest tiles come first.
struct AttPlace {
    RowSpan span;
    int64_t row0;   // the tile's first row in the example
    int kv, head;   // heads of keys, of queries
    bool there;
    __device__ __forceinline__ AttPlace(const TokenRows &tok, const AttHeads &a, bool backwards, bool members) {
        const int64_t padded = (a.pairs + 7) & ~(int64_t)7;
        const int64_t pair = blockIdx.x % padded, member = members ? blockIdx.x / padded : 0;
        there = pair < a.pairs;
        if (!there) return;
        span = rows_of(tok, tok.base + pair / a.kv_heads);
        kv = (int)(pair % a.kv_heads);
        head = kv * a.group + (int)member;
        row0 = (int64_t)(backwards ? gridDim.y - 1 - blockIdx.y : blockIdx.y) * kAttRows;
        there = row0 < span.count;
    }
};

constexpr float kLog2E = 1.44269504088896341f, kLn2 = 0.693147180559945309f;

// p is held 2^shift times as large: fp16 has room for that above (the forward pass's p reach 2^8, the backward pass's 1), and
// below 2^-14 its numbers lose digits.
template <typename T> constexpr float kAttShiftForward = 0.f;
template <> constexpr float kAttShiftForward<f16_t> = 7.f;
template <typename T> constexpr float kAttShiftBack = 0.f;
template <> constexpr float kAttShiftBack<f16_t> = 14.f;

// A staged tile's rows; LDS for two of them, all planes.
template <typename T> constexpr int att_step() { return LinearPlanes<T>::N == 1 ? 64 : 32; }

template <typename T, int D>
__global__ __launch_bounds__(kAttThreads, LinearPlanes<T>::N == 1 ? 2 : 1) void attention_forward(
    TokenRows tok, AttHeads a, const T *__restrict__ Q, int64_t q_stride, const T *__restrict__ K, int64_t k_stride,
    const T *__restrict__ V, int64_t v_stride, T *__restrict__ O, int64_t o_stride, float *__restrict__ lse, int64_t q_heads)
{
    typedef typename LinearPlanes<T>::elem E;
    constexpr int STEP = att_step<T>(), KB = STEP / 32, DB = D / 32;
    typedef AttStage<T, D, STEP> Stage;
    __shared__ __align__(16) E lds[2 * Stage::LEN];
    const AttPlace at(tok, a, true, true);
    if (!at.there) return;  // uniform
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t first = at.row0 + wave * 32, mine = first + (lane & 31), count = at.span.count;
    const T *q = Q + (at.span.first + (mine < count ? mine : 0)) * q_stride + (int64_t)at.head * a.dim;
    const T *k = K + at.span.first * k_stride + (int64_t)at.kv * a.dim, *v = V + at.span.first * v_stride + (int64_t)at.kv * a.dim;
    AttColumns<T, D> cols;
    cols.load(q, lane, a.dim, mine < count);
    const AttRead<T, D, STEP> read(lane);
    f32x16 acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) acc[d] = zero16();
    float most = -INFINITY, sum = 0.f;  // (of the lane's own rows)
    const float c = a.scale * kLog2E;
    const int64_t end = at.row0 + kAttRows < count ? at.row0 + kAttRows : count;  // keys
    Stage sk, sv;
    sk.load(k, k_stride, 0, end, a.dim);
    sv.load(v, v_stride, 0, end, a.dim);
    for (int64_t t = 0; t < end; t += STEP) {
        __syncthreads();  // (the last tile has been read)
        sk.store(lds);
        sv.store(lds + Stage::LEN);
        __syncthreads();
        if (t + STEP < end) {
            sk.load(k, k_stride, t + STEP, end, a.dim);
            sv.load(v, v_stride, t + STEP, end, a.dim);
        }
        if (t > first + 31) continue;  // all later than this wavefront's queries
        f32x16 s[KB];
#pragma unroll
        for (int b = 0; b < KB; ++b) {
            s[b] = zero16();
#pragma unroll
            for (int d = 0; d < D / 16; ++d) s[b] = att_mfma<T>(read.along(lds, b * 32, d), cols.k[d], s[b]);
        }
        if (t + STEP - 1 > first) {
            const int left = (int)(mine - t);  // rows of the tile up to this query
#pragma unroll
            for (int b = 0; b < KB; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[b][r] = b * 32 + att_row(r, lane) <= left ? s[b][r] : -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[b][r]);
        top = fmaf(both_max(top), c, -kAttShiftForward<T>);
        // (The maximum may lag behind by 2^8, the sums have room for that: they are seldom scaled.)
        if (__any(top > most + 8.f)) {
            const float next = fmaxf(most, top), down = __builtin_amdgcn_exp2f(most - next);
            most = next;
            sum *= down;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[d][r] *= down;
        }
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int r = 0; r < 16; r += 8) {
                float p[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    p[j] = __builtin_amdgcn_exp2f(fmaf(s[b][r + j], c, -most));
                    sum += p[j];
                }
                AttFrag<T> w;
                w.set(p);
#pragma unroll
                for (int d = 0; d < DB; ++d) acc[d] = att_mfma<T>(read.across(lds + Stage::LEN, b * 32 + r * 2, d), w, acc[d]);
            }
    }
    sum = both_sum(sum);
    if (mine < count) {
        att_write<T, D>(O + (at.span.first + mine) * o_stride + (int64_t)at.head * a.dim, acc, 1.f / sum, a.dim, lane);
        if (lse && lane < 32) lse[(at.span.first + mine) * q_heads + at.head] = (most + __builtin_amdgcn_logf(sum)) * kLn2;
    }
}

// Products with ds: of fp16 elements they are scaled by a power of two per column, so that small gradients keep their digits; when a column's
// values outgrow it, what has been summed is scaled down.
template <typename T, int DB>
struct AttScaled {
    float scale = 1.f;
    __device__ __forceinline__ void fit(f32x16 &, f32x16 (&)[DB]) {}
};
template <int DB>
struct AttScaled<f16_t, DB> {
    float scale = 0x1p80f;
    __device__ __forceinline__ void fit(f32x16 &ds, f32x16 (&acc)[DB]) {
        float top = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, fabsf(ds[r]));
        top = both_max(top);
        if (__any(top * scale > 0x1p15f)) {
            // 2^14 / 2^e, 2^e the top's exponent (values that are not finite: as it is)
            const int e = (int)(__float_as_uint(top) >> 23);
            const float want = e == 255 ? scale : __uint_as_float((uint32_t)(268 - e < 254 ? 268 - e : 254) << 23);
            const float next = fminf(scale, want), by = next / scale;
            scale = next;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[d][r] *= by;
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) ds[r] *= scale;
    }
};

// dq by queries; leaves D_i for the other kernel.
template <typename T, int D>
__global__ __launch_bounds__(kAttThreads, LinearPlanes<T>::N == 1 ? 2 : 1) void attention_backward_q(
    TokenRows tok, AttHeads a, const T *__restrict__ Q, int64_t q_stride, const T *__restrict__ K, int64_t k_stride,
    const T *__restrict__ V, int64_t v_stride, const T *__restrict__ O, int64_t o_stride, const float *__restrict__ lse,
    const T *__restrict__ DO, int64_t do_stride, T *__restrict__ DQ, int64_t dq_stride, float *__restrict__ delta, int64_t q_heads)
{
    typedef typename LinearPlanes<T>::elem E;
    constexpr int STEP = att_step<T>(), KB = STEP / 32, DB = D / 32;
    typedef AttStage<T, D, STEP> Stage;
    __shared__ __align__(16) E lds[2 * Stage::LEN];
    const AttPlace at(tok, a, true, true);
    if (!at.there) return;  // uniform
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t first = at.row0 + wave * 32, mine = first + (lane & 31), count = at.span.count;
    const bool live = mine < count;
    const int64_t row = at.span.first + (live ? mine : 0);
    const T *k = K + at.span.first * k_stride + (int64_t)at.kv * a.dim, *v = V + at.span.first * v_stride + (int64_t)at.kv * a.dim;
    AttColumns<T, D> q, g;
    q.load(Q + row * q_stride + (int64_t)at.head * a.dim, lane, a.dim, live);
    float dot = 0.f;
    {
        const T *o = O + row * o_stride + (int64_t)at.head * a.dim, *d = DO + row * do_stride + (int64_t)at.head * a.dim;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            T x[8], y[8];
            att_piece<T>(o, s * 16 + (lane >> 5) * 8, a.dim, live, x);
            att_piece<T>(d, s * 16 + (lane >> 5) * 8, a.dim, live, y);
            g.k[s].set(y);
#pragma unroll
            for (int j = 0; j < 8; ++j) dot = fmaf((float)x[j], (float)y[j], dot);
        }
        dot = both_sum(dot);
        if (live && lane < 32) delta[row * q_heads + at.head] = dot;
    }
    const AttRead<T, D, STEP> read(lane);
    f32x16 acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) acc[d] = zero16();
    AttScaled<T, DB> scaled;
    const float c = a.scale * kLog2E, most = live ? lse[row * q_heads + at.head] * kLog2E : INFINITY;
    const int64_t end = at.row0 + kAttRows < count ? at.row0 + kAttRows : count;
    Stage sk, sv;
    sk.load(k, k_stride, 0, end, a.dim);
    sv.load(v, v_stride, 0, end, a.dim);
    for (int64_t t = 0; t < end; t += STEP) {
        __syncthreads();
        sk.store(lds);
        sv.store(lds + Stage::LEN);
        __syncthreads();
        if (t + STEP < end) {
            sk.load(k, k_stride, t + STEP, end, a.dim);
            sv.load(v, v_stride, t + STEP, end, a.dim);
        }
        if (t > first + 31) continue;
        const bool edge = t + STEP - 1 > first;
        const int left = (int)(mine - t);
#pragma unroll
        for (int b = 0; b < KB; ++b) {
            f32x16 s = zero16(), ds = zero16();
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
                s = att_mfma<T>(read.along(lds, b * 32, d), q.k[d], s);
                ds = att_mfma<T>(read.along(lds + Stage::LEN, b * 32, d), g.k[d], ds);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float p = __builtin_amdgcn_exp2f(fmaf(s[r], c, -most));
                ds[r] = !edge || b * 32 + att_row(r, lane) <= left ? p * (ds[r] - dot) : 0.f;
            }
            scaled.fit(ds, acc);
#pragma unroll
            for (int r = 0; r < 16; r += 8) {
                float x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = ds[r + j];
                AttFrag<T> w;
                w.set(x);
#pragma unroll
                for (int d = 0; d < DB; ++d) acc[d] = att_mfma<T>(read.across(lds, b * 32 + r * 2, d), w, acc[d]);
            }
        }
    }
    if (live) att_write<T, D>(DQ + row * dq_stride + (int64_t)at.head * a.dim, acc, a.scale / scaled.scale, a.dim, lane);
}

// dk and dv by keys, over all heads that share them.
template <typename T, int D>
__global__ __launch_bounds__(kAttThreads, 1) void attention_backward_kv(
    TokenRows tok, AttHeads a, const T *__restrict__ Q, int64_t q_stride, const T *__restrict__ K, int64_t k_stride,
    const T *__restrict__ V, int64_t v_stride, const float *__restrict__ lse, const T *__restrict__ DO, int64_t do_stride,
    const float *__restrict__ delta, T *__restrict__ DK, int64_t dk_stride, T *__restrict__ DV, int64_t dv_stride, int64_t q_heads)
{
    typedef typename LinearPlanes<T>::elem E;
    constexpr int STEP = att_step<T>(), QB = STEP / 32, DB = D / 32;
    typedef AttStage<T, D, STEP> Stage;
    __shared__ __align__(16) E lds[2 * Stage::LEN];
    __shared__ __align__(16) float most[STEP], dots[STEP];
    const AttPlace at(tok, a, false, false);
    if (!at.there) return;  // uniform
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t first = at.row0 + wave * 32, mine = first + (lane & 31), count = at.span.count;
    const bool live = mine < count;
    const int64_t row = at.span.first + (live ? mine : 0);
    AttColumns<T, D> k, v;
    k.load(K + row * k_stride + (int64_t)at.kv * a.dim, lane, a.dim, live);
    v.load(V + row * v_stride + (int64_t)at.kv * a.dim, lane, a.dim, live);
    const AttRead<T, D, STEP> read(lane);
    f32x16 dk[DB], dv[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) dk[d] = dv[d] = zero16();
    AttScaled<T, DB> scaled;
    const float c = a.scale * kLog2E;
    Stage sq, sg;
    float next_most = 0.f, next_dot = 0.f;
    const auto fetch = [&](int64_t t, int64_t head) {
        sq.load(Q + at.span.first * q_stride + head * a.dim, q_stride, t, count, a.dim);
        sg.load(DO + at.span.first * do_stride + head * a.dim, do_stride, t, count, a.dim);
        if (threadIdx.x < STEP) {
            const bool there = t + threadIdx.x < count;
            const int64_t r = (at.span.first + t + threadIdx.x) * q_heads + head;
            next_most = there ? fmaf(lse[r], kLog2E, -kAttShiftBack<T>) : INFINITY;  // (a row that is not there: p = 0)
            next_dot = there ? delta[r] : 0.f;
        }
    };
    int64_t t = at.row0, next_t = t;
    int head = at.head, next_head = head;
    const auto advance = [&]() {
        next_t += STEP;
        if (next_t >= count) {
            next_t = at.row0;
            ++next_head;
        }
    };
    fetch(t, head);
    for (; head < at.head + a.group; t = next_t, head = next_head) {
        __syncthreads();
        sq.store(lds);
        sg.store(lds + Stage::LEN);
        if (threadIdx.x < STEP) {
            most[threadIdx.x] = next_most;
            dots[threadIdx.x] = next_dot;
        }
        __syncthreads();
        advance();
        if (next_head < at.head + a.group) fetch(next_t, next_head);
#pragma unroll
        for (int b = 0; b < QB; ++b) {
            if (t + b * 32 + 31 < first) continue;  // all earlier than this wavefront's keys
            f32x16 s = zero16(), ds = zero16();
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
                s = att_mfma<T>(read.along(lds, b * 32, d), k.k[d], s);
                ds = att_mfma<T>(read.along(lds + Stage::LEN, b * 32, d), v.k[d], ds);
            }
            const bool edge = t + b * 32 < first + 31;
            const int from = (int)(mine - t) - b * 32;  // the first of the rows that sees this key
            const float *m = most + b * 32 + 4 * (lane >> 5), *dot = dots + b * 32 + 4 * (lane >> 5);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float p = __builtin_amdgcn_exp2f(fmaf(s[r], c, -m[8 * (r >> 2) + (r & 3)]));
                const bool seen = !edge || att_row(r, lane) >= from;
                s[r] = seen ? p : 0.f;
                ds[r] = seen ? p * (ds[r] - dot[8 * (r >> 2) + (r & 3)]) : 0.f;
            }
            scaled.fit(ds, dk);
#pragma unroll
            for (int r = 0; r < 16; r += 8) {
                float x[8], y[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    x[j] = s[r + j];
                    y[j] = ds[r + j];
                }
                AttFrag<T> w, z;
                w.set(x);
                z.set(y);
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    dv[d] = att_mfma<T>(read.across(lds + Stage::LEN, b * 32 + r * 2, d), w, dv[d]);
                    dk[d] = att_mfma<T>(read.across(lds, b * 32 + r * 2, d), z, dk[d]);
                }
            }
        }
    }
    constexpr float unshift = kAttShiftBack<T> == 0.f ? 1.f : 0x1p-14f;
    if (live) {
        att_write<T, D>(DK + row * dk_stride + (int64_t)at.kv * a.dim, dk, a.scale * unshift / scaled.scale, a.dim, lane);
        att_write<T, D>(DV + row * dv_stride + (int64_t)at.kv * a.dim, dv, unshift, a.dim, lane);
    }
}

}  // namespace cdgrab
