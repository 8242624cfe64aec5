// Layer norm: forward, and backward with the gain's and the bias's gradient of every example.
//
//   mu = mean(x), s2 = mean((x - mu)^2), r = 1/sqrt(s2 + eps), h = (x - mu) r, y = gain h + bias
//   g = gain dy, dx = r (g - mean(g) - h mean(g h)); per example dgain = sum_t dy h, dbias = sum_t dy
//
// Both are bound by bytes, in fp32: x in and y out; x and dy in, dx out.  In 16 bits the arithmetic is near (VALU busy 79 and 74 % of the
// cycles at a width of 768, 4.6 and 4.4 TB/s), and at odd widths, where threads beyond the row compute what they discard, it is
// what they wait for as much as bytes (61 and 69 % at 515, 2.1 and 1.9 TB/s).  A row stays in the registers of the LANES threads that
// share it between the read and the write, sixteen bytes a thread and access, so that nothing is read twice; the backward
// pass takes mean and deviation from the row it has to read anyway instead of from a forward pass's arrays.
// Statistics and sums in fp32: the mean is taken first and corrected by the mean of what is left, so that a row far from
// zero keeps its digits; results are rounded once, to the rows' type.  A row whose sum of squares is beyond fp32 becomes NaN: with
// a deviation of infinity it would become the bias.
#pragma once
#include "layer_common.hpp"

namespace cdgrab {

constexpr int kNormThreads = 256;
constexpr int64_t kNormMaxWidth = 16384;  // what the registers of a workgroup hold

// Sums of N values each over the threads of a row.
template <int LANES, int N>
struct RowSums {
    static __device__ __forceinline__ void take(float (&s)[N], float *lds) {
        if constexpr (LANES <= 64) {
#pragma unroll
            for (int q = 0; q < N; ++q) s[q] = lanes_sum<LANES>(s[q]);
        } else {  // the whole workgroup shares the row
            constexpr int WAVES = LANES / 64;
            const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
            for (int q = 0; q < N; ++q) s[q] = lanes_sum<64>(s[q]);
            __syncthreads();  // (what an earlier call left there has been read)
            if (lane == 0)
#pragma unroll
                for (int q = 0; q < N; ++q) lds[q * WAVES + wave] = s[q];
            __syncthreads();
#pragma unroll
            for (int q = 0; q < N; ++q) {
                s[q] = 0.f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) s[q] += lds[q * WAVES + w];
            }
        }
    }
};

// The elements of a row that a thread holds: K groups of VEC, group k at element (k LANES + t) VEC.  Only the last
// can reach beyond the row: it is moved back to the row's last VEC elements, of which the first `skip` belong to
// other threads as well (VEC: all of them).
template <int VEC, int LANES, int K>
struct NormSlice {
    int pos[K], skip;
    __device__ __forceinline__ explicit NormSlice(int t, int width) {
#pragma unroll
        for (int k = 0; k < K; ++k) pos[k] = (k * LANES + t) * VEC;
        const int at = pos[K - 1], last = width - VEC;
        skip = at >= width ? VEC : at > last ? at - last : 0;
        if (at > last) pos[K - 1] = last;
    }
    __device__ __forceinline__ bool own(int k, int j) const { return k < K - 1 || j >= skip; }
    __device__ __forceinline__ bool any(int k) const { return k < K - 1 || skip < VEC; }
};

template <typename T, int VEC, int K>
struct NormRow {
    T v[K][VEC];
    template <bool ONCE>
    __device__ __forceinline__ void load(const T *row, const int (&pos)[K]) {
#pragma unroll
        for (int k = 0; k < K; ++k) load_any<T, VEC, ONCE>(row + pos[k], v[k]);
    }
};

// x - mu and 1 / deviation of a row in registers.
template <typename T, int VEC, int LANES, int K>
__device__ __forceinline__ float norm_mean(const NormRow<T, VEC, K> &x, const NormSlice<VEC, LANES, K> &sl, float inv_width,
                                           float *lds) {
    float s[1] = {0.f};
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < VEC; ++j) s[0] += sl.own(k, j) ? (float)x.v[k][j] : 0.f;
    RowSums<LANES, 1>::take(s, lds);
    return s[0] * inv_width;
}

template <typename T, int VEC, int LANES, int K, bool ONCE>
__global__ __launch_bounds__(LANES > kNormThreads ? LANES : kNormThreads) void norm_forward(
    const T *__restrict__ X, int64_t x_stride, const float *__restrict__ gain, const float *__restrict__ bias, T *__restrict__ Y,
    int64_t y_stride, int64_t rows, int width, float eps)
{
    constexpr int THREADS = LANES > kNormThreads ? LANES : kNormThreads, PER = THREADS / LANES;
    __shared__ float lds[LANES > 64 ? 2 * LANES / 64 : 1];
    const int t = threadIdx.x % LANES, mine = threadIdx.x / LANES;
    const NormSlice<VEC, LANES, K> sl(t, width);
    const float inv_width = 1.f / (float)width;
    float w[K][VEC], b[K][VEC];
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            w[k][j] = gain ? gain[sl.pos[k] + j] : 1.f;
            b[k][j] = bias ? bias[sl.pos[k] + j] : 0.f;
        }
    const int64_t step = (int64_t)gridDim.x * PER;
    int64_t row = (int64_t)blockIdx.x * PER + mine;
    NormRow<T, VEC, K> next;
    next.template load<ONCE>(X + (row < rows ? row : rows - 1) * x_stride, sl.pos);
    for (int64_t base = (int64_t)blockIdx.x * PER; base < rows; base += step, row += step) {  // (uniform: rows beyond the last are not written)
        const NormRow<T, VEC, K> x = next;
        if (base + step < rows) next.template load<ONCE>(X + (row + step < rows ? row + step : rows - 1) * x_stride, sl.pos);
        const float mu = norm_mean<T, VEC, LANES, K>(x, sl, inv_width, lds);
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float d = sl.own(k, j) ? (float)x.v[k][j] - mu : 0.f;
                s[0] += d;
                s[1] = fmaf(d, d, s[1]);
            }
        RowSums<LANES, 2>::take(s, lds);
        const float left = s[0] * inv_width, var = fmaxf(fmaf(-left, left, s[1] * inv_width), 0.f);
        const float r = 1.f / sqrtf(var + eps) + (s[1] - s[1]);  // (NaN of a sum that is not finite)
        if (row < rows)
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (sl.any(k)) {
                    T y[VEC];
#pragma unroll
                    for (int j = 0; j < VEC; ++j)
                        y[j] = (T)fmaf(((float)x.v[k][j] - mu - left) * r, w[k][j], b[k][j]);
                    store_any<T, VEC>(Y + row * y_stride + sl.pos[k], y);
                }
    }
}

// Workgroup b takes chunk b % chunks of the rows of example b / chunks; a thread adds up its columns' gradients in registers,
// the workgroup's groups of threads add theirs through LDS in order.  One chunk: to the example's row of G; else to `partial`
// [examples][chunks][1 or 2][width], which norm_grad_finish adds up in order.  So the sums do not depend on what else runs.
template <typename T, int VEC, int LANES, int K, bool ONCE>
__global__ __launch_bounds__(LANES > kNormThreads ? LANES : kNormThreads) void norm_backward(
    TokenRows tok, int chunks, const T *__restrict__ X, int64_t x_stride, const T *__restrict__ DY, int64_t dy_stride,
    const float *__restrict__ gain, T *__restrict__ DX, int64_t dx_stride, float *__restrict__ G, int64_t g_stride, int with_bias,
    float *__restrict__ partial, int width, float eps)
{
    constexpr int THREADS = LANES > kNormThreads ? LANES : kNormThreads, PER = THREADS / LANES, COLS = LANES * VEC * K;
    __shared__ float lds[LANES > 64 ? 4 * LANES / 64 : 1];
    __shared__ float part[PER > 1 ? PER * COLS : 1];
    const int t = threadIdx.x % LANES, mine = threadIdx.x / LANES;
    const int64_t e = tok.base + blockIdx.x / chunks;
    const int c = (int)(blockIdx.x % chunks);
    const RowSpan span = rows_of(tok, e);
    const int64_t per = (span.count + chunks - 1) / chunks;
    const int64_t t0 = c * per < span.count ? c * per : span.count, t1 = t0 + per < span.count ? t0 + per : span.count;
    const NormSlice<VEC, LANES, K> sl(t, width);
    const float inv_width = 1.f / (float)width;
    float w[K][VEC], dw[K][VEC], db[K][VEC];
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            w[k][j] = gain ? gain[sl.pos[k] + j] : 1.f;
            dw[k][j] = db[k][j] = 0.f;
        }
    if (t0 < t1) {  // uniform
        NormRow<T, VEC, K> next_x, next_y;
        const auto fetch = [&](int64_t at) {
            const int64_t row = span.first + (at < t1 ? at : t1 - 1);
            next_x.template load<ONCE>(X + row * x_stride, sl.pos);
            next_y.template load<ONCE>(DY + row * dy_stride, sl.pos);
        };
        fetch(t0 + mine);
        for (int64_t base = t0; base < t1; base += PER) {
            const int64_t at = base + mine;
            const NormRow<T, VEC, K> x = next_x, dy = next_y;
            if (base + PER < t1) fetch(at + PER);
            const bool live = at < t1;
            const float mu = norm_mean<T, VEC, LANES, K>(x, sl, inv_width, lds);
            float s[4] = {0.f, 0.f, 0.f, 0.f};  // sums of d, d^2, g, g d
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const bool own = sl.own(k, j);
                    const float d = own ? (float)x.v[k][j] - mu : 0.f, g = own ? w[k][j] * (float)dy.v[k][j] : 0.f;
                    s[0] += d;
                    s[1] = fmaf(d, d, s[1]);
                    s[2] += g;
                    s[3] = fmaf(g, d, s[3]);
                }
            RowSums<LANES, 4>::take(s, lds);
            const float left = s[0] * inv_width, var = fmaxf(fmaf(-left, left, s[1] * inv_width), 0.f);
            const float r = 1.f / sqrtf(var + eps) + (s[1] - s[1]);
            const float mean_g = s[2] * inv_width, mean_gh = r * fmaf(-left, s[2], s[3]) * inv_width;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                T out[VEC];
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float y = (float)dy.v[k][j], hat = ((float)x.v[k][j] - mu - left) * r;
                    out[j] = (T)(r * (fmaf(w[k][j], y, -mean_g) - hat * mean_gh));
                    if (live) {
                        dw[k][j] = fmaf(y, hat, dw[k][j]);
                        db[k][j] += y;
                    }
                }
                if (DX && live && sl.any(k)) store_any<T, VEC>(DX + (span.first + at) * dx_stride + sl.pos[k], out);
            }
        }
    }
    if (!G && !partial) return;
    float *to = chunks > 1 ? partial + (e * chunks + c) * (1 + with_bias) * width : G + e * g_stride;
    if constexpr (PER == 1) {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (sl.own(k, j)) {
                    to[sl.pos[k] + j] = dw[k][j];
                    if (with_bias) to[width + sl.pos[k] + j] = db[k][j];
                }
    } else {
        for (int which = 0; which <= with_bias; ++which) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int j = 0; j < VEC; ++j)
                    if (sl.own(k, j)) part[mine * COLS + sl.pos[k] + j] = which ? db[k][j] : dw[k][j];
            __syncthreads();
            for (int col = threadIdx.x; col < width; col += THREADS) {
                float sum = 0.f;
#pragma unroll
                for (int g = 0; g < PER; ++g) sum += part[g * COLS + col];
                to[which * width + col] = sum;
            }
        }
    }
}

// G[e][col] = sum over the chunks, in order and in double: 32 columns a workgroup, eight threads a column.
__global__ __launch_bounds__(256) void norm_grad_finish(const float *__restrict__ partial, int chunks, int cols,
                                                        float *__restrict__ G, int64_t g_stride)
{
    __shared__ double part[8][33];
    const int groups = (cols + 31) / 32, lane = threadIdx.x & 31, sub = threadIdx.x >> 5;
    const int64_t e = blockIdx.x / groups;
    const int col = (int)(blockIdx.x - e * groups) * 32 + lane, cc = col < cols ? col : cols - 1;
    const float *from = partial + e * chunks * (int64_t)cols + cc;
    const int c0 = (int)((int64_t)sub * chunks / 8), c1 = (int)((int64_t)(sub + 1) * chunks / 8);
    double acc = 0.0;
#pragma unroll 8
    for (int c = c0; c < c1; ++c) acc += (double)from[(int64_t)c * cols];
    part[sub][lane] = acc;
    __syncthreads();
    if (sub == 0 && col < cols) {
        double sum = 0.0;
#pragma unroll
        for (int q = 0; q < 8; ++q) sum += part[q][lane];
        G[e * g_stride + col] = (float)sum;
    }
}

}  // namespace cdgrab
