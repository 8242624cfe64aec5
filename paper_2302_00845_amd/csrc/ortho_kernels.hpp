// Orthogonalised updates: X_0 = M / ||M||_F (the shorter side as rows), then `steps` times
//     A = X X^T,  X <- a X + (b A + c A^2) X,
// which takes every singular value s to a s + b s^3 + c s^5 and leaves the singular vectors.
//
// Small singular values grow by a factor of a per step (3.4 by default), and so does what rounding does to their vectors:
// products in fp32, or as good, are needed between steps even for results of fewer bits (with one product of bf16 factors the
// result is off by some percent).  Three forms:
//   - short side up to 32, and up to kOrthoNarrow where the matrix does not fit in LDS: X_K = P_K X_0 with P_K a polynomial in
//     A_0 = X_0 X_0^T.  One pass over the matrix for A_0 in double, the recurrence on matrices of the short side (all of which
//     commute), one pass for the product: bytes of the matrix twice.  (In fp32 this form loses too much: the small
//     eigenvalues of A_0 are the squares of the singular values.)
//     Where the matrix lacks rank A_0 has eigenvalues that are rounding, of either sign, and the recurrence makes them grow by a^2
//     per step; for a negative one near -1 the polynomial has no bound.  So one A_0 serves as many steps as keep them small
//     (ortho_gram_steps: eleven with the default coefficients); then X is made, in double, and its Gram matrix anew.
//   - short side up to 128 of a matrix that fits in LDS as pairs with its Gram matrix (OrthoSmall): the products as they stand,
//     all steps in one workgroup.
//   - else the products as they stand, three launches a step.  A and A^2 are symmetric: half of their tiles are computed.
// Pairs: in the last two forms factors are held as the sum of two fp16 (22 bits), and of the four products of the parts the three
// larger are taken: errors as of fp32 products (simulated on matrices of 256 .. 2048: 1.0 to 1.1 times), at a third of the fp16
// MFMA rate, five times the fp32 MFMA's.  fp16 has the digits but not the range: the norm bounds every element, a fixed power of two
// in front uses the range, and the small part is held kOrthoLift times as large, so that it has its eleven bits as long as the
// large part has.  Elements of X from 2^-27 of the norm on have 22 bits, smaller ones are off by about 2^-49 of the norm (with
// the small part as it is: from 2^-16 on, and by 2^-38; rows 1e-7 of the others came out half a percent off).
#pragma once
#include "narrow_common.hpp"
#include "mfma_tiles.hpp"

namespace cdgrab {

typedef double f64x4 __attribute__((ext_vector_type(4)));

template <typename T> __device__ __forceinline__ double ortho_double(T v) { return (double)(float)v; }
__device__ __forceinline__ double ortho_double(double v) { return v; }

// Where a matrix's elements lie and where results go: element (i, j), i along the short side, at i * si + j * sj.
// `sub`: instead of storing O, subtract rate * O from the fp32 array of the same strides (an optimiser's step).
template <typename T>
struct OrthoIo {
    const T *M;
    T *O;
    float *sub;
    float rate;
    int64_t m_i, m_j, m_matrix, o_i, o_j, o_matrix;
    int short_side, long_side;
    __device__ __forceinline__ double at(int64_t b, int i, int64_t j) const { return ortho_double(M[b * m_matrix + i * m_i + j * m_j]); }
    __device__ __forceinline__ void put(int64_t b, int i, int64_t j, double v) const {  // (rounded to fp32, unless O is of doubles)
        const int64_t p = b * o_matrix + i * o_i + j * o_j;
        if (sub) sub[p] = sub[p] - rate * (float)v;
        else if constexpr (sizeof(T) == 8) O[p] = v;
        else O[p] = (T)(float)v;
    }
    // Eight results side by side in memory, from element p on, of which the first n are there.
    __device__ __forceinline__ void put8(int64_t p, const float (&v)[8], int n) const {
        if (!sub && n >= 8) {
            T x[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) x[q] = (T)v[q];
            store_any<T, 8>(O + p, x);
        } else {
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (q < n) {
                    if (sub) sub[p + q] = sub[p + q] - rate * v[q];
                    else O[p + q] = (T)v[q];
                }
        }
    }
};

struct OrthoCoeffs {
    double a, b, c;
    int64_t per_gram;  // steps that one Gram matrix serves
};

// 1 / sqrt of a sum of squares: zero of zero (such a matrix stays as it is), NaN of infinity.
__device__ __forceinline__ double ortho_root(double t) { return t == 0.0 ? 0.0 : 1.0 / sqrt(t) + (t - t); }

// ---- short side up to kOrthoNarrow -----------------------------------------------------------------------------------------
constexpr int kOrthoNarrow = 64;
constexpr int kOrthoThreads = 1024;

// Symmetric matrices of NT x NT tiles of 16 x 16, a tile as a 16 x 16 x 4 MFMA leaves it: lane l holds entries (4 v + l / 16, l % 16),
// v = 0 .. 3, and they lie in LDS in that order, [tile][v][lane].  Read as an operand, entry v of tile (k, i) is what the v-th
// MFMA of a product wants of tile (i, k), its transpose, on the left and of tile (k, i) itself on the right: no other layout
// is needed, and neither shuffles nor padding.
template <int NT>
struct OrthoTiles {
    static_assert(NT * NT <= kOrthoThreads / 64, "a wavefront per tile");
    static constexpr int LEN = NT * NT * 256;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool mine = wave < NT * NT;
    const int ti = wave / NT, tj = wave % NT;

    // this wavefront's tile of X^T Y (X Y where X is symmetric), X and Y in LDS
    __device__ __forceinline__ f64x4 product(const double *X, const double *Y) const {
        f64x4 even = {0.0, 0.0, 0.0, 0.0}, odd = {0.0, 0.0, 0.0, 0.0};
        if (mine) {
            const double *x = X + ti * 256 + lane, *y = Y + tj * 256 + lane;
#pragma unroll
            for (int k = 0; k < NT; ++k)
#pragma unroll
                for (int v = 0; v < 4; v += 2) {
                    even = __builtin_amdgcn_mfma_f64_16x16x4f64(x[k * NT * 256 + v * 64], y[k * NT * 256 + v * 64], even, 0, 0, 0);
                    odd = __builtin_amdgcn_mfma_f64_16x16x4f64(x[k * NT * 256 + v * 64 + 64], y[k * NT * 256 + v * 64 + 64], odd, 0, 0, 0);
                }
        }
        return even + odd;
    }
    static __device__ __forceinline__ f64x4 product(f64x4 x, f64x4 y) {  // (of single tiles in registers)
        f64x4 even = {0.0, 0.0, 0.0, 0.0}, odd = {0.0, 0.0, 0.0, 0.0};
        even = __builtin_amdgcn_mfma_f64_16x16x4f64(x[0], y[0], even, 0, 0, 0);
        odd = __builtin_amdgcn_mfma_f64_16x16x4f64(x[1], y[1], odd, 0, 0, 0);
        even = __builtin_amdgcn_mfma_f64_16x16x4f64(x[2], y[2], even, 0, 0, 0);
        odd = __builtin_amdgcn_mfma_f64_16x16x4f64(x[3], y[3], odd, 0, 0, 0);
        return even + odd;
    }
    __device__ __forceinline__ f64x4 load(const double *X) const {
        f64x4 x = {0.0, 0.0, 0.0, 0.0};
        if (mine)
#pragma unroll
            for (int v = 0; v < 4; ++v) x[v] = X[wave * 256 + v * 64 + lane];
        return x;
    }
    __device__ __forceinline__ void store(double *X, f64x4 x) const {
        if (mine)
#pragma unroll
            for (int v = 0; v < 4; ++v) X[wave * 256 + v * 64 + lane] = x[v];
    }
    // s on the diagonal, for the first n rows
    __device__ __forceinline__ f64x4 diagonal(double s, int n) const {
        f64x4 x;
#pragma unroll
        for (int v = 0; v < 4; ++v) x[v] = ti == tj && 4 * v + (lane >> 4) == (lane & 15) && ti * 16 + (lane & 15) < n ? s : 0.0;
        return x;
    }
    // where entry (i, j) lies
    static __device__ __forceinline__ int at(int i, int j) {
        return ((i >> 4) * NT + (j >> 4)) * 256 + ((i & 15) >> 2) * 64 + (i & 3) * 16 + (j & 15);
    }
};

// P (in LDS) from the Gram matrix of M in A (in LDS), entries beyond the short side zero:
//   A <- A / trace(A), P <- I / sqrt(trace) (not for an X that steps have made: `first`); steps times:
//   Q = a I + b A + c A^2, P <- Q P, A <- Q A Q.
// Everything commutes and is symmetric, but for rounding, which Q A Q takes between eigenvalues l and k to (f(l) - f(k)) / (l - k) of it,
// f(l) = l q(l)^2, while A Q Q would take it to q(k)^2, a^2 for any l beside a small k.  (785 x 10 of rank nine, twenty steps of
// 15/8, -10/8, 3/8: norm 1.0015 by A Q Q.)  A single tile stays in one wavefront's registers; more go through LDS, three
// rounds per step.
template <int NT>
struct OrthoChain {
    typedef OrthoTiles<NT> Tiles;
    double A[Tiles::LEN], Q[Tiles::LEN], P[Tiles::LEN];
    double trace;

    __device__ __forceinline__ void run(int n, int steps, int first, OrthoCoeffs c) {
        const Tiles tiles;
        __syncthreads();
        if (threadIdx.x < 64) {
            double t = (int)threadIdx.x < n ? A[Tiles::at(threadIdx.x, threadIdx.x)] : 0.0;
            t = sum_across_32(sum_across_16(dpp_add<0x140>(sum_of_eight(t))));
            if (threadIdx.x == 0) trace = t;
        }
        __syncthreads();
        const double t = first ? trace : 1.0, inv = t == 0.0 ? 0.0 : 1.0 / t;
        f64x4 a = tiles.load(A), p = tiles.diagonal(ortho_root(t), n);
        const f64x4 one = tiles.diagonal(c.a, NT * 16);
#pragma unroll
        for (int v = 0; v < 4; ++v) a[v] = a[v] * inv;
        if constexpr (NT == 1) {
            if (tiles.wave == 0)
                for (int s = 0; s < steps; ++s) {
                    f64x4 q = Tiles::product(a, a);
#pragma unroll
                    for (int v = 0; v < 4; ++v) q[v] = one[v] + c.b * a[v] + c.c * q[v];
                    p = Tiles::product(q, p);
                    a = Tiles::product(q, Tiles::product(a, q));
                }
            tiles.store(P, p);
        } else {
            tiles.store(A, a);
            tiles.store(P, p);
            __syncthreads();
            for (int s = 0; s < steps; ++s) {
                f64x4 q = tiles.product(A, A);
#pragma unroll
                for (int v = 0; v < 4; ++v) q[v] = one[v] + c.b * a[v] + c.c * q[v];
                tiles.store(Q, q);
                __syncthreads();
                if (s == 0) {  // (P is a multiple of I)
#pragma unroll
                    for (int v = 0; v < 4; ++v) p[v] = q[v] * ortho_root(t);
                } else {
                    p = tiles.product(Q, P);
                }
                const bool more = s + 1 < steps;  // (the last step's A is for nobody)
                if (more) a = tiles.product(A, Q);
                __syncthreads();
                tiles.store(P, p);
                if (more) {
                    tiles.store(A, a);
                    __syncthreads();
                    a = tiles.product(Q, A);
                    __syncthreads();
                    tiles.store(A, a);
                }
                __syncthreads();
            }
        }
        __syncthreads();
    }
};

// Gram matrix of columns j0 .. j1 - 1 (those of the long side), by the workgroup: wavefront w takes every sixteenth group of
// four columns and keeps all tiles on or above the diagonal; `to`(i, j, value) receives sums over the wavefronts, in order.
template <int NT, typename T, typename F>
__device__ __forceinline__ void ortho_gram(const OrthoIo<T> &io, int64_t b, int64_t j0, int64_t j1, double *lds, F &&to) {
    constexpr int TILES = NT * (NT + 1) / 2, WAVES = kOrthoThreads / 64, UN = 4;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, k = lane >> 4;
    f64x4 acc[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) acc[t] = f64x4{0.0, 0.0, 0.0, 0.0};
    for (int64_t jw = j0 + wave * 4; jw < j1; jw += 4 * WAVES * UN) {  // (the same for all lanes)
        const int64_t j = jw + k;
        T raw[UN][NT];
#pragma unroll
        for (int u = 0; u < UN; ++u)  // (clamped, not branched: all loads on their way together)
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int64_t jj = j + u * 4 * WAVES;
                const int i = t * 16 + r;
                raw[u][t] = io.M[b * io.m_matrix + (i < io.short_side ? i : 0) * io.m_i + (jj < j1 ? jj : j0) * io.m_j];
            }
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            double x[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t)
                x[t] = t * 16 + r < io.short_side && j + u * 4 * WAVES < j1 ? ortho_double(raw[u][t]) : 0.0;
            int at = 0;
#pragma unroll
            for (int ti = 0; ti < NT; ++ti)
#pragma unroll
                for (int tj = ti; tj < NT; ++tj, ++at) acc[at] = __builtin_amdgcn_mfma_f64_16x16x4f64(x[ti], x[tj], acc[at], 0, 0, 0);
        }
        // Where the compiler copies the results at the loop's head it has put 4 wait states instead of 18 between the last product and
        // the copy of its last two registers: rows 28 .. 31 of a tile missed products.  (As this stands it does not copy them.)
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_nop 15\n\ts_nop 15");
        __builtin_amdgcn_sched_barrier(0);
    }
    int at = 0;
#pragma unroll
    for (int ti = 0; ti < NT; ++ti)
#pragma unroll
        for (int tj = ti; tj < NT; ++tj, ++at) {
            __syncthreads();
#pragma unroll
            for (int v = 0; v < 4; ++v) lds[wave * 256 + v * 64 + lane] = acc[at][v];
            __syncthreads();
            if (threadIdx.x < 256) {
                double sum = 0.0;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) sum += lds[w * 256 + threadIdx.x];
                const int v = threadIdx.x >> 6, l = threadIdx.x & 63;
                to(ti * 16 + 4 * v + (l >> 4), tj * 16 + (l & 15), sum);
            }
        }
}

// O = P X for columns j0 .. j1 - 1, in double (P's large entries cancel): a wavefront takes sixteen columns at a time, and has
// read them before it writes them (O may be M).
template <int NT, typename T>
__device__ __forceinline__ void ortho_apply(const OrthoIo<T> &io, int64_t b, int64_t j0, int64_t j1, const double *P) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, k = lane >> 4;
    for (int64_t jw = j0 + wave * 16; jw < j1; jw += 16 * (kOrthoThreads / 64)) {
        const int64_t j = jw + r;
        T raw[NT][4];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int i = t * 16 + 4 * v + k;
                raw[t][v] = io.M[b * io.m_matrix + (i < io.short_side ? i : 0) * io.m_i + (j < j1 ? j : j0) * io.m_j];
            }
#pragma unroll
        for (int ti = 0; ti < NT; ++ti) {
            f64x4 even = {0.0, 0.0, 0.0, 0.0}, odd = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int v = 0; v < 4; v += 2) {
                    const double *p = P + (t * NT + ti) * 256 + v * 64 + lane;
                    const bool here = t * 16 + 4 * v + k < io.short_side, next = t * 16 + 4 * v + 4 + k < io.short_side;
                    even = __builtin_amdgcn_mfma_f64_16x16x4f64(p[0], here ? ortho_double(raw[t][v]) : 0.0, even, 0, 0, 0);
                    odd = __builtin_amdgcn_mfma_f64_16x16x4f64(p[64], next ? ortho_double(raw[t][v + 1]) : 0.0, odd, 0, 0, 0);
                }
            const f64x4 sum = even + odd;
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int i = ti * 16 + 4 * v + k;
                if (i < io.short_side && j < j1) io.put(b, i, j, sum[v]);
            }
        }
    }
}

// One workgroup per matrix.
template <int NT, typename T>
__global__ __launch_bounds__(kOrthoThreads) void ortho_narrow(OrthoIo<T> io, int steps, int first, OrthoCoeffs c)
{
    __shared__ OrthoChain<NT> s;
    __shared__ double lds[kOrthoThreads * 4];
    const int64_t b = blockIdx.x;
    ortho_gram<NT>(io, b, 0, io.long_side, lds, [&](int i, int j, double v) {
        s.A[OrthoTiles<NT>::at(i, j)] = v;
        s.A[OrthoTiles<NT>::at(j, i)] = v;
    });
    s.run(io.short_side, steps, first, c);
    ortho_apply<NT>(io, b, 0, io.long_side, s.P);
}

// Long matrices: chunks of columns for the Gram matrix, then the recurrence, then chunks of columns for the product.
template <int NT, typename T>
__global__ __launch_bounds__(kOrthoThreads) void ortho_narrow_gram(OrthoIo<T> io, int chunks, int64_t per, double *__restrict__ parts)
{
    __shared__ double lds[kOrthoThreads * 4];
    const int64_t b = blockIdx.x / chunks, c = blockIdx.x % chunks;
    const int64_t j1 = (c + 1) * per < io.long_side ? (c + 1) * per : io.long_side;
    double *to = parts + (int64_t)blockIdx.x * OrthoTiles<NT>::LEN;
    ortho_gram<NT>(io, b, c * per, j1, lds, [&](int i, int j, double v) { to[OrthoTiles<NT>::at(i, j)] = v; });
}
template <int NT>
__global__ __launch_bounds__(kOrthoThreads) void ortho_narrow_chain(int n, int chunks, const double *__restrict__ parts, int steps,
                                                                    int first, OrthoCoeffs c, double *__restrict__ out)
{
    __shared__ OrthoChain<NT> s;
    typedef OrthoTiles<NT> Tiles;
    const double *from = parts + (int64_t)blockIdx.x * chunks * Tiles::LEN;
    for (int q = threadIdx.x; q < Tiles::LEN; q += kOrthoThreads) {
        const int ti = q / 256 / NT, tj = q / 256 % NT;
        if (ti > tj) continue;
        double sum = 0.0;
#pragma unroll 8
        for (int p = 0; p < chunks; ++p) sum += from[(int64_t)p * Tiles::LEN + q];
        s.A[q] = sum;
        const int i = ti * 16 + (q % 256 / 64) * 4 + q % 64 / 16, j = tj * 16 + q % 16;
        if (ti < tj) s.A[Tiles::at(j, i)] = sum;
    }
    s.run(n, steps, first, c);
    for (int q = threadIdx.x; q < Tiles::LEN; q += kOrthoThreads) out[(int64_t)blockIdx.x * Tiles::LEN + q] = s.P[q];
}
template <int NT, typename T>
__global__ __launch_bounds__(kOrthoThreads) void ortho_narrow_apply(OrthoIo<T> io, int chunks, int64_t per, const double *__restrict__ P)
{
    __shared__ double p[OrthoTiles<NT>::LEN];
    const int64_t b = blockIdx.x / chunks, c = blockIdx.x % chunks;
    for (int q = threadIdx.x; q < OrthoTiles<NT>::LEN; q += kOrthoThreads) p[q] = P[b * OrthoTiles<NT>::LEN + q];
    __syncthreads();
    ortho_apply<NT>(io, b, c * per, (c + 1) * per < io.long_side ? (c + 1) * per : io.long_side, p);
}

// More steps than one Gram matrix serves: X between stretches of steps, [matrix] and as the caller's rows lie, dense.  OUT: from X
// to where the results go.
template <typename T, bool OUT>
__global__ __launch_bounds__(256) void ortho_doubles(OrthoIo<T> io, uint32_t groups, double *__restrict__ X)
{
    const int64_t b = blockIdx.x / groups, cells = (int64_t)io.short_side * io.long_side;
    const bool turn = (OUT ? io.o_i : io.m_i) < (OUT ? io.o_j : io.m_j);
    for (int64_t q = (blockIdx.x - b * groups) * 256 + threadIdx.x; q < cells; q += (int64_t)groups * 256) {
        const int i = (int)(turn ? q % io.short_side : q / io.long_side);
        const int64_t j = turn ? q / io.short_side : q % io.long_side;
        if constexpr (OUT) io.put(b, i, j, X[b * cells + q]);
        else X[b * cells + q] = io.at(b, i, j);
    }
}

// ---- longer sides: products of pairs of fp16 --------------------------------------------------------------------------------
constexpr float kOrthoScaleX = 8192.f, kOrthoScaleA = 2048.f;  // X up to 7.9, A and b A + c A^2 up to 31 (the host sees to it)
constexpr float kOrthoLift = 2048.f;  // of the small parts
constexpr int kOrthoSums = 64;  // sums of squares per matrix

// Sums of squares of matrix b of `rows` x `cols` as it lies in memory; a wavefront takes every 256th row.
template <typename T>
__global__ __launch_bounds__(256) void ortho_squares(const T *__restrict__ M, int64_t matrix, int64_t rows, int64_t cols, int64_t stride,
                                                     double *__restrict__ sums)
{
    __shared__ double part[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t b = blockIdx.x / kOrthoSums, c = blockIdx.x % kOrthoSums;
    double acc = 0.0;
    for (int64_t r = c * 4 + wave; r < rows; r += 4 * kOrthoSums) {
        const T *row = M + b * matrix + r * stride;
#pragma unroll 8
        for (int64_t q = lane; q < cols; q += 64) {
            const double x = (double)(float)row[q];
            acc = __builtin_fma(x, x, acc);
        }
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) acc += __shfl_xor(acc, off, 64);
    if (lane == 0) part[wave] = acc;
    __syncthreads();
    if (threadIdx.x == 0) sums[blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

// v as a pair of fp16, and what is made of pairs: a value, a product from its large and its small terms.
__device__ __forceinline__ void ortho_split(float v, f16_t &hi, f16_t &lo) {
    hi = (f16_t)v;
    lo = (f16_t)((v - (float)hi) * kOrthoLift);
}
__device__ __forceinline__ float ortho_join(float large, float small) { return fmaf(small, 1.f / kOrthoLift, large); }

// X_0 as pairs, [short][long] padded with zeros to sp x lp: 32 x 32 elements a workgroup, turned through LDS where the rows
// of M are the long side.
template <typename T>
__global__ __launch_bounds__(256) void ortho_begin(OrthoIo<T> io, const double *__restrict__ sums, f16_t *__restrict__ X, int sp, int lp)
{
    __shared__ float tile[32][33];
    __shared__ double norm;
    const int ti = sp / 32, tj = lp / 32;
    const int64_t b = blockIdx.x / (ti * tj);
    const int at = (int)(blockIdx.x % (ti * tj)), i0 = at / tj * 32, j0 = at % tj * 32;
    if (threadIdx.x < 64) {
        double t = sums[b * kOrthoSums + threadIdx.x];
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) t += __shfl_xor(t, off, 64);
        if (threadIdx.x == 0) norm = ortho_root(t);
    }
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const bool turn = io.m_i < io.m_j;
    float v[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int i = i0 + (turn ? x : y + 8 * q), j = j0 + (turn ? y + 8 * q : x);
        v[q] = i < io.short_side && j < io.long_side ? (float)io.M[b * io.m_matrix + i * io.m_i + j * io.m_j] : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float n = (float)((double)v[q] * norm);
        if (turn) tile[x][y + 8 * q] = n;
        else tile[y + 8 * q][x] = n;
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int64_t p = b * 2 * sp * (int64_t)lp + pair_at(i0 + y + 8 * q, j0 + x, lp);
        f16_t hi, lo;
        ortho_split(tile[y + 8 * q][x] * kOrthoScaleX, hi, lo);
        X[p] = hi;
        X[p + 32] = lo;
    }
}

enum OrthoWhat { kOrthoGram, kOrthoShare, kOrthoPoly, kOrthoStep, kOrthoLast };

// One tile of a product of pairs, L R^T (Gram, Poly: R's rows, both with their elements along k) or L R (Step, Last: R's rows
// along k), then
//   Gram: A = X X^T;  Share: the sums of a share of k, for ortho_gram_finish;  Poly: B = b A + c A A;  Step: X' = a X + B X;  Last: O = (a X + B X) to the caller's array.
// K is a multiple of 32, the tile's sides T of 32: nothing to clip but O.
struct OrthoProduct {
    const f16_t *L, *R, *E;  // factors, what is added: matrices of pairs
    f16_t *C;                // the result
    int64_t l_ld, r_ld, c_ld, l_matrix, r_matrix, c_matrix;  // (E lies as C does; fp16 from matrix to matrix)
    int k, tiles_m, tiles_n;
    float alpha, beta;  // result = alpha E + beta (product as multiplied)
    int shares;         // Share: of k, and where their sums go: [matrix][share][tile][T][T]
    float *sums;
};

// The t-th of the tiles on or above the diagonal, column after column.
__device__ __forceinline__ void ortho_upper_tile(int t, int &tm, int &tn) {
    tn = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
    while ((tn + 1) * (tn + 2) / 2 <= t) ++tn;
    while (tn * (tn + 1) / 2 > t) --tn;
    tm = t - tn * (tn + 1) / 2;
}

// Eight neighbours of a row of a matrix of pairs.
__device__ __forceinline__ void ortho_store_pairs(f16_t *p, const float (&v)[8]) {
    f16x8 hi, lo;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        f16_t x, y;
        ortho_split(v[j], x, y);
        hi[j] = x;
        lo[j] = y;
    }
    *reinterpret_cast<f16x8 *>(p) = hi;
    *reinterpret_cast<f16x8 *>(p + 32) = lo;
}

// QUADS: that many times four wavefronts share a tile, each four with every QUADS-th stage of k and stages of their own (for where
// tiles are fewer than CUs and a tile's time is a chain of stages).
template <int T, int NS, int QUADS, int WHAT, typename U>
__global__ __launch_bounds__(256 * QUADS, NS * T * 256 > 80 * 1024 ? 1 : 2) void ortho_product_tile(OrthoProduct p, OrthoIo<U> io)
{
    constexpr bool ACROSS = WHAT == kOrthoStep || WHAT == kOrthoLast, SYM = !ACROSS;
    typedef PairTile<T> O;
    constexpr int MB = T / 64, LD = T + 1;  // (eight rows further is eight banks further)
    constexpr int STAGE = 2 * O::LEN, BYTES = QUADS * NS * STAGE * 2, OUT = T / 2 * LD * 4, LOADS = 2 * O::CALLS;
    __shared__ __align__(16) char lds[BYTES > OUT ? BYTES : OUT];
    const int lane = threadIdx.x & 63, quad = QUADS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);
    const int tid = threadIdx.x & 255, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave >> 1, wn = wave & 1;
    f16_t *stage = reinterpret_cast<f16_t *>(lds) + quad * NS * STAGE;
    const int per = SYM ? p.tiles_m * (p.tiles_m + 1) / 2 : p.tiles_m * p.tiles_n;
    const uint32_t id = xcd_neighbours(blockIdx.x, gridDim.x);
    const uint32_t group = id / (uint32_t)per;  // matrix, or matrix and share
    const int64_t b = WHAT == kOrthoShare ? group / (uint32_t)p.shares : group;
    int tm, tn;
    if constexpr (SYM) {
        ortho_upper_tile((int)(id - group * per), tm, tn);
    } else {
        const int t = (int)(id - group * per);
        tm = t % p.tiles_m;
        tn = t / p.tiles_m;
    }
    int stages = p.k / O::KC, begin = 0;
    if constexpr (WHAT == kOrthoShare) {  // (a share has a multiple of QUADS stages, and one at least)
        const int units = stages / QUADS, share = (int)(group % (uint32_t)p.shares);
        begin = (int)((int64_t)units * share / p.shares) * QUADS;
        stages = (int)((int64_t)units * (share + 1) / p.shares) * QUADS - begin;
    }
    stages /= QUADS;
    const f16_t *const left = p.L + b * p.l_matrix + (int64_t)tm * T * 2 * p.l_ld + begin * 64;
    const f16_t *const right = p.R + b * p.r_matrix + begin * 64 + (ACROSS ? (int64_t)tn * T * 2 : (int64_t)tn * T * 2 * p.r_ld);
    // (the products with the small parts in sums of their own, of another scale; and as parts of one sum each would round it once
    // more, 2468 columns 3.3e-6 off instead of 1.9e-6)
    f32x16 acc[MB][MB], low[MB][MB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < MB; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[i][j][q] = low[i][j][q] = 0.f;
    const PairFetch<T, false> fetch_l(p.l_ld, wave, lane);
    const PairFetch<T, ACROSS> fetch_r(p.r_ld, wave, lane);
    const auto fetch = [&](int q, int buf) {
        f16_t *s = stage + buf * STAGE;
        q = q * QUADS + quad;
        fetch_l(left + q * 64, s, wave);
        fetch_r(right + (ACROSS ? q * O::KC * 2 * p.r_ld : q * 64), s + O::LEN, wave);
    };
    struct Operands { f16x8 lh[MB], ll[MB], rh[MB], rl[MB]; };
    const PairRead<T, false> read_l(wm * (T / 2), lane);
    const PairRead<T, ACROSS> read_r(wn * (T / 2), lane);
    const auto read = [&](Operands &o, int buf, int h) {
        const f16_t *s = stage + buf * STAGE;
#pragma unroll
        for (int i = 0; i < MB; ++i) {
            o.lh[i] = read_l.high(s, h, i);
            o.rl[i] = read_r.low(s + O::LEN, h, i);
            o.rh[i] = read_r.high(s + O::LEN, h, i);
            o.ll[i] = read_l.low(s, h, i);
        }
    };
    const auto multiply = [&](const Operands &o) {  // (products that add to the same sum apart from each other)
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < MB; ++j) low[i][j] = mfma32(o.lh[i], o.rl[j], low[i][j]);
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < MB; ++j) acc[i][j] = mfma32(o.lh[i], o.rh[j], acc[i][j]);
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < MB; ++j) low[i][j] = mfma32(o.ll[i], o.rh[j], low[i][j]);
    };
    const auto interleave = [] {  // a few reads, a few products, and so on (left alone, the compiler puts the reads last)
#pragma unroll
        for (int q = 0; q < 6; ++q) {
            __builtin_amdgcn_sched_group_barrier(0x100, ACROSS ? 3 : 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x8, MB, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // Half a stage's operands are read while the other half's products run; between the halves the workgroup meets: the next
    // stage is there, and everybody has read this one, whose place the next loads take.
    int sent = 0;
    for (; sent < NS && sent < stages; ++sent) fetch(sent, sent);
    if (sent == NS) stage_barrier<(NS - 1) * LOADS>();
    else stage_barrier<0>();
    Operands first, second;
    read(first, 0, 0);
    for (int q0 = 0; q0 + 1 < stages; q0 += NS)
#pragma unroll
        for (int buf = 0; buf < NS; ++buf) {  // (a constant: so are the places in LDS)
            const int q = q0 + buf;
            if (q + 1 >= stages) break;
            read(second, buf, 1);
            multiply(first);
            interleave();
            if (q + NS <= stages) stage_barrier<(NS - 2) * LOADS>();
            else stage_barrier<0>();
            if (sent < stages) fetch(sent++, buf);
            read(first, (buf + 1) % NS, 0);
            multiply(second);
            interleave();
        }
    read(second, (stages - 1) % NS, 1);
    multiply(first);
    multiply(second);
    if constexpr (QUADS > 1) {  // the second four's sums to the first
        static_assert(QUADS == 2 && MB == 1 && BYTES >= 256 * 32 * 4, "");
        float *const sums = reinterpret_cast<float *>(lds) + wave * 32 * 64 + lane;
        __syncthreads();
        if (quad == 1)
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                sums[q * 64] = acc[0][0][q];
                sums[(q + 16) * 64] = low[0][0][q];
            }
        __syncthreads();
        if (quad == 0)
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                acc[0][0][q] += sums[q * 64];
                low[0][0][q] += sums[(q + 16) * 64];
            }
    }
    if constexpr (WHAT == kOrthoShare) {
        static_assert(MB == 1, "");
        float *const to = p.sums + (int64_t)id * T * T;
        if (quad == 0)
#pragma unroll
            for (int q = 0; q < 16; ++q)
                to[(wm * 32 + 8 * (q >> 2) + 4 * (lane >> 5) + (q & 3)) * T + wn * 32 + (lane & 31)] = ortho_join(acc[0][0][q], low[0][0][q]);
        return;
    }
    // The tile goes out through LDS, half its rows at a time, so that every thread stores eight neighbours of a row; a tile
    // above the diagonal also to its mirror image.  What is added is requested before the first half is written.
    constexpr int TASKS = T / 2 * T / 8 / 256;  // of a thread, per half
    const auto place = [&](int64_t row, int64_t col) { return b * p.c_matrix + pair_at(row, col, p.c_ld); };
    f16x8 e_hi[2][TASKS], e_lo[2][TASKS];
    if constexpr (WHAT != kOrthoGram)
        if (quad == 0)
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int u = 0; u < TASKS; ++u) {
                const int q = tid + u * 256;
                const int64_t at = place(tm * T + half * (T / 2) + q / (T / 8), tn * T + q % (T / 8) * 8);
                e_hi[half][u] = *reinterpret_cast<const f16x8 *>(p.E + at);
                e_lo[half][u] = *reinterpret_cast<const f16x8 *>(p.E + at + 32);
            }
    float *out = reinterpret_cast<float *>(lds);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        __syncthreads();
        if (wm == half && quad == 0)
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < MB; ++j)
#pragma unroll
                    for (int q = 0; q < 16; ++q)
                        out[(i * 32 + 8 * (q >> 2) + 4 * (lane >> 5) + (q & 3)) * LD + wn * (T / 2) + j * 32 + (lane & 31)] =
                            p.beta * ortho_join(acc[i][j][q], low[i][j][q]);
        __syncthreads();
        // the values are read from LDS once more, along the other side
        const bool turn = WHAT == kOrthoLast && io.o_i < io.o_j;  // (the caller's rows are the long side)
        const bool again = turn || (SYM && tm != tn);
        const int m0 = tm * T + half * (T / 2), n0 = tn * T;
#pragma unroll
        for (int u = 0; u < TASKS; ++u) {
            if (quad != 0) break;
            const int q = tid + u * 256, r = q / (T / 8), c = q % (T / 8) * 8;
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = out[r * LD + c + j];
                if constexpr (WHAT != kOrthoGram) {
                    v[j] = fmaf(p.alpha, ortho_join((float)e_hi[half][u][j], (float)e_lo[half][u][j]), v[j]);
                    if (again) out[r * LD + c + j] = v[j];
                }
            }
            if constexpr (WHAT != kOrthoLast) {
                ortho_store_pairs(p.C + place(m0 + r, n0 + c), v);
            } else if (!turn && m0 + r < io.short_side) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] *= 1.f / kOrthoScaleX;
                io.put8(b * io.o_matrix + (m0 + r) * io.o_i + (n0 + c), v, io.long_side - n0 - c);
            }
        }
        if (!again) continue;
        __syncthreads();
#pragma unroll
        for (int u = 0; u < TASKS; ++u) {
            if (quad != 0) break;
            const int q = tid + u * 256, c = q / (T / 16), r = q % (T / 16) * 8;
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = out[(r + j) * LD + c];
            if constexpr (WHAT != kOrthoLast) {
                ortho_store_pairs(p.C + place(n0 + c, m0 + r), v);
            } else if (n0 + c < io.long_side) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] *= 1.f / kOrthoScaleX;
                io.put8(b * io.o_matrix + (n0 + c) * io.o_j + (m0 + r), v, io.short_side - m0 - r);
            }
        }
    }
}

// A = X X^T from the sums of the shares, in order.  A workgroup takes a tile.
template <int T>
__global__ __launch_bounds__(256) void ortho_gram_finish(OrthoProduct p)
{
    constexpr int LD = T + 1, TASKS = T * T / 8 / 256;
    __shared__ float out[T * LD];
    const int per = p.tiles_m * (p.tiles_m + 1) / 2;
    const int64_t b = blockIdx.x / (uint32_t)per;
    const int t = (int)(blockIdx.x - b * per);
    int tm, tn;
    ortho_upper_tile(t, tm, tn);
    const float *from = p.sums + (b * p.shares * per + t) * T * T;
    f16_t *const C = p.C + b * p.c_matrix;
#pragma unroll
    for (int u = 0; u < TASKS; ++u) {
        const int q = threadIdx.x + u * 256, r = q / (T / 8), c = q % (T / 8) * 8;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int share = 0; share < p.shares; ++share) {
            float x[8];
            load_any<float, 8>(from + (int64_t)share * per * T * T + r * T + c, x);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += x[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) out[r * LD + c + j] = v[j] = p.beta * v[j];
        ortho_store_pairs(C + pair_at(tm * T + r, tn * T + c, p.c_ld), v);
    }
    if (tm == tn) return;  // uniform
    __syncthreads();
#pragma unroll
    for (int u = 0; u < TASKS; ++u) {
        const int q = threadIdx.x + u * 256, c = q / (T / 8), r = q % (T / 8) * 8;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = out[(r + j) * LD + c];
        ortho_store_pairs(C + pair_at(tn * T + c, tm * T + r, p.c_ld), v);
    }
}

// A matrix that fits in LDS as pairs, with its Gram matrix: all steps in one workgroup.  Launches and what lies between them are
// what the products of such matrices take else: 8 matrices of 128 x 128 in 17 launches 76 us, like this 60 us; 64 x 64 in double 64
// us, like this 20.  A wavefront
// computes 32 x 32 blocks, PER of them with the same left rows, holds them while others still read what they replace, and writes
// them in pairs.  (All blocks of A and A^2: those below the diagonal would be written two bytes at a time, and eight wavefronts
// have two blocks each either way.)  X and A have rows of lp and sp elements and eight more, so that the sixteen lanes of a read
// hit different banks.
constexpr int kOrthoSmallThreads = 512;

template <typename T, int BYTES, int PER>
__global__ __launch_bounds__(kOrthoSmallThreads) void ortho_small(OrthoIo<T> io, int sp, int lp, int steps, OrthoCoeffs c)
{
    constexpr int WAVES = kOrthoSmallThreads / 64, MOST = PER == 1 ? 1 : 2;  // units of PER blocks of a wavefront at most
    __shared__ __align__(16) f16_t lds[BYTES / 2];
    __shared__ double part[WAVES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t b = blockIdx.x;
    const int xs = lp + 8, as = sp + 8, s = io.short_side, l = io.long_side;
    f16_t *const Xh = lds, *const Xl = Xh + sp * xs, *const Ah = Xl + sp * xs, *const Al = Ah + sp * as;

    // The caller's rows, whatever side they are: a wavefront takes every eighth, and eight of its rows at a time.
    constexpr int UN = 8;
    const bool turn = io.m_i < io.m_j;  // the rows of M are the long side
    const int inner = turn ? s : l, outer = turn ? l : s, inner_p = turn ? sp : lp, outer_p = turn ? lp : sp;
    const T *from = io.M + b * io.m_matrix;
    const int64_t m_row = turn ? io.m_j : io.m_i;
    const auto each = [&](int rows, int cols, auto &&use) {  // use(row, column, element), rows beyond the matrix: zero
        for (int o = wave; o < rows; o += WAVES * UN)
            for (int q = lane; q < cols; q += 64) {
                T raw[UN];
#pragma unroll
                for (int u = 0; u < UN; ++u) {
                    const int row = o + u * WAVES;
                    raw[u] = from[(row < outer ? row : 0) * m_row + (q < inner ? q : 0)];
                }
#pragma unroll
                for (int u = 0; u < UN; ++u) {
                    const int row = o + u * WAVES;
                    if (row < rows) use(row, q, row < outer && q < inner ? (double)(float)raw[u] : 0.0);
                }
            }
    };
    double sum = 0.0;
    each(outer, inner, [&](int, int, double x) { sum = __builtin_fma(x, x, sum); });
    sum = sum_across_32(sum_across_16(dpp_add<0x140>(sum_of_eight(sum))));
    if (lane == 0) part[wave] = sum;
    __syncthreads();
    sum = 0.0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) sum += part[w];
    const double norm = ortho_root(sum) * (double)kOrthoScaleX;
    each(outer_p, inner_p, [&](int o, int q, double x) {
        f16_t hi, lo;
        ortho_split((float)(x * norm), hi, lo);
        const int at = turn ? q * xs + o : o * xs + q;
        Xh[at] = hi;
        Xl[at] = lo;
    });
    __syncthreads();

    // Blocks (i0, j0), (i0, j0 + 32), .. of a product, turned: a lane's sixteen entries of each are in row lane % 32, at columns
    // 8 (q / 4) + 4 (lane / 32) + q % 4.  left: rows along k; right: rows along k (its transpose is the factor), or across.
    const int row = lane & 31, quad = 4 * (lane >> 5);
    typedef __attribute__((ext_vector_type(4))) f16_t f16x4;
    struct Blocks { f32x16 v[PER]; };
    const auto along = [&](const f16_t *m, int stride, int first, int k) {
        return *reinterpret_cast<const f16x8 *>(m + (first + row) * stride + k + 8 * (lane >> 5));
    };
    const auto across = [&](const f16_t *m, int stride, int first, int k) {  // rows k .., columns first ..
        typedef __attribute__((address_space(3))) s16x4 *Ptr;
        const f16_t *p = m + (k + (lane >> 5) * 8 + ((lane & 15) >> 2)) * stride + first + (lane & 16) + (lane & 3) * 4;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)p), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(p + 4 * stride));
        return __builtin_bit_cast(f16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    const auto product = [&](const f16_t *lh_, const f16_t *ll_, int ls, int i0, auto &&right, const f16_t *rh_, const f16_t *rl_, int rs,
                             int j0, int length) {
        Blocks out;
        f32x16 low[PER];
#pragma unroll
        for (int u = 0; u < PER; ++u)
#pragma unroll
            for (int q = 0; q < 16; ++q) out.v[u][q] = low[u][q] = 0.f;
        struct Operands { f16x8 lh, ll, rh[PER], rl[PER]; };
        const auto read = [&](Operands &o, int k) {
            o.lh = along(lh_, ls, i0, k);
            o.ll = along(ll_, ls, i0, k);
#pragma unroll
            for (int u = 0; u < PER; ++u) {
                o.rl[u] = right(rl_, rs, j0 + 32 * u, k);
                o.rh[u] = right(rh_, rs, j0 + 32 * u, k);
            }
        };
        const auto multiply = [&](const Operands &o) {
#pragma unroll
            for (int u = 0; u < PER; ++u) low[u] = mfma32(o.rl[u], o.lh, low[u]);
#pragma unroll
            for (int u = 0; u < PER; ++u) out.v[u] = mfma32(o.rh[u], o.lh, out.v[u]);
#pragma unroll
            for (int u = 0; u < PER; ++u) low[u] = mfma32(o.rh[u], o.ll, low[u]);
        };
        for (int k = 0; k < length; k += 16) {  // (not unrolled: the transposing reads are convergent, the length is known at run time only)
            Operands o;
            read(o, k);
            multiply(o);
        }
#pragma unroll
        for (int u = 0; u < PER; ++u)
#pragma unroll
            for (int q = 0; q < 16; ++q) out.v[u][q] = ortho_join(out.v[u][q], low[u][q]);
        return out;
    };
    const auto put = [&](f16_t *mh, f16_t *ml, int stride, int i0, int j0, const Blocks &x) {
#pragma unroll
        for (int u = 0; u < PER; ++u)
#pragma unroll
            for (int q = 0; q < 16; q += 4) {
                f16x4 hi, lo;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    f16_t y, z;
                    ortho_split(x.v[u][q + e], y, z);
                    hi[e] = y;
                    lo[e] = z;
                }
                const int at = (i0 + row) * stride + j0 + 32 * u + 2 * q + quad;
                *reinterpret_cast<f16x4 *>(mh + at) = hi;
                *reinterpret_cast<f16x4 *>(ml + at) = lo;
            }
    };
    const auto plus = [&](const f16_t *mh, const f16_t *ml, int stride, int i0, int j0, float alpha, float beta, Blocks &x) {
#pragma unroll
        for (int u = 0; u < PER; ++u)
#pragma unroll
            for (int q = 0; q < 16; q += 4) {
                const int at = (i0 + row) * stride + j0 + 32 * u + 2 * q + quad;
                const f16x4 hi = *reinterpret_cast<const f16x4 *>(mh + at), lo = *reinterpret_cast<const f16x4 *>(ml + at);
#pragma unroll
                for (int e = 0; e < 4; ++e) x.v[u][q + e] = fmaf(alpha, ortho_join((float)hi[e], (float)lo[e]), beta * x.v[u][q + e]);
            }
    };
    const int nb = sp / 32, units = nb * (lp / 32 / PER);
    const bool sym = wave < nb * nb / PER;  // this wavefront's blocks of A and A^2
    const int si = wave % nb * 32, sj = wave / nb * 32 * PER;
    for (int step = 0; step < steps; ++step) {
        Blocks y;
        if (sym) {
            y = product(Xh, Xl, xs, si, along, Xh, Xl, xs, sj, lp);
#pragma unroll
            for (int u = 0; u < PER; ++u)
#pragma unroll
                for (int q = 0; q < 16; ++q) y.v[u][q] *= kOrthoScaleA / (kOrthoScaleX * kOrthoScaleX);
            put(Ah, Al, as, si, sj, y);
        }
        __syncthreads();
        if (sym) {
            y = product(Ah, Al, as, si, along, Ah, Al, as, sj, sp);
            plus(Ah, Al, as, si, sj, (float)c.b, (float)(c.c / kOrthoScaleA), y);
        }
        __syncthreads();
        if (sym) put(Ah, Al, as, si, sj, y);
        __syncthreads();
        Blocks x[MOST];
#pragma unroll
        for (int u = 0; u < MOST; ++u) {
            const int t = wave + u * WAVES, i0 = t % nb * 32, j0 = t / nb * 32 * PER;
            if (t < units) {
                x[u] = product(Ah, Al, as, i0, across, Xh, Xl, xs, j0, sp);
                plus(Xh, Xl, xs, i0, j0, (float)c.a, 1.f / kOrthoScaleA, x[u]);
            }
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < MOST; ++u) {
            const int t = wave + u * WAVES, i0 = t % nb * 32, j0 = t / nb * 32 * PER;
            if (t < units) put(Xh, Xl, xs, i0, j0, x[u]);
        }
        __syncthreads();
    }
    const int64_t o_row = turn ? io.o_j : io.o_i;
    for (int o = wave; o < outer; o += WAVES)
        for (int q = lane; q < inner; q += 64) {
            const int at = turn ? q * xs + o : o * xs + q;
            const float v = ortho_join((float)Xh[at], (float)Xl[at]) * (1.f / kOrthoScaleX);
            const int64_t p = b * io.o_matrix + o * o_row + q;
            if (io.sub) io.sub[p] = io.sub[p] - io.rate * v;
            else io.O[p] = (T)v;
        }
}

// No step at all: O = X_0.
template <typename T>
__global__ __launch_bounds__(256) void ortho_scaled(OrthoIo<T> io, const double *__restrict__ sums)
{
    const int64_t b = blockIdx.y;
    double t = 0.0;
    for (int q = 0; q < kOrthoSums; ++q) t += sums[b * kOrthoSums + q];
    const double norm = ortho_root(t);
    const int64_t cells = (int64_t)io.short_side * io.long_side;
    const bool turn = io.o_i < io.o_j;
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < cells; q += (int64_t)gridDim.x * 256) {
        const int i = (int)(turn ? q % io.short_side : q / io.long_side);
        const int64_t j = turn ? q / io.short_side : q % io.long_side;
        io.put(b, i, j, io.at(b, i, j) * norm);
    }
}

}  // namespace cdgrab
