// Orthogonalised updates: X_0 = M / ||M||_F (the shorter side as rows), then `steps` times
//     A = X X^T,  X <- a X + (b A + c A^2) X,
// which takes every singular value s to a s + b s^3 + c s^5 and leaves the singular vectors.
//
// Small singular values grow by a factor of a per step (3.4 by default), and so does what rounding does to their vectors:
// products in fp32, or as good, are needed between steps even for results of fewer bits (with one product of bf16 factors the
// result is off by some percent).  Two forms:
//   - short side up to kOrthoNarrow: X_K = P_K X_0 with P_K a polynomial in A_0 = X_0 X_0^T.  One pass over the matrix for A_0 in
//     double, the recurrence on matrices of the short side (all of which commute), one pass for the product: bytes of the matrix
//     twice.  (In fp32 this form loses too much: the small eigenvalues of A_0 are the squares of the singular values.)
//   - else the products as they stand.  Factors are held as the sum of two fp16 (22 bits), and of the four products of the
//     parts the three larger are taken: errors as of fp32 products (simulated on matrices of 256 .. 2048: 1.0 to 1.1 times), at a
//     third of the fp16 MFMA rate, five times the fp32 MFMA's.  fp16 has the digits but not the range: the norm bounds every
//     element, and a fixed power of two in front keeps the parts normal.  A and A^2 are symmetric: half of their tiles are
//     computed.
#pragma once
#include "linear_kernels.hpp"

namespace cdgrab {

typedef double f64x4 __attribute__((ext_vector_type(4)));

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
    __device__ __forceinline__ double at(int64_t b, int i, int64_t j) const { return (double)(float)M[b * m_matrix + i * m_i + j * m_j]; }
    __device__ __forceinline__ void put(int64_t b, int i, int64_t j, float v) const {
        const int64_t p = b * o_matrix + i * o_i + j * o_j;
        if (sub) sub[p] = sub[p] - rate * v;
        else O[p] = (T)v;
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

struct OrthoCoeffs { double a, b, c; };

// 1 / sqrt of a sum of squares: zero of zero (such a matrix stays as it is), NaN of infinity.
__device__ __forceinline__ double ortho_root(double t) { return t == 0.0 ? 0.0 : 1.0 / sqrt(t) + (t - t); }

// ---- short side up to kOrthoNarrow -----------------------------------------------------------------------------------------
constexpr int kOrthoNarrow = 64;
constexpr int kOrthoThreads = 1024;

// A product of NT x NT tiles of 16 x 16 in LDS (row-major, row length LD): wavefront w takes tile w, if there is one.  Lane l
// holds entries (4 v + l / 16, l % 16), v = 0 .. 3, of its tile.
template <int NT, int LD>
struct OrthoTiles {
    static_assert(NT * NT <= kOrthoThreads / 64, "a wavefront per tile");
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const bool mine = wave < NT * NT;
    const int row = (wave / NT) * 16 + (lane >> 4), col = (wave % NT) * 16 + (lane & 15);  // of entry v = 0

    __device__ __forceinline__ f64x4 product(const double *A, const double *B) const {
        f64x4 acc = {0.0, 0.0, 0.0, 0.0};
        if (mine) {
            const double *a = A + ((wave / NT) * 16 + (lane & 15)) * LD + (lane >> 4), *b = B + (lane >> 4) * LD + col;
#pragma unroll
            for (int q = 0; q < NT * 4; ++q)
                acc = __builtin_amdgcn_mfma_f64_16x16x4f64(a[q * 4], b[q * 4 * LD], acc, 0, 0, 0);
        }
        return acc;
    }
    __device__ __forceinline__ void store(double *C, f64x4 x) const {
        if (mine)
#pragma unroll
            for (int v = 0; v < 4; ++v) C[(row + 4 * v) * LD + col] = x[v];
    }
};

// P (in LDS) from the Gram matrix of M in A (in LDS), entries beyond the short side zero:
//   A <- A / trace(A), P <- I / sqrt(trace); steps times: Q = a I + b A + c A^2, P <- Q P, A <- Q A Q.
// Everything commutes and is symmetric, so that the order of factors does not matter.
template <int NT>
struct OrthoChain {
    static constexpr int N = NT * 16, LD = N + 2;  // (rows an even number of banks apart would share them)
    double A[N * LD], Q[N * LD], P[N * LD];
    double trace;

    __device__ __forceinline__ void run(int n, int steps, OrthoCoeffs c) {
        const int tid = threadIdx.x;
        const OrthoTiles<NT, LD> tiles;
        __syncthreads();
        if (tid < 64) {
            double t = 0.0;
            for (int i = tid; i < n; i += 64) t += A[i * LD + i];
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) t += __shfl_xor(t, off, 64);
            if (tid == 0) trace = t;
        }
        __syncthreads();
        const double t = trace, inv = t == 0.0 ? 0.0 : 1.0 / t, root = ortho_root(t);
        for (int q = tid; q < N * N; q += kOrthoThreads) {
            const int i = q / N, j = q % N;
            A[i * LD + j] = A[i * LD + j] * inv;
            P[i * LD + j] = i == j && i < n ? root : 0.0;
        }
        __syncthreads();
        for (int s = 0; s < steps; ++s) {
            f64x4 x = tiles.product(A, A);
            if (tiles.mine)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const int i = tiles.row + 4 * v, j = tiles.col;
                    Q[i * LD + j] = (i == j ? c.a : 0.0) + c.b * A[i * LD + j] + c.c * x[v];
                }
            __syncthreads();
            x = tiles.product(Q, P);
            const f64x4 y = tiles.product(Q, A);
            __syncthreads();
            tiles.store(P, x);
            tiles.store(A, y);
            __syncthreads();
            if (s + 1 < steps) {  // (the last step's A is for nobody)
                x = tiles.product(A, Q);
                __syncthreads();
                tiles.store(A, x);
                __syncthreads();
            }
        }
    }
};

// Gram matrix of columns j0 .. j1 - 1 (those of the long side), by the workgroup: wavefront w takes every sixteenth group of
// four columns and keeps all tiles on or above the diagonal; `to`(i, j, value) receives sums over the wavefronts, in order.
template <int NT, typename T, typename F>
__device__ __forceinline__ void ortho_gram(const OrthoIo<T> &io, int64_t b, int64_t j0, int64_t j1, double *lds, F &&to) {
    constexpr int TILES = NT * (NT + 1) / 2, WAVES = kOrthoThreads / 64, UN = 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, k = lane >> 4;
    f64x4 acc[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) acc[t] = f64x4{0.0, 0.0, 0.0, 0.0};
    for (int64_t j = j0 + wave * 4 + k; __any(j < j1); j += 4 * WAVES * UN) {
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
                x[t] = t * 16 + r < io.short_side && j + u * 4 * WAVES < j1 ? (double)(float)raw[u][t] : 0.0;
            int at = 0;
#pragma unroll
            for (int ti = 0; ti < NT; ++ti)
#pragma unroll
                for (int tj = ti; tj < NT; ++tj, ++at) acc[at] = __builtin_amdgcn_mfma_f64_16x16x4f64(x[ti], x[tj], acc[at], 0, 0, 0);
        }
        // The results are copied at the loop's head, and there the compiler puts 4 wait states instead of 18 between the last
        // product and the copy of its last two registers: without the next line rows 28 .. 31 of a tile miss products.
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

// O = P X for columns j0 .. j1 - 1, in double (P's large entries cancel): a thread takes a column and ROWS rows.
template <int NT, typename T>
__device__ __forceinline__ void ortho_apply(const OrthoIo<T> &io, int64_t b, int64_t j0, int64_t j1, const double *P, int ld) {
    constexpr int ROWS = NT == 1 ? 2 : 8;
    const int n = io.short_side, parts = (n + ROWS - 1) / ROWS;
    for (int64_t q = threadIdx.x; q < (j1 - j0) * parts; q += kOrthoThreads) {
        // neighbouring threads take what lies side by side in memory
        const int64_t j = io.o_j < io.o_i ? j0 + q % (j1 - j0) : j0 + q / parts;
        const int i0 = (int)(io.o_j < io.o_i ? q / (j1 - j0) : q % parts) * ROWS;
        double acc[ROWS];
#pragma unroll
        for (int u = 0; u < ROWS; ++u) acc[u] = 0.0;
        for (int k = 0; k < n; ++k) {
            const double x = io.at(b, k, j);
#pragma unroll
            for (int u = 0; u < ROWS; ++u) acc[u] = __builtin_fma(P[(i0 + u) * ld + k], x, acc[u]);
        }
#pragma unroll
        for (int u = 0; u < ROWS; ++u)
            if (i0 + u < n) io.put(b, i0 + u, j, (float)acc[u]);
    }
}

// One workgroup per matrix.
template <int NT, typename T>
__global__ __launch_bounds__(kOrthoThreads) void ortho_narrow(OrthoIo<T> io, int steps, OrthoCoeffs c)
{
    __shared__ OrthoChain<NT> s;
    __shared__ double lds[kOrthoThreads * 4];
    const int64_t b = blockIdx.x;
    ortho_gram<NT>(io, b, 0, io.long_side, lds, [&](int i, int j, double v) {
        s.A[i * s.LD + j] = v;
        s.A[j * s.LD + i] = v;
    });
    s.run(io.short_side, steps, c);
    ortho_apply<NT>(io, b, 0, io.long_side, s.P, s.LD);
}

// Long matrices: chunks of columns for the Gram matrix, then the recurrence, then chunks of columns for the product.
template <int NT, typename T>
__global__ __launch_bounds__(kOrthoThreads) void ortho_narrow_gram(OrthoIo<T> io, int chunks, int64_t per, double *__restrict__ parts)
{
    __shared__ double lds[kOrthoThreads * 4];
    constexpr int N = NT * 16;
    const int64_t b = blockIdx.x / chunks, c = blockIdx.x % chunks;
    const int64_t j1 = (c + 1) * per < io.long_side ? (c + 1) * per : io.long_side;
    double *to = parts + (int64_t)blockIdx.x * N * N;
    ortho_gram<NT>(io, b, c * per, j1, lds, [&](int i, int j, double v) { to[i * N + j] = v; });
}
template <int NT>
__global__ __launch_bounds__(kOrthoThreads) void ortho_narrow_chain(int n, int chunks, const double *__restrict__ parts, int steps,
                                                                    OrthoCoeffs c, double *__restrict__ out)
{
    __shared__ OrthoChain<NT> s;
    constexpr int N = NT * 16;
    const double *from = parts + (int64_t)blockIdx.x * chunks * N * N;
    for (int q = threadIdx.x; q < N * N; q += kOrthoThreads) {
        const int i = q / N, j = q % N;
        if (i / 16 > j / 16) continue;
        double sum = 0.0;
#pragma unroll 8
        for (int p = 0; p < chunks; ++p) sum += from[(int64_t)p * N * N + q];
        s.A[i * s.LD + j] = sum;
        if (i / 16 < j / 16) s.A[j * s.LD + i] = sum;
    }
    s.run(n, steps, c);
    for (int q = threadIdx.x; q < N * N; q += kOrthoThreads) out[(int64_t)blockIdx.x * N * N + q] = s.P[(q / N) * s.LD + q % N];
}
template <int NT, typename T>
__global__ __launch_bounds__(kOrthoThreads) void ortho_narrow_apply(OrthoIo<T> io, int chunks, int64_t per, const double *__restrict__ P)
{
    constexpr int N = NT * 16, LD = N + 2;
    __shared__ double p[N * LD];
    const int64_t b = blockIdx.x / chunks, c = blockIdx.x % chunks;
    for (int q = threadIdx.x; q < N * N; q += kOrthoThreads) p[(q / N) * LD + q % N] = P[b * N * N + q];
    __syncthreads();
    ortho_apply<NT>(io, b, c * per, (c + 1) * per < io.long_side ? (c + 1) * per : io.long_side, p, LD);
}

// ---- longer sides: products of pairs of fp16 --------------------------------------------------------------------------------
constexpr float kOrthoScaleX = 8192.f, kOrthoScaleA = 2048.f;  // X up to 7.9, A and b A + c A^2 up to 31 (the host sees to it)
constexpr int kOrthoSums = 64;  // sums of squares per matrix

// A matrix as pairs of fp16: hi and lo planes, `ld` elements from row to row.
struct OrthoPair { f16_t *hi, *lo; };

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

// v as a pair of fp16.
__device__ __forceinline__ void ortho_split(float v, f16_t &hi, f16_t &lo) {
    hi = (f16_t)v;
    lo = (f16_t)(v - (float)hi);
}

// X_0 as pairs, [short][long] padded with zeros to sp x lp: 32 x 32 elements a workgroup, turned through LDS where the rows
// of M are the long side.
template <typename T>
__global__ __launch_bounds__(256) void ortho_begin(OrthoIo<T> io, const double *__restrict__ sums, OrthoPair X, int sp, int lp)
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
    const int64_t base = b * sp * (int64_t)lp;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int64_t p = base + (int64_t)(i0 + y + 8 * q) * lp + j0 + x;
        f16_t hi, lo;
        ortho_split(tile[y + 8 * q][x] * kOrthoScaleX, hi, lo);
        X.hi[p] = hi;
        X.lo[p] = lo;
    }
}

enum OrthoWhat { kOrthoGram, kOrthoPoly, kOrthoStep, kOrthoLast };

// One tile of a product of pairs, L R^T (Gram, Poly: R's rows, both with their elements along k) or L R (Step, Last: R's rows
// along k), then
//   Gram: A = X X^T;  Poly: B = b A + c A A;  Step: X' = a X + B X;  Last: O = (a X + B X) to the caller's array.
// K is a multiple of 32, the tile's sides T of 32: nothing to clip but O.
// Memory to LDS without registers, sixteen bytes a lane, NS stages of 32 k on their way or in use.  LDS rows are dense (a wave
// fills 1 KB in a row); sixteen-byte pieces are swapped within a row by its number, so that the lanes of a read hit different banks.
template <int T> struct OrthoTile {
    static constexpr int KC = 32, PLANE = T * KC, CALLS = PLANE / 8 / 64 / 4;  // elements; a wavefront's loads per plane
    // piece c of row r of an [T][KC] plane / of a [KC][T] plane (pairs of pieces stay together for the transposing read)
    static __device__ __forceinline__ int along(int r, int c) { return c ^ ((r >> 2) & 3); }
    static __device__ __forceinline__ int across(int r, int c) { return T == 128 ? c ^ ((r & 7) << 1) : c ^ (((r >> 1) & 3) << 1); }
};

// Waits until at most LEFT of this wavefront's loads are on their way and its LDS reads are done, then for the workgroup.
// (By builtins: the compiler then knows that the reads are done, and does not wait for the next ones instead.)
template <int LEFT>
__device__ __forceinline__ void ortho_barrier() {
    static_assert(LEFT < 64, "six bits");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_s_waitcnt((LEFT & 15) | (LEFT >> 4) << 14 | 7 << 4);  // vmcnt LEFT, lgkmcnt 0, expcnt any
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    __builtin_amdgcn_sched_barrier(0);
}

// A wavefront's share of a stage's loads of one plane: `from` is the same for all lanes, a lane adds `at[q]` bytes for its q-th load.
template <int T, bool ACROSS>
struct OrthoFetch {
    typedef OrthoTile<T> O;
    uint32_t at[O::CALLS];
    __device__ __forceinline__ OrthoFetch(int64_t ld, int wave, int lane) {
        constexpr int PIECES = ACROSS ? T / 8 : O::KC / 8, ROWS = 64 / PIECES;
#pragma unroll
        for (int q = 0; q < O::CALLS; ++q) {
            const int row = (q * 4 + wave) * ROWS + lane / PIECES, slot = lane % PIECES;
            at[q] = (uint32_t)(row * (int)ld + (ACROSS ? O::across(row, slot) : O::along(row, slot)) * 8) * 2u;
        }
    }
    __device__ __forceinline__ void operator()(const f16_t *from, f16_t *lds, int wave) const {
        typedef __attribute__((address_space(3))) void *Lds;
        typedef const __attribute__((address_space(1))) void *Mem;
#pragma unroll
        for (int q = 0; q < O::CALLS; ++q)
            __builtin_amdgcn_global_load_lds((Mem)(reinterpret_cast<const char *>(from) + at[q]), (Lds)(lds + (q * 4 + wave) * 512), 16, 0, 0);
    }
};

// A lane's operands of 32 x 32 x 16 MFMAs: `at[k / 16]` is where those of the tile's first 32 rows (columns) lie in a plane,
// those of the i-th next are a constant further, as the planes and stages are.
template <int T, bool ACROSS>
struct OrthoRead {
    typedef OrthoTile<T> O;
    int at[2], at4[2];  // (in elements; at4: the second half of a transposing read)
    __device__ __forceinline__ OrthoRead(int first, int lane) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if constexpr (!ACROSS) {  // row first + lane % 32, elements 16 h + 8 (lane / 32) ..
                const int row = first + (lane & 31);
                at[h] = row * O::KC + O::along(row, 2 * h + (lane >> 5)) * 8;
            } else {
                const int row = 16 * h + (lane >> 5) * 8 + ((lane & 15) >> 2), col = first + (lane & 16) + (lane & 3) * 4;
                at[h] = row * T + O::across(row, col >> 3) * 8 + (col & 4);
                at4[h] = (row + 4) * T + O::across(row + 4, col >> 3) * 8 + (col & 4);
            }
        }
    }
    // (ACROSS: columns are swapped by exclusive or, and so are those 32 further, since `first` is a multiple of 64)
    __device__ __forceinline__ f16x8 operator()(const f16_t *plane, int h, int i) const {
        if constexpr (!ACROSS) {
            return *reinterpret_cast<const f16x8 *>(plane + at[h] + i * 32 * O::KC);
        } else {
            typedef __attribute__((address_space(3))) s16x4 *Ptr;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(plane + (at[h] ^ (i * 32))));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(plane + (at4[h] ^ (i * 32))));
            return __builtin_bit_cast(f16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

struct OrthoProduct {
    OrthoPair L, R, E, C;  // factors, what is added, the result
    int64_t l_ld, r_ld, c_ld, l_matrix, r_matrix, c_matrix;  // (E lies as C does)
    int k, tiles_m, tiles_n;
    float alpha, beta;  // result = alpha E + beta (product as multiplied)
};

template <int T, int NS, int WHAT, typename U>
__global__ __launch_bounds__(256, NS * T * 256 > 80 * 1024 ? 1 : 2) void ortho_product_tile(OrthoProduct p, OrthoIo<U> io)
{
    constexpr bool ACROSS = WHAT == kOrthoStep || WHAT == kOrthoLast, SYM = !ACROSS;
    typedef OrthoTile<T> O;
    constexpr int MB = T / 64, LD = T + 1;  // (eight rows further is eight banks further)
    constexpr int STAGE = 4 * O::PLANE, BYTES = NS * STAGE * 2, OUT = T / 2 * LD * 4, LOADS = 4 * O::CALLS;
    __shared__ __align__(16) char lds[BYTES > OUT ? BYTES : OUT];
    f16_t *stage = reinterpret_cast<f16_t *>(lds);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave >> 1, wn = wave & 1;
    const int per = SYM ? p.tiles_m * (p.tiles_m + 1) / 2 : p.tiles_m * p.tiles_n;
    const uint32_t id = xcd_neighbours(blockIdx.x, gridDim.x);
    const int64_t b = id / (uint32_t)per;
    int tm, tn;
    if constexpr (SYM) {  // tiles on or above the diagonal, column after column
        const int t = (int)(id - b * per);
        tn = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
        while ((tn + 1) * (tn + 2) / 2 <= t) ++tn;
        while (tn * (tn + 1) / 2 > t) --tn;
        tm = t - tn * (tn + 1) / 2;
    } else {
        const int t = (int)(id - b * per);
        tm = t % p.tiles_m;
        tn = t / p.tiles_m;
    }
    const f16_t *src[4] = {p.L.hi + b * p.l_matrix + (int64_t)tm * T * p.l_ld, p.L.lo + b * p.l_matrix + (int64_t)tm * T * p.l_ld,
                           p.R.hi + b * p.r_matrix + (ACROSS ? (int64_t)tn * T : (int64_t)tn * T * p.r_ld),
                           p.R.lo + b * p.r_matrix + (ACROSS ? (int64_t)tn * T : (int64_t)tn * T * p.r_ld)};
    // (the products with the small parts in sums of their own: as parts of one sum each would round it once more, 2468
    // columns 3.3e-6 off instead of 1.9e-6)
    f32x16 acc[MB][MB], low[MB][MB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < MB; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[i][j][q] = low[i][j][q] = 0.f;
    const OrthoFetch<T, false> fetch_l(p.l_ld, wave, lane);
    const OrthoFetch<T, ACROSS> fetch_r(p.r_ld, wave, lane);
    const auto fetch = [&](int q, int buf) {
        f16_t *s = stage + buf * STAGE;
        const int k = q * O::KC;
        const int64_t off = ACROSS ? k * p.r_ld : k;
        fetch_l(src[0] + k, s, wave);
        fetch_l(src[1] + k, s + O::PLANE, wave);
        fetch_r(src[2] + off, s + 2 * O::PLANE, wave);
        fetch_r(src[3] + off, s + 3 * O::PLANE, wave);
    };
    struct Operands { f16x8 lh[MB], ll[MB], rh[MB], rl[MB]; };
    const OrthoRead<T, false> read_l(wm * (T / 2), lane);
    const OrthoRead<T, ACROSS> read_r(wn * (T / 2), lane);
    const auto read = [&](Operands &o, int buf, int h) {
        const f16_t *s = stage + buf * STAGE;
#pragma unroll
        for (int i = 0; i < MB; ++i) {
            o.lh[i] = read_l(s, h, i);
            o.rl[i] = read_r(s + 3 * O::PLANE, h, i);
            o.rh[i] = read_r(s + 2 * O::PLANE, h, i);
            o.ll[i] = read_l(s + O::PLANE, h, i);
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
    const int stages = p.k / O::KC;
    int sent = 0;
    for (; sent < NS && sent < stages; ++sent) fetch(sent, sent);
    if (sent == NS) ortho_barrier<(NS - 1) * LOADS>();
    else ortho_barrier<0>();
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
            if (q + NS <= stages) ortho_barrier<(NS - 2) * LOADS>();
            else ortho_barrier<0>();
            if (sent < stages) fetch(sent++, buf);
            read(first, (buf + 1) % NS, 0);
            multiply(second);
            interleave();
        }
    read(second, (stages - 1) % NS, 1);
    multiply(first);
    multiply(second);
    // The tile goes out through LDS, half its rows at a time, so that every thread stores eight neighbours of a row; a tile
    // above the diagonal also to its mirror image.  What is added is requested before the first half is written.
    constexpr int TASKS = T / 2 * T / 8 / 256;  // of a thread, per half
    const int64_t c_tile = b * p.c_matrix + (int64_t)tm * T * p.c_ld + tn * T;
    f16x8 e_hi[2][TASKS], e_lo[2][TASKS];
    if constexpr (WHAT != kOrthoGram)
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int u = 0; u < TASKS; ++u) {
                const int q = threadIdx.x + u * 256;
                const int64_t at = c_tile + (int64_t)(half * (T / 2) + q / (T / 8)) * p.c_ld + q % (T / 8) * 8;
                e_hi[half][u] = *reinterpret_cast<const f16x8 *>(p.E.hi + at);
                e_lo[half][u] = *reinterpret_cast<const f16x8 *>(p.E.lo + at);
            }
    float *out = reinterpret_cast<float *>(lds);
    const auto store = [&](const float (&v)[8], int64_t at) {
        f16x8 hi, lo;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            f16_t x, y;
            ortho_split(v[j], x, y);
            hi[j] = x;
            lo[j] = y;
        }
        *reinterpret_cast<f16x8 *>(p.C.hi + at) = hi;
        *reinterpret_cast<f16x8 *>(p.C.lo + at) = lo;
    };
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        __syncthreads();
        if (wm == half)
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < MB; ++j)
#pragma unroll
                    for (int q = 0; q < 16; ++q)
                        out[(i * 32 + 8 * (q >> 2) + 4 * (lane >> 5) + (q & 3)) * LD + wn * (T / 2) + j * 32 + (lane & 31)] =
                            p.beta * (acc[i][j][q] + low[i][j][q]);
        __syncthreads();
        // the values are read from LDS once more, along the other side
        const bool turn = WHAT == kOrthoLast && io.o_i < io.o_j;  // (the caller's rows are the long side)
        const bool again = turn || (SYM && tm != tn);
        const int m0 = tm * T + half * (T / 2), n0 = tn * T;
#pragma unroll
        for (int u = 0; u < TASKS; ++u) {
            const int q = threadIdx.x + u * 256, r = q / (T / 8), c = q % (T / 8) * 8;
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = out[r * LD + c + j];
                if constexpr (WHAT != kOrthoGram) {
                    v[j] = fmaf(p.alpha, (float)e_hi[half][u][j] + (float)e_lo[half][u][j], v[j]);
                    if (again) out[r * LD + c + j] = v[j];
                }
            }
            if constexpr (WHAT != kOrthoLast) {
                store(v, c_tile + (int64_t)(half * (T / 2) + r) * p.c_ld + c);
            } else if (!turn && m0 + r < io.short_side) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] *= 1.f / kOrthoScaleX;
                io.put8(b * io.o_matrix + (m0 + r) * io.o_i + (n0 + c), v, io.long_side - n0 - c);
            }
        }
        if (!again) continue;
        __syncthreads();
        const int64_t mirror = b * p.c_matrix + (int64_t)n0 * p.c_ld + m0;
#pragma unroll
        for (int u = 0; u < TASKS; ++u) {
            const int q = threadIdx.x + u * 256, c = q / (T / 16), r = q % (T / 16) * 8;
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = out[(r + j) * LD + c];
            if constexpr (WHAT != kOrthoLast) {
                store(v, mirror + (int64_t)c * p.c_ld + r);
            } else if (n0 + c < io.long_side) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] *= 1.f / kOrthoScaleX;
                io.put8(b * io.o_matrix + (n0 + c) * io.o_j + (m0 + r), v, io.short_side - m0 - r);
            }
        }
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
        io.put(b, i, j, (float)(io.at(b, i, j) * norm));
    }
}

}  // namespace cdgrab
