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
//
// Measured: forward 2 x 8192 tokens, 32 heads on 8 of 128, bf16 1110 to 1270 us by the card, 990 to 870 TFLOP/s (a large product reaches 1100
// to 1150); with heads of 64, where there is one exponential for half as many products, 64 x 1024 tokens, 12 heads 190 to 198 us, 530 TFLOP/s:
// VALU 66 % of the cycles, MFMA 30 %.  Back, the same: dq 270 us, dk and dv 300, 575 and 685 TFLOP/s of the products that they take; half of
// the wavefronts' time is waiting, and registers allow no more of them (dk, dv: one, two, three per SIMD 668, 420, 400 us).  fp32 64 x 128
// tokens, 4 heads of 32 11 us, dq 14, dk and dv 16; 16 x 1024, 8 heads of 64 121, 207 and 252 us; 8 x 1024, 16 heads on 4 of 128 290, 400 and 870.
//
// What is far from that: dk and dv where keys are shared or examples are few or uneven, since a workgroup goes over all heads of the group and all
// later queries of its 128 keys by itself (24 examples of up to 1500 tokens, 8 heads on 2 of 80, fp16 250 us, CUs busy for 60 % of it; 1 x 2048,
// 32 heads on 1 of 128, bf16, 16 workgroups, 2500 us for what its products take 60), and at more than 64 features, of which one workgroup
// fits a CU; forward and dq of fewer than eight pairs (example, head of keys), each of which runs on one XCD: 1 x 8192, 32 heads on 1 of 128
// forward 4100 us, on 4 of 128 1110, on 8 all XCDs are in use.
#pragma once
#include "linear_kernels.hpp"

namespace cdgrab {

constexpr int kAttThreads = 256;
constexpr int kAttRows = 128;  // queries (keys) of a workgroup, 32 a wavefront
constexpr int kAttMaxDim = 128;

struct AttHeads {
    int64_t pairs, unit0;  // examples * kv_heads; the launch's first workgroup
    int tiles;             // of kAttRows rows that an example has at most
    int kv_heads, group;   // queries' heads that share keys and values
    bool by_pair;          // order of the workgroups
    const uint64_t *list;  // or NULL: the number of tiles that there are, and then example and number in it of each
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
    __device__ __forceinline__ void load(const T *base, int64_t stride, int at, int end, int dim) {
#pragma unroll
        for (int q = 0; q < PER; ++q) {
            const int i = threadIdx.x + q * kAttThreads, r = i / USED, piece = i % USED;
            att_piece<T>(base + (int64_t)(at + r) * stride, piece * 8, dim, (TOTAL % kAttThreads == 0 || i < TOTAL) && at + r < end, v[q]);
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

// Two operands' tiles of ROWS rows on their way to LDS.  DIRECT (16-bit elements in whole, aligned pieces): from memory to LDS without
// registers, a tile ahead, into the other of two buffers (2 x 8192 tokens, 32 heads on 8 of 128: 2177 -> 1128 us); otherwise through
// registers, where fp32 elements are split.  Rows from `end` on
// are zero, or with DIRECT the last one again: they meet weights of zero.
template <typename T, int D, int ROWS, bool DIRECT>
struct AttPipe {
    typedef AttStage<T, D, ROWS> Stage;
    typedef typename Stage::E E;
    static constexpr int LEN = 2 * Stage::LEN, LDS = LEN;
    Stage a, b;
    E *lds;
    int dim;
    __device__ __forceinline__ AttPipe(E *lds, int dim, int64_t, int64_t) : lds(lds), dim(dim) {}
    __device__ __forceinline__ void fetch(const T *A, int64_t a_stride, const T *B, int64_t b_stride, int at, int end) {
        a.load(A, a_stride, at, end, dim);
        b.load(B, b_stride, at, end, dim);
    }
    // The tile fetched last, for the whole workgroup; then the next one may be fetched.
    __device__ __forceinline__ const E *turn() {
        __syncthreads();  // (the last tile has been read)
        a.store(lds);
        b.store(lds + Stage::LEN);
        __syncthreads();
        return lds;
    }
};
template <typename T, int D, int ROWS>
struct AttPipe<T, D, ROWS, true> {
    typedef AttLayout<D> L;
    typedef typename LinearPlanes<T>::elem E;
    static constexpr int ONE = ROWS * L::LD, LEN = 2 * ONE, LDS = 2 * LEN, CALLS = ROWS * L::PIECES / kAttThreads;
    static_assert(LinearPlanes<T>::N == 1 && CALLS * kAttThreads == ROWS * L::PIECES, "");
    E *lds;
    int buf = 0, row[CALLS];
    uint32_t piece[CALLS], at_a[CALLS], at_b[CALLS];  // bytes
    bool there[CALLS];
    __device__ __forceinline__ AttPipe(E *lds, int dim, int64_t a_stride, int64_t b_stride) : lds(lds) {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (int q = 0; q < CALLS; ++q) {
            const int slot = (q * (kAttThreads / 64) + wave) * 64 + lane;
            row[q] = slot / L::PIECES;
            const int p = slot % L::PIECES ^ L::swap(row[q]);
            there[q] = p * 8 < dim;
            piece[q] = p * 16;
            at_a[q] = (uint32_t)(row[q] * (int)a_stride * 2) + piece[q];
            at_b[q] = (uint32_t)(row[q] * (int)b_stride * 2) + piece[q];
        }
        if (dim < D) {  // uniform: what is never loaded is zero
            typedef uint32_t words __attribute__((ext_vector_type(4)));
            for (int i = threadIdx.x; i < LDS / 8; i += kAttThreads) reinterpret_cast<words *>(lds)[i] = words{0, 0, 0, 0};
            __syncthreads();
        }
    }
    __device__ __forceinline__ void one(const T *from, int64_t stride, const uint32_t (&offset)[CALLS], E *to, int at, int end) const {
        typedef __attribute__((address_space(3))) void *Lds;
        typedef const __attribute__((address_space(1))) void *Mem;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const char *base = reinterpret_cast<const char *>(from + at * stride);
        const bool whole = at + ROWS <= end;  // uniform
#pragma unroll
        for (int q = 0; q < CALLS; ++q) {
            uint32_t o = offset[q];
            if (!whole) o = (uint32_t)((row[q] < end - at ? row[q] : end - at - 1) * (int)stride * 2) + piece[q];
            if (there[q]) __builtin_amdgcn_global_load_lds((Mem)(base + o), (Lds)(to + (q * (kAttThreads / 64) + wave) * 512), 16, 0, 0);
        }
    }
    __device__ __forceinline__ void fetch(const T *A, int64_t a_stride, const T *B, int64_t b_stride, int at, int end) const {
        one(A, a_stride, at_a, lds + buf * LEN, at, end);
        one(B, b_stride, at_b, lds + buf * LEN + ONE, at, end);
    }
    __device__ __forceinline__ const E *turn() {
        stage_barrier<0>();
        const E *now = lds + buf * LEN;
        buf ^= 1;
        return now;
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

// The `across` operands of 32 rows, all features.  DIRECT: read at once and waited for, in one piece of assembly each 32 or 64 features:
// in front of a transposing read by its builtin the compiler waits for all loads to LDS that are on their way, the next tile's
// (it cannot see that they go elsewhere), which took away what fetching ahead brings.
template <typename T, int D, int ROWS, bool DIRECT>
struct AttAcross {
    const AttRead<T, D, ROWS> &read;
    const typename AttRead<T, D, ROWS>::E *tile;
    int first;
    __device__ __forceinline__ AttAcross(const AttRead<T, D, ROWS> &read, const typename AttRead<T, D, ROWS>::E *tile, int first)
        : read(read), tile(tile), first(first) {}
    __device__ __forceinline__ AttFrag<T> get(int step, int d) const { return read.across(tile, first + step * 16, d); }
};
template <typename T, int D, int ROWS>
struct AttAcross<T, D, ROWS, true> {
    typedef AttLayout<D> L;
    typedef typename LinearPlanes<T>::elem E;
    s16x4 v[2][D / 32][2];
    __device__ __forceinline__ AttAcross(const AttRead<T, D, ROWS> &read, const E *tile, int first) {
        typedef const __attribute__((address_space(3))) E *Ptr;
        constexpr int ROW = L::LD * 2;  // bytes
        const uint32_t base = (uint32_t)(uintptr_t)(Ptr)(tile + first * L::LD + read.token);
#pragma unroll
        for (int d = 0; d < D / 32; d += 2) {
            const uint32_t lo = base + 2 * (read.lo ^ (d * 32)), hi = base + 2 * (read.hi ^ (d * 32));
            if constexpr (D == 32) {
                asm volatile("ds_read_b64_tr_b16 %0, %4\n\tds_read_b64_tr_b16 %1, %5 offset:%6\n\t"
                             "ds_read_b64_tr_b16 %2, %4 offset:%7\n\tds_read_b64_tr_b16 %3, %5 offset:%8\n\ts_waitcnt lgkmcnt(0)"
                             : "=&v"(v[0][0][0]), "=&v"(v[0][0][1]), "=&v"(v[1][0][0]), "=&v"(v[1][0][1])
                             : "v"(lo), "v"(hi), "n"(8 * ROW), "n"(16 * ROW), "n"(24 * ROW)
                             : "memory");
            } else if (d + 1 < D / 32) {
                const uint32_t lo1 = base + 2 * (read.lo ^ (d * 32 + 32)), hi1 = base + 2 * (read.hi ^ (d * 32 + 32));
                asm volatile("ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %9 offset:%12\n\t"
                             "ds_read_b64_tr_b16 %2, %10\n\tds_read_b64_tr_b16 %3, %11 offset:%12\n\t"
                             "ds_read_b64_tr_b16 %4, %8 offset:%13\n\tds_read_b64_tr_b16 %5, %9 offset:%14\n\t"
                             "ds_read_b64_tr_b16 %6, %10 offset:%13\n\tds_read_b64_tr_b16 %7, %11 offset:%14\n\ts_waitcnt lgkmcnt(0)"
                             : "=&v"(v[0][d][0]), "=&v"(v[0][d][1]), "=&v"(v[0][d + 1][0]), "=&v"(v[0][d + 1][1]), "=&v"(v[1][d][0]),
                               "=&v"(v[1][d][1]), "=&v"(v[1][d + 1][0]), "=&v"(v[1][d + 1][1])
                             : "v"(lo), "v"(hi), "v"(lo1), "v"(hi1), "n"(8 * ROW), "n"(16 * ROW), "n"(24 * ROW)
                             : "memory");
            } else {
                asm volatile("ds_read_b64_tr_b16 %0, %4\n\tds_read_b64_tr_b16 %1, %5 offset:%6\n\t"
                             "ds_read_b64_tr_b16 %2, %4 offset:%7\n\tds_read_b64_tr_b16 %3, %5 offset:%8\n\ts_waitcnt lgkmcnt(0)"
                             : "=&v"(v[0][d][0]), "=&v"(v[0][d][1]), "=&v"(v[1][d][0]), "=&v"(v[1][d][1])
                             : "v"(lo), "v"(hi), "n"(8 * ROW), "n"(16 * ROW), "n"(24 * ROW)
                             : "memory");
            }
        }
    }
    __device__ __forceinline__ AttFrag<T> get(int step, int d) const {
        AttFrag<T> f;
        f.v[0] = __builtin_bit_cast(typename AttFrag<T>::vec, __builtin_shufflevector(v[step][d][0], v[step][d][1], 0, 1, 2, 3, 4, 5, 6, 7));
        return f;
    }
};

// The `across` operands of 16 rows of two tiles, `apart` elements from each other; DIRECT as above.
template <typename T, int D, int ROWS, bool DIRECT>
struct AttAcrossBoth {
    const AttRead<T, D, ROWS> &read;
    const typename AttRead<T, D, ROWS>::E *a, *b;
    int first;
    __device__ __forceinline__ AttAcrossBoth(const AttRead<T, D, ROWS> &read, const typename AttRead<T, D, ROWS>::E *a,
                                             const typename AttRead<T, D, ROWS>::E *b, int first) : read(read), a(a), b(b), first(first) {}
    __device__ __forceinline__ AttFrag<T> get_a(int d) const { return read.across(a, first, d); }
    __device__ __forceinline__ AttFrag<T> get_b(int d) const { return read.across(b, first, d); }
};
template <typename T, int D, int ROWS>
struct AttAcrossBoth<T, D, ROWS, true> {
    typedef AttLayout<D> L;
    typedef typename LinearPlanes<T>::elem E;
    s16x4 v[2][D / 32][2];
    // (b lies behind a in AttPipe's buffers)
    __device__ __forceinline__ AttAcrossBoth(const AttRead<T, D, ROWS> &read, const E *a, const E *, int first) {
        typedef const __attribute__((address_space(3))) E *Ptr;
        constexpr int ROW = L::LD * 2, APART = ROWS * ROW;  // bytes
        const uint32_t base = (uint32_t)(uintptr_t)(Ptr)(a + first * L::LD + read.token);
#pragma unroll
        for (int d = 0; d < D / 32; d += 2) {
            const uint32_t lo = base + 2 * (read.lo ^ (d * 32)), hi = base + 2 * (read.hi ^ (d * 32));
            if (d + 1 < D / 32) {
                const int e = d + 1 < D / 32 ? d + 1 : d;  // (the compiler looks at it for D = 32 as well)
                const uint32_t lo1 = base + 2 * (read.lo ^ (e * 32)), hi1 = base + 2 * (read.hi ^ (e * 32));
                asm volatile("ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %9 offset:%12\n\t"
                             "ds_read_b64_tr_b16 %2, %10\n\tds_read_b64_tr_b16 %3, %11 offset:%12\n\t"
                             "ds_read_b64_tr_b16 %4, %8 offset:%13\n\tds_read_b64_tr_b16 %5, %9 offset:%14\n\t"
                             "ds_read_b64_tr_b16 %6, %10 offset:%13\n\tds_read_b64_tr_b16 %7, %11 offset:%14\n\ts_waitcnt lgkmcnt(0)"
                             : "=&v"(v[0][d][0]), "=&v"(v[0][d][1]), "=&v"(v[0][e][0]), "=&v"(v[0][e][1]), "=&v"(v[1][d][0]),
                               "=&v"(v[1][d][1]), "=&v"(v[1][e][0]), "=&v"(v[1][e][1])
                             : "v"(lo), "v"(hi), "v"(lo1), "v"(hi1), "n"(8 * ROW), "n"(APART), "n"(APART + 8 * ROW)
                             : "memory");
            } else {
                asm volatile("ds_read_b64_tr_b16 %0, %4\n\tds_read_b64_tr_b16 %1, %5 offset:%6\n\t"
                             "ds_read_b64_tr_b16 %2, %4 offset:%7\n\tds_read_b64_tr_b16 %3, %5 offset:%8\n\ts_waitcnt lgkmcnt(0)"
                             : "=&v"(v[0][d][0]), "=&v"(v[0][d][1]), "=&v"(v[1][d][0]), "=&v"(v[1][d][1])
                             : "v"(lo), "v"(hi), "n"(8 * ROW), "n"(APART), "n"(APART + 8 * ROW)
                             : "memory");
            }
        }
    }
    __device__ __forceinline__ AttFrag<T> get(int which, int d) const {
        AttFrag<T> f;
        f.v[0] = __builtin_bit_cast(typename AttFrag<T>::vec, __builtin_shufflevector(v[which][d][0], v[which][d][1], 0, 1, 2, 3, 4, 5, 6, 7));
        return f;
    }
    __device__ __forceinline__ AttFrag<T> get_a(int d) const { return get(0, d); }
    __device__ __forceinline__ AttFrag<T> get_b(int d) const { return get(1, d); }
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

// The tiles of examples of uneven length, the longest first: list[0] of them, list[1 ..] = example << 32 | number in the example.  One
// workgroup: it counts the tiles of each number and hands out places behind those of higher ones (which tile of a number gets which place
// is open: it is only the order in which they run).
// Examples that share no rows have at most rows / kAttRows + 1 whole tiles and one that is not whole each, which is the list's room.  Where
// there are more, some share rows, and outputs of those are not defined: each whole tile claims the multiple of kAttRows among its
// rows, the first example that claims one keeps its tile, and other tiles are left out.  A tile of an example that shares no rows is never
// one of them, and there is room for what is left.  claims [rows / kAttRows + 1].
__global__ __launch_bounds__(1024) void attention_list(TokenRows tok, int tiles, int64_t room, uint64_t *__restrict__ list,
                                                       uint32_t *__restrict__ claims)
{
    extern __shared__ int place[];  // [tiles]
    __shared__ int sums[1024];
    // f(example, its rows, tile's number)
    const auto each = [&](auto &&f) {
        for (int64_t e = threadIdx.x; e < tok.examples; e += 1024) {
            const RowSpan span = rows_of(tok, e);
            const int mine = (int)((span.count + kAttRows - 1) / kAttRows);  // (at most `tiles`)
            for (int j = 0; j < mine; ++j) f(e, span, j);
        }
    };
    const auto claim = [&](const RowSpan &span, int j) -> uint32_t * {  // (NULL: not a whole tile)
        return (j + 1) * kAttRows <= span.count ? claims + (span.first + j * kAttRows + kAttRows - 1) / kAttRows : nullptr;
    };
    bool shared = false;  // uniform
    const auto kept = [&](int64_t e, const RowSpan &span, int j) {
        if (!shared) return true;
        const uint32_t *c = claim(span, j);
        return !c || __hip_atomic_load(c, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)e;
    };
    // The first place of each number, into `place`; how many there are.
    const auto hand_out = [&]() {
        for (int j = threadIdx.x; j < tiles; j += 1024) place[j] = 0;
        __syncthreads();
        each([&](int64_t e, const RowSpan &span, int j) {
            if (kept(e, span, j)) atomicAdd(place + j, 1);
        });
        __syncthreads();
        // a thread's share of the numbers, from the highest on: its sum, the sums before it, its places
        const int per = (tiles + 1023) / 1024, hi = tiles - threadIdx.x * per;
        int sum = 0;
        for (int j = hi - 1; j >= 0 && j >= hi - per; --j) sum += place[j];
        sums[threadIdx.x] = sum;
        __syncthreads();
        for (int gap = 1; gap < 1024; gap *= 2) {
            const int before = (int)threadIdx.x >= gap ? sums[threadIdx.x - gap] : 0;
            __syncthreads();
            sums[threadIdx.x] += before;
            __syncthreads();
        }
        int at = sums[threadIdx.x] - sum;
        for (int j = hi - 1; j >= 0 && j >= hi - per; --j) {
            const int n = place[j];
            place[j] = at;
            at += n;
        }
        const int total = sums[1023];
        __syncthreads();
        return total;
    };
    int total = hand_out();  // uniform
    if (total > room) {
        for (int64_t i = threadIdx.x; i < tok.rows / kAttRows + 1; i += 1024) claims[i] = ~0u;
        __threadfence();
        __syncthreads();
        each([&](int64_t e, const RowSpan &span, int j) {
            if (uint32_t *c = claim(span, j)) atomicMin(c, (uint32_t)e);
        });
        __threadfence();
        __syncthreads();
        shared = true;
        total = hand_out();
    }
    if (threadIdx.x == 0) list[0] = (uint64_t)(total < room ? total : room);
    each([&](int64_t e, const RowSpan &span, int j) {
        if (!kept(e, span, j)) return;
        const int to = atomicAdd(place + j, 1);
        if (to < room) list[1 + to] = (uint64_t)e << 32 | (uint64_t)j;
    });
}

// What a workgroup works on.  All of a pair (example, head of keys) run on one XCD: workgroups go round the XCDs, so every eighth belongs
// to the same pair.  The longest tiles of all pairs come first: a long one that starts late keeps the others waiting.  Or, by_pair, those of
// a pair one after the other, so that the XCD's L2 holds what they share.  (us, tile by tile and by pair: forward 64 x 1024 tokens, 12
// heads of 64, bf16, 6144 workgroups 191 and 183; 16 x 1024, 8 heads of 64, fp32, 1024 workgroups 117 and 177; dk and dv of 16 x 1024, 16
// heads on 4 of 128, 512 workgroups 250 and 383.)
struct AttPlace {
    RowSpan span;
    int row0, count;  // the tile's first row in the example, the example's rows
    int kv, head;     // heads of keys, of queries
    bool there;
    // QUERIES: a workgroup per tile and head of queries, later tiles are the longer ones.  Otherwise one per tile of keys.
    template <bool QUERIES>
    __device__ __forceinline__ AttPlace(const TokenRows &tok, const AttHeads &a, std::integral_constant<bool, QUERIES>) {
        const int members = QUERIES ? a.group : 1;
        if (a.list) {  // uniform: the heads of a tile side by side
            const int64_t unit = a.unit0 + blockIdx.x, heads = (int64_t)a.kv_heads * members, slot = unit / heads;
            there = slot < (int64_t)a.list[0];
            if (!there) return;
            const uint64_t entry = a.list[1 + slot];
            const int which = (int)(unit - slot * heads), j = (int)(uint32_t)entry;
            span = rows_of(tok, (int64_t)(entry >> 32));
            count = (int)span.count;
            kv = which / members;
            head = kv * a.group + (which - kv * members);
            row0 = (QUERIES ? j : (count + kAttRows - 1) / kAttRows - 1 - j) * kAttRows;
            return;
        }
        const int64_t unit = a.unit0 + blockIdx.x, turn = unit >> 3, per = a.by_pair ? (int64_t)a.tiles * members : (a.pairs + 7) >> 3;
        const int64_t whole = turn / per, part = turn - whole * per, pair = (a.by_pair ? whole : part) * 8 + (unit & 7);
        const int rest = (int)(a.by_pair ? part : whole), tile = rest / members;
        there = pair < a.pairs;
        if (!there) return;
        const int64_t e = pair / a.kv_heads;
        span = rows_of(tok, tok.base + e);
        kv = (int)(pair - e * a.kv_heads);
        head = kv * a.group + (rest - tile * members);
        row0 = (QUERIES ? a.tiles - 1 - tile : tile) * kAttRows;
        count = (int)span.count;  // (at most kAttMaxTokens)
        there = row0 < count;
    }
};

constexpr float kLog2E = 1.44269504088896341f, kLn2 = 0.693147180559945309f;

// p is held 2^shift times as large: fp16 has room for that above (the forward pass's p reach 2^8, the backward pass's 1), and
// below 2^-14 its numbers lose digits.
template <typename T> constexpr float kAttShiftForward = 0.f;
template <> constexpr float kAttShiftForward<f16_t> = 7.f;
template <typename T> constexpr float kAttShiftBack = 0.f;
template <> constexpr float kAttShiftBack<f16_t> = 14.f;

template <typename T> constexpr bool kAttExact = LinearPlanes<T>::N > 1;  // fp32

// A staged tile's rows; LDS for two of them, all planes.
template <typename T> constexpr int att_step() { return LinearPlanes<T>::N == 1 ? 64 : 32; }

// Exponents of the forward pass: s c - most, where most is the rounded product of c and the row's maximum.  That all of a row are off by half a
// step of `most` is nothing while it is small, since a factor of all weights goes out with their sum, but from 2^24 on it takes them out
// of fp16 and from 2^31 on out of fp32.  So where it would pass kAttFar a wavefront goes over to (s - ref) c - most for the rest of its rows,
// ref the maximum in the scores' units and most the shift alone: a difference of scores is as exact as they are, at any scale.
// (One branch a tile: 64 x 1024 tokens, 12 heads of 64, bf16 196 -> 198 us, 2 x 8192, 32 heads on 8 of 128 1264 -> 1272 on the same card.)
constexpr float kAttFar = 0x1p20f;

template <typename T, int D, bool DIRECT>
__global__ __launch_bounds__(kAttThreads, LinearPlanes<T>::N == 1 ? 2 : 1) void attention_forward(
    TokenRows tok, AttHeads a, const T *__restrict__ Q, int64_t q_stride, const T *__restrict__ K, int64_t k_stride,
    const T *__restrict__ V, int64_t v_stride, T *__restrict__ O, int64_t o_stride, float *__restrict__ lse)
{
    typedef typename LinearPlanes<T>::elem E;
    constexpr int STEP = att_step<T>(), KB = STEP / 32, DB = D / 32;
    typedef AttPipe<T, D, STEP, DIRECT> Pipe;
    __shared__ __align__(16) E lds[Pipe::LDS];
    const AttPlace at(tok, a, std::true_type{});
    if (!at.there) return;  // uniform
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int first = at.row0 + wave * 32, mine = first + (lane & 31), count = at.count;
    const T *q = Q + (at.span.first + (mine < count ? mine : 0)) * q_stride + (int64_t)at.head * a.dim;
    const T *k = K + at.span.first * k_stride + (int64_t)at.kv * a.dim, *v = V + at.span.first * v_stride + (int64_t)at.kv * a.dim;
    AttColumns<T, D> cols;
    cols.load(q, lane, a.dim, mine < count);
    const AttRead<T, D, STEP> read(lane);
    f32x16 acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) acc[d] = zero16();
    float most = -INFINITY, sum = 0.f, ref = 0.f;  // (`sum` of the lane's own rows)
    const float c = a.scale * kLog2E;
    bool far = false;  // uniform
    const int end = at.row0 + kAttRows < count ? at.row0 + kAttRows : count;  // keys
    Pipe pipe(lds, a.dim, k_stride, v_stride);
    pipe.fetch(k, k_stride, v, v_stride, 0, end);
    for (int t = 0; t < end; t += STEP) {
        const E *tk = pipe.turn(), *tv = tk + Pipe::LEN / 2;
        if (t + STEP < end) pipe.fetch(k, k_stride, v, v_stride, t + STEP, end);
        if (t > first + 31) continue;  // all later than this wavefront's queries
        f32x16 s[KB];
#pragma unroll
        for (int b = 0; b < KB; ++b) {
            s[b] = zero16();
#pragma unroll
            for (int d = 0; d < D / 16; ++d) s[b] = att_mfma<T>(read.along(tk, b * 32, d), cols.k[d], s[b]);
        }
        if (t + STEP - 1 > first) {
            const int left = mine - t;  // rows of the tile up to this query
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
        const float raw = both_max(top);
        top = fmaf(raw, c, -kAttShiftForward<T>);
        // (The maximum may lag behind by 2^8, the sums have room for that: they are seldom scaled.)
        if (__any(far ? (raw - ref) * c > 8.f : top > most + 8.f)) {
            float next = fmaxf(most, top), down = __builtin_amdgcn_exp2f(most - next);
            if (far || __any(fabsf(next) > kAttFar && next > -INFINITY)) {  // (-inf: a row that is NaN so far)
                float by = 0.f;  // what the exponents of the sums change by for the other form
                if (!far) {
                    far = true;
                    ref = most / c;
                    by = most > -INFINITY ? fmaf(-ref, c, most) + kAttShiftForward<T> : 0.f;
                }
                next = -kAttShiftForward<T>;
                const float peak = fmaxf(ref, raw);
                down = __builtin_amdgcn_exp2f(fmaf(ref - peak, c, by));
                ref = peak;
            }
            most = next;
            sum *= down;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[d][r] *= down;
        }
        if (far)
#pragma unroll
            for (int b = 0; b < KB; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[b][r] -= ref;
#pragma unroll
        for (int b = 0; b < KB; ++b) {
            const AttAcross<T, D, STEP, DIRECT> values(read, tv, b * 32);
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
                for (int d = 0; d < DB; ++d) acc[d] = att_mfma<T>(values.get(r / 8, d), w, acc[d]);
            }
        }
    }
    sum = both_sum(sum);
    if (mine < count) {
        att_write<T, D>(O + (at.span.first + mine) * o_stride + (int64_t)at.head * a.dim, acc, 1.f / sum, a.dim, lane);
        if (lse && lane < 32)
            lse[at.head * tok.rows + at.span.first + mine] = fmaf(ref, a.scale, (most + __builtin_amdgcn_logf(sum)) * kLn2);
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
template <typename T, int D, bool DIRECT>
__global__ __launch_bounds__(kAttThreads, LinearPlanes<T>::N > 1 ? 1 : D <= 64 ? 4 : 2) void attention_backward_q(
    TokenRows tok, AttHeads a, const T *__restrict__ Q, int64_t q_stride, const T *__restrict__ K, int64_t k_stride,
    const T *__restrict__ V, int64_t v_stride, const T *__restrict__ O, int64_t o_stride, const float *__restrict__ lse,
    const T *__restrict__ DO, int64_t do_stride, T *__restrict__ DQ, int64_t dq_stride, float *__restrict__ delta)
{
    typedef typename LinearPlanes<T>::elem E;
    constexpr int STEP = att_step<T>(), KB = STEP / 32, DB = D / 32;
    typedef AttPipe<T, D, STEP, DIRECT> Pipe;
    __shared__ __align__(16) E lds[Pipe::LDS];
    const AttPlace at(tok, a, std::true_type{});
    if (!at.there) return;  // uniform
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int first = at.row0 + wave * 32, mine = first + (lane & 31), count = at.count;
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
    }
    const AttRead<T, D, STEP> read(lane);
    const float c = a.scale * kLog2E, most = live ? lse[at.head * tok.rows + row] * kLog2E : INFINITY;
    const int end = at.row0 + kAttRows < count ? at.row0 + kAttRows : count;
    Pipe pipe(lds, a.dim, k_stride, v_stride);
    pipe.fetch(k, k_stride, v, v_stride, 0, end);
    // p (do v - D) of 32 keys
    const auto weights = [&](const E *tk, const E *tv, int t, int b) {
        f32x16 s = zero16(), ds = zero16();
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
            s = att_mfma<T>(read.along(tk, b * 32, d), q.k[d], s);
            ds = att_mfma<T>(read.along(tv, b * 32, d), g.k[d], ds);
        }
        if (t + b * 32 + 31 > first)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = b * 32 + att_row(r, lane) <= mine - t ? s[r] : -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; ++r) ds[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c, -most)) * (ds[r] - dot);
        return ds;
    };
    // The first rows of an example go over their keys twice: o is rounded to 16 bits, and D with it, and for a row of few keys that is
    // as much as p (do v - D) itself (which is nothing for the first).  What sum_j p_ij (do_i v_j - D_i) leaves is D's error.  (dq, relative,
    // without and with: 2 tokens of fp16 5.1e-4 and 2.9e-4, 1024 of bf16 2.50e-3 and 2.38e-3; the outputs' rounding alone is 2.1e-4 and
    // 1.66e-3.  Of rows of many keys D's error is a part of that of p, by the root of their number.)
    if (LinearPlanes<T>::N == 1 && at.row0 == 0) {
        float rest = 0.f;
        for (int t = 0; t < end; t += STEP) {
            const E *tk = pipe.turn(), *tv = tk + Pipe::LEN / 2;
            pipe.fetch(k, k_stride, v, v_stride, t + STEP < end ? t + STEP : 0, end);  // (behind the last the first again)
            if (t > first + 31) continue;
#pragma unroll 1
            for (int b = 0; b < KB; ++b) {
                const f32x16 ds = weights(tk, tv, t, b);
#pragma unroll
                for (int r = 0; r < 16; ++r) rest += ds[r];
            }
        }
        dot += both_sum(rest);
    }
    f32x16 acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) acc[d] = zero16();
    AttScaled<T, DB> scaled;
    for (int t = 0; t < end; t += STEP) {
        const E *tk = pipe.turn(), *tv = tk + Pipe::LEN / 2;
        if (t + STEP < end) pipe.fetch(k, k_stride, v, v_stride, t + STEP, end);
        if (t > first + 31) continue;
#pragma unroll 1
        for (int b = 0; b < KB; ++b) {
            f32x16 ds = weights(tk, tv, t, b);
            scaled.fit(ds, acc);
            const AttAcross<T, D, STEP, DIRECT> keys(read, tk, b * 32);
#pragma unroll
            for (int r = 0; r < 16; r += 8) {
                float x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = ds[r + j];
                AttFrag<T> w;
                w.set(x);
#pragma unroll
                for (int d = 0; d < DB; ++d) acc[d] = att_mfma<T>(keys.get(r / 8, d), w, acc[d]);
            }
        }
    }
    if (live && lane < 32) delta[at.head * tok.rows + row] = dot;
    if (live) att_write<T, D>(DQ + row * dq_stride + (int64_t)at.head * a.dim, acc, a.scale / scaled.scale, a.dim, lane);
}

// dk and dv by keys, over all heads that share them.  A block of 32 queries at a time: two at a time need registers that are not there (620 us
// against 430 for the case above).  Spilled: 62 registers of fp32 at 128 features, at 64 of 16 bits 3 (whole pieces; dq too) or 4 to 15.
template <typename T, int D, bool DIRECT>
__global__ __launch_bounds__(kAttThreads, LinearPlanes<T>::N == 1 && D <= 64 ? 3 : 1) void attention_backward_kv(
    TokenRows tok, AttHeads a, const T *__restrict__ Q, int64_t q_stride, const T *__restrict__ K, int64_t k_stride,
    const T *__restrict__ V, int64_t v_stride, const float *__restrict__ lse, const T *__restrict__ DO, int64_t do_stride,
    const float *__restrict__ delta, T *__restrict__ DK, int64_t dk_stride, T *__restrict__ DV, int64_t dv_stride)
{
    typedef typename LinearPlanes<T>::elem E;
    constexpr int STEP = att_step<T>(), QB = STEP / 32, DB = D / 32;
    typedef AttPipe<T, D, STEP, DIRECT> Pipe;
    // (One array: with several the compiler waits for all loads to LDS in front of each read.)
    __shared__ __align__(16) E lds[Pipe::LDS + 8 * STEP];
    float *const row_values = reinterpret_cast<float *>(lds + Pipe::LDS);  // [2][2][STEP]
    const AttPlace at(tok, a, std::false_type{});
    if (!at.there) return;  // uniform
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int first = at.row0 + wave * 32, mine = first + (lane & 31), count = at.count;
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
    Pipe pipe(lds, a.dim, q_stride, do_stride);
    int which = 0;
    float next_most = 0.f, next_dot = 0.f;
    const auto fetch = [&](int t, int64_t head) {
        pipe.fetch(Q + at.span.first * q_stride + head * a.dim, q_stride, DO + at.span.first * do_stride + head * a.dim, do_stride, t, count);
        if (threadIdx.x < STEP) {  // (nothing is done with them here: that would wait for them)
            const int64_t r = head * tok.rows + at.span.first + (t + (int)threadIdx.x < count ? t + threadIdx.x : count - 1);
            next_most = lse[r];
            next_dot = delta[r];
        }
    };
    int t = at.row0, next_t = t;
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
        if (threadIdx.x < STEP) {  // (the other one may still be read)
            // (a row that is not there: p = 0)
            row_values[which * 2 * STEP + threadIdx.x] = 
                t + (int)threadIdx.x >= count ? -INFINITY : kAttExact<T> ? -next_most * kLog2E : (kAttShiftBack<T> * kLn2 - next_most) / a.scale;
            row_values[which * 2 * STEP + STEP + threadIdx.x] = -next_dot;
        }
        const E *tq = pipe.turn(), *tg = tq + Pipe::LEN / 2;
        const float *most = row_values + which * 2 * STEP, *dots = most + STEP;
        which ^= 1;
        advance();
        if (next_head < at.head + a.group) fetch(next_t, next_head);
        if (t + STEP - 1 < first) continue;  // all earlier than this wavefront's keys
#pragma unroll 1
        for (int b = 0; b < QB; ++b) {
            // (sums that begin at -L / scale and -D: the exponent and do v - D without further instructions.  fp32: L / scale would take
            // digits from the scores, dk 1.2e-6 off instead of 0.7e-6)
            const float *m = most + b * 32 + 4 * (lane >> 5), *dot = dots + b * 32 + 4 * (lane >> 5);
            f32x16 s, ds;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[r] = kAttExact<T> ? 0.f : m[8 * (r >> 2) + (r & 3)];
                ds[r] = dot[8 * (r >> 2) + (r & 3)];
            }
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
                s = att_mfma<T>(read.along(tq, b * 32, d), k.k[d], s);
                ds = att_mfma<T>(read.along(tg, b * 32, d), v.k[d], ds);
            }
            const int from = mine - t - b * 32;  // the first of the rows that sees this key
            if (t + b * 32 < first + 31)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = att_row(r, lane) >= from ? s[r] : -INFINITY;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[r] = __builtin_amdgcn_exp2f(kAttExact<T> ? fmaf(s[r], c, m[8 * (r >> 2) + (r & 3)]) : s[r] * c);
                ds[r] *= s[r];
            }
            scaled.fit(ds, dk);
            AttFrag<T> w[2], z[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float x[8], y[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    x[j] = s[8 * h + j];
                    y[j] = ds[8 * h + j];
                }
                w[h].set(x);
                z[h].set(y);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const AttAcrossBoth<T, D, STEP, DIRECT> rows(read, tq, tg, b * 32 + h * 16);
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    dv[d] = att_mfma<T>(rows.get_b(d), w[h], dv[d]);
                    dk[d] = att_mfma<T>(rows.get_a(d), z[h], dk[d]);
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
