// Embedding of token ids: y_t = scale table[id_t], and per example the table's gradient
//   G_e[v] = scale sum over the example's rows t with id_t = v of dy_t.
//
// Both are bound by bytes: forward a row of the table in and a row out, backward every row of dy in and all of G out, most of which are
// rows of zeros.  G is written once: a workgroup that owns rows of G knows which rows of dy belong there, in order.  So nothing is added
// up by atomics, and the sums do not depend on what else runs.
#pragma once
#include "layer_common.hpp"

namespace cdgrab {

constexpr int kEmbedThreads = 256;
constexpr int kEmbedList = 2048;    // ids of an example that a workgroup looks through by itself
constexpr int kEmbedElems = 16384;  // elements of G that a workgroup writes, about
constexpr int kEmbedSpan = 2048;    // rows of G at most
constexpr int kEmbedLong = 32;      // rows of dy from which on all threads of a workgroup share a row of G
constexpr int kEmbedChunk = 4096;   // keys that a workgroup sorts
constexpr int kEmbedFan = 16;       // sorted runs that are merged at a time
constexpr int kEmbedPiece = 64;     // sorted keys that a group of threads adds up

// Threads that share a row: 1 << shift of them, VEC elements each at a time.
template <typename TT, typename T, int VEC>
__global__ __launch_bounds__(kEmbedThreads) void embed_forward(const int32_t *__restrict__ ids, int64_t rows, int64_t vocab, int width,
                                                               int shift, const TT *__restrict__ table, int64_t t_stride, float scale,
                                                               T *__restrict__ Y, int64_t y_stride)
{
    const int lanes = 1 << shift, t = threadIdx.x & (lanes - 1);
    const int64_t per = kEmbedThreads >> shift, step = (int64_t)gridDim.x * per;
    for (int64_t row = (int64_t)blockIdx.x * per + (threadIdx.x >> shift); row < rows; row += step) {
        const int64_t id = ids[row];
        const bool known = id >= 0 && id < vocab;
        const TT *from = table + (known ? id : 0) * t_stride;
        T *to = Y + row * y_stride;
#pragma unroll 2
        for (int col = t * VEC; col < width; col += lanes * VEC) {
            const int at = col + VEC <= width ? col : width - VEC;  // (the last ones twice, with the same values)
            TT x[VEC];
            T y[VEC];
            load_any<TT, VEC>(from + at, x);
#pragma unroll
            for (int j = 0; j < VEC; ++j) y[j] = known ? (T)((float)x[j] * scale) : (T)0.f;
            store_any<T, VEC>(to + at, y);
        }
    }
}

// Sum of `n` rows of dy, row(j) the j-th, at columns col ..; eight loads on their way.
template <typename T, int VEC, typename F>
__device__ __forceinline__ void embed_sum(const T *DY, int64_t stride, int col, int n, F &&row, float (&sum)[VEC]) {
#pragma unroll 8
    for (int j = 0; j < n; ++j) {
        T x[VEC];
        load_any<T, VEC>(DY + row(j) * stride + col, x);
#pragma unroll
        for (int i = 0; i < VEC; ++i) sum[i] += (float)x[i];
    }
}

// The same of a long list by all threads of the workgroup: shares of the list by its groups of threads, which the first adds up in
// order and hands to `put`.  `part` holds kEmbedThreads * VEC floats.
template <int VEC, typename S, typename P>
__device__ __forceinline__ void embed_shared(int shift, int width, int n, float *part, S &&sum_of, P &&put) {
    const int lanes = 1 << shift, t = threadIdx.x & (lanes - 1), mine = threadIdx.x >> shift, groups = kEmbedThreads >> shift;
    const int per = (n + groups - 1) / groups, j0 = mine * per < n ? mine * per : n, j1 = j0 + per < n ? j0 + per : n;
    for (int base = 0; base < width; base += lanes * VEC) {
        const int col = base + t * VEC, at = col + VEC <= width ? col : width - VEC;
        float sum[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) sum[i] = 0.f;
        if (col < width) sum_of(at, j0, j1 - j0, sum);
#pragma unroll
        for (int i = 0; i < VEC; ++i) part[threadIdx.x * VEC + i] = sum[i];
        __syncthreads();
        if (mine == 0 && col < width) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) sum[i] = 0.f;
            for (int g = 0; g < groups; ++g)
#pragma unroll
                for (int i = 0; i < VEC; ++i) sum[i] += part[((g << shift) + t) * VEC + i];
            put(at, sum);
        }
        __syncthreads();
    }
}

// Examples of at most kEmbedList rows.  Workgroup b writes rows v0 .. v0 + span - 1 of example b / units: it picks the ids in that range,
// sorts them (id and row, by counting the smaller ones), and its groups of threads take the rows of G in turn.
template <typename T, int VEC>
__global__ __launch_bounds__(kEmbedThreads) void embed_grad_few(TokenRows tok, uint32_t units, int span, int shift,
                                                                const int32_t *__restrict__ ids, int64_t vocab, int width,
                                                                const T *__restrict__ DY, int64_t dy_stride, float scale,
                                                                float *__restrict__ G, int64_t g_stride)
{
    __shared__ uint32_t found[kEmbedList], sorted[kEmbedList];
    __shared__ uint16_t start[kEmbedSpan], stop[kEmbedSpan], longs[kEmbedList / kEmbedLong];
    __shared__ float part[kEmbedThreads * VEC];
    __shared__ int have, many;
    const uint32_t local = blockIdx.x / units;
    const int64_t e = tok.base + local, v0 = (int64_t)(blockIdx.x - local * units) * span;
    const RowSpan rows = rows_of(tok, e);
    const int n = (int)rows.count, own = (int)(vocab - v0 < span ? vocab - v0 : span);
    if (threadIdx.x == 0) have = many = 0;
    for (int v = threadIdx.x; v < own; v += kEmbedThreads) start[v] = stop[v] = 0;
    __syncthreads();
    for (int t = threadIdx.x; t < n; t += kEmbedThreads) {
        const int64_t v = ids[rows.first + t] - v0;
        if (v >= 0 && v < own) found[atomicAdd(&have, 1)] = (uint32_t)v << 16 | (uint32_t)t;  // (in any order: they are sorted)
    }
    __syncthreads();
    const int m = have;
    for (int i = threadIdx.x; i < m; i += kEmbedThreads) {
        const uint32_t key = found[i];
        int rank = 0;
#pragma unroll 4
        for (int j = 0; j < m; ++j) rank += found[j] < key;
        sorted[rank] = key;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < m; i += kEmbedThreads) {
        const uint32_t v = sorted[i] >> 16;
        if (i == 0 || sorted[i - 1] >> 16 != v) start[v] = (uint16_t)i;
        if (i == m - 1 || sorted[i + 1] >> 16 != v) stop[v] = (uint16_t)(i + 1);
    }
    __syncthreads();
    const int lanes = 1 << shift, t = threadIdx.x & (lanes - 1), groups = kEmbedThreads >> shift;
    float *to = G + e * g_stride + v0 * width;
    const T *dy = DY + rows.first * dy_stride;
    const auto sum_of = [&](int at, int j0, int count, float (&sum)[VEC]) {
        embed_sum<T, VEC>(dy, dy_stride, at, count, [&](int j) { return (int64_t)(sorted[j0 + j] & 0xffff); }, sum);
    };
    for (int v = threadIdx.x >> shift; v < own; v += groups) {
        const int j0 = start[v], count = stop[v] - j0;
        if (count >= kEmbedLong) {
            if (t == 0) longs[atomicAdd(&many, 1)] = (uint16_t)v;
            continue;
        }
        for (int col = t * VEC; col < width; col += lanes * VEC) {
            const int at = col + VEC <= width ? col : width - VEC;
            float sum[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) sum[i] = 0.f;
            if (count > 0) sum_of(at, j0, count, sum);
#pragma unroll
            for (int i = 0; i < VEC; ++i) sum[i] *= scale;
            store_any<float, VEC>(to + (int64_t)v * width + at, sum);
        }
    }
    __syncthreads();
    for (int q = 0; q < many; ++q) {  // uniform
        const int v = longs[q], j0 = start[v];
        embed_shared<VEC>(shift, width, stop[v] - j0, part,
                          [&](int at, int from, int count, float (&sum)[VEC]) { sum_of(at, j0 + from, count, sum); },
                          [&](int at, float (&sum)[VEC]) {
#pragma unroll
                              for (int i = 0; i < VEC; ++i) sum[i] *= scale;
                              store_any<float, VEC>(to + (int64_t)v * width + at, sum);
                          });
    }
}

// ---- longer examples: all (id, row) keys of an example in order -------------------------------------

constexpr uint64_t kEmbedNone = ~(uint64_t)0;  // of no row, or an id that is not in the table

// Chunk b % chunks of example b / chunks: its keys, sorted.  keys [examples of the launch][chunks * kEmbedChunk]
__global__ __launch_bounds__(1024) void embed_sort(TokenRows tok, int chunks, const int32_t *__restrict__ ids, int64_t vocab,
                                                   uint64_t *__restrict__ keys)
{
    __shared__ uint64_t part[kEmbedChunk];
    const int64_t local = blockIdx.x / chunks, c = blockIdx.x - local * chunks;
    const RowSpan rows = rows_of(tok, tok.base + local);
    for (int i = threadIdx.x; i < kEmbedChunk; i += 1024) {
        const int64_t t = c * kEmbedChunk + i;
        const int64_t id = t < rows.count ? ids[rows.first + t] : -1;
        part[i] = id >= 0 && id < vocab ? (uint64_t)id << 32 | (uint64_t)t : kEmbedNone;
    }
    for (int size = 2; size <= kEmbedChunk; size *= 2)
        for (int gap = size / 2; gap > 0; gap /= 2) {
            __syncthreads();
            for (int i = threadIdx.x; i < kEmbedChunk / 2; i += 1024) {
                const int lo = 2 * i - (i & (gap - 1)), hi = lo + gap;
                const uint64_t a = part[lo], b = part[hi];
                const bool up = (lo & size) == 0;
                if ((a > b) == up) {
                    part[lo] = b;
                    part[hi] = a;
                }
            }
        }
    __syncthreads();
    uint64_t *to = keys + (local * chunks + c) * kEmbedChunk;
    for (int i = threadIdx.x; i < kEmbedChunk; i += 1024) to[i] = part[i];
}

// Number of keys below `key` among the n sorted ones.
__device__ __forceinline__ int64_t embed_below(const uint64_t *keys, int64_t n, uint64_t key) {
    int64_t lo = 0, hi = n;
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (keys[mid] < key) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

// kEmbedFan sorted runs of `run` keys each become one: a key's place is the number of smaller ones in all of them.  (Keys are distinct but
// for those of no row, which keep the runs' order.)
__global__ __launch_bounds__(256) void embed_merge(const uint64_t *__restrict__ from, uint64_t *__restrict__ to, int64_t len, int64_t run)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= len) return;
    const uint64_t *keys = from + blockIdx.y * len;
    const uint64_t key = keys[i];
    const int64_t mine = i / run, group = mine / kEmbedFan * kEmbedFan;
    int64_t at = i - mine * run;
#pragma unroll
    for (int r = 0; r < kEmbedFan; ++r) {
        const int64_t begin = (group + r) * run;
        if (group + r == mine || begin >= len) continue;
        const int64_t n = len - begin < run ? len - begin : run;
        at += key != kEmbedNone ? embed_below(keys + begin, n, key) : group + r < mine ? n : embed_below(keys + begin, n, key);
    }
    to[blockIdx.y * len + group * run + at] = key;
}

// A group of threads adds up the rows of kEmbedPiece sorted keys.  Runs of one id that lie within the piece go to G; of the others the
// sums go to parts [piece][2][width]: 0 of a run that has begun in an earlier piece, 1 of one that begins here and goes on.
template <typename T, int VEC>
__global__ __launch_bounds__(kEmbedThreads) void embed_grad_pieces(TokenRows tok, int64_t pieces, int shift, const uint64_t *__restrict__ keys,
                                                                   int64_t len, int width, const T *__restrict__ DY, int64_t dy_stride,
                                                                   float scale, float *__restrict__ G, int64_t g_stride,
                                                                   float *__restrict__ parts)
{
    const int lanes = 1 << shift, t = threadIdx.x & (lanes - 1);
    const int64_t unit = (int64_t)blockIdx.x * (kEmbedThreads >> shift) + (threadIdx.x >> shift);
    if (unit >= pieces * tok.examples) return;
    const int64_t local = unit / pieces, piece = unit - local * pieces, e = tok.base + local;
    const RowSpan rows = rows_of(tok, e);
    const uint64_t *list = keys + local * len, *k = list + piece * kEmbedPiece;
    if (k[0] == kEmbedNone) return;
    const bool before = piece > 0 && k[-1] >> 32 == k[0] >> 32;
    const T *dy = DY + rows.first * dy_stride;
    float *g = G + e * g_stride, *part = parts + unit * 2 * width;
    for (int col = t * VEC; col < width; col += lanes * VEC) {
        const int at = col + VEC <= width ? col : width - VEC;
        float sum[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) sum[i] = 0.f;
        bool begun = before;
        uint64_t key = k[0];
        for (int j0 = 0; j0 < kEmbedPiece; j0 += 8) {
            if (k[j0] == kEmbedNone) break;
            T x[8][VEC];
            uint64_t next[9];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                next[j] = k[j0 + j];
                if (next[j] != kEmbedNone) load_any<T, VEC>(dy + (int64_t)(next[j] & 0xffffffffu) * dy_stride + at, x[j]);
            }
            const int64_t behind = piece * kEmbedPiece + j0 + 8;
            next[8] = behind < len ? list[behind] : kEmbedNone;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (next[j] == kEmbedNone) break;
                key = next[j];
#pragma unroll
                for (int i = 0; i < VEC; ++i) sum[i] += (float)x[j][i];
                const bool same = next[j + 1] >> 32 == key >> 32;
                if (same && j0 + j + 1 < kEmbedPiece) continue;
                if (!begun && !same) {
#pragma unroll
                    for (int i = 0; i < VEC; ++i) sum[i] *= scale;
                    store_any<float, VEC>(g + (int64_t)(key >> 32) * width + at, sum);
                } else {
                    store_any<float, VEC>(part + (begun ? 0 : width) + at, sum);
                }
                begun = false;
#pragma unroll
                for (int i = 0; i < VEC; ++i) sum[i] = 0.f;
            }
        }
    }
}

// The rest of G: zeros, and runs of several pieces.
template <int VEC>
__global__ __launch_bounds__(kEmbedThreads) void embed_grad_rest(TokenRows tok, uint32_t units, int span, int shift, int64_t pieces,
                                                                 const uint64_t *__restrict__ keys, int64_t len, int64_t vocab, int width,
                                                                 float scale, const float *__restrict__ parts, float *__restrict__ G,
                                                                 int64_t g_stride)
{
    __shared__ int64_t start[kEmbedSpan + 1];
    __shared__ float part[kEmbedThreads * VEC];
    const uint32_t local = blockIdx.x / units;
    const int64_t e = tok.base + local, v0 = (int64_t)(blockIdx.x - local * units) * span;
    const int own = (int)(vocab - v0 < span ? vocab - v0 : span);
    const uint64_t *list = keys + local * len;
    for (int v = threadIdx.x; v <= own; v += kEmbedThreads) start[v] = embed_below(list, len, (uint64_t)(v0 + v) << 32);
    __syncthreads();
    const int lanes = 1 << shift, t = threadIdx.x & (lanes - 1), groups = kEmbedThreads >> shift;
    float *to = G + e * g_stride + v0 * width;
    const float *from = parts + local * pieces * 2 * width;
    float none[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) none[i] = 0.f;
    for (int v = threadIdx.x >> shift; v < own; v += groups)
        if (start[v] == start[v + 1])
            for (int col = t * VEC; col < width; col += lanes * VEC)
                store_any<float, VEC>(to + (int64_t)v * width + (col + VEC <= width ? col : width - VEC), none);
    for (int v = 0; v < own; ++v) {  // uniform
        const int64_t first = start[v] / kEmbedPiece, last = (start[v + 1] - 1) / kEmbedPiece;
        if (start[v] == start[v + 1] || first == last) continue;
        embed_shared<VEC>(shift, width, (int)(last - first + 1), part,
                          [&](int at, int j0, int count, float (&sum)[VEC]) {
                              embed_sum<float, VEC>(from, width, at, count,
                                                    [&](int j) { return (first + j0 + j) * 2 + (j0 + j == 0 ? 1 : 0); }, sum);
                          },
                          [&](int at, float (&sum)[VEC]) {
#pragma unroll
                              for (int i = 0; i < VEC; ++i) sum[i] *= scale;
                              store_any<float, VEC>(to + (int64_t)v * width + at, sum);
                          });
    }
}

}  // namespace cdgrab
