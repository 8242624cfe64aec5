// Embedding of token ids: y_t = scale table[id_t], and per example the table's gradient
//   G_e[v] = scale sum over the example's rows t with id_t = v of dy_t.
//
// Both are bound by bytes: forward a row of the table in and a row out, backward every row of dy in and all of G out, most of which are
// rows of zeros.  G is written once: a workgroup that owns rows of G knows which rows of dy belong there, in order.  So nothing is added
// up by atomics, and the sums do not depend on what else runs.  Measured: 65 536 rows of 768, bf16 31 us (4.8 TB/s: of ids by rank in
// 50 000 15 700 are different, 48 MB of the table are read and 101 MB written); gradients of 64 examples of 128 rows, 5000 x 128 33 us, 5.1 TB/s; of one of 65 536 rows, 50 000 x 768 135 us,
// of which sorting the ids 15, merging them 21, frequent ids 12 and the rest, where G is written, 62.
#pragma once
#include "layer_common.hpp"

namespace cdgrab {

constexpr int kEmbedThreads = 256;
constexpr int kEmbedList = 2048;    // ids of an example that a workgroup looks through by itself
constexpr int kEmbedElems = 16384;  // elements of G that a workgroup writes, about
constexpr int kEmbedSpan = 2048;    // rows of G at most
constexpr int kEmbedLong = 32;      // rows of dy from which on all threads of a workgroup share a row of G
constexpr int kEmbedPiece = 16;     // longer examples: the same, and sorted keys of one id that are added up beforehand
constexpr int kEmbedChunk = 1024;   // keys that a workgroup sorts (of 4096: 40 us for 16 of them, of 1024 a quarter of that)
constexpr int kEmbedFan = 16;       // sorted runs that are merged at a time

// Threads that share a row: 1 << shift of them, VEC elements each at a time.  ONCE, here and below: what is written is more than the caches
// hold, and goes past them (65 536 rows of 768, bf16, with other inputs every time 45 -> 32 us; 64 examples of 5000 x 128 46 -> 33).
template <typename TT, typename T, int VEC, bool ONCE>
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
            store_any<T, VEC, ONCE>(to + at, y);
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
template <typename T, int VEC, bool ONCE>
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
            store_any<float, VEC, ONCE>(to + (int64_t)v * width + at, sum);
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

// ---- longer examples: all (id, row) keys of an example in order, then as above --------------------------

constexpr uint64_t kEmbedNone = ~(uint64_t)0;  // of no row, or an id that is not in the table

// Chunk b % chunks of example b / chunks: its keys, sorted.  keys [examples of the launch][chunks * kEmbedChunk]
__global__ __launch_bounds__(kEmbedThreads) void embed_sort(TokenRows tok, int chunks, const int32_t *__restrict__ ids, int64_t vocab,
                                                            uint64_t *__restrict__ keys)
{
    __shared__ uint64_t part[kEmbedChunk];
    const int64_t local = blockIdx.x / chunks, c = blockIdx.x - local * chunks;
    const RowSpan rows = rows_of(tok, tok.base + local);
    for (int i = threadIdx.x; i < kEmbedChunk; i += kEmbedThreads) {
        const int64_t t = c * kEmbedChunk + i;
        const int64_t id = t < rows.count ? ids[rows.first + t] : -1;
        part[i] = id >= 0 && id < vocab ? (uint64_t)id << 32 | (uint64_t)t : kEmbedNone;
    }
    for (int size = 2; size <= kEmbedChunk; size *= 2)
        for (int gap = size / 2; gap > 0; gap /= 2) {
            __syncthreads();
#pragma unroll
            for (int i = threadIdx.x; i < kEmbedChunk / 2; i += kEmbedThreads) {
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
    for (int i = threadIdx.x; i < kEmbedChunk; i += kEmbedThreads) to[i] = part[i];
}

// kEmbedFan sorted runs of `run` keys each become one: a key's place is the number of smaller ones in all of them.  A wavefront counts
// those of one run, for 64 keys side by side, whose searches go the same way and read the same lines (a lane per run instead: 18 us a
// pass over 65 536 keys).  (Keys are distinct but for those of no row, which keep the runs' order.)
__global__ __launch_bounds__(64 * kEmbedFan) void embed_merge(const uint64_t *__restrict__ from, uint64_t *__restrict__ to, int64_t len,
                                                              int64_t run)
{
    __shared__ int below[kEmbedFan][64];
    const int lane = threadIdx.x & 63, r = threadIdx.x >> 6;
    const int64_t i = (int64_t)blockIdx.x * 64 + lane;  // (len and run are multiples of 64)
    const uint64_t *keys = from + blockIdx.y * len;
    const uint64_t key = keys[i];
    const int64_t mine = i / run, group = mine / kEmbedFan * kEmbedFan, begin = (group + r) * run;
    const int64_t n = begin >= len ? 0 : len - begin < run ? len - begin : run;
    int64_t lo = 0, hi = n;
    if (group + r == mine) lo = hi = i - begin;
    if (group + r < mine && key == kEmbedNone) lo = hi;
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (keys[begin + mid] < key) lo = mid + 1;
        else hi = mid;
    }
    below[r][lane] = (int)lo;
    __syncthreads();
    if (r == 0) {
        int64_t at = group * run;
#pragma unroll
        for (int q = 0; q < kEmbedFan; ++q) at += below[q][lane];
        to[blockIdx.y * len + at] = key;
    }
}

// Of a piece of sorted keys that all have one id a group of threads adds up the rows, to parts [piece][width]: frequent ids are shared by
// many workgroups so.
template <typename T, int VEC>
__global__ __launch_bounds__(kEmbedThreads) void embed_grad_pieces(TokenRows tok, int64_t pieces, int shift, const uint64_t *__restrict__ keys,
                                                                   int64_t len, int width, const T *__restrict__ DY, int64_t dy_stride,
                                                                   float *__restrict__ parts)
{
    const int lanes = 1 << shift, t = threadIdx.x & (lanes - 1);
    const int64_t unit = (int64_t)blockIdx.x * (kEmbedThreads >> shift) + (threadIdx.x >> shift);
    if (unit >= pieces * tok.examples) return;
    const int64_t local = unit / pieces, piece = unit - local * pieces;
    const uint64_t *k = keys + local * len + piece * kEmbedPiece;
    if (k[kEmbedPiece - 1] == kEmbedNone || k[0] >> 32 != k[kEmbedPiece - 1] >> 32) return;
    const T *dy = DY + rows_of(tok, tok.base + local).first * dy_stride;
    for (int col = t * VEC; col < width; col += lanes * VEC) {
        const int at = col + VEC <= width ? col : width - VEC;
        float sum[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) sum[i] = 0.f;
        embed_sum<T, VEC>(dy, dy_stride, at, kEmbedPiece, [&](int j) { return (int64_t)(k[j] & 0xffffffffu); }, sum);
        store_any<float, VEC>(parts + unit * width + at, sum);
    }
}

// Number of the n sorted keys below `key`: all threads of the workgroup look at once, 256 places at a time.
__device__ __forceinline__ int64_t embed_below(const uint64_t *keys, int64_t n, uint64_t key) {
    int64_t lo = 0;
    while (n > 0) {  // uniform
        const int64_t gap = (n + kEmbedThreads - 1) / kEmbedThreads, at = threadIdx.x * gap;
        const int below = __syncthreads_count(at < n && keys[lo + at] < key);
        if (below == 0) break;  // (the first place is not below)
        // places 0 .. below - 1 are: the answer lies behind the last of them, within its gap
        const int64_t last = (below - 1) * gap;
        lo += last + 1;
        n = (last + gap < n ? last + gap : n) - last - 1;
    }
    return lo;
}

// embed_grad_few for sorted keys, but for the ids of many rows.
template <typename T, int VEC, bool ONCE>
__device__ __forceinline__ void embed_span(uint32_t *lds, const uint64_t *list, int64_t len, int64_t v0, int own, int shift, int width,
                                           const T *dy, int64_t dy_stride, float scale, float *g)
{
    uint32_t *const start = lds, *const stop = lds + kEmbedSpan, *const found = lds + 2 * kEmbedSpan;
    for (int v = threadIdx.x; v < own; v += kEmbedThreads) start[v] = stop[v] = 0;
    const int64_t begin = embed_below(list, len, (uint64_t)v0 << 32);
    const int64_t m = embed_below(list + begin, len - begin, (uint64_t)(v0 + own) << 32);
    list += begin;
    __syncthreads();
    for (int64_t i = threadIdx.x; i < m; i += kEmbedThreads) {
        const uint64_t key = list[i];
        const int v = (int)((int64_t)(key >> 32) - v0);
        if (i < kEmbedList) found[i] = (uint32_t)key;
        if (i == 0 || list[i - 1] >> 32 != key >> 32) start[v] = (uint32_t)i;
        if (i == m - 1 || list[i + 1] >> 32 != key >> 32) stop[v] = (uint32_t)i + 1;
    }
    __syncthreads();
    const int lanes = 1 << shift, t = threadIdx.x & (lanes - 1), groups = kEmbedThreads >> shift;
    float *to = g + v0 * width;
    const bool here = m <= kEmbedList;  // uniform
    for (int v = threadIdx.x >> shift; v < own; v += groups) {
        const int64_t j0 = start[v], count = stop[v] - j0;
        if (count >= kEmbedPiece) continue;
        for (int col = t * VEC; col < width; col += lanes * VEC) {
            const int at = col + VEC <= width ? col : width - VEC;
            float sum[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) sum[i] = 0.f;
            if (count > 0) {
                if (here) embed_sum<T, VEC>(dy, dy_stride, at, (int)count, [&](int j) { return (int64_t)found[j0 + j]; }, sum);
                else embed_sum<T, VEC>(dy, dy_stride, at, (int)count, [&](int j) { return (int64_t)(uint32_t)list[j0 + j]; }, sum);
            }
#pragma unroll
            for (int i = 0; i < VEC; ++i) sum[i] *= scale;
            store_any<float, VEC, ONCE>(to + (int64_t)v * width + at, sum);
        }
    }
}

// Ids of kEmbedPiece rows and more: a workgroup each, that of the piece in which the id's keys begin (of no two ids: the first would
// fill the piece).  Rows up to the first whole piece, whole pieces, the rest; in this order.
template <typename T, int VEC>
__device__ __forceinline__ void embed_long(float *part, const uint64_t *list, int64_t len, int64_t piece, int shift, int width, const T *dy,
                                           int64_t dy_stride, float scale, const float *parts, float *g)
{
    int64_t j0 = -1;
#pragma unroll
    for (int j = 0; j < kEmbedPiece; ++j) {  // (uniform, and at most one)
        const int64_t i = piece * kEmbedPiece + j, last = i + kEmbedPiece - 1;
        if (last < len && list[last] != kEmbedNone && list[last] >> 32 == list[i] >> 32 && (i == 0 || list[i - 1] >> 32 != list[i] >> 32))
            j0 = i;
    }
    if (j0 < 0) return;
    const uint64_t id = list[j0] >> 32;
    const int64_t j1 = j0 + embed_below(list + j0, len - j0, (id + 1) << 32);
    const int64_t p0 = (j0 + kEmbedPiece - 1) / kEmbedPiece, p1 = j1 / kEmbedPiece;
    const int whole = p1 > p0 ? (int)(p1 - p0) : 0;
    const int head = (int)(whole ? p0 * kEmbedPiece - j0 : j1 - j0), tail = (int)(whole ? j1 - p1 * kEmbedPiece : 0);
    const float *from = parts + p0 * width;
    float *to = g + (int64_t)id * width;
    const auto rows_sum = [&](int at, const uint64_t *k, int count, float (&sum)[VEC]) {
        embed_sum<T, VEC>(dy, dy_stride, at, count, [&](int j) { return (int64_t)(uint32_t)k[j]; }, sum);
    };
    embed_shared<VEC>(shift, width, head + whole + tail, part,
                      [&](int at, int a, int count, float (&sum)[VEC]) {
                          const int b = a + count;
                          if (a < head) rows_sum(at, list + j0 + a, (b < head ? b : head) - a, sum);
                          const int pa = a > head ? a - head : 0, pb = b - head < whole ? b - head : whole;
                          if (pb > pa) embed_sum<float, VEC>(from, width, at, pb - pa, [&](int j) { return (int64_t)(pa + j); }, sum);
                          const int ta = a > head + whole ? a - head - whole : 0, tb = b - head - whole;
                          if (tb > ta) rows_sum(at, list + p1 * kEmbedPiece + ta, tb - ta, sum);
                      },
                      [&](int at, float (&sum)[VEC]) {
#pragma unroll
                          for (int i = 0; i < VEC; ++i) sum[i] *= scale;
                          store_any<float, VEC>(to + at, sum);
                      });
}

// Both, the ids of many rows first: they take longest, and the others fill the chip beside them (one after the other 50 + 24 us).
template <typename T, int VEC, bool ONCE>
__global__ __launch_bounds__(kEmbedThreads) void embed_grad_many(TokenRows tok, uint32_t units, int span, int shift, uint32_t pieces,
                                                                 const uint64_t *__restrict__ keys, int64_t len, int64_t vocab, int width,
                                                                 const T *__restrict__ DY, int64_t dy_stride, float scale,
                                                                 const float *__restrict__ parts, float *__restrict__ G, int64_t g_stride)
{
    __shared__ uint32_t lds[2 * kEmbedSpan + kEmbedList];
    static_assert(sizeof(lds) >= kEmbedThreads * VEC * sizeof(float), "");
    const uint32_t longs = pieces * (uint32_t)tok.examples;  // workgroups
    const bool many = blockIdx.x < longs;                    // uniform
    const uint32_t b = many ? blockIdx.x : blockIdx.x - longs, local = b / (many ? pieces : units), at = b - local * (many ? pieces : units);
    const int64_t e = tok.base + local;
    const uint64_t *list = keys + local * len;
    const T *dy = DY + rows_of(tok, e).first * dy_stride;
    float *g = G + e * g_stride;
    if (many) {
        embed_long<T, VEC>(reinterpret_cast<float *>(lds), list, len, at, shift, width, dy, dy_stride, scale,
                           parts + (int64_t)local * pieces * width, g);
    } else {
        const int64_t v0 = (int64_t)at * span;
        embed_span<T, VEC, ONCE>(lds, list, len, v0, (int)(vocab - v0 < span ? vocab - v0 : span), shift, width, dy, dy_stride, scale, g);
    }
}

}  // namespace cdgrab
