// Host side of the sequence operators (embedding, norms of heads with the position rotation, attention): argument checks, choice of the
// kernel, launches.  Included by cdgrab.hip behind layer_entries.hpp.
#pragma once

namespace {

constexpr int64_t kEmbedBytes = (int64_t)1 << 30;  // keys and sums of pieces: as many examples at a time
constexpr int64_t kMaxHeads = 4096;
constexpr int64_t kAttMaxTokens = (int64_t)1 << 22;
constexpr int64_t kAttListTiles = 8192;  // of an example (LDS of the kernel that lists tiles)

// An array of rows as the checks take it.
struct Rows {
    const char *name;
    const void *p;
    int64_t rows, bytes, stride;  // bytes of a row, from row to row
    bool meets(const Rows &o) const { return rows_overlap(p, rows, bytes, stride, o.p, o.rows, o.bytes, o.stride); }
};

// No output shares a byte with an input or with another output.
int check_apart(cdgrab_handle *h, const char *who, std::initializer_list<Rows> in, std::initializer_list<Rows> out) {
    for (const Rows &o : out) {
        for (const Rows &i : in)
            if (o.meets(i)) return fail(h, CDGRAB_EINVAL, "%s: %s must not overlap %s", who, o.name, i.name);
        for (const Rows &other : out)
            if (&other != &o && o.meets(other)) return fail(h, CDGRAB_EINVAL, "%s: %s must not overlap %s", who, o.name, other.name);
    }
    return CDGRAB_OK;
}

template <typename F>
int by_elem(int32_t type, F &&f) {
    if (type == CDGRAB_F32) return f(float{});
    return type == CDGRAB_BF16 ? f(bf16_t{}) : f(f16_t{});
}

// Threads that share a row of `width`, as a power of two: what holds it in pieces of `vec`, a workgroup at the most.
int row_shift(int64_t width, int64_t vec) {
    int s = 0;
    while (s < 8 && (vec << s) < width) ++s;
    return s;
}

constexpr int64_t kOnceBytes = (int64_t)64 << 20;  // of an array from which on it is written past the caches

template <typename TT, typename T>
int run_embed(cdgrab_handle *h, const int32_t *ids, int64_t rows, int64_t vocab, int64_t width, const void *table, int64_t t_stride,
              float scale, void *Y, int64_t y_stride) {
    constexpr int VEC = 16 / (int)sizeof(T);
    const auto launch = [&](auto vec, auto once) {
        constexpr int V = decltype(vec)::value;
        const int shift = row_shift(width, V);
        const int64_t per = kEmbedThreads >> shift, groups = std::min<int64_t>((rows + per - 1) / per, 8 * (int64_t)h->num_cu);
        hipLaunchKernelGGL((embed_forward<TT, T, V, decltype(once)::value>), dim3((unsigned)groups), dim3(kEmbedThreads), 0, h->stream, ids, rows, vocab, (int)width,
                           shift, (const TT *)table, t_stride, scale, (T *)Y, y_stride);
    };
    if (width < VEC) launch(std::integral_constant<int, 1>{}, std::false_type{});
    else if (rows * width * (int64_t)sizeof(T) < kOnceBytes) launch(std::integral_constant<int, VEC>{}, std::false_type{});
    else launch(std::integral_constant<int, VEC>{}, std::true_type{});
    HIP_TRY(h, hipGetLastError());
    return CDGRAB_OK;
}

template <typename T, int VEC, bool ONCE>
int run_embed_grad(cdgrab_handle *h, const char *who, const TokenRows &tok, int64_t vocab, int64_t width, const int32_t *ids, const T *DY,
                   int64_t dy_stride, float scale, float *G, int64_t g_stride) {
    const int shift = row_shift(width, VEC);
    const int64_t tokens = std::min(tok.tokens, tok.rows);
    // rows of G per workgroup: stretches of kEmbedElems, or shorter ones until there are 32 workgroups per CU (the first ids are the
    // frequent ones of most vocabularies: a workgroup that has many of them is the last to end)
    const int64_t elems = std::max<int64_t>(1024, std::min<int64_t>(kEmbedElems, tok.examples * vocab * width / (32 * (int64_t)h->num_cu)));
    const int64_t span = std::min<int64_t>(std::max<int64_t>(1, elems / width), std::min<int64_t>(kEmbedSpan, vocab));
    const int64_t units = (vocab + span - 1) / span;
    if (tokens <= kEmbedList) {
        const int64_t per = std::max<int64_t>(1, kMaxGroups / units);
        for (int64_t e0 = 0; e0 < tok.examples; e0 += per) {
            TokenRows part = tok;
            part.examples = std::min(per, tok.examples - e0);
            part.base = e0;
            hipLaunchKernelGGL((embed_grad_few<T, VEC, ONCE>), dim3((unsigned)(part.examples * units)), dim3(kEmbedThreads), 0, h->stream, part,
                               (uint32_t)units, (int)span, shift, ids, vocab, (int)width, DY, dy_stride, scale, G, g_stride);
        }
        HIP_TRY(h, hipGetLastError());
        return CDGRAB_OK;
    }
    const int64_t chunks = (tokens + kEmbedChunk - 1) / kEmbedChunk, len = chunks * kEmbedChunk, pieces = len / kEmbedPiece;
    const int64_t bytes = len * 16 + pieces * width * 4;  // of an example
    const int64_t lanes = kEmbedThreads >> shift;
    const int64_t at_once = std::max<int64_t>(1, std::min({tok.examples, kEmbedBytes / bytes, kMaxGroups / (units + pieces),
                                                           (int64_t)65535, kMaxGroups * lanes / pieces}));
    char *ws = nullptr;
    const int rc = layer_room(h, who, at_once * bytes, &ws);
    if (rc) return rc;
    uint64_t *const keys = reinterpret_cast<uint64_t *>(ws), *const other = keys + at_once * len;
    float *const parts = reinterpret_cast<float *>(other + at_once * len);
    for (int64_t e0 = 0; e0 < tok.examples; e0 += at_once) {
        TokenRows part = tok;
        part.examples = std::min(at_once, tok.examples - e0);
        part.base = e0;
        hipLaunchKernelGGL(embed_sort, dim3((unsigned)(part.examples * chunks)), dim3(kEmbedThreads), 0, h->stream, part, (int)chunks, ids, vocab,
                           keys);
        uint64_t *from = keys, *to = other;
        for (int64_t run = kEmbedChunk; run < len; run *= kEmbedFan) {
            hipLaunchKernelGGL(embed_merge, dim3((unsigned)(len / 64), (unsigned)part.examples), dim3(64 * kEmbedFan), 0, h->stream, from, to, len, run);
            std::swap(from, to);
        }
        hipLaunchKernelGGL((embed_grad_pieces<T, VEC>), dim3((unsigned)((part.examples * pieces + lanes - 1) / lanes)), dim3(kEmbedThreads), 0,
                           h->stream, part, pieces, shift, from, len, (int)width, DY, dy_stride, parts);
        hipLaunchKernelGGL((embed_grad_many<T, VEC, ONCE>), dim3((unsigned)(part.examples * (pieces + units))), dim3(kEmbedThreads), 0, h->stream,
                           part, (uint32_t)units, (int)span, shift, (uint32_t)pieces, from, len, vocab, (int)width, DY, dy_stride, scale, parts,
                           G, g_stride);
    }
    HIP_TRY(h, hipGetLastError());
    return CDGRAB_OK;
}

// f(threads per head, elements per access) for half a head's features
template <typename T, typename F>
int by_head_shape(int half, F &&f) {
    constexpr int VEC = 16 / (int)sizeof(T);
    const int groups = (half + VEC - 1) / VEC;
#define HEAD_SHAPE(V, L) return f(std::integral_constant<int, V>{}, std::integral_constant<int, L>{})
    if (half < VEC) HEAD_SHAPE(1, 8);
    if (groups <= 1) HEAD_SHAPE(VEC, 1);
    if (groups <= 2) HEAD_SHAPE(VEC, 2);
    if (groups <= 4) HEAD_SHAPE(VEC, 4);
    if (groups <= 8) HEAD_SHAPE(VEC, 8);
    if (groups <= 16) HEAD_SHAPE(VEC, 16);
    if (VEC == 8 || groups <= 32) HEAD_SHAPE(VEC, 32);
    HEAD_SHAPE(VEC, 64);
#undef HEAD_SHAPE
}

HeadTurns head_turns(int half, double base) {
    HeadTurns t{};
    if (base == 0.0) return t;
    // (powers of the ratio one after the other: 64 bits, of which 256 products leave 56)
    const long double ratio = powl((long double)base, -1.0L / half);
    long double turn = 18446744073709551616.0L / (2.0L * 3.14159265358979323846264338327950288L);  // of one radian per position
    for (int i = 0; i < half; ++i, turn *= ratio) t.turn[i] = (uint64_t)turn;
    return t;
}

int check_heads(cdgrab_handle *h, const char *who, const cdgrab_heads *s, int32_t type) {
    if (!s) return fail(h, CDGRAB_EINVAL, "%s: the heads are NULL", who);
    if (s->q_heads < 0 || s->k_heads < 0 || s->q_heads + s->k_heads < 1 || s->q_heads > kMaxHeads || s->k_heads > kMaxHeads || s->dim < 2 ||
        s->dim > kHeadMaxDim || s->dim % 2 != 0 || bad_type(type) || !(s->eps >= 0.f) ||
        !(s->base == 0.0 || (s->base >= 1.0 && std::isfinite(s->base))))
        return fail(h, CDGRAB_EINVAL, "%s: bad arguments q_heads=%lld k_heads=%lld (0 .. %lld) dim=%lld (even, 2 .. %d) type=%d eps=%g base=%g "
                    "(0, or 1 at least)", who, (long long)s->q_heads, (long long)s->k_heads, (long long)kMaxHeads, (long long)s->dim,
                    kHeadMaxDim, (int)type, (double)s->eps, s->base);
    return CDGRAB_OK;
}

template <typename T, bool BACKWARD>
int run_heads(cdgrab_handle *h, const char *who, const TokenRows &tok, const cdgrab_heads &s, const T *X, int64_t x_stride, const T *DY,
              int64_t dy_stride, const float *gain_q, const float *gain_k, T *Y, int64_t y_stride, float *G, int64_t g_stride) {
    const int half = (int)s.dim / 2, heads = (int)(s.q_heads + s.k_heads);
    const HeadTurns turns = head_turns(half, s.base);
    const int64_t width = heads * s.dim, size = sizeof(T);
    // (pieces of heads in whole lines: else a line that both halves share is read twice, 257 examples of 200 rows of 10 heads of 80, fp16
    // 46 -> 55 us; 65 536 rows of 24 heads of 64, bf16 95 -> 91, 20 000 of 40 of 128 back 133 -> 118)
    const bool once = half * size % 64 == 0 && norm_once(tok.rows, width, size, X, x_stride) && (!BACKWARD || norm_once(tok.rows, width, size, DY, dy_stride));
    return by_head_shape<T>(half, [&](auto vec, auto lanes) {
        constexpr int VEC = decltype(vec)::value, LANES = decltype(lanes)::value;
        // an example's rows in chunks until the chip is full, of a round of the groups of threads at least
        constexpr int GROUPS = kHeadThreads / LANES;
        const int64_t tokens = std::min(tok.tokens, tok.rows), fill = 8 * (int64_t)h->num_cu, least = std::max(1, GROUPS / heads);
        const int64_t chunks = std::min(std::max<int64_t>(1, tokens / least), std::max<int64_t>(1, (fill + tok.examples - 1) / tok.examples));
        const int64_t each = (tokens + chunks - 1) / chunks;
        const HeadShape sh{(int)s.q_heads, heads, half, (int)std::max<int64_t>(1, std::min<int64_t>({kHeadTable / half, each, 64})), s.eps};
        float *partial = nullptr;
        if (BACKWARD && G && chunks > 1) {
            const int rc = layer_room(h, who, tok.examples * chunks * 2 * s.dim, &partial);
            if (rc) return rc;
        }
        const int64_t per = std::max<int64_t>(1, kMaxGroups / chunks);
        for (int64_t e0 = 0; e0 < tok.examples; e0 += per) {
            TokenRows part = tok;
            part.examples = std::min(per, tok.examples - e0);
            part.base = e0;
            const auto launch = [&](auto kernel) {
                hipLaunchKernelGGL(kernel, dim3((unsigned)(part.examples * chunks)), dim3(kHeadThreads), 0, h->stream, part, (int)chunks, sh,
                                   turns, X, x_stride, DY, dy_stride, gain_q, gain_k, Y, y_stride, G, g_stride, partial);
            };
            if constexpr (!std::is_same<T, f16_t>::value) {
                if (s.eps < kHeadTiny) {
                    launch(head_norm<T, VEC, LANES, BACKWARD, false, true>);
                    continue;
                }
            }
            if constexpr (VEC > 1) {
                if (once) {
                    launch(head_norm<T, VEC, LANES, BACKWARD, true, false>);
                    continue;
                }
            }
            launch(head_norm<T, VEC, LANES, BACKWARD, false, false>);
        }
        if (partial)  // (fewer than `fill` examples of at most 32 groups of columns: one launch)
            hipLaunchKernelGGL(norm_grad_finish, dim3((unsigned)(tok.examples * ((2 * s.dim + 31) / 32))), dim3(256), 0, h->stream, partial,
                               (int)chunks, (int)(2 * s.dim), G, g_stride);
        HIP_TRY(h, hipGetLastError());
        return (int)CDGRAB_OK;
    });
}

int check_attention(cdgrab_handle *h, const char *who, const cdgrab_token_rows *t, int64_t q_heads, int64_t kv_heads, int64_t dim,
                    int32_t type, float scale) {
    const int rc = check_tokens(h, who, t);
    if (rc) return rc;
    if (q_heads < 1 || kv_heads < 1 || q_heads > kMaxHeads || q_heads % kv_heads != 0 || dim < 1 || dim > kAttMaxDim || bad_type(type) ||
        !(scale >= 1e-30f && scale <= 1e30f))
        return fail(h, CDGRAB_EINVAL, "%s: bad arguments q_heads=%lld (a multiple of kv_heads, at most %lld) kv_heads=%lld dim=%lld (1 .. %d) "
                    "type=%d scale=%g (1e-30 .. 1e30)", who, (long long)q_heads, (long long)kMaxHeads, (long long)kv_heads, (long long)dim,
                    kAttMaxDim, (int)type, (double)scale);
    if (std::min(t->tokens, t->rows) > kAttMaxTokens)
        return fail(h, CDGRAB_EINVAL, "%s: %lld tokens of an example, and at most 2^22", who, (long long)std::min(t->tokens, t->rows));
    return CDGRAB_OK;
}

// f(widest head that the kernel has room for)
template <typename F>
int by_head_dim(int64_t dim, F &&f) {
    if (dim <= 32) return f(std::integral_constant<int, 32>{});
    if (dim <= 64) return f(std::integral_constant<int, 64>{});
    if (dim <= 96) return f(std::integral_constant<int, 96>{});
    return f(std::integral_constant<int, 128>{});
}

// Rows that go to LDS in whole pieces of 16 bytes, 64 of them within 2 GB; f(whether all of the arrays are such).
struct Pieces {
    const void *p;
    int64_t stride;
};
template <typename T, typename F>
int by_pieces(int64_t dim, std::initializer_list<Pieces> arrays, F &&f) {
    if constexpr (sizeof(T) == 2) {
        bool whole = dim % 8 == 0;
        for (const Pieces &a : arrays)
            whole = whole && reinterpret_cast<uintptr_t>(a.p) % 16 == 0 && a.stride % 8 == 0 && a.stride < ((int64_t)1 << 24);
        if (whole) return f(std::true_type{});
    }
    return f(std::false_type{});
}

int64_t att_tiles(const TokenRows &tok) { return (std::min(tok.tokens, tok.rows) + kAttRows - 1) / kAttRows; }

// Room of the list of tiles: what examples that share no rows can have at most, if a list pays (else 0): where the longest example is much longer
// than the others most of [examples][tiles] is empty, and a workgroup that finds nothing costs about a nanosecond (1000 examples of 100 tokens and
// one of 8192, 12 heads of 64, bf16: forward 1141 -> 342 us, back 2855 -> 966).  Of packed rows only: with the rows of a padded batch there
// may be as many tiles as there are workgroups, and `count` is not known here.
int64_t att_list(const TokenRows &tok) {
    const int64_t tiles = att_tiles(tok), most = tok.rows / kAttRows + tok.examples;
    const bool pays = tok.count && tiles > 1 && tiles <= kAttListTiles && tok.examples < INT32_MAX / tiles && most < INT32_MAX / 2 &&
                      tok.examples >= 2 * most / tiles + 64;
    return pays ? most + 1 : 0;
}

// The list, and what its kernel takes besides (claims), whole words of eight bytes.
int64_t att_list_bytes(const TokenRows &tok) {
    const int64_t most = att_list(tok);
    return most ? (most + 1) * 8 + round_up((tok.rows / kAttRows + 1) * 4, 8) : 0;
}

void make_att_list(cdgrab_handle *h, const TokenRows &tok, uint64_t *list) {
    const int64_t most = att_list(tok), tiles = att_tiles(tok);
    if (most)
        hipLaunchKernelGGL(attention_list, dim3(1), dim3(1024), (size_t)tiles * sizeof(int), h->stream, tok, (int)tiles, most, list,
                           reinterpret_cast<uint32_t *>(list + most + 1));
}

// launch(heads, workgroups) for as many workgroups at a time as a grid holds; `members`: one per tile and head of queries, else of keys.
// By pairs if there are so many that the last long ones do not count.
template <typename F>
void by_units(cdgrab_handle *h, const TokenRows &tok, int64_t q_heads, int64_t kv_heads, int64_t dim, float scale, bool members,
              const uint64_t *list, F &&launch) {
    const int64_t tiles = att_tiles(tok), group = q_heads / kv_heads, pairs = tok.examples * kv_heads, most = att_list(tok);
    const int64_t units = most ? most * (members ? q_heads : kv_heads) : round_up(pairs, 8) * tiles * (members ? group : 1);
    for (int64_t u = 0; u < units; u += kMaxGroups)  // (a multiple of eight)
        launch(AttHeads{pairs, u, (int)tiles, (int)kv_heads, (int)group, members && units >= 8 * (int64_t)h->num_cu, most ? list : nullptr,
                        (int)dim, scale},
               dim3((unsigned)std::min(kMaxGroups, units - u)));
}

}  // namespace

extern "C" int cdgrab_embed(cdgrab_handle *h, int64_t rows, int64_t vocab, int64_t width, const int32_t *ids, int32_t table_type,
                            const void *table, int64_t t_stride, float scale, int32_t type, void *Y, int64_t y_stride) {
    if (!h) return CDGRAB_EINVAL;
    static const char *who = "cdgrab_embed";
    if (rows < 0 || rows > ((int64_t)1 << 40) || vocab < 1 || vocab > INT32_MAX || width < 1 || width > (1 << 20) || bad_type(type) ||
        (table_type != type && table_type != CDGRAB_F32) || !std::isfinite(scale))
        return fail(h, CDGRAB_EINVAL, "%s: bad arguments rows=%lld vocab=%lld width=%lld (1 .. 2^20) table_type=%d (fp32 or type) type=%d scale=%g",
                    who, (long long)rows, (long long)vocab, (long long)width, (int)table_type, (int)type, (double)scale);
    if (rows == 0) return CDGRAB_OK;
    if (!ids || !table || !Y) return fail(h, CDGRAB_EINVAL, "%s: null pointer", who);
    const int64_t size = elem_size(type), t_size = elem_size(table_type);
    if (bad_rows(table, vocab, width, t_stride, t_size) || bad_rows(Y, rows, width, y_stride, size) || bad_rows(ids, rows, 1, 1, 4))
        return fail(h, CDGRAB_EINVAL, "%s: a stride below the width, or a misaligned or too long array", who);
    const int rc = check_apart(h, who, {{"ids", ids, 1, rows * 4, rows * 4}, {"table", table, vocab, width * t_size, t_stride * t_size}},
                               {{"Y", Y, rows, width * size, y_stride * size}});
    if (rc) return rc;
    const OnDevice on(h->device);
    HIP_TRY(h, on.err);
    return by_elem(type, [&](auto elem) {
        typedef decltype(elem) T;
        if (table_type == CDGRAB_F32) return run_embed<float, T>(h, ids, rows, vocab, width, table, t_stride, scale, Y, y_stride);
        return run_embed<T, T>(h, ids, rows, vocab, width, table, t_stride, scale, Y, y_stride);
    });
}

extern "C" int cdgrab_pergrad_embed(cdgrab_handle *h, const cdgrab_token_rows *t, int64_t vocab, int64_t width, int32_t type,
                                    const int32_t *ids, const void *DY, int64_t dy_stride, float scale, float *G, int64_t g_stride) {
    if (!h) return CDGRAB_EINVAL;
    static const char *who = "cdgrab_pergrad_embed";
    int rc = check_tokens(h, who, t);
    if (rc) return rc;
    if (vocab < 1 || vocab > INT32_MAX || width < 1 || width > (1 << 20) || vocab * width > kMaxCells || bad_type(type) || !std::isfinite(scale) ||
        std::min(t->tokens, t->rows) > ((int64_t)1 << 26))
        return fail(h, CDGRAB_EINVAL, "%s: bad arguments vocab=%lld width=%lld (1 .. 2^20, 2^32 elements) type=%d scale=%g tokens=%lld (2^26)", who,
                    (long long)vocab, (long long)width, (int)type, (double)scale, (long long)t->tokens);
    if (t->examples == 0) return CDGRAB_OK;
    if (!G || (t->rows > 0 && t->tokens > 0 && (!ids || !DY))) return fail(h, CDGRAB_EINVAL, "%s: null pointer", who);
    const int64_t size = elem_size(type), d = vocab * width;
    if (bad_rows(DY, t->rows, width, dy_stride, size) || bad_rows(G, t->examples, d, g_stride, 4) || bad_rows(ids, t->rows, 1, 1, 4))
        return fail(h, CDGRAB_EINVAL, "%s: a stride below the width, or a misaligned or too long array", who);
    rc = check_apart(h, who, {{"ids", ids, 1, t->rows * 4, t->rows * 4}, {"DY", DY, t->rows, width * size, dy_stride * size}},
                     {{"G", G, t->examples, d * 4, g_stride * 4}});
    if (rc) return rc;
    const OnDevice on(h->device);
    HIP_TRY(h, on.err);
    const TokenRows tok{t->examples, t->rows, t->tokens, t->first, t->count, 0};
    return by_elem(type, [&](auto elem) {
        typedef decltype(elem) T;
        const T *dy = (const T *)DY;
        if (width < 4) return run_embed_grad<T, 1, false>(h, who, tok, vocab, width, ids, dy, dy_stride, scale, G, g_stride);
        if (d > kOnceBytes / 4 / t->examples) return run_embed_grad<T, 4, true>(h, who, tok, vocab, width, ids, dy, dy_stride, scale, G, g_stride);
        return run_embed_grad<T, 4, false>(h, who, tok, vocab, width, ids, dy, dy_stride, scale, G, g_stride);
    });
}

extern "C" int cdgrab_headnorm(cdgrab_handle *h, const cdgrab_token_rows *t, const cdgrab_heads *s, int32_t type, const void *X,
                               int64_t x_stride, const float *gain_q, const float *gain_k, void *Y, int64_t y_stride) {
    if (!h) return CDGRAB_EINVAL;
    static const char *who = "cdgrab_headnorm";
    int rc = check_tokens(h, who, t);
    if (rc || (rc = check_heads(h, who, s, type))) return rc;
    if (t->examples == 0 || t->rows == 0 || t->tokens == 0) return CDGRAB_OK;
    if (!X || !Y) return fail(h, CDGRAB_EINVAL, "%s: null pointer", who);
    const int64_t size = elem_size(type), width = (s->q_heads + s->k_heads) * s->dim;
    if (bad_rows(X, t->rows, width, x_stride, size) || bad_rows(Y, t->rows, width, y_stride, size))
        return fail(h, CDGRAB_EINVAL, "%s: a stride below the width, or a misaligned or too long array", who);
    if ((rc = check_apart(h, who, {{"X", X, t->rows, width * size, x_stride * size}}, {{"Y", Y, t->rows, width * size, y_stride * size}})))
        return rc;
    const OnDevice on(h->device);
    HIP_TRY(h, on.err);
    const TokenRows tok{t->examples, t->rows, t->tokens, t->first, t->count, 0};
    return by_elem(type, [&](auto elem) {
        typedef decltype(elem) T;
        return run_heads<T, false>(h, who, tok, *s, (const T *)X, x_stride, nullptr, 0, gain_q, gain_k, (T *)Y, y_stride, nullptr, 0);
    });
}

extern "C" int cdgrab_pergrad_headnorm(cdgrab_handle *h, const cdgrab_token_rows *t, const cdgrab_heads *s, int32_t type, const void *X,
                                       int64_t x_stride, const void *DY, int64_t dy_stride, const float *gain_q, const float *gain_k,
                                       void *DX, int64_t dx_stride, float *G, int64_t g_stride) {
    if (!h) return CDGRAB_EINVAL;
    static const char *who = "cdgrab_pergrad_headnorm";
    int rc = check_tokens(h, who, t);
    if (rc || (rc = check_heads(h, who, s, type))) return rc;
    if (t->examples == 0) return CDGRAB_OK;
    if (!DX && !G) return fail(h, CDGRAB_EINVAL, "%s: neither DX nor G is wanted", who);
    if (t->rows > 0 && t->tokens > 0 && (!X || !DY)) return fail(h, CDGRAB_EINVAL, "%s: null pointer", who);
    const int64_t size = elem_size(type), width = (s->q_heads + s->k_heads) * s->dim;
    if (bad_rows(X, t->rows, width, x_stride, size) || bad_rows(DY, t->rows, width, dy_stride, size) ||
        (DX && bad_rows(DX, t->rows, width, dx_stride, size)) || (G && bad_rows(G, t->examples, 2 * s->dim, g_stride, 4)))
        return fail(h, CDGRAB_EINVAL, "%s: a stride below the width, or a misaligned or too long array", who);
    rc = check_apart(h, who, {{"X", X, t->rows, width * size, x_stride * size}, {"DY", DY, t->rows, width * size, dy_stride * size}},
                     {{"DX", DX, t->rows, width * size, dx_stride * size}, {"G", G, t->examples, 2 * s->dim * 4, g_stride * 4}});
    if (rc) return rc;
    const OnDevice on(h->device);
    HIP_TRY(h, on.err);
    const TokenRows tok{t->examples, t->rows, t->tokens, t->first, t->count, 0};
    return by_elem(type, [&](auto elem) {
        typedef decltype(elem) T;
        return run_heads<T, true>(h, who, tok, *s, (const T *)X, x_stride, (const T *)DY, dy_stride, gain_q, gain_k, (T *)DX, dx_stride, G,
                                  g_stride);
    });
}

extern "C" int cdgrab_attention(cdgrab_handle *h, const cdgrab_token_rows *t, int64_t q_heads, int64_t kv_heads, int64_t dim, int32_t type,
                                float scale, const void *Q, int64_t q_stride, const void *K, int64_t k_stride, const void *V,
                                int64_t v_stride, void *O, int64_t o_stride, float *lse) {
    if (!h) return CDGRAB_EINVAL;
    static const char *who = "cdgrab_attention";
    int rc = check_attention(h, who, t, q_heads, kv_heads, dim, type, scale);
    if (rc) return rc;
    if (t->examples == 0 || t->rows == 0 || t->tokens == 0) return CDGRAB_OK;
    if (!Q || !K || !V || !O) return fail(h, CDGRAB_EINVAL, "%s: null pointer", who);
    const int64_t size = elem_size(type), qw = q_heads * dim, kw = kv_heads * dim, rows = t->rows;
    if (bad_rows(Q, rows, qw, q_stride, size) || bad_rows(K, rows, kw, k_stride, size) || bad_rows(V, rows, kw, v_stride, size) ||
        bad_rows(O, rows, qw, o_stride, size) || bad_rows(lse, q_heads, rows, rows, 4))
        return fail(h, CDGRAB_EINVAL, "%s: a stride below the width, or a misaligned or too long array", who);
    rc = check_apart(h, who, {{"Q", Q, rows, qw * size, q_stride * size}, {"K", K, rows, kw * size, k_stride * size},
                              {"V", V, rows, kw * size, v_stride * size}},
                     {{"O", O, rows, qw * size, o_stride * size}, {"lse", lse, 1, rows * q_heads * 4, rows * q_heads * 4}});
    if (rc) return rc;
    const OnDevice on(h->device);
    HIP_TRY(h, on.err);
    const TokenRows tok{t->examples, rows, t->tokens, t->first, t->count, 0};
    uint64_t *list = nullptr;
    if (att_list_bytes(tok) && (rc = layer_room(h, who, att_list_bytes(tok) / 8, &list))) return rc;
    make_att_list(h, tok, list);
    return by_elem(type, [&](auto elem) {
        typedef decltype(elem) T;
        return by_head_dim(dim, [&](auto room) { return by_pieces<T>(dim, {{K, k_stride}, {V, v_stride}}, [&](auto direct) {
            by_units(h, tok, q_heads, kv_heads, dim, scale, true, list, [&](const AttHeads &a, dim3 grid) {
                hipLaunchKernelGGL((attention_forward<T, decltype(room)::value, decltype(direct)::value>), grid, dim3(kAttThreads), 0, h->stream, tok, a, (const T *)Q,
                                   q_stride, (const T *)K, k_stride, (const T *)V, v_stride, (T *)O, o_stride, lse);
            });
            HIP_TRY(h, hipGetLastError());
            return (int)CDGRAB_OK;
        }); });
    });
}

extern "C" int cdgrab_attention_backward(cdgrab_handle *h, const cdgrab_token_rows *t, int64_t q_heads, int64_t kv_heads, int64_t dim,
                                         int32_t type, float scale, const void *Q, int64_t q_stride, const void *K, int64_t k_stride,
                                         const void *V, int64_t v_stride, const void *O, int64_t o_stride, const float *lse,
                                         const void *DO, int64_t do_stride, void *DQ, int64_t dq_stride, void *DK, int64_t dk_stride,
                                         void *DV, int64_t dv_stride) {
    if (!h) return CDGRAB_EINVAL;
    static const char *who = "cdgrab_attention_backward";
    int rc = check_attention(h, who, t, q_heads, kv_heads, dim, type, scale);
    if (rc) return rc;
    if (t->examples == 0 || t->rows == 0 || t->tokens == 0) return CDGRAB_OK;
    if (!Q || !K || !V || !O || !lse || !DO || !DQ || !DK || !DV) return fail(h, CDGRAB_EINVAL, "%s: null pointer", who);
    const int64_t size = elem_size(type), qw = q_heads * dim, kw = kv_heads * dim, rows = t->rows;
    if (bad_rows(Q, rows, qw, q_stride, size) || bad_rows(K, rows, kw, k_stride, size) || bad_rows(V, rows, kw, v_stride, size) ||
        bad_rows(O, rows, qw, o_stride, size) || bad_rows(DO, rows, qw, do_stride, size) || bad_rows(lse, q_heads, rows, rows, 4) ||
        bad_rows(DQ, rows, qw, dq_stride, size) || bad_rows(DK, rows, kw, dk_stride, size) || bad_rows(DV, rows, kw, dv_stride, size))
        return fail(h, CDGRAB_EINVAL, "%s: a stride below the width, or a misaligned or too long array", who);
    rc = check_apart(h, who, {{"Q", Q, rows, qw * size, q_stride * size}, {"K", K, rows, kw * size, k_stride * size},
                              {"V", V, rows, kw * size, v_stride * size}, {"O", O, rows, qw * size, o_stride * size},
                              {"DO", DO, rows, qw * size, do_stride * size}, {"lse", lse, 1, rows * q_heads * 4, rows * q_heads * 4}},
                     {{"DQ", DQ, rows, qw * size, dq_stride * size}, {"DK", DK, rows, kw * size, dk_stride * size},
                      {"DV", DV, rows, kw * size, dv_stride * size}});
    if (rc) return rc;
    const OnDevice on(h->device);
    HIP_TRY(h, on.err);
    const TokenRows tok{t->examples, rows, t->tokens, t->first, t->count, 0};
    char *ws = nullptr;
    if ((rc = layer_room(h, who, att_list_bytes(tok) + rows * q_heads * 4, &ws))) return rc;
    uint64_t *const list = reinterpret_cast<uint64_t *>(ws);
    float *const delta = reinterpret_cast<float *>(ws + att_list_bytes(tok));
    make_att_list(h, tok, list);
    return by_elem(type, [&](auto elem) {
        typedef decltype(elem) T;
        return by_head_dim(dim, [&](auto room) {
            constexpr int D = decltype(room)::value;
            by_pieces<T>(dim, {{K, k_stride}, {V, v_stride}}, [&](auto direct) {
                by_units(h, tok, q_heads, kv_heads, dim, scale, true, list, [&](const AttHeads &a, dim3 grid) {
                    hipLaunchKernelGGL((attention_backward_q<T, D, decltype(direct)::value>), grid, dim3(kAttThreads), 0, h->stream, tok, a,
                                       (const T *)Q, q_stride, (const T *)K, k_stride, (const T *)V, v_stride, (const T *)O, o_stride, lse,
                                       (const T *)DO, do_stride, (T *)DQ, dq_stride, delta);
                });
                return 0;
            });
            by_pieces<T>(dim, {{Q, q_stride}, {DO, do_stride}}, [&](auto direct) {
                by_units(h, tok, q_heads, kv_heads, dim, scale, false, list, [&](const AttHeads &a, dim3 grid) {
                    hipLaunchKernelGGL((attention_backward_kv<T, D, decltype(direct)::value>), grid, dim3(kAttThreads), 0, h->stream, tok, a,
                                       (const T *)Q, q_stride, (const T *)K, k_stride, (const T *)V, v_stride, lse, (const T *)DO, do_stride,
                                       delta, (T *)DK, dk_stride, (T *)DV, dv_stride);
                });
                return 0;
            });
            HIP_TRY(h, hipGetLastError());
            return (int)CDGRAB_OK;
        });
    });
}
