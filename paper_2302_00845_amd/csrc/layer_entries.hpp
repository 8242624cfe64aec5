// Host side of the layer operators: argument checks, choice of the kernel, launches.  Included by cdgrab.hip.
#pragma once

namespace {

constexpr int64_t kMaxGroups = (int64_t)1 << 22;  // workgroups per launch (a grid dimension holds fewer than 2^32 threads)

// Workspace of the layer operators.  What a recorded call has used is kept until the handle goes, also when a larger
// buffer takes its place: the recording holds its address.  A recorded call allocates nothing.
template <typename T>
int layer_room(cdgrab_handle *h, const char *who, int64_t want, T **out) {
    const int64_t bytes = want * (int64_t)sizeof(T);
    const bool recorded = capturing(h);
    if (h->layer_ws_cap < bytes) {
        if (recorded)
            return fail(h, CDGRAB_ENOMEM, "%s: needs %lld bytes of workspace, and none can be allocated while the stream is "
                        "captured: make the call once before", who, (long long)bytes);
        if (h->layer_ws && h->layer_ws_in_graphs) {
            try {
                h->layer_kept.push_back(h->layer_ws);
            } catch (...) {
                return fail(h, CDGRAB_ENOMEM, "%s: out of host memory", who);
            }
            h->layer_ws = nullptr;
            h->layer_ws_cap = 0;
            h->layer_ws_in_graphs = false;
        }
        const int rc = ensure(h, h->layer_ws, h->layer_ws_cap, bytes);
        if (rc) return rc;
    }
    if (recorded) h->layer_ws_in_graphs = true;
    *out = reinterpret_cast<T *>(h->layer_ws);
    return CDGRAB_OK;
}

// The handle's device for the length of a call.
struct OnDevice {
    int before = -1;
    hipError_t err;
    explicit OnDevice(int device) {
        err = hipGetDevice(&before);
        if (err == hipSuccess && before != device) err = hipSetDevice(device);
        else before = -1;
    }
    ~OnDevice() { if (before >= 0) (void)hipSetDevice(before); }
};

int64_t elem_size(int32_t type) { return type == CDGRAB_F32 ? 4 : 2; }

// Do na rows of wa bytes from a, sa bytes apart, and nb rows from b share a byte?  (Of unequal strides: could they?)
bool rows_overlap(const void *a, int64_t na, int64_t wa, int64_t sa, const void *b, int64_t nb, int64_t wb, int64_t sb) {
    if (!a || !b || na < 1 || nb < 1) return false;
    if (!ranges_overlap(a, (na - 1) * sa + wa, b, (nb - 1) * sb + wb)) return false;
    if (sa != sb || na == 1 || nb == 1) return true;
    const int64_t off = (int64_t)(reinterpret_cast<intptr_t>(b) - reinterpret_cast<intptr_t>(a)), at = ((off % sa) + sa) % sa;
    return at < wa || at + wb > sa;
}

bool bad_type(int32_t type) { return type != CDGRAB_F32 && type != CDGRAB_BF16 && type != CDGRAB_F16; }

// An array of rows: a size, a stride of at least the width, addresses that 64 bits hold, elements at element addresses.
bool bad_rows(const void *p, int64_t rows, int64_t width, int64_t stride, int64_t size) {
    return stride < width || reinterpret_cast<uintptr_t>(p) % (uintptr_t)size != 0 ||
           (rows > 0 && stride > (INT64_MAX >> 4) / rows);
}

int check_tokens(cdgrab_handle *h, const char *who, const cdgrab_token_rows *t) {
    if (!t) return fail(h, CDGRAB_EINVAL, "%s: the examples' rows are NULL", who);
    if (t->examples < 0 || t->rows < 0 || t->tokens < 0 || t->examples > ((int64_t)1 << 40) || t->tokens > ((int64_t)1 << 40) ||
        t->rows > ((int64_t)1 << 40))
        return fail(h, CDGRAB_EINVAL, "%s: bad sizes examples=%lld rows=%lld tokens=%lld", who, (long long)t->examples,
                    (long long)t->rows, (long long)t->tokens);
    if (!t->first && t->tokens > 0 && t->examples > t->rows / t->tokens)
        return fail(h, CDGRAB_EINVAL, "%s: %lld examples of %lld rows each do not fit in %lld rows", who, (long long)t->examples,
                    (long long)t->tokens, (long long)t->rows);
    return CDGRAB_OK;
}

// f(threads per row, groups of VEC per thread): the fewest threads that hold the row in few groups.
template <int VEC, typename F>
void by_norm_shape(int64_t width, F &&f) {
    const int64_t groups = (width + VEC - 1) / VEC;
    const auto go = [&](auto lanes, auto k) { f(lanes, k); };
#define NORM_SHAPE(L, K) go(std::integral_constant<int, L>{}, std::integral_constant<int, K>{})
    if constexpr (VEC == 1) {
        NORM_SHAPE(8, 1);
    } else {
        if (groups <= 8) NORM_SHAPE(8, 1);
        else if (groups <= 16) NORM_SHAPE(16, 1);
        else if (groups <= 32) NORM_SHAPE(32, 1);
        else if (groups <= 64) NORM_SHAPE(64, 1);
        else if (groups <= 128) NORM_SHAPE(64, 2);
        else if (groups <= 192) NORM_SHAPE(64, 3);
        else if (groups <= 256) NORM_SHAPE(64, 4);
        else if (groups <= 512) NORM_SHAPE(256, 2);
        else if (groups <= 768) NORM_SHAPE(256, 3);
        else if (groups <= 1024) NORM_SHAPE(256, 4);
        else if (groups <= 2048) NORM_SHAPE(1024, 2);
        else if constexpr (VEC == 4) {
            if (groups <= 3 * 1024) NORM_SHAPE(1024, 3);
            else NORM_SHAPE(1024, 4);
        }
    }
#undef NORM_SHAPE
}

// f(element type, elements per access)
template <typename F>
void by_norm_type(int32_t type, int64_t width, F &&f) {
    const auto pick = [&](auto elem) {
        typedef decltype(elem) T;
        constexpr int VEC = 16 / (int)sizeof(T);
        if (width < VEC) f(elem, std::integral_constant<int, 1>{});
        else f(elem, std::integral_constant<int, VEC>{});
    };
    if (type == CDGRAB_F32) pick(float{});
    else if (type == CDGRAB_BF16) pick(bf16_t{});
    else pick(f16_t{});
}

template <typename T, int BM, int BN, int WM, int WN>
int run_linear(cdgrab_handle *h, const TokenRows &tok, const T *X, int64_t x_stride, const T *D, int64_t d_stride, int64_t in_dim,
               int64_t out_dim, int with_bias, float *G, int64_t g_stride) {
    const int64_t tiles = ((in_dim + BM - 1) / BM) * ((out_dim + BN - 1) / BN);
    const int64_t d = (in_dim + with_bias) * out_dim;
    // few tiles and many tokens: shares of the tokens, of at least eight steps of the kernel, until the chip is full
    const int64_t fill = 2 * (int64_t)h->num_cu;
    const int64_t most = std::max<int64_t>(1, tok.tokens / (8 * LinearPlanes<T>::KC));
    int64_t shares = tok.examples * tiles >= fill ? 1 : std::min(most, (fill + tok.examples * tiles - 1) / (tok.examples * tiles));
    float *parts = nullptr;
    if (shares > 1) {
        const int rc = layer_room(h, "cdgrab_pergrad_linear", shares * tok.examples * d, &parts);
        if (rc) return rc;
    }
    const int64_t per = std::max<int64_t>(1, kMaxGroups / (tiles * shares));  // examples per launch
    for (int64_t e0 = 0; e0 < tok.examples; e0 += per) {
        const int64_t n = std::min(per, tok.examples - e0);
        TokenRows part = tok;
        part.examples = n;
        part.base = e0;
        hipLaunchKernelGGL((linear_grad<T, BM, BN, WM, WN>), dim3((unsigned)(n * tiles * shares)), dim3(kLinearThreads), 0, h->stream,
                           part, (int)shares, X, x_stride, D, d_stride, (int)in_dim, (int)out_dim, with_bias,
                           shares > 1 ? parts : G, shares > 1 ? d : g_stride, tok.examples * d);
    }
    if (shares > 1)
        hipLaunchKernelGGL(linear_grad_finish, dim3((unsigned)((d + 255) / 256), (unsigned)std::min<int64_t>(tok.examples, 1024)),
                           dim3(256), 0, h->stream, parts, (int)shares, tok.examples * d, tok.examples, d, G, g_stride);
    HIP_TRY(h, hipGetLastError());
    return CDGRAB_OK;
}

}  // namespace

extern "C" int cdgrab_layernorm(cdgrab_handle *h, int64_t rows, int64_t width, int32_t type, const void *X, int64_t x_stride,
                                const float *gain, const float *bias, float eps, void *Y, int64_t y_stride) {
    if (!h) return CDGRAB_EINVAL;
    static const char *who = "cdgrab_layernorm";
    if (rows < 0 || rows > ((int64_t)1 << 40) || width < 1 || width > kNormMaxWidth || bad_type(type) || !(eps >= 0.f))
        return fail(h, CDGRAB_EINVAL, "%s: bad arguments rows=%lld width=%lld (1 .. %lld) type=%d eps=%g", who, (long long)rows,
                    (long long)width, (long long)kNormMaxWidth, (int)type, (double)eps);
    if (rows == 0) return CDGRAB_OK;
    if (!X || !Y) return fail(h, CDGRAB_EINVAL, "%s: null pointer", who);
    const int64_t size = elem_size(type);
    if (bad_rows(X, rows, width, x_stride, size) || bad_rows(Y, rows, width, y_stride, size))
        return fail(h, CDGRAB_EINVAL, "%s: a stride below the width, or a misaligned or too long array", who);
    if (rows_overlap(X, rows, width * size, x_stride * size, Y, rows, width * size, y_stride * size))
        return fail(h, CDGRAB_EINVAL, "%s: X and Y must not overlap", who);
    const OnDevice on(h->device);
    HIP_TRY(h, on.err);
    by_norm_type(type, width, [&](auto elem, auto vec) {
        typedef decltype(elem) T;
        constexpr int VEC = decltype(vec)::value;
        by_norm_shape<VEC>(width, [&](auto lanes, auto k) {
            constexpr int LANES = decltype(lanes)::value, K = decltype(k)::value;
            constexpr int THREADS = LANES > kNormThreads ? LANES : kNormThreads, PER = THREADS / LANES;
            const int64_t groups = std::min<int64_t>((rows + PER - 1) / PER, (int64_t)h->num_cu * (2048 / THREADS));
            hipLaunchKernelGGL((norm_forward<T, VEC, LANES, K>), dim3((unsigned)groups), dim3(THREADS), 0, h->stream,
                               (const T *)X, x_stride, gain, bias, (T *)Y, y_stride, rows, (int)width, eps);
        });
    });
    HIP_TRY(h, hipGetLastError());
    return CDGRAB_OK;
}

extern "C" int cdgrab_pergrad_layernorm(cdgrab_handle *h, const cdgrab_token_rows *t, int64_t width, int32_t type, const void *X,
                                        int64_t x_stride, const void *DY, int64_t dy_stride, const float *gain, float eps, void *DX,
                                        int64_t dx_stride, int32_t with_bias, float *G, int64_t g_stride) {
    if (!h) return CDGRAB_EINVAL;
    static const char *who = "cdgrab_pergrad_layernorm";
    int rc = check_tokens(h, who, t);
    if (rc) return rc;
    if (width < 1 || width > kNormMaxWidth || bad_type(type) || !(eps >= 0.f) || (with_bias != 0 && with_bias != 1))
        return fail(h, CDGRAB_EINVAL, "%s: bad arguments width=%lld (1 .. %lld) type=%d eps=%g with_bias=%d", who, (long long)width,
                    (long long)kNormMaxWidth, (int)type, (double)eps, (int)with_bias);
    const int64_t size = elem_size(type), cols = width * (1 + with_bias);
    if (t->examples == 0) return CDGRAB_OK;
    if (!DX && !G) return fail(h, CDGRAB_EINVAL, "%s: neither DX nor G is wanted", who);
    if (t->rows > 0 && t->tokens > 0 && (!X || !DY)) return fail(h, CDGRAB_EINVAL, "%s: null pointer", who);
    if (bad_rows(X, t->rows, width, x_stride, size) || bad_rows(DY, t->rows, width, dy_stride, size) ||
        (DX && bad_rows(DX, t->rows, width, dx_stride, size)) || (G && bad_rows(G, t->examples, cols, g_stride, 4)))
        return fail(h, CDGRAB_EINVAL, "%s: a stride below the width, or a misaligned or too long array", who);
    if (DX && (rows_overlap(X, t->rows, width * size, x_stride * size, DX, t->rows, width * size, dx_stride * size) ||
               rows_overlap(DY, t->rows, width * size, dy_stride * size, DX, t->rows, width * size, dx_stride * size)))
        return fail(h, CDGRAB_EINVAL, "%s: DX must not overlap X or DY", who);
    if (G && (rows_overlap(X, t->rows, width * size, x_stride * size, G, t->examples, cols * 4, g_stride * 4) ||
              rows_overlap(DY, t->rows, width * size, dy_stride * size, G, t->examples, cols * 4, g_stride * 4) ||
              (DX && rows_overlap(DX, t->rows, width * size, dx_stride * size, G, t->examples, cols * 4, g_stride * 4))))
        return fail(h, CDGRAB_EINVAL, "%s: G must not overlap X, DY or DX", who);
    const OnDevice on(h->device);
    HIP_TRY(h, on.err);
    const TokenRows tok{t->examples, t->rows, t->tokens, t->first, t->count, 0};
    rc = CDGRAB_OK;
    by_norm_type(type, width, [&](auto elem, auto vec) {
        typedef decltype(elem) T;
        constexpr int VEC = decltype(vec)::value;
        by_norm_shape<VEC>(width, [&](auto lanes, auto k) {
            constexpr int LANES = decltype(lanes)::value, K = decltype(k)::value;
            constexpr int THREADS = LANES > kNormThreads ? LANES : kNormThreads, PER = THREADS / LANES;
            // an example's rows in chunks until the chip is full, of eight rows per group of threads at least
            const int64_t fill = (int64_t)h->num_cu * (2048 / THREADS);
            const int64_t most = std::max<int64_t>(1, tok.tokens / (8 * PER));
            const int64_t chunks = std::min(most, std::max<int64_t>(1, (fill + tok.examples - 1) / tok.examples));
            float *partial = nullptr;
            if (G && chunks > 1 && (rc = layer_room(h, who, tok.examples * chunks * cols, &partial))) return;
            const int64_t per = std::max<int64_t>(1, kMaxGroups / chunks);  // examples per launch
            for (int64_t e0 = 0; e0 < tok.examples; e0 += per) {
                TokenRows part = tok;
                part.examples = std::min(per, tok.examples - e0);
                part.base = e0;
                hipLaunchKernelGGL((norm_backward<T, VEC, LANES, K>), dim3((unsigned)(part.examples * chunks)), dim3(THREADS), 0,
                                   h->stream, part, (int)chunks, (const T *)X, x_stride, (const T *)DY, dy_stride, gain, (T *)DX,
                                   dx_stride, G, g_stride, (int)with_bias, partial, (int)width, eps);
            }
            if (partial) {
                const int64_t groups = (cols + 31) / 32;
                const int64_t most_e = std::max<int64_t>(1, kMaxGroups / groups);
                for (int64_t e0 = 0; e0 < tok.examples; e0 += most_e)
                    hipLaunchKernelGGL(norm_grad_finish, dim3((unsigned)(std::min(most_e, tok.examples - e0) * groups)), dim3(256), 0,
                                       h->stream, partial + e0 * chunks * cols, (int)chunks, (int)cols, G + e0 * g_stride, g_stride);
            }
        });
    });
    if (rc) return rc;
    HIP_TRY(h, hipGetLastError());
    return CDGRAB_OK;
}

extern "C" int cdgrab_pergrad_linear(cdgrab_handle *h, const cdgrab_token_rows *t, int64_t in_dim, int64_t out_dim, int32_t type,
                                     const void *X, int64_t x_stride, const void *D, int64_t d_stride, int32_t with_bias, float *G,
                                     int64_t g_stride) {
    if (!h) return CDGRAB_EINVAL;
    static const char *who = "cdgrab_pergrad_linear";
    const int rc = check_tokens(h, who, t);
    if (rc) return rc;
    if (in_dim < 1 || out_dim < 1 || in_dim > (1 << 20) || out_dim > (1 << 20) || bad_type(type) || (with_bias != 0 && with_bias != 1))
        return fail(h, CDGRAB_EINVAL, "%s: bad arguments in_dim=%lld out_dim=%lld (1 .. 2^20) type=%d with_bias=%d", who,
                    (long long)in_dim, (long long)out_dim, (int)type, (int)with_bias);
    const int64_t size = elem_size(type), d = (in_dim + with_bias) * out_dim;
    if (t->examples == 0) return CDGRAB_OK;
    if (!G || (t->rows > 0 && t->tokens > 0 && (!X || !D))) return fail(h, CDGRAB_EINVAL, "%s: null pointer", who);
    if (bad_rows(X, t->rows, in_dim, x_stride, size) || bad_rows(D, t->rows, out_dim, d_stride, size) ||
        bad_rows(G, t->examples, d, g_stride, 4))
        return fail(h, CDGRAB_EINVAL, "%s: a stride below the width, or a misaligned or too long array", who);
    if (rows_overlap(X, t->rows, in_dim * size, x_stride * size, G, t->examples, d * 4, g_stride * 4) ||
        rows_overlap(D, t->rows, out_dim * size, d_stride * size, G, t->examples, d * 4, g_stride * 4))
        return fail(h, CDGRAB_EINVAL, "%s: G must not overlap X or D", who);
    const OnDevice on(h->device);
    HIP_TRY(h, on.err);
    const TokenRows tok{t->examples, t->rows, t->tokens, t->first, t->count, 0};
    const auto by_type = [&](auto elem) {
        typedef decltype(elem) T;
        const T *x = (const T *)X, *dl = (const T *)D;
        const auto tiles = [&](int64_t bm, int64_t bn) { return ((in_dim + bm - 1) / bm) * ((out_dim + bn - 1) / bn) * tok.examples; };
        if (out_dim <= 32)
            return run_linear<T, 128, 32, 4, 1>(h, tok, x, x_stride, dl, d_stride, in_dim, out_dim, with_bias, G, g_stride);
        if (in_dim <= 32)
            return run_linear<T, 32, 128, 1, 4>(h, tok, x, x_stride, dl, d_stride, in_dim, out_dim, with_bias, G, g_stride);
        if (in_dim <= 64 || out_dim <= 64 || tiles(128, 128) < h->num_cu)
            return run_linear<T, 64, 64, 2, 2>(h, tok, x, x_stride, dl, d_stride, in_dim, out_dim, with_bias, G, g_stride);
        return run_linear<T, 128, 128, 2, 2>(h, tok, x, x_stride, dl, d_stride, in_dim, out_dim, with_bias, G, g_stride);
    };
    if (type == CDGRAB_F32) return by_type(float{});
    return type == CDGRAB_BF16 ? by_type(bf16_t{}) : by_type(f16_t{});
}
