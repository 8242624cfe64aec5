// Host side of the layer operators: argument checks, choice of the kernel, launches.  Included by cdgrab.hip.
#pragma once

namespace {

constexpr int64_t kOrthoSmallLds = 152 * 1024, kOrthoSmallLdsHalf = 76 * 1024;  // of a matrix that one workgroup holds
constexpr int64_t kOrthoBytes = (int64_t)4 << 30;            // workspace of the products' form: as many matrices at a time
constexpr int64_t kOrthoMaxShort = 16384;
constexpr int64_t kOrthoMaxSide = (int64_t)1 << 20;
constexpr int64_t kMaxGroups = (int64_t)1 << 21;  // workgroups per launch, of up to 1024 threads (a grid dimension holds fewer than 2^32)
constexpr int64_t kMaxCells = (int64_t)1 << 32;   // elements of a matrix, of a gradient row: 2^22 workgroups of 256 threads at the most

// Workspace of the layer operators.  A recorded call allocates nothing.
template <typename T>
int layer_room(cdgrab_handle *h, const char *who, int64_t want, T **out) {
    const int64_t bytes = want * (int64_t)sizeof(T);
    const bool recorded = capturing(h);
    if (recorded && h->layer_ws_cap < bytes)
        return fail(h, CDGRAB_ENOMEM, "%s: needs %lld bytes of workspace, and none can be allocated while the stream is "
                    "captured: make the call once before", who, (long long)bytes);
    if (recorded) h->recorded = true;
    const int rc = ensure(h, h->layer_ws, h->layer_ws_cap, bytes);
    if (rc) return rc;
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

// Do na rows of wa bytes from a, sa bytes apart, and nb rows from b share a byte?  (Of unequal strides: could they?  A single row
// has the other array's.)
bool rows_overlap(const void *a, int64_t na, int64_t wa, int64_t sa, const void *b, int64_t nb, int64_t wb, int64_t sb) {
    if (!a || !b || na < 1 || nb < 1) return false;
    if (!ranges_overlap(a, (na - 1) * sa + wa, b, (nb - 1) * sb + wb)) return false;
    if (na == 1) sa = sb;
    if (nb == 1) sb = sa;
    if (sa != sb || (na == 1 && nb == 1)) return true;
    const int64_t off = (int64_t)(reinterpret_cast<intptr_t>(b) - reinterpret_cast<intptr_t>(a)), at = ((off % sa) + sa) % sa;
    return at < wa || at + wb > sa;
}

// The same of `batch` matrices of rows x width bytes each, s bytes from row to row and t from matrix to matrix: they share nothing if
// their stretches do not, taken as rows, or if all their rows lie at whole multiples of s and these do not.
bool matrices_overlap(int64_t batch, int64_t rows, int64_t width, const void *a, int64_t sa, int64_t ta, const void *b, int64_t sb,
                      int64_t tb) {
    const int64_t la = (rows - 1) * sa + width, lb = (rows - 1) * sb + width;  // of a matrix
    if (!rows_overlap(a, batch, la, ta, b, batch, lb, tb)) return false;
    if (batch == 1) return rows_overlap(a, rows, width, sa, b, rows, width, sb);
    if (rows == 1 || ta % sa != 0 || tb % sb != 0) return true;
    return rows_overlap(a, (batch - 1) * (ta / sa) + rows, width, sa, b, (batch - 1) * (tb / sb) + rows, width, sb);
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

// Rows that the caches do not hold anyway are read past them, if their pieces are whole (a line that two rows share would be read
// twice).  65 536 rows of 768 fp32: forward 79 -> 66 us, backward 127 -> 106; in bf16 47 and 79 -> 77; 51 400 rows of 515 fp16,
// which are not, forward 35 -> 43.
bool norm_once(int64_t rows, int64_t width, int64_t size, const void *p, int64_t stride) {
    return rows * width * size >= ((int64_t)64 << 20) && reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * size % 16 == 0;
}

// f(threads per row, groups of VEC per thread): the fewest threads that hold the row in few groups.  The backward pass, which has
// two reductions and twice the arithmetic per row, takes narrower ones where its rows then fill them: two rows of 768 bf16 a
// wavefront instead of one 74 -> 68 us (65 536 rows), the forward pass 45 -> 59.
template <int VEC, bool BACKWARD, typename F>
void by_norm_shape(int64_t width, F &&f) {
    const int64_t groups = (width + VEC - 1) / VEC;
    const auto go = [&](auto lanes, auto k) { f(lanes, k); };
#define NORM_SHAPE(L, K) go(std::integral_constant<int, L>{}, std::integral_constant<int, K>{})
    if constexpr (VEC == 1) {
        NORM_SHAPE(8, 1);
    } else {
        constexpr int HALF = BACKWARD ? 2 : 1;
        if (groups <= 8) NORM_SHAPE(8, 1);
        else if (groups <= 16) NORM_SHAPE(16, 1);
        else if (groups <= 32) NORM_SHAPE(32 / HALF, HALF);
        else if (groups <= 64) NORM_SHAPE(64 / HALF, HALF);
        else if (groups <= 96 && BACKWARD) NORM_SHAPE(32, 3);
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

// Stores of four elements until they start at the same column again.
int64_t flat_period(int64_t out_dim) { return out_dim / std::gcd<int64_t>(out_dim, 4); }

// Floats of LDS that a stretch of linear_flat needs at most.
int64_t flat_lds(int64_t tok, int64_t in_dim, int64_t out_dim, int64_t with_bias) {
    return tok * (std::min<int64_t>(in_dim + with_bias, (kFlatElems + out_dim - 1) / out_dim + 1) + 1 + out_dim);
}

template <typename T, int TOK, int THREADS>
int run_flat(cdgrab_handle *h, const TokenRows &tok, const T *X, int64_t x_stride, const T *D, int64_t d_stride, int64_t in_dim,
             int64_t out_dim, int with_bias, float *G, int64_t g_stride) {
    const int64_t d = (in_dim + with_bias) * out_dim, units = (d + 3 + kFlatElems - 1) / kFlatElems;
    const int64_t per = std::max<int64_t>(1, kMaxGroups / units);
    // threads whose stores of four elements make whole rows
    const int period = (int)flat_period(out_dim), active = THREADS / period * period;
    const auto launch = [&](auto kernel) {
        for (int64_t e0 = 0; e0 < tok.examples; e0 += per) {
            TokenRows part = tok;
            part.examples = std::min(per, tok.examples - e0);
            part.base = e0;
            hipLaunchKernelGGL(kernel, dim3((unsigned)(part.examples * units)), dim3(THREADS),
                               (size_t)flat_lds(TOK, in_dim, out_dim, with_bias) * sizeof(float), h->stream, part, (uint32_t)units, X, x_stride,
                               D, d_stride, (int)in_dim, (int)out_dim, with_bias, active, G, g_stride);
        }
    };
    if (out_dim < 4) launch(linear_flat<T, TOK, THREADS, true>);
    else launch(linear_flat<T, TOK, THREADS, false>);
    HIP_TRY(h, hipGetLastError());
    return CDGRAB_OK;
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
    // Neighbouring tiles along G's rows write whole lines between them (200 examples of one token, 768 -> 2304: 319 -> 267 us); along
    // the side of fewer tiles they read less, which counts with many tokens (32 of 1024: 236 -> 212).
    const int down = tok.tokens >= 512 && in_dim < out_dim;
    const int64_t per = std::max<int64_t>(1, kMaxGroups / (tiles * shares));  // examples per launch
    for (int64_t e0 = 0; e0 < tok.examples; e0 += per) {
        const int64_t n = std::min(per, tok.examples - e0);
        TokenRows part = tok;
        part.examples = n;
        part.base = e0;
        hipLaunchKernelGGL((linear_grad<T, BM, BN, WM, WN>), dim3((unsigned)(n * tiles * shares)), dim3(kLinearThreads), 0, h->stream,
                           part, (int)shares, X, x_stride, D, d_stride, (int)in_dim, (int)out_dim, with_bias, down,
                           shares > 1 ? parts : G, shares > 1 ? d : g_stride, tok.examples * d);
    }
    if (shares > 1)
        hipLaunchKernelGGL(linear_grad_finish, dim3((unsigned)((d + 255) / 256), (unsigned)std::min<int64_t>(tok.examples, 1024)),
                           dim3(256), 0, h->stream, parts, (int)shares, tok.examples * d, tok.examples, d, G, g_stride);
    HIP_TRY(h, hipGetLastError());
    return CDGRAB_OK;
}

// The largest singular value that the steps can make of values up to 1: they are refused beyond what the kernels' scales
// have room for (X up to 3.5, the factor b A + c A^2 up to 30).  With l = s^2 a step takes s to s (a + b l + c l^2); both that
// and the factor are largest at an end of 0 .. most^2 or where their slopes are zero.
bool ortho_in_range(int64_t steps, const OrthoCoeffs &c, double *largest) {
    *largest = 1.0001;
    if (!std::isfinite(c.a) || !std::isfinite(c.b) || !std::isfinite(c.c)) return false;
    double most = 1.0001;
    for (int64_t s = 0; s < steps; ++s) {
        const double end = most * most;
        double at[4] = {end, end, end, end};
        const double square = 9.0 * c.b * c.b - 20.0 * c.a * c.c;
        if (c.c != 0.0) {
            at[0] = -c.b / (2.0 * c.c);
            if (square >= 0.0) {
                at[1] = (-3.0 * c.b + std::sqrt(square)) / (10.0 * c.c);
                at[2] = (-3.0 * c.b - std::sqrt(square)) / (10.0 * c.c);
            }
        } else if (c.b != 0.0) {
            at[1] = -c.a / (3.0 * c.b);
        }
        double next = 0.0;
        for (double l : at) {
            l = std::max(0.0, std::min(l, end));
            const double factor = c.b * l + c.c * l * l, y = std::abs(std::sqrt(l) * (c.a + factor));
            if (!(std::abs(factor) <= 30.0 && y <= 3.5)) return false;
            next = std::max(next, y);
        }
        most = 1.001 * next;
        *largest = std::max(*largest, most);
    }
    return most <= 3.51;
}

// Steps that one Gram matrix serves.  A step takes an eigenvalue l of it to l q(l)^2, q = a + b l + c l^2, and what rounding has added
// to the matrix grows by the slope of that, q (a + 3 b l + 5 c l^2), at the most: 2^-52 of the trace stays below 2^-12, which is little
// beside 1, where the polynomial's range ends.  (Default coefficients: a^2 = 11.9 at l = 0, eleven steps; matrices that lack rank,
// and with singular values down to 1e-4 .. 1e-9, are then off by 5e-6 at the most, where products in fp32 are by 5e-3 .. 3e-2.  Of
// 15/8, -10/8, 3/8 it is 22 steps, and 8e-6.  Simulated further: twelve steps 1e-5, fourteen 1e-3, sixteen diverge.)  A further
// stretch costs what the first one did: 785 x 10, 5 / 7 / 12 / 20 steps 13 / 14 / 33 / 37 us.
int64_t ortho_gram_steps(const OrthoCoeffs &c, double largest) {
    double slope = 1.0;
    for (int q = 0; q <= 64; ++q) {
        const double l = largest * largest * q / 64;
        slope = std::max(slope, std::abs((c.a + c.b * l + c.c * l * l) * (c.a + 3.0 * c.b * l + 5.0 * c.c * l * l)));
    }
    return slope > 1.25 ? std::max<int64_t>(1, (int64_t)(40.0 / std::log2(slope))) : 64;
}

// `chunks` of `per` columns with their sums in `parts`; none: one workgroup per matrix.
template <int NT, typename T>
void launch_ortho_narrow(cdgrab_handle *h, int64_t batch, const OrthoIo<T> &io, int64_t steps, int first, const OrthoCoeffs &c, int chunks,
                         int64_t per, double *parts) {
    if (!parts) {
        hipLaunchKernelGGL((ortho_narrow<NT, T>), dim3((unsigned)batch), dim3(kOrthoThreads), 0, h->stream, io, (int)steps, first, c);
        return;
    }
    double *P = parts + batch * chunks * NT * NT * 256;
    hipLaunchKernelGGL((ortho_narrow_gram<NT, T>), dim3((unsigned)(batch * chunks)), dim3(kOrthoThreads), 0, h->stream, io, chunks, per, parts);
    hipLaunchKernelGGL((ortho_narrow_chain<NT>), dim3((unsigned)batch), dim3(kOrthoThreads), 0, h->stream, io.short_side, chunks, parts,
                       (int)steps, first, c, P);
    hipLaunchKernelGGL((ortho_narrow_apply<NT, T>), dim3((unsigned)(batch * chunks)), dim3(kOrthoThreads), 0, h->stream, io, chunks, per, P);
}

template <int NT, typename T>
int run_ortho_narrow(cdgrab_handle *h, const char *who, int64_t batch, const OrthoIo<T> &io, int64_t steps, const OrthoCoeffs &c,
                     bool launch) {
    // one workgroup per matrix while a matrix is short or there are enough of them (us of one launch -> three: 12 x 4000 46 -> 27, 30 x
    // 1000 37 -> 27, 64 x 512 111 -> 73)
    const bool whole = io.long_side <= 1024 / (NT * NT) * 2 || batch >= h->num_cu;
    const int64_t fill = whole ? 1 : std::min<int64_t>(std::max<int64_t>(1, h->num_cu / batch), 128);
    const int64_t per = round_up((io.long_side + fill - 1) / fill, 256);
    const int chunks = whole ? 0 : (int)((io.long_side + per - 1) / per);
    // steps in stretches, of one Gram matrix each, with X in between
    const int64_t stretches = std::max<int64_t>(1, (steps + c.per_gram - 1) / c.per_gram), cells = (int64_t)io.short_side * io.long_side;
    const int64_t x_len = stretches > 1 ? batch * cells : 0, parts_len = whole ? 0 : batch * (chunks + 1) * NT * NT * 256;
    double *X = nullptr;
    if (x_len + parts_len > 0) {
        const int rc = layer_room(h, who, x_len + parts_len, &X);
        if (rc) return rc;
    }
    if (!launch) return CDGRAB_OK;
    double *const parts = whole ? nullptr : X + x_len;
    if (stretches == 1) {
        launch_ortho_narrow<NT>(h, batch, io, steps, 1, c, chunks, per, parts);
    } else {
        const bool turn = io.m_i < io.m_j;
        const int64_t x_i = turn ? 1 : io.long_side, x_j = turn ? io.short_side : 1;
        const OrthoIo<double> between{X, X, nullptr, 0.f, x_i, x_j, cells, x_i, x_j, cells, io.short_side, io.long_side};
        const uint32_t groups = (uint32_t)std::min((cells + 1023) / 1024, std::max<int64_t>(1, kMaxGroups / batch));
        hipLaunchKernelGGL((ortho_doubles<T, false>), dim3((unsigned)(batch * groups)), dim3(256), 0, h->stream, io, groups, X);
        for (int64_t s = 0; s < stretches; ++s)
            launch_ortho_narrow<NT>(h, batch, between, steps * (s + 1) / stretches - steps * s / stretches, s == 0, c, chunks, per, parts);
        hipLaunchKernelGGL((ortho_doubles<T, true>), dim3((unsigned)(batch * groups)), dim3(256), 0, h->stream, io, groups, X);
    }
    HIP_TRY(h, hipGetLastError());
    return CDGRAB_OK;
}

template <int TILE, typename T>
int run_ortho_products(cdgrab_handle *h, const char *who, int64_t batch, OrthoIo<T> io, int64_t steps, const OrthoCoeffs &c, bool launch) {
    const int64_t sp = round_up(io.short_side, TILE), lp = round_up(io.long_side, TILE);
    const int64_t x_len = 2 * sp * lp, a_len = 2 * sp * sp, per_matrix = 2 * x_len + 2 * a_len + kOrthoSums * 4;  // fp16 elements
    const int64_t tm = sp / TILE, tn = lp / TILE;
    const int64_t most = std::max<int64_t>(1, std::min(kOrthoBytes / 2 / per_matrix,
                                                       kMaxGroups / std::max(tm * tn, (sp / 32) * (lp / 32))));
    const int64_t at_once = std::min(batch, most);
    // Few tiles and a long side: the Gram matrix in shares of it, of 24 stages at least, until there is a workgroup for every CU (us,
    // whole -> in shares: 2 x 200 x 12000 542 -> 251, 1 x 768 x 2304 251 -> 233)
    const int64_t half = tm * (tm + 1) / 2;
    const int64_t shares = TILE == 64 ? std::max<int64_t>(1, std::min(h->num_cu / (at_once * half), lp / (24 * 32))) : 1;
    const int64_t shares_len = shares > 1 ? at_once * half * shares * TILE * TILE * 2 : 0;  // (in fp16 elements)
    f16_t *ws = nullptr;
    const int rc = layer_room(h, who, at_once * per_matrix + shares_len, &ws);
    if (rc || !launch) return rc;
    float *const parts = reinterpret_cast<float *>(ws + at_once * per_matrix);
    double *sums = reinterpret_cast<double *>(ws);
    f16_t *at = ws + at_once * kOrthoSums * 4;
    const auto take = [&](int64_t len) {
        f16_t *p = at;
        at += at_once * len;
        return p;
    };
    f16_t *X = take(x_len), *Y = take(x_len), *const A = take(a_len), *const B = take(a_len);
    const int64_t rows = io.m_i < io.m_j ? io.long_side : io.short_side, cols = io.m_i < io.m_j ? io.short_side : io.long_side;
    for (int64_t b0 = 0; b0 < batch; b0 += at_once) {
        const int64_t n = std::min(at_once, batch - b0);
        OrthoIo<T> part = io;
        part.M += b0 * io.m_matrix;
        if (part.O) part.O += b0 * io.o_matrix;
        if (part.sub) part.sub += b0 * io.o_matrix;
        hipLaunchKernelGGL((ortho_squares<T>), dim3((unsigned)(n * kOrthoSums)), dim3(256), 0, h->stream, part.M, io.m_matrix, rows, cols,
                           std::max(io.m_i, io.m_j), sums);
        hipLaunchKernelGGL((ortho_begin<T>), dim3((unsigned)(n * (sp / 32) * (lp / 32))), dim3(256), 0, h->stream, part, sums, X, (int)sp, (int)lp);
        const auto go = [&](auto kernel, const OrthoProduct &p, int64_t tiles) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)(n * tiles)), dim3(256), 0, h->stream, p, part);
        };
        constexpr int Q = TILE == 64 ? 2 : 1;
        // Tiles that leave CUs idle are computed by eight wavefronts, from ten stages on (768 x 768 201 -> 179 us, 512 x 512 150 -> 135; with
        // four to six stages 130 x 70 81 -> 89).
        const auto wide = [&](const OrthoProduct &p, int64_t tiles) { return Q == 2 && p.k >= 320 && n * tiles <= h->num_cu; };
        const auto go2 = [&](auto kernel, const OrthoProduct &p, int64_t tiles) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)(n * tiles)), dim3(256 * Q), 0, h->stream, p, part);
        };
        // Stages of LDS: two leave room for two workgroups per CU, four for one, which is what there is when the tiles are few.  (24
        // matrices of 768 x 768 945 us with two, 1030 with four; 12 of 768 x 2304, whose Gram matrices have 252 tiles, 1203 and 1194.)
        for (int64_t s = 0; s < steps; ++s) {
            const auto sym = [&](auto kernel2, auto kernel4, auto kernel8, const OrthoProduct &p) {
                if (wide(p, half)) go2(kernel8, p, half);
                else if (TILE == 64 || n * half <= h->num_cu) go(kernel4, p, half);
                else go(kernel2, p, half);
            };
            const OrthoProduct gram{X, X, A, A, lp, lp, sp, x_len, x_len, a_len, (int)lp, (int)tm, (int)tm, 0.f,
                                    kOrthoScaleA / (kOrthoScaleX * kOrthoScaleX), (int)shares, parts};
            if constexpr (TILE == 64) {
                if (shares > 1) {
                    go2(ortho_product_tile<TILE, 4, Q, kOrthoShare, T>, gram, half * shares);
                    hipLaunchKernelGGL((ortho_gram_finish<TILE>), dim3((unsigned)(n * half)), dim3(256), 0, h->stream, gram);
                }
            }
            if (shares == 1)
                sym(ortho_product_tile<TILE, 2, 1, kOrthoGram, T>, ortho_product_tile<TILE, 4, 1, kOrthoGram, T>,
                    ortho_product_tile<TILE, 4, Q, kOrthoGram, T>, gram);
            sym(ortho_product_tile<TILE, 2, 1, kOrthoPoly, T>, ortho_product_tile<TILE, 4, 1, kOrthoPoly, T>,
                ortho_product_tile<TILE, 4, Q, kOrthoPoly, T>,
                OrthoProduct{A, A, A, B, sp, sp, sp, a_len, a_len, a_len, (int)sp, (int)tm, (int)tm, (float)c.b,
                             (float)(c.c / kOrthoScaleA), 1, nullptr});
            const OrthoProduct step{B, X, X, Y, sp, lp, lp, a_len, x_len, x_len, (int)sp, (int)tm, (int)tn, (float)c.a, 1.f / kOrthoScaleA,
                                    1, nullptr};
            constexpr int NS = TILE == 64 ? 4 : 2;
            if (wide(step, tm * tn)) {
                if (s + 1 < steps) go2(ortho_product_tile<TILE, NS, Q, kOrthoStep, T>, step, tm * tn);
                else go2(ortho_product_tile<TILE, NS, Q, kOrthoLast, T>, step, tm * tn);
            } else if (s + 1 < steps) go(ortho_product_tile<TILE, NS, 1, kOrthoStep, T>, step, tm * tn);
            else go(ortho_product_tile<TILE, NS, 1, kOrthoLast, T>, step, tm * tn);
            std::swap(X, Y);
        }
    }
    HIP_TRY(h, hipGetLastError());
    return CDGRAB_OK;
}

// The padded sides of a matrix for ortho_small, and whether it takes one: a short side above 32 (below, the narrow form is as
// fast) and at most 128, at most 32 blocks, LDS for all of it.  Blocks in units of one as long as there is a wavefront for each.
struct OrthoSmall {
    int64_t sp, lp, bytes;
    int per;
    bool fits;
    OrthoSmall(int64_t s, int64_t l) {
        sp = round_up(s, 32);
        lp = round_up(l, 32);
        per = sp * lp <= 8 * 1024 && sp <= 64 ? 1 : 2;
        if (per == 2) {  // (whole units)
            sp = round_up(s, 64);
            lp = round_up(l, 64);
        }
        bytes = 4 * sp * (lp + 8 + sp + 8);
        fits = s > 32 && s <= 128 && sp * lp <= 32 * 1024 && bytes <= kOrthoSmallLds;
    }
};

// M and O (or `sub`) of `batch` matrices of rows x cols, `m_row` / `o_row` elements from row to row.  Without `launch`: the workspace
// is made as large as such a call needs it, and nothing is enqueued.
template <typename T>
int run_ortho(cdgrab_handle *h, const char *who, int64_t batch, int64_t rows, int64_t cols, const T *M, int64_t m_row, int64_t m_matrix,
              int64_t steps, const OrthoCoeffs &c, T *O, float *sub, float rate, int64_t o_row, int64_t o_matrix,
              bool launch = true) {
    const bool wide = rows <= cols;
    const OrthoIo<T> io{M, O, sub, rate, wide ? m_row : 1, wide ? 1 : m_row, m_matrix, wide ? o_row : 1, wide ? 1 : o_row, o_matrix,
                        (int)std::min(rows, cols), (int)std::max(rows, cols)};
    if (io.short_side <= 16) return run_ortho_narrow<1>(h, who, batch, io, steps, c, launch);
    if (io.short_side <= 32) return run_ortho_narrow<2>(h, who, batch, io, steps, c, launch);
    if (io.short_side <= kOrthoNarrow && (steps == 0 || !OrthoSmall(io.short_side, io.long_side).fits))
        return run_ortho_narrow<4>(h, who, batch, io, steps, c, launch);
    if (steps == 0) {
        for (int64_t b0 = 0; b0 < batch; b0 += 32768) {
            const int64_t n = std::min<int64_t>(32768, batch - b0);
            double *sums = nullptr;
            const int rc = layer_room(h, who, n * kOrthoSums, &sums);
            if (rc || !launch) return rc;
            OrthoIo<T> part = io;
            part.M += b0 * io.m_matrix;
            if (part.O) part.O += b0 * io.o_matrix;
            if (part.sub) part.sub += b0 * io.o_matrix;
            hipLaunchKernelGGL((ortho_squares<T>), dim3((unsigned)(n * kOrthoSums)), dim3(256), 0, h->stream, part.M, m_matrix, rows, cols,
                               m_row, sums);
            hipLaunchKernelGGL((ortho_scaled<T>), dim3((unsigned)std::min<int64_t>((rows * cols + 1023) / 1024, 4096), (unsigned)n), dim3(256),
                               0, h->stream, part, sums);
        }
        HIP_TRY(h, hipGetLastError());
        return CDGRAB_OK;
    }
    const OrthoSmall small(io.short_side, io.long_side);
    if (small.fits) {
        if (!launch) return CDGRAB_OK;
        const auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)batch), dim3(kOrthoSmallThreads), 0, h->stream, io, (int)small.sp, (int)small.lp,
                               (int)steps, c);
        };
        if (small.per == 1) go(ortho_small<T, kOrthoSmallLdsHalf, 1>);
        else if (small.bytes <= kOrthoSmallLdsHalf) go(ortho_small<T, kOrthoSmallLdsHalf, 2>);
        else go(ortho_small<T, kOrthoSmallLds, 2>);
        HIP_TRY(h, hipGetLastError());
        return CDGRAB_OK;
    }
    const int64_t s = io.short_side, tiles = batch * ((s + 127) / 128) * ((s + 127) / 128 + 1) / 2;
    if (tiles >= h->num_cu / 2) return run_ortho_products<128>(h, who, batch, io, steps, c, launch);
    return run_ortho_products<64>(h, who, batch, io, steps, c, launch);
}

int ortho_coeffs(cdgrab_handle *h, const char *who, int64_t steps, const double *coeffs, OrthoCoeffs *c) {
    *c = coeffs ? OrthoCoeffs{coeffs[0], coeffs[1], coeffs[2], 1} : OrthoCoeffs{3.4445, -4.775, 2.0315, 1};
    if (steps < 0 || steps > 64) return fail(h, CDGRAB_EINVAL, "%s: steps=%lld (0 .. 64)", who, (long long)steps);
    double largest = 0.0;
    if (!ortho_in_range(steps, *c, &largest))
        return fail(h, CDGRAB_EINVAL, "%s: with coefficients %g %g %g the steps can take a singular value beyond 3.5", who, c->a, c->b, c->c);
    c->per_gram = ortho_gram_steps(*c, largest);
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
    const bool once = norm_once(rows, width, size, X, x_stride);
    by_norm_type(type, width, [&](auto elem, auto vec) {
        typedef decltype(elem) T;
        constexpr int VEC = decltype(vec)::value;
        by_norm_shape<VEC, false>(width, [&](auto lanes, auto k) {
            constexpr int LANES = decltype(lanes)::value, K = decltype(k)::value;
            constexpr int THREADS = LANES > kNormThreads ? LANES : kNormThreads, PER = THREADS / LANES;
            // (at least four rows per group of threads, which reads its columns' parameters once, if that leaves two workgroups per CU)
            const int64_t all = (rows + PER - 1) / PER, most = (int64_t)h->num_cu * (2048 / THREADS);
            const int64_t groups = std::min(std::min(all, most), std::max<int64_t>(2 * (int64_t)h->num_cu, all / 4));
            const auto launch = [&](auto kernel) {
                hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(THREADS), 0, h->stream, (const T *)X, x_stride, gain, bias, (T *)Y,
                                   y_stride, rows, (int)width, eps);
            };
            if constexpr (VEC > 1) {
                if (once) return launch(norm_forward<T, VEC, LANES, K, true>);
            }
            launch(norm_forward<T, VEC, LANES, K, false>);
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
    const bool once = norm_once(t->rows, width, size, X, x_stride) && norm_once(t->rows, width, size, DY, dy_stride);
    by_norm_type(type, width, [&](auto elem, auto vec) {
        typedef decltype(elem) T;
        constexpr int VEC = decltype(vec)::value;
        by_norm_shape<VEC, true>(width, [&](auto lanes, auto k) {
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
                const auto launch = [&](auto kernel) {
                    hipLaunchKernelGGL(kernel, dim3((unsigned)(part.examples * chunks)), dim3(THREADS), 0, h->stream, part, (int)chunks,
                                       (const T *)X, x_stride, (const T *)DY, dy_stride, gain, (T *)DX, dx_stride, G, g_stride,
                                       (int)with_bias, partial, (int)width, eps);
                };
                if constexpr (VEC > 1) {
                    if (once) {
                        launch(norm_backward<T, VEC, LANES, K, true>);
                        continue;
                    }
                }
                launch(norm_backward<T, VEC, LANES, K, false>);
            }
            if (partial)  // (fewer than `fill` examples, 2^11, of at most 2^10 groups of columns: one launch)
                hipLaunchKernelGGL(norm_grad_finish, dim3((unsigned)(tok.examples * ((cols + 31) / 32))), dim3(256), 0, h->stream, partial,
                                   (int)chunks, (int)cols, G, g_stride);
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
    if (d > kMaxCells) return fail(h, CDGRAB_EINVAL, "%s: %lld elements per gradient row, and at most 2^32", who, (long long)d);
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
        // Few rows per example as outer products, us tiles -> stretches: one row, 784 -> 10, 60 000 examples 2496 -> 451, 768 -> 768, 500
        // examples 244 -> 206; two rows, 768 -> 768 262 -> 268, 300 -> 250 173 -> 119; four rows, 300 -> 64 133 -> 113, 128 -> 128
        // 76 -> 94; eight rows, 300 -> 40 115 -> 93, 50 -> 20 141 -> 36, 128 -> 128 76 -> 126.
        const int64_t flat_tok = tok.tokens <= 2 ? tok.tokens : tok.tokens <= 4 ? 4 : 8;
        if ((tok.tokens <= 2 || (tok.tokens <= 8 && tok.tokens * out_dim <= 384)) && d < ((int64_t)1 << 31) - 2 * kFlatElems &&
            flat_period(out_dim) <= 256 && flat_lds(flat_tok, in_dim, out_dim, with_bias) <= kFlatLds) {
            const auto flat = [&](auto t) {
                constexpr int TOK = decltype(t)::value;
                if (d <= 2048 && flat_period(out_dim) <= 64) return run_flat<T, TOK, 64>(h, tok, x, x_stride, dl, d_stride, in_dim, out_dim, with_bias, G, g_stride);
                return run_flat<T, TOK, 256>(h, tok, x, x_stride, dl, d_stride, in_dim, out_dim, with_bias, G, g_stride);
            };
            if (flat_tok <= 1) return flat(std::integral_constant<int, 1>{});
            if (flat_tok == 2) return flat(std::integral_constant<int, 2>{});
            if (flat_tok == 4) return flat(std::integral_constant<int, 4>{});
            return flat(std::integral_constant<int, 8>{});
        }
        if (out_dim <= 32)
            return run_linear<T, 128, 32, 4, 1>(h, tok, x, x_stride, dl, d_stride, in_dim, out_dim, with_bias, G, g_stride);
        if (in_dim <= 32)
            return run_linear<T, 32, 128, 1, 4>(h, tok, x, x_stride, dl, d_stride, in_dim, out_dim, with_bias, G, g_stride);
        // Small tiles where large ones, even in shares of the tokens, would not fill the chip, and where small ones fill it without
        // shares (64 examples of 1024 tokens, 128 -> 384: 26 us against 33; one of 65 536, 768 -> 2304: large ones in shares 414, small 800).
        const bool few = tiles(128, 128) * std::max<int64_t>(1, tok.tokens / 256) < 2 * h->num_cu;
        if (in_dim <= 64 || out_dim <= 64 || few || (tiles(128, 128) < h->num_cu && tiles(64, 64) >= 2 * h->num_cu))
            return run_linear<T, 64, 64, 2, 2>(h, tok, x, x_stride, dl, d_stride, in_dim, out_dim, with_bias, G, g_stride);
        return run_linear<T, 128, 128, 2, 2>(h, tok, x, x_stride, dl, d_stride, in_dim, out_dim, with_bias, G, g_stride);
    };
    if (type == CDGRAB_F32) return by_type(float{});
    return type == CDGRAB_BF16 ? by_type(bf16_t{}) : by_type(f16_t{});
}

extern "C" int cdgrab_orthogonalize(cdgrab_handle *h, int64_t batch, int64_t rows, int64_t cols, int32_t type, const void *M,
                                    int64_t m_stride, int64_t m_matrix, int32_t steps, const double *coeffs, void *O, int64_t o_stride,
                                    int64_t o_matrix) {
    if (!h) return CDGRAB_EINVAL;
    static const char *who = "cdgrab_orthogonalize";
    if (batch < 0 || batch > kMaxGroups || rows < 1 || cols < 1 || rows > kOrthoMaxSide || cols > kOrthoMaxSide || bad_type(type))
        return fail(h, CDGRAB_EINVAL, "%s: bad arguments batch=%lld rows=%lld cols=%lld (1 .. 2^20) type=%d", who, (long long)batch,
                    (long long)rows, (long long)cols, (int)type);
    if (std::min(rows, cols) > kOrthoMaxShort || rows * cols > kMaxCells)
        return fail(h, CDGRAB_EINVAL, "%s: a shorter side of %lld (at most %lld) or %lld elements (2^32)", who,
                    (long long)std::min(rows, cols), (long long)kOrthoMaxShort, (long long)(rows * cols));
    OrthoCoeffs c{};
    const int rc = ortho_coeffs(h, who, steps, coeffs, &c);
    if (rc) return rc;
    if (batch == 0) return CDGRAB_OK;
    if (!M || !O) return fail(h, CDGRAB_EINVAL, "%s: null pointer", who);
    const int64_t size = elem_size(type);
    if (bad_rows(M, rows, cols, m_stride, size) || bad_rows(O, rows, cols, o_stride, size) ||
        (batch > 1 && (m_matrix < (rows - 1) * m_stride + cols || o_matrix < (rows - 1) * o_stride + cols ||
                       m_matrix > (INT64_MAX >> 4) / batch || o_matrix > (INT64_MAX >> 4) / batch)))
        return fail(h, CDGRAB_EINVAL, "%s: a stride below the size, or a misaligned or too long array", who);
    if (batch == 1) m_matrix = o_matrix = 0;
    if (matrices_overlap(batch, rows, cols * size, M, m_stride * size, m_matrix * size, O, o_stride * size, o_matrix * size))
        return fail(h, CDGRAB_EINVAL, "%s: M and O must not overlap", who);
    const OnDevice on(h->device);
    HIP_TRY(h, on.err);
    const auto by_type = [&](auto elem) {
        typedef decltype(elem) T;
        return run_ortho<T>(h, who, batch, rows, cols, (const T *)M, m_stride, m_matrix, steps, c, (T *)O, nullptr, 0.f, o_stride, o_matrix);
    };
    if (type == CDGRAB_F32) return by_type(float{});
    return type == CDGRAB_BF16 ? by_type(bf16_t{}) : by_type(f16_t{});
}
