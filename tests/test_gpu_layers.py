"""GPU tests of the layer operators against plain formulas in 64 bits: layer norm, its backward pass with per-example
parameter gradients, and per-example gradients of linear layers; dense, padded and packed examples, odd sizes, strides,
empty examples, garbage in rows of no example, other streams, recorded calls."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24  # half a step of fp32, relative
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def lib():
    import paper_2302_00845_amd as p
    return p


def rand(seed, *shape, scale=1.0, offset=0.0, dtype=torch.float32):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=gen, dtype=torch.float64) * scale + offset).to(dtype).cuda()


def step(dtype):
    return torch.finfo(dtype).eps / 2


def close(got, want, tol, what):
    """|got - want| <= tol, element by element; the worst as a share of its tolerance is printed."""
    got, want, tol = got.double().cpu(), want.cpu(), tol.cpu()
    share = ((got - want).abs() / tol.clamp_min(1e-300)).max().item() if got.numel() else 0.0
    print("%s: at most %.3f of the tolerance" % (what, share))
    assert torch.isfinite(got).all() and share <= 1.0


def norm64(x, w, b, eps):
    x = x.double()
    mean = x.mean(-1, keepdim=True)
    r = 1.0 / ((x - mean).square().mean(-1, keepdim=True) + eps).sqrt()
    return (x - mean) * r, r


# A thread adds at most 32 elements of a row in order, then at most ten more additions join the threads: 42 roundings on a
# sum of squares, 21 on the deviation; the mean's correction is as much of the mean absolute difference, below the
# deviation.  80 U of |gain| (|hat| + 1) covers both and the handful of roundings of the formula itself.
def norm_tol(hat, w, b, dtype):
    y = (hat * w + b).abs()
    return 80 * U * w.abs() * (hat.abs() + 1) + 2 * U * (b.abs() + y) + step(dtype) * y * (1 + 80 * U) + tiny(dtype)


def tiny(dtype):
    return torch.finfo(dtype).tiny * torch.finfo(dtype).eps  # a step of the numbers below the normal ones


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width", [(1, 1), (5, 3), (3, 4), (2, 7), (9, 8), (33, 63), (4, 64), (7, 65), (130, 128), (3, 255),
                                        (5, 515), (2, 1000), (3, 1027), (2, 1536), (3, 2049), (2, 4100), (2, 6001), (1, 8200),
                                        (2, 12289), (1, 16384)])
def test_layernorm(lib, rows, width, dtype):
    x = rand(width, rows, width, offset=3.0, dtype=dtype)
    w, b = rand(1, width, offset=1.0, scale=0.3), rand(2, width)
    h = lib.Handle()
    y = lib.cdgrab_layernorm(h, x, w, b, eps=1e-5)
    hat, _ = norm64(x, w, b, 1e-5)
    close(y, hat * w.double() + b.double(), norm_tol(hat, w.double(), b.double(), dtype), "y")
    plain = lib.cdgrab_layernorm(h, x)  # neither gain nor bias
    one, zero = torch.ones_like(w).double(), torch.zeros_like(w).double()
    close(plain, hat, norm_tol(hat, one, zero, dtype), "without parameters")


def test_layernorm_far_from_zero(lib):
    # 4096 is 2^12, so that differences of 2^-11 are exact in fp32: the digits that are there must survive
    x = (4096.0 + torch.randint(-8, 9, (64, 300), generator=torch.Generator().manual_seed(5)).double() / 2048).float().cuda()
    h = lib.Handle()
    y = lib.cdgrab_layernorm(h, x, eps=1e-12)
    hat, _ = norm64(x, None, None, 1e-12)
    # (a mean's rounding of at most 2^-12 of 4096 U is taken out by the correction; what stays is its own rounding)
    one, zero = torch.ones(300, dtype=torch.float64, device="cuda"), torch.zeros(300, dtype=torch.float64, device="cuda")
    close(y, hat, norm_tol(hat, one, zero, torch.float32), "y")


def spans_of(kind, counts, tokens):
    n = len(counts)
    if kind == "dense":
        return [(e * tokens, tokens) for e in range(n)], n * tokens, None, None
    if kind == "padded":
        return [(e * tokens, c) for e, c in enumerate(counts)], n * tokens, None, counts
    first, at = [], 0
    for c in counts:
        first.append(at)
        at += c
    return list(zip(first, counts)), at, first, counts


def device_spans(first, count):
    return (None if first is None else torch.tensor(first, dtype=torch.int64, device="cuda"),
            None if count is None else torch.tensor(count, dtype=torch.int32, device="cuda"))


def grad64(x, dy, w, eps, spans, dtype):
    """dX, G and their tolerances."""
    width = x.shape[-1]
    hat, r = norm64(x, None, None, eps)
    dy, w = dy.double(), w.double()
    g = dy * w
    mg, mgh = g.mean(-1, keepdim=True), (g * hat).mean(-1, keepdim=True)
    dx = r * (g - mg - hat * mgh)
    # as norm_tol: 42 roundings per sum, 21 on the deviation (which enters three times), a few on each product
    ag = g.abs().mean(-1, keepdim=True)
    tol_dx = 160 * U * r * (g.abs() + ag + (hat.abs() + 1) * ((g * hat).abs().mean(-1, keepdim=True) + ag)) + \
        step(dtype) * dx.abs() * 1.01 + tiny(dtype)
    G, tol = [], []
    for first, count in spans:
        rows = slice(first, first + count)
        G.append(torch.cat([(dy[rows] * hat[rows]).sum(0), dy[rows].sum(0)]))
        # each term's own error, and one rounding per addition at the most
        a = (dy[rows].abs() * (hat[rows].abs() + 1)).sum(0)
        tol.append(torch.cat([(80 + count + 16) * U * a, (count + 16) * U * dy[rows].abs().sum(0)]) + 1e-38)
    return dx, tol_dx, torch.stack(G), torch.stack(tol)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind,counts,tokens,width", [
    ("dense", [1], 1, 8), ("dense", [5] * 3, 5, 33), ("dense", [64] * 4, 64, 128), ("dense", [1] * 40, 1, 515),
    ("padded", [0, 7, 3, 7, 1], 7, 64), ("padded", [0, 0], 9, 100), ("packed", [4, 0, 11, 1], 11, 259),
    ("packed", [300, 2, 0, 77], 300, 65), ("dense", [2000], 2000, 40), ("padded", [1999, 3], 2000, 771), ("dense", [40] * 2, 40, 2050),
    ("packed", [9, 12], 12, 5003), ("dense", [3] * 2, 3, 9000), ("padded", [2], 3, 16384), ("dense", [9] * 2, 9, 12290),
    ("dense", [700] * 3, 700, 1030),
])
def test_layernorm_backward(lib, kind, counts, tokens, width, dtype):
    spans, rows, first, count = spans_of(kind, counts, tokens)
    x, dy = rand(width, rows, width, offset=0.5, dtype=dtype), rand(width + 1, rows, width, scale=0.1, dtype=dtype)
    w = rand(3, width, offset=1.0, scale=0.2)
    want_dx, tol_dx, want_g, tol_g = grad64(x, dy, w, 1e-5, spans, dtype)
    inside = torch.zeros(rows, dtype=torch.bool, device="cuda")
    for a, c in spans:
        inside[a:a + c] = True
    x[~inside] = float("nan")  # nobody's rows may hold anything, and are left alone
    dy[~inside] = float("inf")
    dx = torch.full_like(x, 7.0)
    shape = (len(counts), tokens, width) if kind != "packed" else (rows, width)
    f, c = device_spans(first, count)
    h = lib.Handle()
    got, g = lib.cdgrab_pergrad_layernorm(h, x.view(shape), dy.view(shape), w, eps=1e-5, first=f, count=c, tokens=tokens,
                                          dX=dx.view(shape))
    assert (dx[~inside] == 7.0).all()
    close(dx[inside], want_dx[inside], tol_dx[inside], "dX")
    close(g, want_g, tol_g, "G")
    # each output alone, and without the bias's gradient: the same bits
    only, none = lib.cdgrab_pergrad_layernorm(h, x.view(shape), dy.view(shape), w, eps=1e-5, first=f, count=c, tokens=tokens,
                                              want_grads=False)
    assert none is None and torch.equal(only.view(rows, width)[inside], dx[inside])
    none, gain_only = lib.cdgrab_pergrad_layernorm(h, x.view(shape), dy.view(shape), w, eps=1e-5, first=f, count=c, tokens=tokens,
                                                   want_dx=False, with_bias=False)
    assert none is None and torch.equal(gain_only, g[:, :width])


@pytest.mark.parametrize("width", [2, 24])
def test_layernorm_gradient_is_the_slope(lib, width):
    """Differences of the loss sum(dy * y), y in double from the definition, against dX and G."""
    x, dy, w = rand(1, 1, 3, width), rand(2, 1, 3, width), rand(3, width, offset=1.0)
    b = rand(4, width)
    h = lib.Handle()
    dx, g = lib.cdgrab_pergrad_layernorm(h, x, dy, w, eps=0.1)

    def loss(x, w, b):
        hat, _ = norm64(x, None, None, 0.1)
        return (dy.double() * (hat * w + b)).sum().item()

    e = 1e-4  # (central differences: error of order e^2 times a third derivative of order ten)
    x64, w64, b64 = x.double(), w.double(), b.double()
    for i in range(3):
        for j in range(width):
            d = torch.zeros_like(x64)
            d[0, i, j] = e
            assert abs((loss(x64 + d, w64, b64) - loss(x64 - d, w64, b64)) / (2 * e) - dx[0, i, j].item()) < 1e-5
    for j in range(width):
        d = torch.zeros_like(w64)
        d[j] = e
        assert abs((loss(x64, w64 + d, b64) - loss(x64, w64 - d, b64)) / (2 * e) - g[0, j].item()) < 1e-5
        assert abs((loss(x64, w64, b64 + d) - loss(x64, w64, b64 - d)) / (2 * e) - g[0, width + j].item()) < 1e-5


def linear64(x, d, spans, dtype, shares=64):
    G, tol = [], []
    x, d = x.double(), d.double()
    for first, count in spans:
        a, c = x[first:first + count], d[first:first + count]
        G.append(torch.cat([(a.t() @ c).reshape(-1), c.sum(0)]))
        # fp32 sums: two roundings per term at the most; fp32 factors: dropped parts and their own sums, 2^-21 of a term
        mass = torch.cat([(a.abs().t() @ c.abs()).reshape(-1), c.abs().sum(0)])
        tol.append(((2 * count + shares) * U + (2.0 ** -21 if dtype == torch.float32 else 0.0)) * mass + 1e-38)
    return torch.stack(G), torch.stack(tol)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind,counts,tokens,n_in,n_out", [
    ("dense", [1] * 3, 1, 1, 1), ("dense", [1] * 70, 1, 40, 10), ("dense", [3] * 5, 3, 130, 7), ("dense", [16] * 2, 16, 32, 32),
    ("padded", [0, 5, 2], 5, 129, 33), ("packed", [7, 0, 40, 1], 40, 65, 31), ("padded", [33, 64, 0], 64, 300, 131),
    ("packed", [100, 37], 100, 257, 260), ("dense", [2100], 2100, 70, 90), ("padded", [1999, 4], 2000, 5, 200),
    ("dense", [2] * 300, 2, 150, 140), ("dense", [4] * 6, 4, 785, 10), ("dense", [1] * 9, 1, 20, 2049), ("packed", [31, 33], 33, 1, 500),
    ("dense", [48] * 40, 48, 384, 256), ("padded", [1, 0, 1], 1, 9000, 3), ("padded", [2, 1, 0], 2, 700, 50), ("packed", [3, 1, 4], 4, 5001, 2),
    ("padded", [8, 0, 5], 8, 900, 40), ("dense", [1] * 5, 1, 3, 255), ("dense", [1] * 3, 1, 33, 1021), ("padded", [6, 7], 7, 1300, 1),
    ("dense", [2] * 3, 2, 8191, 1), ("packed", [0, 2], 2, 16, 514),
])
def test_linear(lib, kind, counts, tokens, n_in, n_out, dtype):
    spans, rows, first, count = spans_of(kind, counts, tokens)
    x, d = rand(n_in, rows, n_in, offset=0.3, dtype=dtype), rand(n_out, rows, n_out, scale=0.1, dtype=dtype)
    want, tol = linear64(x, d, spans, dtype)
    inside = torch.zeros(rows, dtype=torch.bool, device="cuda")
    for a, c in spans:
        inside[a:a + c] = True
    x[~inside] = float("nan")
    d[~inside] = float("inf")
    lead = (len(counts), tokens) if kind != "packed" else (rows,)
    f, c = device_spans(first, count)
    h = lib.Handle()
    g = lib.cdgrab_pergrad_linear(h, x.view(*lead, n_in), d.view(*lead, n_out), first=f, count=c, tokens=tokens)
    close(g, want, tol, "G")
    bare = lib.cdgrab_pergrad_linear(h, x.view(*lead, n_in), d.view(*lead, n_out), with_bias=False, first=f, count=c, tokens=tokens)
    assert torch.equal(bare, g[:, :n_in * n_out])


def test_linear_agrees_with_the_softmax_gradient(lib):
    """cdgrab_pergrad is this with one row per example and delta = softmax - onehot."""
    import workloads
    X, y, W = (torch.from_numpy(a).cuda() for a in workloads.softmax_problem(0, 200, 50, 7))
    h = lib.Handle()
    G = lib.cdgrab_pergrad(h, X, y, W)
    z = X.double() @ W[:-1].double() + W[-1].double()
    delta = (torch.softmax(z, 1) - torch.nn.functional.one_hot(y.long(), 7)).float()
    g = lib.cdgrab_pergrad_linear(h, X.unsqueeze(1), delta.unsqueeze(1))
    # a softmax in fp32 against one in double: 50 roundings of the logits, which are below 1, and a few more
    assert (g - G).abs().max().item() <= 100 * U * 1.01


@pytest.mark.parametrize("dtype", TYPES)
def test_strided_rows_and_a_stretch_of_longer_gradient_rows(lib, dtype):
    n, t, width, n_out = 5, 6, 37, 50
    wide = rand(1, n, t, 200, dtype=dtype)
    x, dy, d = wide[..., 3:3 + width], wide[..., 60:60 + width], wide[..., 110:110 + n_out]
    all_g = torch.full((n, 5000), -3.0, device="cuda")
    g1, g2 = all_g[:, 11:11 + 2 * width], all_g[:, 200:200 + (width + 1) * n_out]
    h = lib.Handle()
    dx_all = torch.full((n, t, 100), 9.0, dtype=dtype, device="cuda")
    lib.cdgrab_pergrad_layernorm(h, x, dy, dX=dx_all[..., 13:13 + width], G_out=g1)
    lib.cdgrab_pergrad_linear(h, x, d, G_out=g2)
    dx, ga = lib.cdgrab_pergrad_layernorm(h, x.contiguous(), dy.contiguous())
    gb = lib.cdgrab_pergrad_linear(h, x.contiguous(), d.contiguous())
    assert torch.equal(dx_all[..., 13:13 + width], dx) and torch.equal(g1, ga) and torch.equal(g2, gb)
    rest = torch.ones(5000, dtype=torch.bool, device="cuda")
    rest[11:11 + 2 * width] = False
    rest[200:200 + (width + 1) * n_out] = False
    assert (all_g[:, rest] == -3.0).all() and (dx_all[..., :13] == 9.0).all() and (dx_all[..., 13 + width:] == 9.0).all()
    y_all = torch.full((n, t, 64), 9.0, dtype=dtype, device="cuda")
    lib.cdgrab_layernorm(h, x, Y=y_all[..., 5:5 + width])
    assert torch.equal(y_all[..., 5:5 + width], lib.cdgrab_layernorm(h, x.contiguous()))
    assert (y_all[..., :5] == 9.0).all() and (y_all[..., 5 + width:] == 9.0).all()


@pytest.mark.parametrize("tokens,n_in,n_out", [(1, 70, 10), (1, 900, 33), (2, 40, 3), (4, 5000, 7), (5, 40, 50), (40, 130, 140)])
def test_gradient_rows_at_any_element(lib, tokens, n_in, n_out):
    """Rows of G that start at any multiple of four bytes, one after the other or with room between them."""
    x, d = rand(1, 5, tokens, n_in), rand(2, 5, tokens, n_out)
    h = lib.Handle()
    want = lib.cdgrab_pergrad_linear(h, x, d)
    size = want.shape[1]
    for gap in (0, 1, 2, 3, 6):
        for start in (0, 1, 2, 3):
            whole = torch.full((start + 5 * (size + gap) + 8,), 9.0, device="cuda")
            G = torch.as_strided(whole, (5, size), (size + gap, 1), start)
            lib.cdgrab_pergrad_linear(h, x, d, G_out=G)
            assert torch.equal(G, want)
            G.fill_(9.0)
            assert (whole == 9.0).all()


def test_spans_that_leave_the_arrays_are_cut(lib):
    x, d = rand(1, 20, 40), rand(2, 20, 50)
    first = torch.tensor([-5, 18, 25, 0, 3, 20, 19], dtype=torch.int64, device="cuda")
    count = torch.tensor([4, 10, 3, -2, 1000, 5, 1], dtype=torch.int32, device="cuda")
    spans = [(0, 0), (18, 2), (0, 0), (0, 0), (3, 8), (0, 0), (19, 1)]  # (8: `tokens`)
    h = lib.Handle()
    want, tol = linear64(x, d, spans, torch.float32)
    close(lib.cdgrab_pergrad_linear(h, x, d, first=first, count=count, tokens=8), want, tol, "linear")
    dy = rand(3, 20, 40)
    _, _, want_g, tol_g = grad64(x, dy, torch.ones(40, device="cuda"), 1e-5, spans, torch.float32)
    dx, g = lib.cdgrab_pergrad_layernorm(h, x, dy, first=first, count=count, tokens=8)
    close(g, want_g, tol_g, "norm")
    assert (dx[:3] == 0).all() and (dx[11:18] == 0).all()


def test_no_examples_and_no_rows(lib):
    h = lib.Handle()
    x = torch.empty(0, 5, 12, device="cuda")
    assert lib.cdgrab_pergrad_linear(h, x, torch.empty(0, 5, 7, device="cuda")).shape == (0, 13 * 7)
    assert lib.cdgrab_pergrad_layernorm(h, x, x)[1].shape == (0, 24)
    assert lib.cdgrab_layernorm(h, x).shape == x.shape
    x = torch.empty(3, 0, 12, device="cuda")  # three examples without a row: zero gradients
    G = torch.full((3, 13 * 7), 5.0, device="cuda")
    lib.cdgrab_pergrad_linear(h, x, torch.empty(3, 0, 7, device="cuda"), G_out=G)
    assert (G == 0).all()
    assert (lib.cdgrab_pergrad_layernorm(h, x, x)[1] == 0).all()


def test_not_finite_rows_stay_among_themselves(lib):
    x, dy, d = rand(1, 4, 3, 20), rand(2, 4, 3, 20), rand(3, 4, 3, 9)
    x[1, 2, 4] = float("inf")
    x[2, 0, 0] = float("nan")
    h = lib.Handle()
    y = lib.cdgrab_layernorm(h, x)
    bad = torch.zeros(4, 3, dtype=torch.bool, device="cuda")
    bad[1, 2] = bad[2, 0] = True
    assert torch.isnan(y[bad]).all() and torch.isfinite(y[~bad]).all()
    dx, g = lib.cdgrab_pergrad_layernorm(h, x, dy)
    assert torch.isnan(dx[bad]).all() and torch.isfinite(dx[~bad]).all()
    assert torch.isnan(g[1:3, :20]).all() and torch.isfinite(g[[0, 3]]).all() and torch.isfinite(g[:, 20:]).all()
    gl = lib.cdgrab_pergrad_linear(h, x, d).view(4, 21, 9)
    assert torch.isfinite(gl[[0, 3]]).all() and not torch.isfinite(gl[1, 4]).any() and torch.isnan(gl[2, 0]).all()
    assert torch.isfinite(gl[1, :4]).all() and torch.isfinite(gl[1, 5:]).all() and torch.isfinite(gl[2, 1:]).all()


def test_other_stream_and_recorded_calls(lib):
    x, dy, d, w = rand(1, 3, 900, 70), rand(2, 3, 900, 70), rand(3, 3, 900, 45), rand(4, 70)
    base = lib.Handle()
    want = [lib.cdgrab_layernorm(base, x, w), *lib.cdgrab_pergrad_layernorm(base, x, dy, w), lib.cdgrab_pergrad_linear(base, x, d)]
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        h = lib.Handle(stream=stream)
        out = [torch.empty_like(t) for t in want]

        def call():
            lib.cdgrab_layernorm(h, x, w, Y=out[0])
            lib.cdgrab_pergrad_layernorm(h, x, dy, w, dX=out[1], G_out=out[2])
            lib.cdgrab_pergrad_linear(h, x, d, G_out=out[3])

        call()
        stream.synchronize()
        for o, t in zip(out, want):
            assert torch.equal(o, t)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call()
        # a larger call in between takes a larger workspace; the recording keeps its own
        lib.cdgrab_pergrad_linear(h, rand(5, 2, 20000, 70), rand(6, 2, 20000, 45))
        for k in range(3):
            for o in out:
                o.fill_(float("nan"))
            graph.replay()
            stream.synchronize()
            for o, t in zip(out, want):
                assert torch.equal(o, t)
            lib.cdgrab_pergrad_linear(h, x, d)


def test_refusals(lib):
    h = lib.Handle()
    x, d = rand(1, 2, 3, 8), rand(2, 2, 3, 5)
    for call in (lambda: lib.cdgrab_layernorm(h, x, eps=-1.0), lambda: lib.cdgrab_layernorm(h, x, eps=float("nan")),
                 lambda: lib.cdgrab_layernorm(h, x, Y=x), lambda: lib.cdgrab_layernorm(h, torch.empty(2, 0, device="cuda")),
                 lambda: lib.cdgrab_layernorm(h, torch.zeros(2, 16385, device="cuda")),
                 lambda: lib.cdgrab_pergrad_layernorm(h, x, x, dX=x), lambda: lib.cdgrab_pergrad_layernorm(h, x, x, eps=-1e-9),
                 lambda: lib.cdgrab_pergrad_layernorm(h, x, x, want_dx=False, want_grads=False),
                 lambda: lib.cdgrab_pergrad_linear(h, torch.empty(1, 1, 0, device="cuda"), torch.empty(1, 1, 3, device="cuda"))):
        with pytest.raises(lib.CdgrabError) as err:
            call()
        assert err.value.code == -1 and "cdgrab_" in str(err.value)
    # sizes and addresses that the binding would not make
    import ctypes
    from paper_2302_00845_amd.cdgrab import _TokenRows
    big = torch.zeros(4000, device="cuda")
    p, q = x.data_ptr(), big.data_ptr()
    lib_h, ok = h._lib, _TokenRows(2, 6, 3, None, None)
    assert lib_h.cdgrab_layernorm(h._h, 6, 8, 7, p, 8, None, None, 1e-5, q, 8) == -1  # no such type
    assert lib_h.cdgrab_layernorm(h._h, 6, 8, 0, p, 7, None, None, 1e-5, q, 8) == -1  # rows overlap
    assert lib_h.cdgrab_layernorm(h._h, 6, 8, 0, p + 1, 8, None, None, 1e-5, q, 8) == -1  # between elements
    assert lib_h.cdgrab_layernorm(h._h, -1, 8, 0, p, 8, None, None, 1e-5, q, 8) == -1
    assert lib_h.cdgrab_layernorm(h._h, 6, 8, 0, None, 8, None, None, 1e-5, q, 8) == -1
    for t in (None, _TokenRows(3, 6, 3, None, None), _TokenRows(-1, 6, 3, None, None), _TokenRows(2, 6, -3, None, None)):
        t = ctypes.byref(t) if t is not None else None
        assert lib_h.cdgrab_pergrad_linear(h._h, t, 8, 5, 0, p, 8, d.data_ptr(), 5, 1, q, 45) == -1
        assert lib_h.cdgrab_pergrad_layernorm(h._h, t, 8, 0, p, 8, q, 8, None, 1e-5, None, 8, 1, q + 400, 16) == -1
    for n_in, n_out, bias, g_stride in ((0, 5, 1, 45), (8, 2 ** 20 + 1, 1, 2 ** 30), (2 ** 20, 2 ** 13, 1, 2 ** 40), (8, 5, 2, 45), (8, 5, 1, 44)):
        assert lib_h.cdgrab_pergrad_linear(h._h, ctypes.byref(ok), n_in, n_out, 0, p, 2 ** 20, d.data_ptr(), 2 ** 20, bias, q, g_stride) == -1
    whole = torch.zeros(6, 100, device="cuda")
    with pytest.raises(lib.CdgrabError):  # the gradients' rows lie in the input's
        lib.cdgrab_pergrad_linear(h, whole[:, :4].unsqueeze(0), torch.zeros(1, 6, 3, device="cuda"), G_out=whole[:1, 2:17])
    y = lib.cdgrab_layernorm(h, whole[:, :40], Y=whole[:, 40:80])  # side by side in the same rows is no overlap
    assert torch.isfinite(y).all()
    for bad in (lambda: lib.cdgrab_layernorm(h, x.double()), lambda: lib.cdgrab_pergrad_linear(h, x, d.half())):
        with pytest.raises((TypeError, ValueError)):
            bad()


def test_rows_beyond_31_bits_of_elements(lib):
    """Offsets are 64-bit: rows 2^31 elements and more into an array, and a gradient row that far into G."""
    rows, width = 5, 600_000_000
    big = torch.zeros(rows * width, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(big, (rows, 24), (width, 1))
    d = rand(3, rows, 10, dtype=torch.bfloat16)
    x.copy_(rand(4, rows, 24, dtype=torch.bfloat16))
    h = lib.Handle()
    first = torch.tensor([4, 0], dtype=torch.int64, device="cuda")
    count = torch.tensor([1, 5], dtype=torch.int32, device="cuda")
    g = lib.cdgrab_pergrad_linear(h, x, d, first=first, count=count, tokens=5)
    want, tol = linear64(x.contiguous(), d, [(4, 1), (0, 5)], torch.bfloat16)
    close(g, want, tol, "G")
    far = torch.zeros(4 * width, dtype=torch.float32, device="cuda")
    G_out = torch.as_strided(far, (2, 250), (3 * width, 1))
    lib.cdgrab_pergrad_linear(h, x, d, first=first, count=count, tokens=5, G_out=G_out)
    assert torch.equal(G_out, g)
    assert torch.equal(lib.cdgrab_layernorm(h, x), lib.cdgrab_layernorm(h, x.contiguous()))


def test_a_block_of_layers_makes_the_balancers_rows(lib):
    """Layer norm, then a linear layer, per-example gradients side by side in the rows that are balanced: the same
    order as balancing rows made in double, and the gradients are those of torch's own backward pass."""
    m, n, t, width, n_out = 4, 8, 6, 24, 10
    N, d = m * n, 2 * width + (width + 1) * n_out
    x, w, b = rand(1, N, t, width), rand(2, width, offset=1.0, scale=0.1), rand(3, width, scale=0.1)
    W, target = rand(4, width, n_out, scale=0.2), rand(5, N, t, n_out)
    h = lib.Handle()
    rows = torch.empty(N, d, device="cuda")
    y = lib.cdgrab_layernorm(h, x, w, b)
    delta = (y @ W - target)
    lib.cdgrab_pergrad_linear(h, y, delta, G_out=rows[:, 2 * width:])
    dx, _ = lib.cdgrab_pergrad_layernorm(h, x, delta @ W.t(), w, G_out=rows[:, :2 * width])
    out = lib.cdgrab_balance_epoch(h, m, n, d, grads=rows.view(m, n, d), want_dots=True)
    torch.cuda.synchronize()

    x64, w64, b64, W64 = x.double().cpu(), w.double().cpu(), b.double().cpu(), W.double().cpu()
    want = np.empty((N, d))
    for e in range(N):
        p = [v.clone().requires_grad_() for v in (w64, b64, W64, torch.zeros(n_out, dtype=torch.float64))]
        y64 = torch.nn.functional.layer_norm(x64[e], (width,), p[0], p[1], 1e-5) @ p[2] + p[3]
        (0.5 * (y64 - target[e].double().cpu()).square().sum()).backward()
        want[e] = torch.cat([v.grad.reshape(-1) for v in p]).numpy()
    err = np.linalg.norm(rows.cpu().numpy() - want) / np.linalg.norm(want)
    print("rows against double: %.2e" % err)
    assert err < 1e-5  # the repository's bound for per-example gradients
    from parity import check_epoch
    got = {k: (v.cpu().numpy() if v is not None else None) for k, v in out.items()}
    check_epoch(rows.view(m, n, d).cpu().numpy(), got)


@pytest.mark.parametrize("tokens,n_in,n_out", [(2, 50, 20), (6, 300, 40), (90, 140, 150), (1200, 40, 70)])
def test_the_same_rows_in_several_examples(lib, tokens, n_in, n_out):
    """Examples may share rows, all of them too: each has its own sums, and dX is the row's whoever it belongs to."""
    rows = tokens + 7
    x, d, dy = rand(1, rows, n_in), rand(2, rows, n_out), rand(3, rows, n_in)
    spans = [(3, tokens), (3, tokens), (0, tokens), (5, tokens - 1), (3, tokens)]
    first, count = device_spans(*zip(*spans))
    h = lib.Handle()
    want, tol = linear64(x, d, spans, torch.float32)
    g = lib.cdgrab_pergrad_linear(h, x, d, first=first, count=count, tokens=tokens)
    close(g, want, tol, "linear")
    assert torch.equal(g[0], g[1]) and torch.equal(g[0], g[4])
    want_dx, tol_dx, want_g, tol_g = grad64(x, dy, torch.ones(n_in, device="cuda"), 1e-5, spans, torch.float32)
    dx, g = lib.cdgrab_pergrad_layernorm(h, x, dy, first=first, count=count, tokens=tokens)
    close(g, want_g, tol_g, "norm")
    assert torch.equal(g[0], g[1]) and torch.equal(g[0], g[4])
    inside = torch.zeros(rows, dtype=torch.bool, device="cuda")
    for a, c in spans:
        inside[a:a + c] = True
    close(dx[inside], want_dx[inside], tol_dx[inside], "dX")
    assert (dx[~inside] == 0).all()
