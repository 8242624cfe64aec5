"""GPU tests of the layer operators at the sizes that the small tests do not come to: large tiles of the linear gradients, rows read
past the caches, each split of a row over threads, and calls that take several launches."""
import pytest
import torch

from test_gpu_layers import TYPES, U, close, device_spans, grad64, lib, linear64, norm64, norm_tol, rand, spans_of  # noqa: F401
from test_gpu_orthogonal import check

pytestmark = pytest.mark.gpu


def rows_of_no_example(rows, spans):
    outside = torch.ones(rows, dtype=torch.bool, device="cuda")
    for first, count in spans:
        outside[first:first + count] = False
    return outside


# 128 x 128 tiles: 600 and more of them (odd sizes, examples of no to all tokens); tokens from 512 on and more columns than rows, whose
# tiles are numbered down the columns; few tiles and thousands of tokens, in shares of the tokens.
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind,examples,tokens,n_in,n_out", [
    ("padded", 100, 63, 301, 1001), ("packed", 64, 530, 130, 200), ("dense", 64, 520, 200, 130), ("packed", 3, 16500, 260, 300),
    ("padded", 2, 9000, 300, 260), ("dense", 1, 40000, 129, 385),
])
def test_linear_in_large_tiles(lib, kind, examples, tokens, n_in, n_out, dtype):  # noqa: F811
    counts = [tokens * e // (examples - 1) if examples > 1 else tokens for e in range(examples)][::-1]  # down to none
    spans, rows, first, count = spans_of(kind, counts, tokens)
    x, d = rand(n_in, rows, n_in, offset=0.3, dtype=dtype), rand(n_out, rows, n_out, scale=0.1, dtype=dtype)
    want, tol = linear64(x, d, spans, dtype)
    outside = rows_of_no_example(rows, spans)
    x[outside], d[outside] = float("nan"), float("inf")
    lead = (rows,) if kind == "packed" else (examples, tokens)
    f, c = device_spans(first, count)
    h = lib.Handle()
    g = lib.cdgrab_pergrad_linear(h, x.view(*lead, n_in), d.view(*lead, n_out), first=f, count=c, tokens=tokens)
    close(g, want, tol, "G")
    bare = lib.cdgrab_pergrad_linear(h, x.view(*lead, n_in), d.view(*lead, n_out), with_bias=False, first=f, count=c, tokens=tokens)
    assert torch.equal(bare, g[:, :n_in * n_out])
    assert torch.equal(lib.cdgrab_pergrad_linear(h, x.view(*lead, n_in), d.view(*lead, n_out), first=f, count=c, tokens=tokens), g)


# 67 to 69 MB of rows, whose pieces of sixteen bytes are whole (read past the caches) or not.
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind,whole", [("dense", True), ("padded", True), ("packed", True), ("padded", False)])
def test_layernorm_of_many_rows(lib, kind, whole, dtype):  # noqa: F811
    width = (700 if dtype == torch.float32 else 1400) + (0 if whole else 1)
    examples, tokens = (60, 410) if kind != "packed" else (119, 410)
    counts = [tokens] * examples if kind == "dense" else [tokens * e // (examples - 1) for e in range(examples)]
    spans, rows, first, count = spans_of(kind, counts, tokens)
    assert rows * width * torch.finfo(dtype).bits // 8 >= 64 << 20
    x, dy = rand(1, rows, width, offset=0.5, dtype=dtype), rand(2, rows, width, scale=0.1, dtype=dtype)
    w, b = rand(3, width, offset=1.0, scale=0.2), rand(4, width)
    h = lib.Handle()
    hat, _ = norm64(x, None, None, 1e-5)
    close(lib.cdgrab_layernorm(h, x, w, b), hat * w.double() + b.double(), norm_tol(hat, w.double(), b.double(), dtype), "y")
    want_dx, tol_dx, want_g, tol_g = grad64(x, dy, w, 1e-5, spans, dtype)
    outside = rows_of_no_example(rows, spans)
    x[outside], dy[outside] = float("nan"), float("inf")
    shape = (rows, width) if kind == "packed" else (examples, tokens, width)
    dx = torch.full_like(x, 7.0)
    f, c = device_spans(first, count)
    _, g = lib.cdgrab_pergrad_layernorm(h, x.view(shape), dy.view(shape), w, first=f, count=c, tokens=tokens, dX=dx.view(shape))
    assert (dx[outside] == 7.0).all()
    close(dx[~outside], want_dx[~outside], tol_dx[~outside], "dX")
    close(g, want_g, tol_g, "G")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [100, 200, 450, 700, 900, 1800, 3500, 7000, 11000, 14000])
def test_each_split_of_a_row(lib, width, dtype):  # noqa: F811
    counts, tokens = [9, 0, 4], 9
    spans, rows, first, count = spans_of("padded", counts, tokens)
    x, dy = rand(1, rows, width, offset=0.5, dtype=dtype), rand(2, rows, width, scale=0.1, dtype=dtype)
    w, b = rand(3, width, offset=1.0, scale=0.2), rand(4, width)
    h = lib.Handle()
    hat, _ = norm64(x, None, None, 1e-5)
    close(lib.cdgrab_layernorm(h, x, w, b), hat * w.double() + b.double(), norm_tol(hat, w.double(), b.double(), dtype), "y")
    want_dx, tol_dx, want_g, tol_g = grad64(x, dy, w, 1e-5, spans, dtype)
    outside = rows_of_no_example(rows, spans)
    x[outside] = float("nan")
    _, c = device_spans(None, count)
    dx, g = lib.cdgrab_pergrad_layernorm(h, x.view(3, tokens, width), dy.view(3, tokens, width), w, count=c)
    assert (dx.view(rows, width)[outside] == 0).all()
    close(dx.view(rows, width)[~outside], want_dx[~outside], tol_dx[~outside], "dX")
    close(g, want_g, tol_g, "G")


MANY = (1 << 21) + 60_000  # examples: more than a launch takes


def test_layernorm_backward_of_millions_of_examples(lib):  # noqa: F811
    x, dy = rand(1, MANY, 1, 8, offset=0.5), rand(2, MANY, 1, 8, scale=0.1)
    w = rand(3, 8, offset=1.0, scale=0.2)
    dx, g = lib.cdgrab_pergrad_layernorm(lib.Handle(), x, dy, w)
    want_dx, tol_dx, _, _ = grad64(x, dy, w, 1e-5, [(0, 1)], torch.float32)
    close(dx, want_dx, tol_dx, "dX")
    hat, _ = norm64(x, None, None, 1e-5)
    a = dy.double().abs()
    # (as grad64: one row each)
    close(g, torch.cat([dy.double() * hat, dy.double()], 2).squeeze(1),
          torch.cat([(80 + 17) * U * a * (hat.abs() + 1), 17 * U * a], 2).squeeze(1) + 1e-38, "G")


@pytest.mark.parametrize("tokens,n_in,n_out", [(1, 8, 3), (9, 4, 4)])  # outer products, and tiles
def test_linear_of_millions_of_examples(lib, tokens, n_in, n_out):  # noqa: F811
    x, d = rand(1, MANY, tokens, n_in), rand(2, MANY, tokens, n_out, scale=0.1)
    g = lib.cdgrab_pergrad_linear(lib.Handle(), x, d)
    x, d = torch.cat([x, torch.ones(MANY, tokens, 1, device="cuda")], 2).double(), d.double()
    want = sum(x[:, t].unsqueeze(2) * d[:, t].unsqueeze(1) for t in range(tokens)).flatten(1)
    mass = sum(x[:, t].abs().unsqueeze(2) * d[:, t].abs().unsqueeze(1) for t in range(tokens)).flatten(1)
    close(g, want, ((2 * tokens + 64) * U + 2.0 ** -21) * mass + 1e-38, "G")  # as linear64


def test_more_matrices_than_the_workspace_holds(lib):  # noqa: F811
    """Pairs of 130 x 130 are 1 MB per matrix, and 4094 of them are held at a time."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    m = torch.randn(4100, 130, 130, generator=gen, device="cuda")
    h = lib.Handle()
    out = lib.cdgrab_orthogonalize(h, m)
    for b in (0, 17, 4093, 4094, 4099):
        check(out[b], m[b], torch.float32)
    m[4094:] = m[:6]
    again = lib.cdgrab_orthogonalize(h, m)
    assert torch.equal(again[:4094], out[:4094])
    for b in range(6):
        assert ((again[4094 + b] - out[b]).norm() / out[b].norm()).item() <= 2 * 400 * U  # (other tiles: up to rounding)


def test_no_steps_on_many_matrices(lib):  # noqa: F811
    gen = torch.Generator(device="cuda").manual_seed(2)
    m = torch.randn(33_000, 65, 66, generator=gen, device="cuda")
    m[32_768] *= 1e6
    out = lib.cdgrab_orthogonalize(lib.Handle(), m, steps=0)
    norm = m.flatten(1).double().norm(dim=1).view(-1, 1, 1)
    want = m.double() / norm
    close(out, want, 2 * U * want.abs() + 1e-38, "X0")  # (rounded once, from double)


@pytest.mark.parametrize("tokens,n_in,n_out", [(3, 70, 40), (60, 130, 90)])
def test_first_without_count(lib, tokens, n_in, n_out):  # noqa: F811
    """Examples of `tokens` rows each, wherever they start; the last one is cut by the array's end."""
    rows = 3 * tokens + 2
    x, d, dy = rand(1, rows, n_in), rand(2, rows, n_out), rand(3, rows, n_in)
    first = torch.tensor([2 * tokens, 1, rows - 2], dtype=torch.int64, device="cuda")
    spans = [(2 * tokens, tokens), (1, tokens), (rows - 2, 2)]
    h = lib.Handle()
    want, tol = linear64(x, d, spans, torch.float32)
    close(lib.cdgrab_pergrad_linear(h, x, d, first=first, tokens=tokens), want, tol, "linear")
    _, _, want_g, tol_g = grad64(x, dy, torch.ones(n_in, device="cuda"), 1e-5, spans, torch.float32)
    close(lib.cdgrab_pergrad_layernorm(h, x, dy, first=first, tokens=tokens)[1], want_g, tol_g, "norm")
