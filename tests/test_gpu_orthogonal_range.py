"""GPU tests of the orthogonalised update where its arithmetic is at its limits: many steps on matrices that lack rank."""
import numpy as np
import pytest
import torch

import workloads
from test_gpu_orthogonal import COEFFS, TOL, by_products, check, lib, rand  # noqa: F401

pytestmark = pytest.mark.gpu

POLAR = (1.875, -1.25, 0.375)


def velocity(seed, in_dim, classes):
    """A softmax regression's gradient: its columns add up to zero."""
    X, y, W = workloads.softmax_problem(seed, 400, in_dim, classes)
    X = torch.cat([torch.from_numpy(X), torch.ones(400, 1)], 1)
    delta = torch.softmax(X @ torch.from_numpy(W) * 20, 1)
    delta[torch.arange(400), torch.from_numpy(y).long()] -= 1
    return (X.t() @ delta / 400).cuda()


def of_rank(seed, rank, *shape):
    gen = torch.Generator().manual_seed(seed)
    a = torch.randint(-3, 4, (*shape[:-1], rank), generator=gen).float()
    return (a @ torch.randint(-3, 4, (*shape[:-2], rank, shape[-1]), generator=gen).float()).cuda()  # (exact: small whole numbers)


CASES = [("velocity", (785, 10)), ("velocity", (41, 7)), ("rank 4", (30, 200)), ("rank 3", (50, 20)), ("rank 1", (16, 16)), ("rank 9", (12, 6000)),
         ("rank 5", (5000, 31)), ("rank 6", (60, 900)), ("rank 2", (700, 40)), ("rank 7", (60, 100)), ("rank 20", (130, 200))]


def matrix(kind, shape):
    return velocity(1, shape[0] - 1, shape[1]) if kind == "velocity" else of_rank(2, int(kind[5:]), *shape)


# Errors in double grow by 3.4445 (1.875) per step: 2^-52 3.4445^12 = 6e-10 and 2^-52 1.875^30 = 3e-8, and the results are
# rounded to fp32.  The forms of pairs have the error of fp32 products, 2^-24 per step growing alike, and are not held to that.
@pytest.mark.parametrize("steps,coeffs", [(7, COEFFS), (12, COEFFS), (13, POLAR), (30, POLAR)])
@pytest.mark.parametrize("kind,shape", [c for c in CASES if min(c[1]) <= 32 or max(c[1]) >= 700])
def test_more_steps_than_one_gram_matrix_serves(lib, kind, shape, steps, coeffs):  # noqa: F811
    m = matrix(kind, shape)
    check(lib.cdgrab_orthogonalize(lib.Handle(), m, steps=steps, coeffs=coeffs), m, torch.float32, steps, coeffs)


# With the default coefficients a singular value in 0 .. 1 stays below 1.203, the largest value of the polynomial up to there,
# whatever rounding has put into directions that the matrix does not have; with 15/8, -10/8, 3/8 below 1.  Rounding the results to
# bf16 adds at most 2^-8 of the Frobenius norm, which is at most the root of the short side times the largest.
@pytest.mark.parametrize("steps", [5, 12, 16, 20, 40, 64])
@pytest.mark.parametrize("coeffs", [COEFFS, POLAR])
@pytest.mark.parametrize("kind,shape", CASES)
def test_singular_values_stay_in_range(lib, kind, shape, steps, coeffs):  # noqa: F811
    m = matrix(kind, shape)
    h = lib.Handle()
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        out = lib.cdgrab_orthogonalize(h, m.to(dtype), steps=steps, coeffs=coeffs).double().cpu()
        assert torch.isfinite(out).all()
        most = (1.203 if coeffs == COEFFS else 1.0) * (1.001 + torch.finfo(dtype).eps / 2 * min(shape) ** 0.5)
        assert torch.linalg.matrix_norm(out, 2).item() <= most


@pytest.mark.parametrize("batch,rows,cols,rank", [(300, 6, 9, 2), (3, 20, 7, 3), (2, 9, 9000, 4), (270, 30, 4000, 5), (2, 64, 1500, 10)])
def test_batches_of_many_steps(lib, batch, rows, cols, rank):  # noqa: F811
    m = of_rank(batch, rank, batch, rows, cols)
    m[1] = rand(5, rows, cols)
    m[0] *= 2.0 ** 40
    m[-1] = 0
    h = lib.Handle()
    wide = torch.full((batch, rows + 1, cols + 3), 9.0, device="cuda")
    out = lib.cdgrab_orthogonalize(h, m, steps=12, out=wide[:, 1:, 2:-1])
    for b in {0, 1, batch // 2} - {batch - 1}:
        check(out[b], m[b], torch.float32, 12)
    assert (out[-1] == 0).all()
    assert torch.equal(lib.cdgrab_orthogonalize(h, m, steps=12), out)
    out.fill_(9.0)
    assert (wide == 9.0).all()
    m[0, 1, 2] = float("nan")
    again = lib.cdgrab_orthogonalize(h, m, steps=12)
    assert torch.isnan(again[0]).all() and torch.isfinite(again[1:]).all()


def test_many_steps_recorded(lib):  # noqa: F811
    ms = [velocity(3, 784, 10), of_rank(4, 3, 12, 7000), of_rank(5, 3, 900, 60).half()]
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        h = lib.Handle(stream=stream)
        want = [lib.cdgrab_orthogonalize(h, m, steps=20) for m in ms]
        out = [torch.empty_like(m) for m in ms]
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            for m, o in zip(ms, out):
                lib.cdgrab_orthogonalize(h, m, steps=20, out=o)
        for _ in range(3):
            for o in out:
                o.fill_(float("nan"))
            graph.replay()
            stream.synchronize()
            for o, w in zip(out, want):
                assert torch.equal(o, w)
            lib.cdgrab_orthogonalize(h, rand(1, 80, 3000))


@pytest.mark.parametrize("steps", [5, 20, 64])
def test_training_epoch_of_many_steps(lib, steps):  # noqa: F811
    """The velocity lacks a rank at every step; an update's norm is at most 1.203 times the root of the classes."""
    m, n, in_dim, classes, lr = 4, 16, 30, 5, 0.02
    X, y, W0 = workloads.softmax_problem(7, m * n, in_dim, classes)
    W, v = torch.from_numpy(W0.copy()).cuda(), torch.zeros(W0.size, device="cuda")
    out = lib.cdgrab_train_epoch_softmax_orthogonal(lib.Handle(), torch.from_numpy(X).cuda().view(m, n, in_dim),
                                                    torch.from_numpy(y).cuda().view(m, n), W, v, lr=lr, momentum=0.9, steps=steps)
    assert torch.isfinite(W).all() and torch.isfinite(v).all() and torch.isfinite(out["loss"]).all()
    assert np.linalg.norm(W.cpu().numpy() - W0) <= n * lr * 1.203 * classes ** 0.5 * 1.01


def spread(seed, rows, cols, least):
    """Singular values from 1 down to `least`, evenly over their logarithm."""
    u, _ = torch.linalg.qr(rand(seed, rows, rows, dtype=torch.float64).cpu())
    v, _ = torch.linalg.qr(rand(seed + 1, cols, rows, dtype=torch.float64).cpu())
    return (u * torch.logspace(0, np.log10(least), rows, dtype=torch.float64) @ v.t()).float().cuda()


# The Gram matrix's rounding, 2^-52 of its trace, grows by 3.4445^2 per step, as a part of a singular value's square: at most
# 2^-12 of that, half of it of the value, after the eleven steps that one matrix serves; and of the matrix's norm only
# what the few values have that have grown to about one by then, a fifth of them or less: 5e-5.  (15/8: 22 steps.)
@pytest.mark.parametrize("steps,coeffs", [(11, COEFFS), (12, COEFFS), (22, POLAR), (23, POLAR)])
@pytest.mark.parametrize("rows,cols,least", [(30, 100, 1e-4), (12, 6000, 1e-6), (60, 900, 1e-7), (32, 50, 1e-9)])
def test_singular_values_of_all_sizes(lib, rows, cols, least, steps, coeffs):  # noqa: F811
    m = spread(rows, rows, cols, least)
    check(lib.cdgrab_orthogonalize(lib.Handle(), m, steps=steps, coeffs=coeffs), m, torch.float32, steps, coeffs, tol=5e-5)
