"""GPU tests of the orthogonalised update against its definition in 64 bits, alone and in the training epoch."""
import numpy as np
import pytest
import torch

import workloads
from parity import check_epoch, rel_l2

pytestmark = pytest.mark.gpu

COEFFS = (3.4445, -4.775, 2.0315)
U = 2.0 ** -24


@pytest.fixture(scope="module")
def lib():
    import paper_2302_00845_amd as p
    return p


def rand(seed, *shape, scale=1.0, dtype=torch.float32):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=gen, dtype=torch.float64) * scale).to(dtype).cuda()


def by_products(m, steps=5, coeffs=COEFFS):
    """The definition, in double on the CPU."""
    x = m.double().cpu()
    flip = x.shape[0] > x.shape[1]
    x = x.t() if flip else x
    norm = x.square().sum().sqrt()
    x = x / norm if norm > 0 else x
    a, b, c = coeffs
    for _ in range(steps):
        g = x @ x.t()
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.t() if flip else x


# What rounding does: every step's products are good to about 2 U (two parts of 22 bits, fp32 sums) of the norms that
# enter, and a step's error grows by at most 3.4445 in each later step; the parts that enter are at most the result's own
# norm.  2 U (1 + 3.4445 + .. + 3.4445^4) = 400 U in the worst direction; errors spread over all directions, so this bounds
# the relative Frobenius norm of any matrix whose result is not much smaller than the largest of its singular values.
TOL = 400 * U


def check(got, m, dtype, steps=5, coeffs=COEFFS, tol=TOL):
    want = by_products(m, steps, coeffs)
    got = got.double().cpu()
    assert torch.isfinite(got).all()
    err = ((got - want).norm() / want.norm()).item()
    print("relative error %.2e" % err)
    # (each element is off by at most half a step of its type, relative)
    assert err <= tol + torch.finfo(dtype).eps / 2


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 9), (9, 1), (2, 2), (10, 785), (785, 10), (16, 16), (17, 40), (33, 32), (40, 33),
                                       (64, 64), (5000, 12), (30, 9001), (64, 6000), (65, 65), (128, 128), (70, 300), (300, 70),
                                       (129, 257), (500, 501), (640, 640)])
def test_matches_the_definition(lib, rows, cols, dtype):
    m = rand(rows + cols, rows, cols, scale=0.02, dtype=dtype)
    check(lib.cdgrab_orthogonalize(lib.Handle(), m), m, dtype)


@pytest.mark.parametrize("batch,rows,cols", [(3, 20, 7), (300, 5, 6), (2, 3, 10000), (3, 130, 70), (40, 128, 192), (5, 100, 800),
                                             (260, 12, 5000), (24, 300, 500), (24, 500, 300), (60, 300, 260), (3, 33, 250), (2, 64, 500),
                                             (2, 250, 33), (5, 128, 120), (2, 60, 700), (300, 40, 90)])
def test_batches(lib, batch, rows, cols):
    m = rand(batch, batch, rows, cols)
    m[batch // 2] *= 1e-12  # each matrix has its own norm
    m[0] *= 1e12
    h = lib.Handle()
    out = lib.cdgrab_orthogonalize(h, m)
    for b in {0, batch // 2, batch - 1}:
        check(out[b], m[b], torch.float32)
        if batch < 100:  # (alone a matrix may be cut into other tiles or chunks: the same up to rounding)
            one = lib.cdgrab_orthogonalize(h, m[b])
            assert ((one - out[b]).norm() / one.norm()).item() <= 2 * TOL


@pytest.mark.parametrize("rows,cols", [(12, 40), (40, 12), (50, 60), (100, 200), (200, 100), (256, 256)])
@pytest.mark.parametrize("steps,coeffs", [(0, COEFFS), (1, COEFFS), (2, (1.5, -0.5, 0.0)), (12, (1.5, -0.5, 0.0)), (3, (2.0, -1.5, 0.5))])
def test_steps_and_coefficients(lib, rows, cols, steps, coeffs):
    m = rand(rows, rows, cols)
    # (a factor of a per step instead of 3.4445: 2 U (1 + a + ..) is 400 U or less but for twelve steps of 1.5, 2 U * 258)
    check(lib.cdgrab_orthogonalize(lib.Handle(), m, steps=steps, coeffs=coeffs), m, torch.float32, steps, coeffs, tol=max(TOL, 520 * U))


def test_many_steps_end_in_the_polar_factor(lib):
    """With 15/8, -10/8, 3/8 singular values go to one: O O^T is the identity.  Twenty steps take one of 1/100 of the norm there;
    afterwards the map is flat, so that only the last products' rounding shows."""
    for rows, cols in ((20, 50), (90, 130)):
        u, _ = torch.linalg.qr(rand(1, rows, rows, dtype=torch.float64).cpu())
        v, _ = torch.linalg.qr(rand(2, cols, rows, dtype=torch.float64).cpu())
        s = torch.linspace(0.1, 1.0, rows, dtype=torch.float64)
        m = (u * s @ v.t()).float().cuda()
        o = lib.cdgrab_orthogonalize(lib.Handle(), m, steps=20, coeffs=(1.875, -1.25, 0.375)).double().cpu()
        assert (o @ o.t() - torch.eye(rows, dtype=torch.float64)).abs().max().item() < 64 * U
        assert (o - u @ v.t()).norm().item() / rows ** 0.5 < 64 * U * 10  # (vectors: rounding of m over gaps of a tenth)


@pytest.mark.parametrize("rows,cols", [(8, 30), (30, 8), (60, 61), (150, 100), (100, 150)])
def test_strides(lib, rows, cols):
    wide = rand(5, 4, rows + 3, cols + 11)
    m = wide[1:3, 2:2 + rows, 4:4 + cols]
    all_out = torch.full((2, rows + 5, cols + 7), 3.0, device="cuda")
    out = all_out[:, 1:1 + rows, 6:6 + cols]
    h = lib.Handle()
    lib.cdgrab_orthogonalize(h, m, out=out)
    assert torch.equal(out, lib.cdgrab_orthogonalize(h, m.contiguous()))
    out.fill_(3.0)
    assert (all_out == 3.0).all()


@pytest.mark.parametrize("rows,cols", [(8, 30), (64, 64), (100, 150), (150, 100), (20, 6000)])
def test_zero_and_not_finite_matrices(lib, rows, cols):
    m = rand(1, 5, rows, cols)
    m[1] = 0
    m[2, 3, 4] = float("inf")
    m[3, 1, 1] = float("nan")
    h = lib.Handle()
    for steps in (0, 5):
        out = lib.cdgrab_orthogonalize(h, m, steps=steps)
        assert (out[1] == 0).all()
        assert torch.isnan(out[2]).any() and torch.isnan(out[3]).any()
        if steps:
            assert torch.isnan(out[2]).all() and torch.isnan(out[3]).all()
        for b in (0, 4):  # neighbours in the batch are not touched
            check(out[b], m[b], torch.float32, steps)
    big = torch.full((rows, cols), 3e38, device="cuda")  # squares beyond fp32; rank one: the value itself is taken by the steps
    big[0] *= -1
    want = by_products(big)
    assert (lib.cdgrab_orthogonalize(h, big).double().cpu() - want).norm() / want.norm() <= TOL


def test_same_bits_again_recorded_and_on_a_stream(lib):
    ms = [rand(1, 785, 10), rand(2, 2, 60, 50), rand(3, 3, 200, 300), rand(4, 20, 7000)]
    base = lib.Handle()
    want = [lib.cdgrab_orthogonalize(base, m) for m in ms]
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        h = lib.Handle(stream=stream)
        out = [torch.empty_like(m) for m in ms]

        def call():
            for m, o in zip(ms, out):
                lib.cdgrab_orthogonalize(h, m, out=o)

        call()
        stream.synchronize()
        for o, w in zip(out, want):
            assert torch.equal(o, w)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call()
        lib.cdgrab_orthogonalize(h, rand(9, 4, 700, 600))  # a larger workspace in between
        for _ in range(3):
            for o in out:
                o.fill_(float("nan"))
            graph.replay()
            stream.synchronize()
            for o, w in zip(out, want):
                assert torch.equal(o, w)


def test_a_first_call_is_not_recorded(lib):
    """What has to allocate says so instead of breaking the recording."""
    h = None
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        h = lib.Handle(stream=stream)
        m, out = rand(1, 100, 200), torch.empty(100, 200, device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            with pytest.raises(lib.CdgrabError) as err:
                lib.cdgrab_orthogonalize(h, m, out=out)
            out.zero_()
        assert err.value.code == -2 and "captured" in str(err.value)
        graph.replay()
        stream.synchronize()
        assert (out == 0).all()
        lib.cdgrab_orthogonalize(h, m, out=out)
        stream.synchronize()
    check(out, m, torch.float32)


def test_refusals(lib):
    h = lib.Handle()
    m = rand(1, 20, 30)
    whole = torch.zeros(4000, device="cuda")
    for call in (lambda: lib.cdgrab_orthogonalize(h, m, steps=-1), lambda: lib.cdgrab_orthogonalize(h, m, steps=65),
                 lambda: lib.cdgrab_orthogonalize(h, m, coeffs=(4.0, 0.0, 0.0)),  # 4 > 3.5 after one step
                 lambda: lib.cdgrab_orthogonalize(h, m, coeffs=(float("nan"), 0.0, 0.0)),
                 lambda: lib.cdgrab_orthogonalize(h, m, coeffs=(1.0, 60.0, -60.0)),
                 lambda: lib.cdgrab_orthogonalize(h, m, out=m), lambda: lib.cdgrab_orthogonalize(h, torch.empty(0, 5, device="cuda")),
                 lambda: lib.cdgrab_orthogonalize(h, whole[:2000].view(40, 50), out=whole[1990:3990].view(40, 50))):
        with pytest.raises(lib.CdgrabError) as err:
            call()
        assert err.value.code == -1
    p, lim = m.data_ptr(), 2 ** 21 + 1  # sizes that no array here has: refused before anything is looked at
    for b, r, c in ((lim, 20, 30), (1, 2 ** 20 + 1, 1), (1, 16385, 16385), (1, 8192, 2 ** 20), (-1, 2, 2)):
        assert h._lib.cdgrab_orthogonalize(h._h, b, r, c, 0, p, c, r * c, 5, None, p, c, r * c) == -1
    assert h._lib.cdgrab_orthogonalize(h._h, 1, 20, 30, 3, p, 30, 0, 5, None, p, 30, 0) == -1  # no such type
    assert h._lib.cdgrab_orthogonalize(h._h, 1, 20, 30, 0, p, 29, 0, 5, None, whole.data_ptr(), 30, 0) == -1  # rows overlap
    assert h._lib.cdgrab_orthogonalize(h._h, 2, 20, 30, 0, p, 30, 599, 5, None, whole.data_ptr(), 30, 600) == -1  # matrices do
    assert h._lib.cdgrab_orthogonalize(h._h, 1, 20, 30, 0, p + 2, 30, 0, 5, None, whole.data_ptr(), 30, 0) == -1  # between elements
    assert h._lib.cdgrab_orthogonalize(h._h, 1, 20, 30, 0, None, 30, 0, 5, None, whole.data_ptr(), 30, 0) == -1
    for call in (lambda: lib.cdgrab_orthogonalize(h, m.double()), lambda: lib.cdgrab_orthogonalize(h, m[0]),
                 lambda: lib.cdgrab_orthogonalize(h, m.t()), lambda: lib.cdgrab_orthogonalize(h, m, out=torch.empty(20, 31, device="cuda"))):
        with pytest.raises((TypeError, ValueError)):
            call()
    assert lib.cdgrab_orthogonalize(h, torch.empty(0, 5, 6, device="cuda")).shape == (0, 5, 6)


def train64(X, y, perm, W, momentum, lr, steps):
    """The training epoch with the orthogonalised update, in double."""
    m, n, _ = X.shape
    W, v = torch.from_numpy(W).double(), torch.zeros(W.shape, dtype=torch.float64)
    rows, loss = [], np.empty((m, n))
    for j in range(n):
        ids = perm[:, j]
        x = torch.from_numpy(np.concatenate([X[np.arange(m), ids], np.ones((m, 1))], 1)).double()
        t = torch.from_numpy(y[np.arange(m), ids]).long()
        z = x @ W
        delta = torch.softmax(z, 1) - torch.nn.functional.one_hot(t, W.shape[1])
        loss[:, j] = torch.nn.functional.cross_entropy(z, t, reduction="none").numpy()
        g = x.unsqueeze(2) * delta.unsqueeze(1)
        rows.append(g.reshape(m, -1).numpy())
        v = momentum * v + g.mean(0)
        W = W - lr * by_products(v, steps)
    return W.numpy(), v.numpy(), np.stack(rows, 1), loss


@pytest.mark.parametrize("m,n,in_dim,classes,momentum", [(4, 16, 12, 3, 0.95), (3, 10, 7, 5, 0.0), (16, 12, 40, 10, 0.9), (1, 8, 5, 2, 0.5),
                                                         (32, 4, 784, 10, 0.95), (5, 6, 90, 80, 0.9)])
def test_training_epoch(lib, m, n, in_dim, classes, momentum):
    X, y, W0 = workloads.softmax_problem(m + n, m * n, in_dim, classes)
    X, y, W0 = X.reshape(m, n, in_dim), y.reshape(m, n), (W0 * 10).astype(np.float32)
    perm = workloads.random_perms(3, m, n)
    h = lib.Handle()
    W, v = torch.from_numpy(W0.copy()).cuda(), torch.zeros(W0.size, device="cuda")
    out = lib.cdgrab_train_epoch_softmax_orthogonal(h, torch.from_numpy(X).cuda(), torch.from_numpy(y).cuda(), W, v,
                                                    perm_in=torch.from_numpy(perm).cuda(), lr=0.02, momentum=momentum, want_grads=True)
    torch.cuda.synchronize()
    W64, v64, rows64, loss64 = train64(X, y, perm, W0, momentum, 0.02, 5)
    rows = out["grads"].cpu().numpy()
    row_err = max(rel_l2(rows[:, j], rows64[:, j]) for j in range(n))
    print("W %.2e  v %.2e  rows %.2e" % (rel_l2(W.cpu().numpy(), W64), rel_l2(v.cpu().numpy(), v64.reshape(-1)), row_err))
    # fp32 gradients (1e-7 a step) through updates that enlarge a relative error by 485 at the most, times the rate and the
    # few steps: 1e-5 as for the plain epoch, the weights' rounding included
    assert rel_l2(W.cpu().numpy(), W64) <= 1e-5 and rel_l2(v.cpu().numpy(), v64.reshape(-1)) <= 1e-5 and row_err <= 1e-5
    np.testing.assert_allclose(out["loss"].cpu().numpy(), loss64, rtol=1e-4, atol=1e-6)
    check_epoch(rows, {"signs": out["signs"].cpu().numpy(), "perm": out["perm"].cpu().numpy()}, perm)


def test_training_epoch_refusals_and_steps(lib):
    X, y, W0 = workloads.softmax_problem(0, 8, 6, 3)
    X, y, W = torch.from_numpy(X).cuda().view(2, 4, 6), torch.from_numpy(y).cuda().view(2, 4), torch.from_numpy(W0).cuda()
    h = lib.Handle()
    v = torch.zeros(W.numel(), device="cuda")
    for kw in ({"steps": -1}, {"steps": 100}, {"coeffs": (9.0, 0.0, 0.0)}):
        with pytest.raises(lib.CdgrabError) as err:
            lib.cdgrab_train_epoch_softmax_orthogonal(h, X, y, W, v, **kw)
        assert err.value.code == -1
    with pytest.raises(lib.CdgrabError):
        lib.cdgrab_train_epoch_softmax_orthogonal(h, X, y, W, None)
    assert torch.equal(W.cpu(), torch.from_numpy(W0)) and (v == 0).all()
    # each step of an update of norm one moves the weights by lr at the most
    lib.cdgrab_train_epoch_softmax_orthogonal(h, X, y, W, v, lr=0.5, steps=0)
    assert (W.cpu() - torch.from_numpy(W0)).norm().item() <= 4 * 0.5 * (1 + 100 * U)


def test_training_epoch_velocity_apart_from_the_weights(lib):
    X, y, W0 = workloads.softmax_problem(0, 8, 6, 3)
    X, y = torch.from_numpy(X).cuda().view(2, 4, 6), torch.from_numpy(y).cuda().view(2, 4)
    h = lib.Handle()
    for at in (0, 9, 20):  # 21 elements each
        with pytest.raises(lib.CdgrabError) as err:
            big = torch.zeros(45, device="cuda")
            lib.cdgrab_train_epoch_softmax_orthogonal(h, X, y, big[:21].view(7, 3), big[at:at + 21])
        assert err.value.code == -1 and "overlap" in str(err.value)
    both = torch.zeros(42, device="cuda")
    lib.cdgrab_train_epoch_softmax_orthogonal(h, X, y, both[:21].view(7, 3), both[21:])
    assert torch.isfinite(both).all()


@pytest.mark.parametrize("m,n,in_dim,classes", [(3, 10, 7, 5), (5, 6, 90, 80), (2, 4, 300, 200)])
def test_training_epoch_recorded(lib, m, n, in_dim, classes):
    X, y, W0 = workloads.softmax_problem(m + n, m * n, in_dim, classes)
    X, y, W0 = torch.from_numpy(X).cuda().view(m, n, in_dim), torch.from_numpy(y).cuda().view(m, n), torch.from_numpy(W0).cuda()
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        h = lib.Handle(stream=stream)
        W, v = W0.clone(), torch.zeros(W0.numel(), device="cuda")
        want = lib.cdgrab_train_epoch_softmax_orthogonal(h, X, y, W, v)
        stream.synchronize()
        want_W, want_v = W.clone(), v.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = lib.cdgrab_train_epoch_softmax_orthogonal(h, X, y, W, v)
        lib.cdgrab_orthogonalize(h, rand(1, 2, 500, 400))  # a larger workspace in between
        for _ in range(3):
            W.copy_(W0)
            v.zero_()
            graph.replay()
            stream.synchronize()
            assert torch.equal(W, want_W) and torch.equal(v, want_v)
            for key in ("signs", "perm", "loss"):
                assert torch.equal(got[key], want[key])
            lib.cdgrab_orthogonalize(h, rand(2, 300, 100))


def test_two_recordings_and_two_handles(lib):
    """Recordings of one handle share its workspace and follow one another; another handle's call runs beside them."""
    a, b, c = rand(1, 3, 200, 300), rand(2, 150, 260), rand(3, 4, 140, 200)
    base = lib.Handle()
    want = [lib.cdgrab_orthogonalize(base, t) for t in (a, b, c)]
    torch.cuda.synchronize()
    stream, beside = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(beside):
        other = lib.Handle(stream=beside)
        out_c = torch.empty_like(c)
    with torch.cuda.stream(stream):
        h = lib.Handle(stream=stream)
        out_a, out_b = torch.empty_like(a), torch.empty_like(b)
        graphs = []
        for t, o in ((b, out_b), (a, out_a)):  # (the second takes a larger workspace than the first one has recorded)
            lib.cdgrab_orthogonalize(h, t, out=o)
            stream.synchronize()
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=stream):
                lib.cdgrab_orthogonalize(h, t, out=o)
    for _ in range(4):
        for o in (out_a, out_b, out_c):
            o.fill_(float("nan"))
        torch.cuda.synchronize()
        with torch.cuda.stream(beside):
            lib.cdgrab_orthogonalize(other, c, out=out_c)
        with torch.cuda.stream(stream):
            for g in graphs:
                g.replay()
        torch.cuda.synchronize()
        for o, w in zip((out_a, out_b, out_c), want):
            assert torch.equal(o, w)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("batch,rows,cols", [(2, 200, 12000), (1, 12000, 70), (1, 700, 1600), (1, 66, 1537), (3, 1600, 129), (1, 320, 330),
                                             (2, 500, 319), (1, 100, 40000)])
def test_few_tiles_and_long_sides(lib, batch, rows, cols, dtype):
    """Tiles of eight wavefronts, and Gram matrices in shares of the long side."""
    m = rand(rows + cols, batch, rows, cols, dtype=dtype)
    h = lib.Handle()
    got = lib.cdgrab_orthogonalize(h, m)
    for b in range(batch):
        check(got[b], m[b], dtype)
    assert torch.equal(lib.cdgrab_orthogonalize(h, m), got)
    m[0, -1, -1] = float("nan")
    again = lib.cdgrab_orthogonalize(h, m)
    assert torch.isnan(again[0]).all()
    assert torch.equal(again[1:], got[1:])


def test_shares_recorded(lib):
    m, small = rand(1, 90, 9000), rand(2, 700, 1600)
    want = lib.cdgrab_orthogonalize(lib.Handle(), m)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        h = lib.Handle(stream=stream)
        out = torch.empty_like(m)
        lib.cdgrab_orthogonalize(h, m, out=out)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            lib.cdgrab_orthogonalize(h, m, out=out)
        for _ in range(3):
            out.fill_(float("nan"))
            graph.replay()
            stream.synchronize()
            assert torch.equal(out, want)
            lib.cdgrab_orthogonalize(h, small)
