"""GPU tests of training epochs with the orthogonalised update that take several staging chunks, whose rows are balanced on a
second stream meanwhile."""
import numpy as np
import pytest
import torch

import workloads
from parity import check_epoch, rel_l2
from test_gpu_orthogonal import lib, train64  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n,in_dim,classes", [(4, 1200, 20, 5), (16, 300, 90, 10), (3, 1500, 150, 131)])
def test_several_chunks(lib, m, n, in_dim, classes):  # noqa: F811
    X, y, W0 = workloads.softmax_problem(m + n, m * n, in_dim, classes)
    X, y, W0 = X.reshape(m, n, in_dim), y.reshape(m, n), (W0 * 10).astype(np.float32)
    perm = workloads.random_perms(3, m, n)
    *args, perm_in = (torch.from_numpy(a).cuda() for a in (X, y, perm))
    h = lib.Handle()

    def epoch(h, W, v):
        return lib.cdgrab_train_epoch_softmax_orthogonal(h, *args, W, v, perm_in=perm_in, want_grads=True)

    W, v = torch.from_numpy(W0.copy()).cuda(), torch.zeros(W0.size, device="cuda")
    out = epoch(h, W, v)
    torch.cuda.synchronize()
    rows = out["grads"].cpu().numpy()
    # the first steps against the epoch in double (later ones differ by what rounding has put into the missing direction of
    # every velocity), and the order of all of them
    steps = 24
    at, ids = np.arange(m)[:, None], perm[:, :steps]
    _, _, want, loss = train64(X[at, ids], y[at, ids], np.tile(np.arange(steps), (m, 1)), W0, 0.95, 0.02, 5)
    assert max(rel_l2(rows[:, j], want[:, j]) for j in range(steps)) <= 1e-5
    np.testing.assert_allclose(out["loss"].cpu().numpy()[:, :steps], loss, rtol=1e-4, atol=1e-6)
    assert torch.isfinite(W).all() and torch.isfinite(v).all()
    check_epoch(rows, {"signs": out["signs"].cpu().numpy(), "perm": out["perm"].cpu().numpy()}, perm)
    # the same bits again on another stream, and recorded (a few thousand launches)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        other = lib.Handle(stream=stream)
        W2, v2 = torch.from_numpy(W0.copy()).cuda(), torch.zeros(W0.size, device="cuda")
        again = epoch(other, W2, v2)
        stream.synchronize()
        assert torch.equal(W, W2) and torch.equal(v, v2)
        for key in ("signs", "perm", "grads", "loss"):
            assert torch.equal(out[key], again[key])
        if classes > 32:
            return
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            recorded = epoch(other, W2, v2)
        for _ in range(3):
            W2.copy_(torch.from_numpy(W0))
            v2.zero_()
            graph.replay()
            stream.synchronize()
            assert torch.equal(W, W2) and torch.equal(v, v2)
            for key in ("signs", "perm", "grads", "loss"):
                assert torch.equal(out[key], recorded[key])
            lib.cdgrab_orthogonalize(other, v2.view(-1, classes))


def test_a_single_class(lib):  # noqa: F811
    """Its gradients are zero, and so is every update."""
    X, y, W0 = workloads.softmax_problem(5, 24, 9, 1)
    W, v = torch.from_numpy(W0.copy()).cuda(), torch.zeros(10, device="cuda")
    for steps in (5, 30):
        lib.cdgrab_train_epoch_softmax_orthogonal(lib.Handle(), torch.from_numpy(X).cuda().view(3, 8, 9),
                                                  torch.from_numpy(y).cuda().view(3, 8), W, v, steps=steps)
        assert torch.equal(W.cpu(), torch.from_numpy(W0)) and (v == 0).all()
