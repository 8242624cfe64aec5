"""GPU tests of recorded calls after larger ones on the same handle have taken larger workspaces: a recording keeps its own."""
import pytest
import torch

import workloads
from test_gpu_layers import lib, rand  # noqa: F401

pytestmark = pytest.mark.gpu


def gradients(seed, m, n, d):
    return rand(seed, m, n, d)


def problem(seed, m, n, in_dim, classes):
    X, y, W = (torch.from_numpy(a).cuda() for a in workloads.softmax_problem(seed, m * n, in_dim, classes))
    return X.view(m, n, in_dim), y.view(m, n), W


def balance(lib, m, n, d):  # noqa: F811
    g = gradients(1, m, n, d)
    return lambda h: lib.cdgrab_balance_epoch(h, m, n, d, grads=g, want_r64=True, want_dots=True)


def independent(lib, m, n, d):  # noqa: F811
    g = gradients(2, m, n, d)
    return lambda h: lib.cdgrab_balance_epoch_independent(h, g)


def herding(lib, m, n, d):  # noqa: F811
    g = gradients(3, m, n, d)
    return lambda h: {"bound": lib.cdgrab_herding_bound(h, g)}


def train(lib, m, n, in_dim, classes, orthogonal):  # noqa: F811
    X, y, W0 = problem(4, m, n, in_dim, classes)
    W, v = W0.clone(), torch.zeros(W0.numel(), device="cuda")

    def epoch(h):
        W.copy_(W0)
        v.zero_()
        if orthogonal:
            out = lib.cdgrab_train_epoch_softmax_orthogonal(h, X, y, W, v, want_grads=True)
        else:
            out = lib.cdgrab_train_epoch_softmax(h, X, y, W, velocity=v, momentum=0.9, want_grads=True)
        return {**out, "W": W, "v": v}
    return epoch


CASES = {
    "long rows": (lambda lib: balance(lib, 2, 40, 70_000), lambda lib: balance(lib, 3, 60, 300_000)),
    "short rows": (lambda lib: balance(lib, 4, 200, 500), lambda lib: balance(lib, 8, 1000, 9000)),
    "narrow rows": (lambda lib: balance(lib, 2, 700, 30), lambda lib: balance(lib, 4, 9000, 64)),
    "walks side by side": (lambda lib: independent(lib, 5, 200, 300), lambda lib: independent(lib, 20, 700, 2000)),
    "herding": (lambda lib: herding(lib, 3, 200, 100), lambda lib: herding(lib, 5, 5000, 700)),
    "training": (lambda lib: train(lib, 4, 40, 50, 5, False), lambda lib: train(lib, 8, 400, 300, 10, False)),
    "training, a launch pair per step": (lambda lib: train(lib, 40, 10, 30, 20, False), lambda lib: train(lib, 70, 30, 200, 40, False)),
    "training, orthogonalised": (lambda lib: train(lib, 4, 40, 50, 5, True), lambda lib: train(lib, 8, 400, 300, 10, True)),
    "training, orthogonalised by products": (lambda lib: train(lib, 2, 6, 150, 131, True), lambda lib: train(lib, 4, 8, 400, 300, True)),
}


@pytest.mark.parametrize("name", CASES)
def test_a_recording_keeps_its_workspace(lib, name):  # noqa: F811
    make, make_larger = CASES[name]
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        h = lib.Handle(stream=stream)
        call, larger = make(lib), make_larger(lib)
        want = {k: t.clone() for k, t in call(h).items() if t is not None}
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = call(h)
        first = {k: t.clone() for k, t in larger(h).items() if t is not None}
        stream.synchronize()
        torch.cuda.empty_cache()
        fill = [torch.full((1 << 20,), float("nan"), device="cuda") for _ in range(64)]  # what had been freed would be here
        for _ in range(3):
            graph.replay()
            stream.synchronize()
            for k, t in want.items():
                assert torch.equal(got[k], t), k
            again = larger(h)
            for k, t in first.items():
                assert torch.equal(again[k], t), k
        stream.synchronize()
        assert all(torch.isnan(t).all() for t in fill)
