"""GPU tests of a training epoch whose update finds no workspace: refused as such, before anything has been enqueued."""
import pytest
import torch

import workloads
from test_gpu_orthogonal import lib, rand  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("in_dim,classes,steps", [(300, 200, 5), (150, 130, 5), (5000, 9, 5), (20, 6, 30), (90, 80, 0)])
def test_an_epoch_without_workspace_is_not_begun(lib, in_dim, classes, steps):  # noqa: F811
    m, n = 2, 4
    X, y, W0 = workloads.softmax_problem(3, m * n, in_dim, classes)
    X, y, W0 = torch.from_numpy(X).cuda().view(m, n, in_dim), torch.from_numpy(y).cuda().view(m, n), torch.from_numpy(W0).cuda()
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        h = lib.Handle(stream=stream)
        W, v = W0.clone(), torch.zeros(W0.numel(), device="cuda")
        lib.cdgrab_train_epoch_softmax(h, X, y, W.clone(), velocity=v.clone(), momentum=0.9)  # the rest of the workspace
        mark = torch.zeros(1, device="cuda")
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            with pytest.raises(lib.CdgrabError) as err:
                lib.cdgrab_train_epoch_softmax_orthogonal(h, X, y, W, v, steps=steps)
            mark.add_(1)
        assert err.value.code == -2 and "captured" in str(err.value) and "make the call once before" in str(err.value)
        graph.replay()
        stream.synchronize()
        assert mark.item() == 1 and torch.equal(W, W0) and (v == 0).all()  # nothing but the mark was recorded
        # made once, it may be recorded
        lib.cdgrab_train_epoch_softmax_orthogonal(h, X, y, W, v, steps=steps)
        stream.synchronize()
        want_W, want_v = W.clone(), v.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            lib.cdgrab_train_epoch_softmax_orthogonal(h, X, y, W, v, steps=steps)
        for _ in range(3):
            W.copy_(W0)
            v.zero_()
            graph.replay()
            stream.synchronize()
            assert torch.equal(W, want_W) and torch.equal(v, want_v)
            lib.cdgrab_orthogonalize(h, rand(2, 300, 100))
