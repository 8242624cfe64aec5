"""GPU tests of where a call's outputs are allocated when the handle's stream is not the current one."""
import pytest
import torch

import workloads
from test_gpu_layers import lib, rand  # noqa: F401

pytestmark = pytest.mark.gpu


def let_go_of(device, outputs):
    """Blocks of the outputs' sizes that the current stream has let go of: the allocator would hand these out for an allocation on it.
    Returns their addresses."""
    held = [torch.empty_like(t) for t in outputs]
    at = {t.data_ptr() for t in held}
    del held
    return at


def calls(lib):  # noqa: F811
    x, dy, d, w = rand(1, 8, 40, 100), rand(2, 8, 40, 100), rand(3, 8, 40, 64), rand(4, 100)
    count = torch.full((8,), 11, dtype=torch.int32, device="cuda")
    m = rand(5, 4, 200, 300)
    m, n, in_dim, classes = 4, 16, 50, 7
    X, y, W = (torch.from_numpy(a).cuda() for a in workloads.softmax_problem(1, m * n, in_dim, classes))
    X3, y2, v = X.view(m, n, in_dim), y.view(m, n), torch.zeros(W.numel(), device="cuda")
    g = rand(6, m, n, 600)
    u = torch.rand(m, n // 2, generator=torch.Generator().manual_seed(1)).cuda()
    mats = rand(5, 4, 200, 300)
    signs = torch.where(rand(7, m, n) > 0, 1, -1).to(torch.int8)
    return {
        "layernorm": lambda h: [lib.cdgrab_layernorm(h, x, w)],
        "pergrad_layernorm": lambda h: list(lib.cdgrab_pergrad_layernorm(h, x, dy, w, count=count)),
        "pergrad_linear": lambda h: [lib.cdgrab_pergrad_linear(h, x, d)],
        "orthogonalize": lambda h: [lib.cdgrab_orthogonalize(h, mats)],
        "pergrad": lambda h: [lib.cdgrab_pergrad(h, X, y, W)],
        "balance": lambda h: list(lib.cdgrab_balance_epoch(h, m, n, 600, grads=g, want_r64=True, want_dots=True).values()),
        "independent": lambda h: list(lib.cdgrab_balance_epoch_independent(h, g).values()),
        "stale_mean": lambda h: list(lib.cdgrab_balance_epoch_stale_mean(h, g.view(m * n, 600)).values()),
        "randomized": lambda h: list(lib.cdgrab_balance_epoch_randomized(h, g, u).values()),
        "reorder": lambda h: [lib.cdgrab_reorder(h, signs)],
        "herding": lambda h: [lib.cdgrab_herding_bound(h, g)],
        "train": lambda h: list(lib.cdgrab_train_epoch_softmax(h, X3, y2, W.clone(), want_grads=True).values()),
        "train_orthogonal": lambda h: list(lib.cdgrab_train_epoch_softmax_orthogonal(h, X3, y2, W.clone(), v.clone(),
                                                                                     want_grads=True).values()),
    }


@pytest.mark.parametrize("name", ["layernorm", "pergrad_layernorm", "pergrad_linear", "orthogonalize", "pergrad", "balance", "independent",
                                  "stale_mean", "randomized", "reorder", "herding", "train", "train_orthogonal"])
def test_outputs_do_not_take_the_current_streams_memory(lib, name):  # noqa: F811
    call = calls(lib)[name]
    want = [t.clone() for t in call(lib.Handle())]
    torch.cuda.synchronize()
    h = lib.Handle(stream=torch.cuda.Stream())  # not the current one
    at = let_go_of(h.device, want)
    got = call(h)
    assert not at & {t.data_ptr() for t in got}
    h.stream.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    # on the handle's own stream they come from there as ever
    with torch.cuda.stream(h.stream):
        for a, b in zip(call(h), want):
            assert torch.equal(a, b)
    h.stream.synchronize()


def test_an_output_is_kept_while_the_current_stream_reads_it(lib):  # noqa: F811
    """Let go of by the program, it goes back to the handle's stream only once the current stream has passed that point."""
    x = rand(1, 64, 1000)
    h = lib.Handle(stream=torch.cuda.Stream())
    for busy in (1000, 20_000_000):  # (cycles; the first time loads the kernels, which the host waits for)
        y = lib.cdgrab_layernorm(h, x)
        torch.cuda.current_stream().wait_stream(h.stream)
        at = y.data_ptr()
        torch.cuda._sleep(busy)
        z = y * 2
        read = torch.cuda.Event()
        read.record()
        del y
        again = [lib.cdgrab_layernorm(h, x) for _ in range(4)]
        waiting = not read.query()  # the current stream has not come to its reading yet
        torch.cuda.synchronize()
        assert torch.equal(z, again[0] * 2)
        if waiting:
            assert at not in {t.data_ptr() for t in again}
        del z, again
    assert waiting
