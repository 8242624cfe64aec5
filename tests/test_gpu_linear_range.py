"""GPU tests of per-example linear gradients on values near the ends of their types' ranges."""
import pytest
import torch

from test_gpu_layers import U, close, lib, rand  # noqa: F401

pytestmark = pytest.mark.gpu

SHAPES = [(1, 700, 10), (2, 40, 30), (8, 30, 40), (20, 130, 20), (20, 20, 130), (40, 64, 80), (300, 200, 150)]  # each kernel


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("tokens,n_in,n_out", SHAPES)
def test_linear_of_infinities(lib, tokens, n_in, n_out, dtype):  # noqa: F811
    """What an infinity enters is infinite or NaN, and nothing else is."""
    x, d = rand(1, 3, tokens, n_in, dtype=dtype), rand(2, 3, tokens, n_out, dtype=dtype)
    x[1, 0, 3] = float("inf")
    d[2, tokens - 1, 5] = -float("inf")
    g = lib.cdgrab_pergrad_linear(lib.Handle(), x, d).view(3, n_in + 1, n_out)
    bad = torch.zeros_like(g, dtype=torch.bool)
    bad[1, 3] = True
    bad[2, :, 5] = True
    assert not torch.isfinite(g[bad]).any() and torch.isfinite(g[~bad]).all()


@pytest.mark.parametrize("exponent", [100, 106])
@pytest.mark.parametrize("tokens,n_in,n_out", SHAPES)
def test_linear_of_small_numbers(lib, tokens, n_in, n_out, exponent):  # noqa: F811
    """Products near one of factors near the ends of the range, whose parts are among the numbers below the normal ones."""
    x, d = rand(1, 2, tokens, n_in) * 2.0 ** -exponent, rand(2, 2, tokens, n_out) * 2.0 ** exponent
    g = lib.cdgrab_pergrad_linear(lib.Handle(), x, d, with_bias=False).view(2, n_in, n_out)
    a, c = x.double().transpose(1, 2).contiguous(), d.double()
    close(g, a @ c, ((2 * tokens + 64) * U + 2.0 ** -21) * (a.abs() @ c.abs()), "G")
