"""GPU tests of layer norm on rows whose squares are beyond fp32."""
import pytest
import torch

from test_gpu_layers import lib, rand  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("width", [3, 40, 515, 1000, 6001])
@pytest.mark.parametrize("size", [1e20, 1e38])
def test_layernorm_rows_too_large_for_their_squares(lib, width, size, dtype):  # noqa: F811
    """Squares beyond fp32: the deviation is not known, and the row says so instead of becoming the bias."""
    x, dy = rand(1, 3, 4, width, dtype=dtype), rand(2, 3, 4, width, dtype=dtype)
    x[1, 2] = (torch.arange(width, device="cuda") % 2 * 2 - 1) * size
    w, b = rand(3, width, offset=1.0), rand(4, width)
    h = lib.Handle()
    y = lib.cdgrab_layernorm(h, x, w, b)
    dx, g = lib.cdgrab_pergrad_layernorm(h, x, dy, w)
    bad = torch.zeros(3, 4, dtype=torch.bool, device="cuda")
    bad[1, 2] = True
    assert torch.isnan(y[bad]).all() and torch.isnan(dx[bad]).all() and torch.isnan(g[1, :width]).all()
    assert torch.isfinite(y[~bad]).all() and torch.isfinite(dx[~bad]).all()
    assert torch.isfinite(g[[0, 2]]).all() and torch.isfinite(g[:, width:]).all()
