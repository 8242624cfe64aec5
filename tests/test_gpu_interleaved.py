"""GPU tests of outputs that lie between the rows of an input without sharing an element: no overlap, and not refused."""
import pytest
import torch

from test_gpu_orthogonal import lib, rand  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("batch,rows,cols", [(1, 20, 30), (1, 785, 10), (3, 40, 50), (2, 150, 100), (1, 1, 9)])
def test_orthogonalize_beside_its_matrix(lib, batch, rows, cols):  # noqa: F811
    whole = torch.full((batch, rows, 2 * cols + 5), 3.0, device="cuda")
    m, out = whole[..., 2:2 + cols], whole[..., cols + 4:2 * cols + 4]
    m.copy_(rand(1, batch, rows, cols))
    before = m.clone()
    h = lib.Handle()
    want = lib.cdgrab_orthogonalize(h, before)
    if batch == 1:
        lib.cdgrab_orthogonalize(h, m[0], out=out[0])
    else:
        lib.cdgrab_orthogonalize(h, m, out=out)
    assert torch.equal(out, want) and torch.equal(m, before)
    assert (whole[..., :2] == 3.0).all() and (whole[..., 2 + cols:cols + 4] == 3.0).all() and (whole[..., 2 * cols + 4:] == 3.0).all()
    for shift in (1, cols - 1):  # these share elements
        with pytest.raises(lib.CdgrabError) as err:
            lib.cdgrab_orthogonalize(h, whole[..., :cols], out=whole[..., shift:shift + cols])
        assert err.value.code == -1 and "overlap" in str(err.value)
    if rows == 1:
        return
    with pytest.raises(lib.CdgrabError):  # a row of the output would reach into the next row of the input
        lib.cdgrab_orthogonalize(h, torch.as_strided(whole, (rows, cols), (2 * cols, 1)),
                                 out=torch.as_strided(whole, (rows, cols), (2 * cols, 1), cols + 1))


def test_one_gradient_row_beside_the_inputs(lib):  # noqa: F811
    whole = torch.zeros(6, 200, device="cuda")
    x, d = whole[:, :20], whole[:, 20:33]
    x.copy_(rand(1, 6, 20))
    d.copy_(rand(2, 6, 13))
    h = lib.Handle()
    x1, d1 = x[:, :10], d
    want = lib.cdgrab_pergrad_linear(h, x1.reshape(1, 6, 10), d1.reshape(1, 6, 13))
    G = whole[2:3, 40:40 + 143]  # in the second row, behind what is read
    lib.cdgrab_pergrad_linear(h, x1.unsqueeze(0), d1.unsqueeze(0), G_out=G)
    assert torch.equal(G, want)
    with pytest.raises(lib.CdgrabError):  # and over the row's end
        lib.cdgrab_pergrad_linear(h, x1.unsqueeze(0), d1.unsqueeze(0), G_out=torch.as_strided(whole, (1, 143), (143, 1), 260))
    dy, out = whole[:, 100:110], whole[4:5, 190:200]
    dy.zero_()
    lib.cdgrab_pergrad_layernorm(h, x1.unsqueeze(0), dy.unsqueeze(0), G_out=out, with_bias=False, want_dx=False)
    assert (out == 0).all()
