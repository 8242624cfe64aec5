"""GPU tests of the orthogonalised update on matrices whose rows or columns are of very different sizes, as an embedding's
gradient has them: the small ones keep their digits."""
import pytest
import torch

from test_gpu_orthogonal import COEFFS, TOL, by_products, lib, rand  # noqa: F401

pytestmark = pytest.mark.gpu


def uneven(seed, rows, cols, small, side, dtype=torch.float32):
    """A quarter of the rows (or columns) `small` of the others; and which elements those are."""
    m = rand(seed, rows, cols)
    part = torch.zeros(rows, cols, dtype=torch.bool)
    part[:rows // 4] = side == "rows"
    part[:, :cols // 4] |= side == "cols"
    m[part.cuda()] *= small
    return m.to(dtype), part


SHAPES = [(64, 64), (40, 200), (100, 128), (128, 250), (200, 300), (300, 200), (500, 700), (70, 9000)]


# TOL as there, for the small rows by themselves (a step makes them of terms of their own size), and the smallest number
# that an element is held to, 2^-49 of the matrix's norm each.
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("side,small", [("rows", 1e-3), ("rows", 1e-6), ("rows", 1e-7), ("cols", 1e-6), ("cols", 1e-8)])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_small_rows_and_columns(lib, rows, cols, side, small, dtype):  # noqa: F811
    m, part = uneven(rows, rows, cols, small, side, dtype)
    want = by_products(m)
    got = lib.cdgrab_orthogonalize(lib.Handle(), m).double().cpu()
    m = m.double().cpu()
    for which in (part, ~part):
        err = ((got - want)[which].norm() / want[which].norm()).item()
        least = 2.0 ** -49 * m.norm().item() * which.sum().item() ** 0.5 / m[which].norm().item()
        print("relative error %.2e, least number %.2e" % (err, least))
        assert err <= TOL + least + torch.finfo(dtype).eps / 2


@pytest.mark.parametrize("batch,rows,cols", [(3, 100, 128), (60, 200, 300), (4, 64, 90)])
def test_batches_of_uneven_rows(lib, batch, rows, cols):  # noqa: F811
    ms = [uneven(b, rows, cols, 1e-6, "rows") for b in range(batch)]
    out = lib.cdgrab_orthogonalize(lib.Handle(), torch.stack([m for m, _ in ms])).double().cpu()
    for b in (0, batch - 1):
        m, part = ms[b]
        want = by_products(m)
        assert ((out[b] - want)[part].norm() / want[part].norm()).item() <= TOL + 2.0 ** -28  # (the least number: 2^-49 / 2^-21)


# Over many steps small rows grow to the size of the others, and what was rounded off at the start with them: held to four
# times the error that the definition in fp32 has, and 64 roundings for matrices on which it happens to have none.
@pytest.mark.parametrize("small", [1e-3, 1e-5, 1e-7])
@pytest.mark.parametrize("rows,cols", [(64, 64), (100, 128), (200, 300), (300, 200)])
def test_many_steps_on_uneven_rows(lib, rows, cols, small):  # noqa: F811
    m, _ = uneven(rows, rows, cols, small, "rows")
    want = by_products(m, 16)
    x = m.cpu() if rows <= cols else m.cpu().t()
    x = x / x.square().sum().sqrt()
    for _ in range(16):
        g = x @ x.t()
        x = COEFFS[0] * x + (COEFFS[1] * g + COEFFS[2] * (g @ g)) @ x
    plain = (((x if rows <= cols else x.t()).double() - want).norm() / want.norm()).item()
    err = ((lib.cdgrab_orthogonalize(lib.Handle(), m, steps=16).double().cpu() - want).norm() / want.norm()).item()
    print("relative error %.2e, in fp32 %.2e" % (err, plain))
    assert err <= 4 * plain + 64 * 2.0 ** -24
