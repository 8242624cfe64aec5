"""GPU tests of the orthogonalised update on large arrays, and on numbers below the normal ones."""
import pytest
import torch

from test_gpu_orthogonal import COEFFS, TOL, by_products, check, lib, rand  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols,distance", [(5, 24, 600_000_000), (70, 80, 32_000_000), (80, 70, 28_000_000), (140, 150, 15_500_000),
                                                (60, 900, 36_500_000)])
@pytest.mark.parametrize("steps", [0, 5, 9])
def test_rows_beyond_31_bits_of_elements(lib, rows, cols, distance, steps):  # noqa: F811
    """Rows of M and O as far apart as that, in one array."""
    big = torch.zeros(rows * distance, dtype=torch.bfloat16, device="cuda")
    assert (rows - 1) * distance >= 1 << 31
    m, out = torch.as_strided(big, (rows, cols), (distance, 1)), torch.as_strided(big, (rows, cols), (distance, 1), cols + 3)
    m.copy_(rand(rows, rows, cols, dtype=torch.bfloat16))
    h = lib.Handle()
    lib.cdgrab_orthogonalize(h, m, steps=steps, out=out)
    assert torch.equal(out, lib.cdgrab_orthogonalize(h, m.contiguous(), steps=steps))
    out.zero_()
    m.zero_()
    assert not big.any()


def test_elements_beyond_31_bits(lib):  # noqa: F811
    """2100 x 2^20: offsets of elements and of pairs, and the columns' sums in fp32."""
    rows, cols, part = 2100, 1 << 20, 1 << 17
    gen = torch.Generator(device="cuda").manual_seed(3)
    m = torch.randn(rows, cols, generator=gen, device="cuda")
    out = lib.cdgrab_orthogonalize(lib.Handle(), m, steps=1)
    norm = sum(m[:, c:c + part].double().square().sum() for c in range(0, cols, part)).sqrt()
    gram = torch.zeros(rows, rows, dtype=torch.float64, device="cuda")
    for c in range(0, cols, part):
        x = m[:, c:c + part].double() / norm
        gram += x @ x.t().contiguous()
    factor = COEFFS[1] * gram + COEFFS[2] * (gram @ gram)
    err = total = 0.0
    for c in range(0, cols, part):
        x = m[:, c:c + part].double() / norm
        want = COEFFS[0] * x + factor @ x
        err += (out[:, c:c + part] - want).square().sum().item()
        total += want.square().sum().item()
    print("relative error %.2e" % (err / total) ** 0.5)
    assert (err / total) ** 0.5 <= TOL


@pytest.mark.parametrize("rows,cols", [(3, 1 << 20), (1 << 20, 20), (40, 1 << 19)])
def test_the_longest_sides(lib, rows, cols):  # noqa: F811
    m = rand(1, rows, cols)
    check(lib.cdgrab_orthogonalize(lib.Handle(), m), m, torch.float32)


@pytest.mark.parametrize("size", [1e-38, 1e-41])
@pytest.mark.parametrize("rows,cols", [(12, 40), (64, 64), (60, 900), (100, 128), (200, 150)])
@pytest.mark.parametrize("steps", [0, 5])
def test_numbers_below_the_normal_ones(lib, rows, cols, size, steps):  # noqa: F811
    m = (rand(rows, rows, cols, dtype=torch.float64) * size).float()
    check(lib.cdgrab_orthogonalize(lib.Handle(), m, steps=steps), m, torch.float32, steps)
