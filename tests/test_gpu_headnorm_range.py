"""GPU tests of head norms of small elements: without eps a head is as long as one of ordinary elements, however small its own are."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def lib():
    import paper_2302_00845_amd as p
    return p


def rand(seed, *shape, scale=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64) * scale).to(dtype).cuda()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dim", [6, 32, 80, 512])
@pytest.mark.parametrize("power,eps", [(-20, 0.0), (-50, 0.0), (-60, 0.0), (-72, 0.0), (-80, 0.0), (-100, 0.0), (-118, 0.0), (-72, 1e-43),
                                       (-60, 1e-36), (-70, 1e-42), (-72, 1e-20)])
def test_heads_of_small_elements(lib, power, eps, dim, dtype):
    n, tokens, hq, hk = 2, 9, 2, 1
    x = (rand(1, n, tokens, (hq + hk) * dim).double() * 2.0 ** power).to(dtype)
    x[1, 3, :dim] = rand(2, dim, dtype=dtype)  # a head of ordinary elements beside them
    dy = rand(3, n, tokens, (hq + hk) * dim, dtype=dtype)
    gq, gk = rand(4, dim), rand(5, dim)
    kw = dict(q_heads=hq, k_heads=hk, eps=eps, base=0.0)
    h = lib.Handle()
    y = lib.cdgrab_headnorm(h, x, gq, gk, **kw)
    dx, g = lib.cdgrab_pergrad_headnorm(h, x, dy, gq, gk, **kw)
    e32 = float(torch.tensor(eps, dtype=torch.float32))
    half = torch.finfo(dtype).eps / 2
    v, d = x.double().unflatten(-1, (hq + hk, dim)), dy.double().unflatten(-1, (hq + hk, dim))
    w = torch.cat([gq.double().expand(hq, -1), gk.double().expand(hk, -1)])
    r = 1.0 / (v.square().mean(-1, keepdim=True) + e32).sqrt()
    hat = v * r
    # the sum of squares has at most dim + 8 roundings, half of that on the deviation, which has three of its own
    rt = ((dim + 8) / 2 + 4) * U

    def check(got, want, tol, what):
        got = got.double().view(want.shape)
        inside = want.abs() < torch.finfo(dtype).max if what == "dx" else torch.ones_like(want, dtype=torch.bool)
        share = ((got - want).abs() / tol.clamp_min(1e-300))[inside].max().item() if inside.any() else 0.0
        print("%s: at most %.3f of the tolerance" % (what, share))
        assert torch.isfinite(got[inside]).all() and share <= 1.0
    check(y, hat * w, (hat * w).abs() * (rt + 3 * U + half * 1.01) + 1e-40, "y")
    q = d * w
    mean = (q * hat).mean(-1, keepdim=True)
    mean_err = ((q * hat).abs() * (rt + (dim + 8) * U)).mean(-1, keepdim=True)
    want = r * (q - hat * mean)
    tol = r * (q.abs() * (rt + 5 * U) + hat.abs() * (mean_err + mean.abs() * (2 * rt + 5 * U)))
    # (at these sizes only the largest dx are beyond what the type holds)
    check(dx, want, tol + half * want.abs() * 1.01, "dx")
    each, err = d * hat, (d * hat).abs() * (rt + 2 * U)
    for which, heads in ((0, slice(0, hq)), (1, slice(hq, hq + hk))):
        s, a = each[:, :, heads].sum((1, 2)), each[:, :, heads].abs().sum((1, 2))
        check(g[:, which * dim:(which + 1) * dim], s, err[:, :, heads].sum((1, 2)) + (tokens * hq + 8) * U * a, "G")


def test_heads_of_zeros(lib):
    x = torch.zeros(1, 3, 24, device="cuda")
    x[0, 1, :8] = 2.0 ** -126
    kw = dict(q_heads=3, k_heads=0, base=0.0)
    y = lib.cdgrab_headnorm(lib.Handle(), x, eps=0.0, **kw).view(3, 3, 8)
    assert (y[1, 0] - 1.0).abs().max() <= 8 * U and torch.isnan(y[0]).all() and torch.isnan(y[1, 1:]).all() and torch.isnan(y[2]).all()
    assert (lib.cdgrab_headnorm(lib.Handle(), x, eps=1e-6, **kw).view(3, 3, 8)[[0, 2]] == 0).all()
