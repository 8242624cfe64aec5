"""GPU tests of attention's large scores: weights, sums and gradients against formulas in 64 bits.  The elements are such that a score has
no error of its own: whole numbers and powers of two."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24  # half a step of fp32, relative
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def lib():
    import paper_2302_00845_amd as p
    return p


def step(dtype):
    return torch.finfo(dtype).eps / 2


def tiny(dtype):
    return torch.finfo(dtype).tiny * torch.finfo(dtype).eps  # a step of the numbers below the normal ones


def rand(seed, *shape, dtype, scale=1.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64) * scale).to(dtype).cuda()


def whole(seed, *shape, dtype, most=2, times=1.0):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randint(-most, most + 1, shape, generator=gen).double() * times).to(dtype).cuda()


def close(got, want, tol, what):
    got, want, tol = got.double(), want.double(), tol.double()
    share = ((got - want).abs() / tol.clamp_min(1e-300)).max().item()
    print("%s: at most %.3f of the tolerance" % (what, share))
    assert torch.isfinite(got).all() and share <= 1.0


def weights64(q, k, scale):
    n = q.shape[0]
    seen = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
    s = (q.double() @ k.double().t() * scale).where(seen, -math.inf)
    p = torch.exp(s - s.amax(1, keepdim=True))  # (of scores beyond 2^53 their logarithm's sum would not show in lse)
    return s, torch.logsumexp(s, 1, keepdim=True), p / p.sum(1, keepdim=True)


def check_forward(lib, q, k, v, scale):
    n, dim = q.shape
    dtype = q.dtype
    o, lse = lib.cdgrab_attention(lib.Handle(), q.unsqueeze(0), k.unsqueeze(0), v.unsqueeze(0), q_heads=1, kv_heads=1, scale=scale)
    _, want_lse, p = weights64(q, k, float(torch.tensor(scale)))
    want = p @ v.double()
    # An exponent x is a difference of scores times a factor: with the factor's rounding and its own, and with what a row's maximum
    # is off while it lags behind, 4 U |x| + 4 U in all.  p x has its maximum at 1 / e, and exponents beyond 160 no weight in fp32,
    # so 4 U (160 + 1) of p is ample; an exponential is good to two steps, a sum of n to n U.
    ep = 4 * 161 * U + (2 * n + 8) * U + step(dtype)
    low = 2.0 ** -32 if dtype == torch.float16 else 0.0  # of a weight, absolute: below fp16's normal numbers
    close(o[0], want, (p * ep + low) @ v.double().abs() + step(dtype) * want.abs() * 1.01 + tiny(dtype), "o")
    # the maximum, times the factor, plus the logarithm, each rounded
    close(lse[0, 0], want_lse.squeeze(1), 6 * U * want_lse.squeeze(1).abs() + (2 * n + 700) * U, "lse")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [40, 64, 97])
@pytest.mark.parametrize("times,scale", [(1.0, 10.0), (1.0, 1e3), (1.0, 1e5), (1.0, 1e7), (1.0, 1e9), (1.0, 1e30), (1024.0, 0.125)])
def test_weights_of_large_scores(lib, times, scale, dim, dtype):
    n = 330
    check_forward(lib, whole(1, n, dim, dtype=dtype, times=times), whole(2, n, dim, dtype=dtype, times=times), rand(3, n, dim, dtype=dtype),
                  scale)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_weights_of_scores_that_grow(lib, sign, dtype):
    """Scores from 1 to 2^28 along the keys, or from -2^28 to -1, sixteen of each: the largest ones come last, the smaller ones have
    weights as well while they are small."""
    n, dim = 464, 64
    q, k = torch.zeros(n, dim, dtype=dtype, device="cuda"), torch.zeros(n, dim, dtype=dtype, device="cuda")
    power = torch.arange(n, device="cuda") // 16
    q[:, 5] = 2.0 ** 13
    k[:, 5] = (sign * 2.0 ** ((power if sign > 0 else power.flip(0)) - 13).double()).to(dtype)
    check_forward(lib, q, k, rand(4, n, dim, dtype=dtype), 1.0)
    check_forward(lib, q, k.flip(0).contiguous(), rand(4, n, dim, dtype=dtype), 1.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [40, 64, 128])
@pytest.mark.parametrize("most", [2.0 ** 10, 2.0 ** 16])
def test_gradients_of_large_scores(lib, most, dim, dtype):
    """Up to the largest scores for which gradients are promised."""
    n = 200
    q, k = whole(5, n, dim, dtype=dtype), whole(6, n, dim, dtype=dtype)
    v, do = rand(7, n, dim, dtype=dtype), rand(8, n, dim, dtype=dtype, scale=0.01)
    scale = most / (q.double() @ k.double().t()).tril().abs().max().item()
    scale = float(torch.tensor(scale)) * (1 - 2 * U)
    h = lib.Handle()
    kw = dict(q_heads=1, kv_heads=1, scale=scale)
    x = [t.unsqueeze(0) for t in (q, k, v)]
    o, lse = lib.cdgrab_attention(h, *x, **kw)
    dq, dk, dv = (t[0] for t in lib.cdgrab_attention_backward(h, *x, o, lse, do.unsqueeze(0), **kw))
    check_forward(lib, q, k, v, scale)
    scale = float(torch.tensor(scale))
    s, want_lse, p = weights64(q, k, scale)
    seen = torch.isfinite(s)
    q, k, v, do = (t.double() for t in (q, k, v, do))
    half = step(dtype)
    # a weight that the type does not hold (fp16: 2^-14 times as large), or p (do v - D), is lost: below 2^-126 also those of bf16 and fp32
    low = (2.0 ** -32 if dtype == torch.float16 else 2.0 ** -126) * seen
    o = p @ v
    tol_o = (p * (half + 1100 * U) + low) @ v.abs() + half * o.abs() * 1.01 + tiny(dtype)
    D = (do * o).sum(1, keepdim=True)
    dp = do @ v.t()
    ds = (p * (dp - D)).where(seen, 0.0)
    # the weights' error that is promised, of scores and lse, and two steps of the exponential; relative, as exp(x) - 1
    ep = torch.expm1(2.0 ** -18 * (want_lse.abs() + s.where(seen, 0.0).abs()) + 16 * U)
    eD = (do.abs() * tol_o).sum(1, keepdim=True) + (dim + 2) * U * (do * o).abs().sum(1, keepdim=True)
    # (the first rows take D's error back by the weights' own sum, which is off by as much as they are)
    eD = eD + (p * (ep + half) * (dp - D).abs()).where(seen, 0.0).sum(1, keepdim=True) * (1 + ep.amax())
    eds = p * (1 + ep) * ((dim + 12) * U * (do.abs() @ v.abs().t()) + eD) * (1 + half) + ds.abs() * (ep + 2 * U + half) * (1 + half)
    if dtype == torch.float16:
        eds = eds + 2.0 ** -38 * torch.maximum(ds.abs().amax(0, keepdim=True), ds.abs().amax(1, keepdim=True)) * (1 + ep.amax())
    eds = eds + low * (dp - D).abs() + 2.0 ** -126 if dtype != torch.float16 else eds
    eds = (eds + (n + 4) * U * ds.abs()).where(seen, 0.0)
    for name, got, want, tol in (("dq", dq, ds @ k * scale, scale * eds @ k.abs()), ("dk", dk, ds.t() @ q * scale, scale * eds.t() @ q.abs()),
                                 ("dv", dv, p.t() @ do, (p * (ep + half * (1 + ep) + (n + 4) * U) + low).t() @ do.abs())):
        close(got, want, tol + half * want.abs() * 1.01 + tiny(dtype), name)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_beside_a_query_that_is_not_finite(lib, dtype):
    """Queries share nothing but their keys: the others' rows are as good as without it, at large scores too."""
    n, dim = 330, 40
    q, k, v = whole(1, n, dim, dtype=dtype), whole(2, n, dim, dtype=dtype), rand(3, n, dim, dtype=dtype)
    q[0], q[140] = float("nan"), float("inf")
    others = torch.ones(n, dtype=torch.bool, device="cuda")
    others[0] = others[140] = False
    for scale in (0.5, 1e9):
        o, lse = lib.cdgrab_attention(lib.Handle(), q.unsqueeze(0), k.unsqueeze(0), v.unsqueeze(0), q_heads=1, kv_heads=1, scale=scale)
        s, want_lse, p = weights64(q, k, float(torch.tensor(scale)))
        want, size = (p @ v.double())[others], ((p * (4 * 161 * U + (2 * n + 8) * U + step(dtype)) + 2.0 ** -32) @ v.double().abs())[others]
        close(o[0][others], want, size + step(dtype) * want.abs() * 1.01 + tiny(dtype), "o")
        close(lse[0, 0][others], want_lse.squeeze(1)[others], 6 * U * want_lse.squeeze(1)[others].abs() + (2 * n + 700) * U, "lse")
        assert not torch.isfinite(o[0][~others]).any()
