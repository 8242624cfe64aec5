"""GPU tests of the sequence operators against plain formulas in 64 bits: embedding, norms of heads with the position rotation, causal
attention, forward and backward; dense, padded and packed examples, odd sizes, strides, empty examples, garbage in rows of no example."""
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


def rand(seed, *shape, scale=1.0, offset=0.0, dtype=torch.float32):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=gen, dtype=torch.float64) * scale + offset).to(dtype).cuda()


def step(dtype):
    return torch.finfo(dtype).eps / 2


def tiny(dtype):
    return torch.finfo(dtype).tiny * torch.finfo(dtype).eps  # a step of the numbers below the normal ones


def close(got, want, tol, what):
    """|got - want| <= tol, element by element; the worst as a share of its tolerance is printed."""
    got, want, tol = got.double(), want.double(), tol.double()
    share = ((got - want).abs() / tol.clamp_min(1e-300)).max().item() if got.numel() else 0.0
    print("%s: at most %.3f of the tolerance" % (what, share))
    assert torch.isfinite(got).all() and share <= 1.0


def layout(kind, counts, tokens):
    """(spans, rows, keywords of the call); the packed rows have a row of no example between examples and behind them."""
    n = len(counts)
    if kind == "dense":
        return [(e * tokens, tokens) for e in range(n)], n * tokens, {}
    count = torch.tensor(counts, dtype=torch.int32, device="cuda")
    if kind == "padded":
        return [(e * tokens, c) for e, c in enumerate(counts)], n * tokens, {"count": count}
    first, at = [], 1
    for c in counts:
        first.append(at)
        at += c + 1
    return list(zip(first, counts)), at + 2, {"first": torch.tensor(first, dtype=torch.int64, device="cuda"), "count": count,
                                             "tokens": tokens}


def shaped(kind, rows, n, tokens):
    """[rows][..] as the call takes it."""
    return rows if kind == "packed" else rows.unflatten(0, (n, tokens))


def owned(spans, rows):
    mask = torch.zeros(rows, dtype=torch.bool, device="cuda")
    for at, count in spans:
        mask[at:at + count] = True
    return mask


# ---- embedding --------------------------------------------------------------------------------------

@pytest.mark.parametrize("rows,vocab,width", [(1, 1, 1), (5, 3, 3), (7, 11, 4), (130, 50, 7), (33, 1000, 64), (65, 17, 129),
                                              (3, 5, 1000), (300, 70, 2050), (0, 4, 8)])
@pytest.mark.parametrize("kinds", [(torch.float32, torch.float32), (torch.float32, torch.bfloat16), (torch.float32, torch.float16),
                                   (torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16)])
def test_embed(lib, rows, vocab, width, kinds):
    table = rand(1, vocab, width, dtype=kinds[0])
    ids = torch.randint(-2, vocab + 2, (rows,), generator=torch.Generator().manual_seed(2)).int().cuda()
    y = lib.cdgrab_embed(lib.Handle(), ids, table, scale=1.7, dtype=kinds[1])
    known = (ids >= 0) & (ids < vocab)
    want = torch.where(known.unsqueeze(1), table.double()[ids.long().clamp(0, vocab - 1)] * float(torch.tensor(1.7)), 0.0)
    # the product's rounding, and the type's
    close(y, want, (U + step(kinds[1])) * want.abs() * 1.01 + tiny(kinds[1]), "y")
    assert y.dtype == kinds[1] and (y[~known] == 0).all()


def test_embed_strides_and_shapes(lib):
    h = lib.Handle()
    wide, out = rand(3, 40, 90), torch.full((6, 5, 70), 7.0, device="cuda")
    ids = torch.randint(0, 40, (6, 5), generator=torch.Generator().manual_seed(4)).int().cuda()
    lib.cdgrab_embed(h, ids, wide[:, 11:48], Y=out[..., 3:40])
    assert torch.equal(out[..., 3:40], wide[:, 11:48][ids.long()]) and (out[..., :3] == 7).all() and (out[..., 40:] == 7).all()
    assert lib.cdgrab_embed(h, ids[0, 0], wide).shape == (90,)


def embed_case(lib, n, tokens, vocab, width, kind, dtype, seed=5, same=None, G_out=None):
    gen = torch.Generator().manual_seed(seed)
    counts = torch.randint(0, tokens + 1, (n,), generator=gen).tolist()
    counts[0] = tokens
    if n > 1:
        counts[-1] = 0
    spans, rows, kw = layout(kind, counts, tokens)
    ids = torch.randint(-1, vocab + 1, (rows,), generator=gen).int().cuda()
    if same is not None:
        ids[torch.rand(rows, generator=gen).cuda() < 0.7] = same
    dy = rand(seed + 1, rows, width, dtype=dtype)
    mask = owned(spans, rows)
    dy[~mask] = float("nan")
    want = torch.zeros(n, vocab, width, dtype=torch.float64, device="cuda")
    sums, number = torch.zeros_like(want), torch.zeros(n, vocab, 1, dtype=torch.float64, device="cuda")
    for e, (at, count) in enumerate(spans):
        part, d = ids[at:at + count].long(), dy[at:at + count].double()
        part, d = part[(part >= 0) & (part < vocab)], d[(part >= 0) & (part < vocab)]
        want[e].index_put_((part,), d, accumulate=True)
        sums[e].index_put_((part,), d.abs(), accumulate=True)
        number[e].index_put_((part,), torch.ones_like(d[:, :1]), accumulate=True)
    h = lib.Handle()
    g = lib.cdgrab_pergrad_embed(h, shaped(kind, ids, n, tokens), shaped(kind, dy, n, tokens), vocab, scale=0.3, G_out=G_out, **kw)
    f = float(torch.tensor(0.3))
    # a rounding per addition at the most, and the product's
    close(g.reshape(n, vocab, width), want * f, (number + 2) * U * sums * f + 1e-40, "G")
    assert (g.reshape(n, vocab, width)[number.expand_as(want) == 0] == 0).all()
    again = lib.cdgrab_pergrad_embed(h, shaped(kind, ids, n, tokens), shaped(kind, dy, n, tokens), vocab, scale=0.3, **kw)
    assert torch.equal(g, again)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["dense", "padded", "packed"])
@pytest.mark.parametrize("n,tokens,vocab,width", [(1, 1, 1, 1), (3, 5, 7, 3), (4, 33, 50, 20), (2, 130, 3, 65), (9, 64, 300, 129),
                                                  (2, 2048, 700, 8), (3, 2049, 90, 37)])
def test_pergrad_embed(lib, n, tokens, vocab, width, kind, dtype):
    embed_case(lib, n, tokens, vocab, width, kind, dtype)


@pytest.mark.parametrize("tokens,vocab,width,same", [
    (2000, 40, 130, 7),      # one id nearly everywhere
    (5000, 9, 260, 3), (70000, 5000, 12, 100), (4096, 3000, 1, 0), (20000, 70000, 2, 69999), (9000, 2, 1500, 1)])
@pytest.mark.parametrize("kind", ["dense", "packed"])
def test_pergrad_embed_of_long_examples(lib, tokens, vocab, width, same, kind):
    embed_case(lib, 2, tokens, vocab, width, kind, torch.bfloat16, same=same)


def test_pergrad_embed_into_longer_rows(lib):
    whole = torch.full((4, 1 + 50 * 20 + 6), 5.0, device="cuda")
    embed_case(lib, 4, 33, 50, 20, "padded", torch.float32, G_out=whole[:, 1:1001])
    assert (whole[:, 0] == 5).all() and (whole[:, 1001:] == 5).all()


def test_pergrad_embed_of_overlapping_examples(lib):
    ids = torch.tensor([0, 1, 2, 1, 0, 3], dtype=torch.int32, device="cuda")
    dy = rand(8, 6, 5)
    g = lib.cdgrab_pergrad_embed(lib.Handle(), ids, dy, 4, first=torch.tensor([0, 2, 2], device="cuda"),
                                 count=torch.tensor([4, 4, 2], dtype=torch.int32, device="cuda"), tokens=4).view(3, 4, 5)
    assert torch.equal(g[0], torch.stack([dy[0], dy[1] + dy[3], dy[2], 0 * dy[0]]))
    assert torch.equal(g[1], torch.stack([dy[4], dy[3], dy[2], dy[5]]))
    assert torch.equal(g[2], torch.stack([0 * dy[0], dy[3], dy[2], 0 * dy[0]]))


# ---- norms of heads, with the rotation --------------------------------------------------------------

def turned(u, positions, base, back=False):
    half = u.shape[-1] // 2
    angle = positions.double().view(-1, 1, 1) * (base ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half) if base else 0.0)
    angle = angle.expand(-1, 1, half)
    c, s = angle.cos(), (-angle if back else angle).sin()
    a, b = u[..., :half], u[..., half:]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def pair_sum(u):
    """|u_i| + |u_{i + dim/2}|, of both places."""
    a = u.abs()
    half = a.shape[-1] // 2
    return torch.cat([a[..., :half] + a[..., half:]] * 2, -1)


def heads_case(lib, n, tokens, hq, hk, dim, kind, dtype, base=10000.0, eps=1e-6, gains=True, seed=11):
    gen = torch.Generator().manual_seed(seed)
    counts = torch.randint(0, tokens + 1, (n,), generator=gen).tolist()
    counts[0] = tokens
    if n > 1:
        counts[-1] = 0
    spans, rows, kw = layout(kind, counts, tokens)
    mask = owned(spans, rows)
    width = (hq + hk) * dim
    x = rand(seed + 1, rows, width + 9, offset=0.3, dtype=dtype)[:, 5:5 + width]  # (odd addresses, long strides)
    dy = rand(seed + 2, rows, width, scale=0.1, dtype=dtype)
    x[~mask] = float("nan")
    dy[~mask] = float("nan")
    gq, gk = (rand(seed + 3, dim, scale=0.2, offset=1.0), rand(seed + 4, dim, scale=0.2, offset=-1.0)) if gains else (None, None)
    h = lib.Handle()
    kw = dict(kw, q_heads=hq, k_heads=hk, eps=eps, base=base)
    xx, dd = shaped(kind, x, n, tokens), shaped(kind, dy, n, tokens)
    y = lib.cdgrab_headnorm(h, xx, gq, gk, **kw)
    dx, g = lib.cdgrab_pergrad_headnorm(h, xx, dd, gq, gk, **kw)
    y, dx = y.reshape(rows, hq + hk, dim), dx.reshape(rows, hq + hk, dim)
    if kind != "dense":
        assert (y[~mask] == 0).all() and (dx[~mask] == 0).all()
    e32 = float(torch.tensor(eps))
    one = torch.ones(dim, dtype=torch.float64, device="cuda")
    w = torch.cat([(gq.double() if gains else one).expand(hq, -1), (gk.double() if gains else one).expand(hk, -1)])
    # the sum of squares has at most dim + 8 roundings, half of that on the deviation, which has three of its own
    rt = ((dim + 8) / 2 + 4) * U
    for e, (at, count) in enumerate(spans):
        if not count:
            assert (g[e] == 0).all()
            continue
        part = slice(at, at + count)
        v, d = x[part].double().view(count, hq + hk, dim), dy[part].double().view(count, hq + hk, dim)
        r = 1.0 / (v.square().mean(-1, keepdim=True) + e32).sqrt()
        hat, pos = v * r, torch.arange(count, device="cuda")
        want = turned(hat * w, pos, base)
        # a cosine and a sine are good to 4 U (a term of the series each, the angle); two products and a sum
        close(y[part], want, pair_sum(hat * w) * (rt + 8 * U) + step(dtype) * want.abs() * 1.01 + tiny(dtype), "y")
        u = turned(d, pos, base, back=True)
        eu = pair_sum(d) * 8 * U
        q = u * w
        mean = (q * hat).mean(-1, keepdim=True)
        mean_err = (eu * w.abs() * hat.abs() + (q * hat).abs() * (rt + (dim + 8) * U)).mean(-1, keepdim=True)
        want = r * (q - hat * mean)
        tol = r * (w.abs() * eu + q.abs() * (rt + 4 * U) + hat.abs() * (mean_err + mean.abs() * (2 * rt + 4 * U)))
        close(dx[part], want, tol + step(dtype) * want.abs() * 1.01 + tiny(dtype), "dx")
        each, err = u * hat, eu * hat.abs() + (u * hat).abs() * (rt + 2 * U)
        for which, heads in ((0, slice(0, hq)), (1, slice(hq, hq + hk))):
            s, a = each[:, heads].sum((0, 1)), each[:, heads].abs().sum((0, 1))
            close(g[e, which * dim:(which + 1) * dim], s, err[:, heads].sum((0, 1)) + (count * (hq + hk) + 8) * U * a + 1e-38, "G")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["dense", "padded", "packed"])
@pytest.mark.parametrize("n,tokens,hq,hk,dim", [(1, 1, 1, 0, 2), (3, 7, 2, 1, 6), (2, 33, 4, 2, 22), (5, 40, 3, 3, 32), (2, 130, 12, 12, 64),
                                                (3, 65, 8, 2, 80), (2, 19, 1, 4, 128), (2, 9, 0, 5, 200), (1, 17, 2, 2, 512)])
def test_heads(lib, n, tokens, hq, hk, dim, kind, dtype):
    heads_case(lib, n, tokens, hq, hk, dim, kind, dtype)


@pytest.mark.parametrize("base,eps,gains", [(0.0, 1e-6, True), (1.0, 1e-5, False), (5e5, 0.0, True), (10000.0, 1e-3, False)])
def test_heads_other_parameters(lib, base, eps, gains):
    heads_case(lib, 2, 50, 3, 2, 48, "padded", torch.float32, base=base, eps=eps, gains=gains)


def test_heads_at_far_positions(lib):
    # an fp32 angle of 130 000 radians would be 0.004 off
    heads_case(lib, 1, 130_000, 1, 1, 16, "dense", torch.float32)


def test_heads_by_differences(lib):
    h = lib.Handle()
    x, dy, gq, gk = rand(1, 1, 5, 3 * 8).double(), rand(2, 1, 5, 3 * 8), rand(3, 8, offset=1.0), rand(4, 8, offset=1.0)
    kw = dict(q_heads=2, k_heads=1, eps=1e-3)
    dx, g = lib.cdgrab_pergrad_headnorm(h, x.float(), dy, gq, gk, **kw)
    move = 2.0 ** -6

    def value(xx, q):
        return (lib.cdgrab_headnorm(h, xx.float(), q, gk, **kw).double() * dy.double()).sum().item()
    # central differences: the third derivative, at most about 60 of these terms' size, times move^2 / 6; roundings over move
    size = dy.abs().sum().item()
    for i in range(0, 24, 5):
        d = torch.zeros_like(x)
        d[0, 3, i] = move
        got = (value(x + d, gq) - value(x - d, gq)) / (2 * move)
        assert abs(got - dx[0, 3, i].item()) <= 60 * move ** 2 / 6 * dy[0, 3].abs().max().item() + 8 * U * size / move
    for i in range(8):
        d = torch.zeros_like(gq)
        d[i] = move
        got = (value(x, gq + d) - value(x, gq - d)) / (2 * move)  # (linear in the gain)
        assert abs(got - g[0, i].item()) <= 8 * U * size / move


# ---- attention --------------------------------------------------------------------------------------

def attention64(q, k, v, do, scale, dtype):
    """One head of one example in 64 bits, and tolerances.  q, k, v, do [count][dim]."""
    n, dim = q.shape
    q, k, v, do = (x.double() for x in (q, k, v, do))
    seen = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
    s = (q @ k.t() * scale).where(seen, -math.inf)
    lse = torch.logsumexp(s, 1, keepdim=True)
    p = torch.exp(s - lse)
    o = p @ v
    # A score is a sum of dim products, of fp32 elements each with an error of 2^-22 (six of nine products of parts); its
    # exponent, in base 2, is rounded once and has that of the row's maximum taken off; an exponential has an error of two steps.
    size = ((q.abs() @ k.abs().t()) * scale).where(seen, 0.0)
    ds_ = (dim + 8 + (4 if dtype == torch.float32 else 0)) * U * size + 4 * U * (size.amax(1, keepdim=True) + 1)
    worst = ds_.amax(1, keepdim=True)
    ep = ds_ + worst + (n + 8) * U           # relative, of a normalised weight
    low = 2.0 ** -32 if dtype == torch.float16 else 0.0  # of a weight, absolute: below fp16's normal numbers
    half = step(dtype)
    tol_o = (p * (ep + half + n * U) + low) @ v.abs() + half * o.abs() * 1.01 + tiny(dtype)
    tol_lse = worst + (n + 8) * U + 4 * U * lse.abs()
    # backward: from the rounded outputs and sums
    dp = do @ v.t()
    D = (do * o).sum(1, keepdim=True)
    eD = (do.abs() * tol_o).sum(1, keepdim=True) + (dim + 2) * U * (do * o).abs().sum(1, keepdim=True)
    ds = (p * (dp - D)).where(seen, 0.0)
    p = p.where(seen, 0.0)
    eb = ds_ + tol_lse + 8 * U
    eds = p * ((dim + 12) * U * (do.abs() @ v.abs().t()) + eD) * (1 + half) + ds.abs() * (eb + 2 * U + half)
    if dtype == torch.float16:  # scaled so that a column's largest is 2^14 or more
        eds = eds + 2.0 ** -38 * torch.maximum(ds.abs().amax(0, keepdim=True), ds.abs().amax(1, keepdim=True))
    eds = eds.where(seen, 0.0)
    dq, dk, dv = ds @ k * scale, ds.t() @ q * scale, p.t() @ do
    tol = {
        "o": tol_o, "lse": tol_lse.squeeze(1),
        "dq": scale * (eds + (n + 4) * U * ds.abs()) @ k.abs(),
        "dk": scale * (eds + (n + 4) * U * ds.abs()).t() @ q.abs(),
        "dv": ((p * (eb + half + (n + 4) * U) + low * seen).t()) @ do.abs(),
    }
    return {"o": o, "lse": lse.squeeze(1), "dq": dq, "dk": dk, "dv": dv}, tol


def check_attention(lib, spans, rows, kw, kind, n, tokens, q, k, v, do, hq, hk, scale=None, h=None):
    dim, dtype = q.shape[-1] // hq, q.dtype
    h = h or lib.Handle()
    kw = dict(kw, q_heads=hq, kv_heads=hk, scale=scale)
    qq, kk, vv, dd = (shaped(kind, x, n, tokens) for x in (q, k, v, do))
    o, lse = lib.cdgrab_attention(h, qq, kk, vv, **kw)
    grads = lib.cdgrab_attention_backward(h, qq, kk, vv, o, lse, dd, **kw)
    got = {"o": o.reshape(rows, hq, dim), "lse": lse.reshape(hq, rows).t()}
    got.update(zip(("dq", "dk", "dv"), (x.reshape(rows, -1, dim) for x in grads)))
    scale = float(torch.tensor(scale or dim ** -0.5))
    want = {name: torch.zeros(x.shape, dtype=torch.float64, device="cuda") for name, x in got.items()}
    tols = {name: torch.full(x.shape, 1e-300, dtype=torch.float64, device="cuda") for name, x in got.items()}
    heads = [x.unflatten(1, (-1, dim)) for x in (q, k, v, do)]
    for at, count in spans:
        if not count:
            continue
        part = slice(at, at + count)
        for j in range(hq):
            g = j // (hq // hk)
            w, t = attention64(heads[0][part, j], heads[1][part, g], heads[2][part, g], heads[3][part, j], scale, dtype)
            for name in want:
                to = g if name in ("dk", "dv") else j
                want[name][part, to] += w[name]
                tols[name][part, to] += t[name]
    for name in ("dq", "dk", "dv"):
        tols[name] += step(dtype) * want[name].abs() * 1.01 + tiny(dtype)
    for name in want:
        close(got[name], want[name], tols[name], name)
    again = lib.cdgrab_attention_backward(h, qq, kk, vv, o, lse, dd, **kw)
    assert all(torch.equal(a, b) for a, b in zip(grads, again))
    return got


def attention_inputs(seed, spans, rows, hq, hk, dim, dtype):
    """Queries, keys and values side by side in one array's rows; NaN in rows of no example."""
    every = rand(seed, rows, (hq + 2 * hk) * dim, dtype=dtype)
    do = rand(seed + 1, rows, hq * dim, scale=0.01, dtype=dtype)
    mask = owned(spans, rows)
    every[~mask] = float("nan")
    do[~mask] = float("nan")
    return (*every.split([hq * dim, hk * dim, hk * dim], -1), do)


def attention_case(lib, n, tokens, hq, hk, dim, kind, dtype, seed=21):
    gen = torch.Generator().manual_seed(seed)
    counts = torch.randint(0, tokens + 1, (n,), generator=gen).tolist()
    counts[0] = tokens
    if n > 1:
        counts[-1] = 0
    spans, rows, kw = layout(kind, counts, tokens)
    check_attention(lib, spans, rows, kw, kind, n, tokens, *attention_inputs(seed + 1, spans, rows, hq, hk, dim, dtype), hq, hk)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["dense", "padded", "packed"])
@pytest.mark.parametrize("n,tokens,hq,hk,dim", [(1, 1, 1, 1, 1), (3, 2, 2, 1, 7), (2, 31, 4, 4, 16), (3, 33, 4, 1, 32), (2, 64, 6, 2, 33),
                                                (2, 65, 2, 2, 64), (3, 127, 3, 1, 80), (2, 129, 2, 1, 96), (2, 128, 2, 2, 128),
                                                (2, 200, 3, 3, 97), (2, 300, 4, 2, 64)])
def test_attention(lib, n, tokens, hq, hk, dim, kind, dtype):
    attention_case(lib, n, tokens, hq, hk, dim, kind, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [8, 24, 40, 72, 104, 120])
def test_attention_of_heads_narrower_than_their_tiles(lib, dim, dtype):
    attention_case(lib, 2, 150, 2, 1, dim, "padded", dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [32, 64, 96, 128])
def test_attention_of_rows_at_any_element(lib, dim, dtype):
    """Whole heads, but no row or head at a multiple of sixteen bytes."""
    spans, rows, kw = layout("packed", [130, 0, 70], 140)
    every = rand(3, rows, 4 * dim + 3, dtype=dtype)
    do = rand(4, rows, 2 * dim + 5, scale=0.01, dtype=dtype)
    mask = owned(spans, rows)
    every[~mask] = float("nan")
    do[~mask] = float("nan")
    q, k, v = every[:, 1:2 * dim + 1], every[:, 2 * dim + 1:3 * dim + 1], every[:, 3 * dim + 2:4 * dim + 2]
    check_attention(lib, spans, rows, kw, "packed", 3, 140, q, k, v, do[:, 3:2 * dim + 3], 2, 1)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,hq,hk,dim", [(1000, 2, 1, 128), (1537, 1, 1, 64), (2050, 1, 1, 40)])
def test_attention_over_many_tiles(lib, tokens, hq, hk, dim, dtype):
    attention_case(lib, 1, tokens, hq, hk, dim, "dense", dtype)


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_of_growing_scores(lib, dtype):
    """The maximum moves all along a row, by more than what it may lag behind; most weights are next to nothing."""
    n, dim = 500, 64
    grow = torch.linspace(0, 40, n, device="cuda").unsqueeze(1)
    k = (rand(1, n, dim, scale=0.1) + grow / 8).to(dtype)
    q = (rand(2, n, dim, scale=0.1) + 1.0).to(dtype)
    v, do = rand(3, n, dim, dtype=dtype), rand(4, n, dim, scale=0.01, dtype=dtype)
    check_attention(lib, [(0, n)], n, {}, "dense", 1, n, q, k, v, do, 1, 1)
    check_attention(lib, [(0, n)], n, {}, "dense", 1, n, q, k.flip(0).contiguous(), v, do, 1, 1)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [1e-6, 3.0])
def test_attention_at_other_scales(lib, scale, dtype):
    # (all weights alike; and one weight that is nearly everything)
    n, dim = 150, 40
    q, k, v, do = (rand(s, n, dim, dtype=dtype) for s in (1, 2, 3, 4))
    check_attention(lib, [(0, n)], n, {}, "dense", 1, n, q, k, v, do, 1, 1, scale=scale)


def test_attention_of_small_fp16_gradients(lib):
    # (ds of these is 1e-9 and less, far below fp16's numbers; the gradients are not)
    n, dim = 700, 64
    q, k, v = (rand(s, n, dim, dtype=torch.float16) for s in (1, 2, 3))
    got = check_attention(lib, [(0, n)], n, {}, "dense", 1, n, q * 8, k * 8, v, rand(4, n, dim, scale=2e-4, dtype=torch.float16), 1, 1,
                          scale=1.0 / 512)
    assert got["dq"].abs().max() > 0 and got["dk"].abs().max() > 0
    check_attention(lib, [(0, n)], n, {}, "dense", 1, n, q, k, v, rand(4, n, dim, scale=300.0, dtype=torch.float16), 1, 1)


def test_attention_writes_where_it_is_told(lib):
    """Outputs as stretches of other arrays' rows; rows of no example and the columns beside stay as they were."""
    h = lib.Handle()
    spans, rows, kw = layout("packed", [40, 0, 65, 3], 70)
    q, k, v, do = attention_inputs(7, spans, rows, 4, 2, 24, torch.bfloat16)
    kw = dict(kw, q_heads=4, kv_heads=2)
    plain, lse = lib.cdgrab_attention(h, q, k, v, **kw)
    wide = torch.full((rows, 120), 9.0, dtype=torch.bfloat16, device="cuda")
    o, _ = lib.cdgrab_attention(h, q, k, v, O=wide[:, 3:99], want_lse=False, **kw)
    mask = owned(spans, rows)
    assert torch.equal(o[mask], plain[mask]) and (wide[~mask] == 9).all() and (wide[:, :3] == 9).all() and (wide[:, 99:] == 9).all()
    want = lib.cdgrab_attention_backward(h, q, k, v, o, lse, do, **kw)
    d = torch.full((rows, 4 * 24 + 2 * 48 + 5), 9.0, dtype=torch.bfloat16, device="cuda")
    parts = d[:, 5:].split([96, 48, 48], -1)
    lib.cdgrab_attention_backward(h, q, k, v, o, lse, do, dQ=parts[0], dK=parts[1], dV=parts[2], **kw)
    assert all(torch.equal(a[mask], b[mask]) for a, b in zip(parts, want)) and (d[~mask] == 9).all() and (d[:, :5] == 9).all()


def test_attention_by_differences(lib):
    h = lib.Handle()
    n, dim = 9, 6
    x = [rand(s, 1, n, w * dim).double() for s, w in ((1, 2), (2, 1), (3, 1))]
    do = rand(4, 1, n, 2 * dim)
    kw = dict(q_heads=2, kv_heads=1)
    o, lse = lib.cdgrab_attention(h, *(t.float() for t in x), **kw)
    grads = lib.cdgrab_attention_backward(h, *(t.float() for t in x), o, lse, do, **kw)
    move = 2.0 ** -6

    def value(xs):
        return (lib.cdgrab_attention(h, *(t.float() for t in xs), want_lse=False, **kw)[0].double() * do.double()).sum().item()
    size = do.abs().sum().item()
    most = max(t.abs().max().item() for t in x)
    for which in range(3):
        for row, col in ((0, 1), (4, 0), (8, 5)):
            d = [torch.zeros_like(t) for t in x]
            d[which][0, row, col] = move
            got = (value([a + b for a, b in zip(x, d)]) - value([a - b for a, b in zip(x, d)])) / (2 * move)
            # third derivatives of a softmax are below 6 (a factor of the other operand each, over sqrt(dim)), and every row sees the change
            third = 6 * (most / dim ** 0.5) ** 3 * most * size
            assert abs(got - grads[which][0, row, col].item()) <= third * move ** 2 / 6 + 40 * U * size * most / move


def test_values_that_are_not_finite_stay_in_their_example(lib):
    h = lib.Handle()
    q, k, v = (rand(s, 3, 50, 32) for s in (1, 2, 3))
    clean, _ = lib.cdgrab_attention(h, q, k, v, q_heads=1, kv_heads=1)
    v[1, 20], k[1, 30] = float("inf"), float("nan")
    o, _ = lib.cdgrab_attention(h, q, k, v, q_heads=1, kv_heads=1)
    assert torch.equal(o[0], clean[0]) and torch.equal(o[2], clean[2])
    assert not torch.isfinite(o[1, 20:]).any() and torch.isnan(o[1, 30:]).all()


@pytest.mark.parametrize("kind", ["padded", "packed"])
@pytest.mark.parametrize("counts", [[3] * 200 + [900], [900, 0] + [1, 129, 0, 257] * 80, [0] * 300 + [700]])
def test_attention_of_examples_of_very_different_lengths(lib, kind, counts):
    n, tokens, hq, hk, dim = len(counts), 900, 2, 1, 32
    spans, rows, kw = layout(kind, counts, tokens)
    q, k, v, do = attention_inputs(5, spans, rows, hq, hk, dim, torch.bfloat16)
    q, k, v, do = (x.contiguous() for x in (q, k, v, do))
    kw = dict(kw, q_heads=hq, kv_heads=hk)
    h = lib.Handle()
    x = [shaped(kind, t, n, tokens) for t in (q, k, v, do)]
    o, lse = lib.cdgrab_attention(h, *x[:3], **kw)
    grads = lib.cdgrab_attention_backward(h, *x[:3], o, lse, x[3], **kw)
    again = lib.cdgrab_attention_backward(h, *x[:3], o, lse, x[3], **kw)
    assert all(torch.equal(a, b) for a, b in zip(grads, again))
    got = [t.reshape(rows, -1) for t in (o, *grads)] + [lse.reshape(hq, rows).t()]
    mask = owned(spans, rows)
    assert all((t[~mask] == 0).all() for t in got)
    for at, count in {(a, c) for a, c in spans if c}:  # the same numbers as of the example by itself
        part = [t[at:at + count].unsqueeze(0) for t in (q, k, v, do)]
        o1, l1 = lib.cdgrab_attention(h, *part[:3], q_heads=hq, kv_heads=hk)
        g1 = lib.cdgrab_attention_backward(h, *part[:3], o1, l1, part[3], q_heads=hq, kv_heads=hk)
        for t, want in zip(got, [o1, *g1]):
            assert torch.equal(t[at:at + count], want.reshape(count, -1))
        assert torch.equal(got[4][at:at + count], l1.reshape(hq, count).t())


def test_attention_of_more_examples_than_a_launch_holds(lib):
    # one row each: the only weight is one, o = v, dv = do and the others are zero, exactly
    n, heads, dim = 300_000, 8, 8
    q, k, v, do = (rand(s, 4, heads * dim, dtype=torch.bfloat16).repeat(n // 4, 1).unsqueeze(1) for s in (1, 2, 3, 4))
    h = lib.Handle()
    o, lse = lib.cdgrab_attention(h, q, k, v, q_heads=heads, kv_heads=heads)
    dq, dk, dv = lib.cdgrab_attention_backward(h, q, k, v, o, lse, do, q_heads=heads, kv_heads=heads)
    assert torch.equal(o, v) and torch.equal(dv, do)
    # (do v - do o, both sums of the same eight products in another order: at most 16 roundings of their sizes, times q or k)
    size = (do.float() * v.float()).abs().sum() / n * 8
    assert dq.abs().max() <= 16 * U * size * k.abs().max() and dk.abs().max() <= 16 * U * size * q.abs().max()


# ---- streams, recordings, the run together ----------------------------------------------------------

def every_call(lib, h, s):
    kw = dict(q_heads=4, k_heads=2, first=s["first"], count=s["count"], tokens=70)
    at = dict(q_heads=4, kv_heads=2, first=s["first"], count=s["count"], tokens=70)
    x = lib.cdgrab_embed(h, s["ids"], s["table"], scale=3.0, dtype=torch.bfloat16)
    y = lib.cdgrab_headnorm(h, x[:, :144], s["gq"], s["gk"], **kw)
    o, lse = lib.cdgrab_attention(h, y[:, :96], y[:, 96:], x[:, 144:], **at)
    dq, dk, dv = lib.cdgrab_attention_backward(h, y[:, :96], y[:, 96:], x[:, 144:], o, lse, s["do"], **at)
    dx, g = lib.cdgrab_pergrad_headnorm(h, x[:, :144], torch.cat([dq, dk], 1), s["gq"], s["gk"], **kw)
    e = lib.cdgrab_pergrad_embed(h, s["ids"], torch.cat([dx, dv], 1), 60, scale=3.0, first=s["first"], count=s["count"], tokens=70)
    return [y, o, lse, dq, dk, dv, dx, g, e]


def sequence(seed):
    spans, rows, kw = layout("packed", [40, 0, 65, 3, 70], 70)
    ids = torch.randint(0, 60, (rows,), generator=torch.Generator().manual_seed(seed)).int().cuda()
    return {"ids": ids, "table": rand(seed, 60, 192), "gq": rand(seed + 1, 24, offset=1.0), "gk": rand(seed + 2, 24, offset=1.0),
            "do": rand(seed + 3, rows, 96, scale=0.01, dtype=torch.bfloat16), "first": kw["first"], "count": kw["count"]}


def test_on_another_stream(lib):
    s = sequence(31)
    want = every_call(lib, lib.Handle(), s)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    h = lib.Handle(stream=stream)
    with torch.cuda.stream(stream):
        got = every_call(lib, h, s)
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_recorded_calls(lib):
    s = sequence(41)
    h = lib.Handle(stream=(stream := torch.cuda.Stream()))
    with torch.cuda.stream(stream):
        every_call(lib, h, s)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = every_call(lib, h, s)
        for seed in (51, 52, 53):
            new = sequence(seed)
            for name in s:
                s[name].copy_(new[name])
            want = every_call(lib, h, s)
            stream.synchronize()
            for x in got:
                x.fill_(3.0)
            graph.replay()
            stream.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_recorded_attention_of_other_lengths(lib):
    """What an example has is read when the recording is replayed, the list of tiles is made anew."""
    n, tokens, rows = 300, 500, 3000
    stream = torch.cuda.Stream()
    h = lib.Handle(stream=stream)

    def counts(seed):
        c = torch.randint(0, 8, (n,), generator=torch.Generator().manual_seed(seed))
        c[seed % n] = tokens
        first = c.cumsum(0) - c
        return first.cuda(), c.int().cuda()

    with torch.cuda.stream(stream):
        first, count = counts(1)
        q, do = rand(1, rows, 64, dtype=torch.bfloat16), rand(2, rows, 64, dtype=torch.bfloat16)
        k, v = rand(3, rows, 32, dtype=torch.bfloat16), rand(4, rows, 32, dtype=torch.bfloat16)
        kw = dict(q_heads=2, kv_heads=1, first=first, count=count, tokens=tokens)

        def both():
            o, lse = lib.cdgrab_attention(h, q, k, v, **kw)
            return [o, lse, *lib.cdgrab_attention_backward(h, q, k, v, o, lse, do, **kw)]
        both()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = both()
        for seed in (7, 8, 9):
            for t, new in zip((first, count), counts(seed)):
                t.copy_(new)
            want = both()
            stream.synchronize()
            graph.replay()
            stream.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want)) and (want[0] != 0).any()


def test_a_recording_needs_its_workspace_beforehand(lib):
    s = sequence(61)
    y = lib.cdgrab_embed(lib.Handle(), s["ids"], s["table"], dtype=torch.bfloat16)
    kw = dict(q_heads=4, kv_heads=2, first=s["first"], count=s["count"], tokens=70)
    stream = torch.cuda.Stream()
    h = lib.Handle(stream=stream)
    with torch.cuda.stream(stream):
        o, lse = lib.cdgrab_attention(h, y[:, :96], y[:, 96:144], y[:, 144:], **kw)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            with pytest.raises(lib.CdgrabError) as err:
                lib.cdgrab_attention_backward(h, y[:, :96], y[:, 96:144], y[:, 144:], o, lse, s["do"], **kw)
            assert err.value.code == -2
            o.mul_(1.0)
    stream.synchronize()


def test_rows_of_a_transformer_layer(lib):
    """embedding -> layer norm -> queries, keys, values -> head norms -> attention -> linear: every parameter's gradient for every
    example, side by side in the rows that the balancer reads, against torch's backward pass in double."""
    h = lib.Handle()
    n, tokens, width, vocab, hq, hk, dim = 6, 37, 32, 50, 4, 2, 16
    gen = torch.Generator().manual_seed(71)
    ids = torch.randint(0, vocab, (n, tokens), generator=gen).int().cuda()
    count = torch.tensor([37, 12, 30, 1, 25, 36], dtype=torch.int32, device="cuda")
    mask = torch.arange(tokens, device="cuda") < count.unsqueeze(1)
    qkv_width = (hq + 2 * hk) * dim
    table, gain, bias = rand(1, vocab, width), rand(2, width, offset=1.0, scale=0.1), rand(3, width, scale=0.1)
    w1, b1 = rand(4, width, qkv_width, scale=0.2), rand(5, qkv_width, scale=0.1)
    gq, gk = rand(6, dim, offset=1.0, scale=0.1), rand(7, dim, offset=1.0, scale=0.1)
    w2, b2 = rand(8, hq * dim, width, scale=0.2), rand(9, width, scale=0.1)
    dout = rand(10, n, tokens, width, scale=0.1) * mask.unsqueeze(2)
    at = dict(count=count)
    x = lib.cdgrab_embed(h, ids, table, scale=2.0)
    y = lib.cdgrab_layernorm(h, x, gain, bias)
    qkv = (y.flatten(0, 1) @ w1 + b1).view(n, tokens, -1)
    qk = lib.cdgrab_headnorm(h, qkv[..., :(hq + hk) * dim], gq, gk, q_heads=hq, k_heads=hk, **at)
    q, k, v = qk[..., :hq * dim], qk[..., hq * dim:], qkv[..., (hq + hk) * dim:]
    o, lse = lib.cdgrab_attention(h, q, k, v, q_heads=hq, kv_heads=hk, **at)
    sizes = [vocab * width, 2 * width, (width + 1) * qkv_width, 2 * dim, (hq * dim + 1) * width]
    rows = torch.full((n, sum(sizes)), float("nan"), device="cuda")
    to = rows.split(sizes, 1)
    do = (dout.flatten(0, 1) @ w2.t()).view(n, tokens, -1)
    lib.cdgrab_pergrad_linear(h, o, dout, G_out=to[4], **at)
    dqkv = torch.zeros(n, tokens, qkv_width, device="cuda")
    dqk = torch.zeros(n, tokens, (hq + hk) * dim, device="cuda")
    lib.cdgrab_attention_backward(h, q, k, v, o, lse, do, q_heads=hq, kv_heads=hk, dQ=dqk[..., :hq * dim], dK=dqk[..., hq * dim:],
                                  dV=dqkv[..., (hq + hk) * dim:], **at)
    lib.cdgrab_pergrad_headnorm(h, qkv[..., :(hq + hk) * dim], dqk, gq, gk, q_heads=hq, k_heads=hk, dX=dqkv[..., :(hq + hk) * dim],
                                G_out=to[3], **at)
    lib.cdgrab_pergrad_linear(h, y, dqkv, G_out=to[2], **at)
    dy = (dqkv.flatten(0, 1) @ w1.t()).view(n, tokens, -1)
    dx, _ = lib.cdgrab_pergrad_layernorm(h, x, dy, gain, G_out=to[1], **at)
    lib.cdgrab_pergrad_embed(h, ids, dx, vocab, scale=2.0, G_out=to[0], **at)

    params = [t.double().cpu().requires_grad_() for t in (table, gain, bias, w1, b1, gq, gk, w2, b2)]
    ptable, pgain, pbias, pw1, pb1, pgq, pgk, pw2, pb2 = params
    want = torch.zeros(rows.shape, dtype=torch.float64)
    for e in range(n):
        c = int(count[e])
        xx = ptable[ids[e, :c].cpu().long()] * 2.0
        yy = torch.nn.functional.layer_norm(xx, (width,), pgain, pbias, 1e-5)
        z = (yy @ pw1 + pb1).unflatten(-1, (-1, dim))
        hat = z[:, :hq + hk] / (z[:, :hq + hk].square().mean(-1, keepdim=True) + 1e-6).sqrt()
        u = torch.cat([hat[:, :hq] * pgq, hat[:, hq:] * pgk], 1)
        angle = torch.arange(c).double().view(-1, 1, 1) * 10000.0 ** (-torch.arange(dim // 2).double() / (dim // 2))
        a, b = u.chunk(2, -1)
        u = torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], -1)
        qh, kh = u[:, :hq].transpose(0, 1), u[:, hq:].transpose(0, 1).repeat_interleave(hq // hk, 0)
        vh = z[:, hq + hk:].transpose(0, 1).repeat_interleave(hq // hk, 0)
        s = (qh @ kh.transpose(1, 2) / dim ** 0.5).masked_fill(torch.ones(c, c).triu(1).bool(), -math.inf)
        out = (torch.softmax(s, -1) @ vh).transpose(0, 1).flatten(1) @ pw2 + pb2
        grads = torch.autograd.grad(out, params, dout[e, :c].double().cpu())
        want[e] = torch.cat([grads[i].flatten() for i in (0, 1, 2, 3, 4, 5, 6, 7, 8)])
    # Every gradient has passed at most six operators, none with more than 110 roundings of fp32 per term (rows of at most 100 features);
    # terms cancel, so that the error goes by the largest gradient of a parameter: 6 * 110 U of it, and as much for cancelling
    at_col = 0
    for size in [vocab * width, width, width, width * qkv_width, qkv_width, dim, dim, hq * dim * width, width]:
        part = slice(at_col, at_col + size)
        most = want[:, part].abs().max()
        close(rows[:, part].cpu(), want[:, part], torch.full((n, size), 2 * 6 * 110 * U) * most, "gradient of %d" % size)
        at_col += size
    out = lib.cdgrab_balance_epoch(h, 2, 2, rows.shape[1], grads=rows[:4].view(2, 2, -1))
    assert sorted(out["perm"][0].tolist()) == [0, 1]


# ---- refusals of the library itself -----------------------------------------------------------------

def test_refusals(lib):
    h = lib.Handle()
    x = torch.zeros(2, 8, 64, device="cuda")
    ids = torch.zeros(2, 8, dtype=torch.int32, device="cuda")
    kw = dict(q_heads=1, kv_heads=1)

    def refused(f):
        with pytest.raises(lib.CdgrabError) as err:
            f()
        assert err.value.code == -1
    o, lse = lib.cdgrab_attention(h, x, x.clone(), x.clone(), **kw)
    refused(lambda: lib.cdgrab_attention(h, x, x, x, O=x, **kw))                     # O on its inputs
    refused(lambda: lib.cdgrab_attention(h, x, x, x, scale=-1.0, **kw))
    for scale in (float("inf"), float("nan"), 1e-31, 1e31):
        refused(lambda: lib.cdgrab_attention(h, x, x, x, scale=scale, **kw))
    wide = torch.zeros(1, 4, 129, device="cuda")
    refused(lambda: lib.cdgrab_attention(h, wide, wide, wide, **kw))                 # a head of 129
    refused(lambda: lib.cdgrab_attention_backward(h, x, x, x, o, lse, x, dQ=x.clone(), dK=o, **kw))
    d = torch.zeros(2, 8, 64, device="cuda")
    refused(lambda: lib.cdgrab_attention_backward(h, x, x, x, o, lse, x, dK=d, dV=d, **kw))
    refused(lambda: lib.cdgrab_headnorm(h, x, q_heads=1, k_heads=0, Y=x))
    refused(lambda: lib.cdgrab_headnorm(h, x, q_heads=1, k_heads=0, eps=-1.0))
    refused(lambda: lib.cdgrab_headnorm(h, x, q_heads=1, k_heads=0, base=0.5))
    refused(lambda: lib.cdgrab_headnorm(h, x, q_heads=64, k_heads=0))                # a head of one feature
    refused(lambda: lib.cdgrab_pergrad_headnorm(h, x, x, q_heads=1, k_heads=0, want_dx=False, want_grads=False))
    refused(lambda: lib.cdgrab_embed(h, ids, x[0], scale=float("nan")))
    refused(lambda: lib.cdgrab_pergrad_embed(h, ids, x, 4, scale=float("inf")))
    big = torch.zeros(2, 16, 64, device="cuda")
    refused(lambda: lib.cdgrab_pergrad_embed(h, ids, big.view(4, 8, 64)[:2], 16, G_out=big.view(2, 1024)))  # G on DY


def test_sizes_of_nothing(lib):
    h = lib.Handle()
    kw = dict(q_heads=2, kv_heads=1)
    for shape in ((0, 5), (3, 0)):
        q, k = torch.zeros(*shape, 32, device="cuda"), torch.zeros(*shape, 16, device="cuda")
        o, lse = lib.cdgrab_attention(h, q, k, k, **kw)
        assert o.shape == q.shape and [x.shape for x in lib.cdgrab_attention_backward(h, q, k, k, o, lse, q, **kw)] == [q.shape, k.shape, k.shape]
        assert lib.cdgrab_headnorm(h, q, q_heads=1, k_heads=1).shape == q.shape
        ids = torch.zeros(shape, dtype=torch.int32, device="cuda")
        assert (lib.cdgrab_pergrad_embed(h, ids, q, 7) == 0).all()
        assert (lib.cdgrab_pergrad_headnorm(h, q, q, q_heads=1, k_heads=1)[1] == 0).all()
