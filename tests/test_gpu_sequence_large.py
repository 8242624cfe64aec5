"""GPU tests of the sequence operators where a call is large enough for another order or another number of launches: arrays that are read
and written past the caches, tiles in the order of pairs, lists of more than a thousand tiles, examples in several launches."""
import math

import pytest
import torch

from test_gpu_sequence import U, attention64, check_attention, close, embed_case, attention_inputs, layout, lib, owned, pair_sum, rand, step, \
    tiny, turned  # noqa: F401  (lib: the fixture)

pytestmark = pytest.mark.gpu


# ---- arrays of 64 MB and more: past the caches ------------------------------------------------------

@pytest.mark.parametrize("dtype,rows", [(torch.float32, 17_000), (torch.bfloat16, 33_000), (torch.float16, 33_001)])
def test_embed_of_many_rows(lib, dtype, rows):
    width, vocab = 1027, 700
    table = rand(1, vocab, width + 6)[:, 3:width + 3]
    ids = torch.randint(-1, vocab + 1, (rows,), generator=torch.Generator().manual_seed(2)).int().cuda()
    whole = torch.full((rows, width + 10), 7.0, dtype=dtype, device="cuda")
    y = whole[:, 5:width + 5]
    assert y.numel() * y.element_size() >= 1 << 26
    lib.cdgrab_embed(lib.Handle(), ids, table, scale=1.7, Y=y)
    known = ((ids >= 0) & (ids < vocab)).unsqueeze(1)
    want = torch.where(known, table[ids.long().clamp(0, vocab - 1)].double() * float(torch.tensor(1.7)), 0.0)
    close(y, want, (U + step(dtype)) * want.abs() * 1.01 + tiny(dtype), "y")
    assert (whole[:, :5] == 7).all() and (whole[:, width + 5:] == 7).all()


@pytest.mark.parametrize("n,tokens,vocab,width", [(3, 700, 6000, 1027), (40, 60, 900, 515), (2, 3000, 9000, 1027), (1, 5000, 70_000, 261)])
@pytest.mark.parametrize("kind,dtype", [("dense", torch.bfloat16), ("packed", torch.float32), ("padded", torch.float16)])
def test_pergrad_embed_of_large_tables(lib, n, tokens, vocab, width, kind, dtype):
    assert n * vocab * width * 4 > 1 << 26
    whole = torch.full((n, vocab * width + 9), 5.0, device="cuda")
    embed_case(lib, n, tokens, vocab, width, kind, dtype, same=vocab // 2, G_out=whole[:, 4:vocab * width + 4])
    assert (whole[:, :4] == 5).all() and (whole[:, vocab * width + 4:] == 5).all()


@pytest.mark.parametrize("dtype,n,tokens,hq,hk,dim", [(torch.bfloat16, 90, 300, 16, 4, 64), (torch.float32, 41, 340, 20, 20, 32),
                                                      (torch.float16, 35, 800, 4, 3, 192), (torch.bfloat16, 3, 5000, 9, 1, 256)])
@pytest.mark.parametrize("kind", ["dense", "padded"])
def test_heads_of_many_rows(lib, dtype, n, tokens, hq, hk, dim, kind):
    width = (hq + hk) * dim
    counts = [(n - i) * tokens // n for i in range(n)] if kind == "padded" else [tokens] * n
    spans, rows, kw = layout(kind, counts, tokens)
    assert rows * width * torch.empty((), dtype=dtype).element_size() >= 1 << 26
    x = rand(1, rows, width + 16, offset=0.3, dtype=dtype)[:, 8:width + 8].unflatten(0, (n, tokens))
    dy = rand(2, rows, width + 8, scale=0.1, dtype=dtype)[:, :width].unflatten(0, (n, tokens))
    gq, gk = rand(3, dim, scale=0.2, offset=1.0), rand(4, dim, scale=0.2, offset=-1.0)
    h = lib.Handle()
    kw = dict(kw, q_heads=hq, k_heads=hk)
    out = torch.full((n, tokens, width + 3), 5.0, dtype=dtype, device="cuda")
    back = torch.full((n, tokens, width + 5), 5.0, dtype=dtype, device="cuda")
    y, dx = out[..., 1:width + 1], back[..., 2:width + 2]
    lib.cdgrab_headnorm(h, x, gq, gk, Y=y, **kw)
    _, g = lib.cdgrab_pergrad_headnorm(h, x, dy, gq, gk, dX=dx, **kw)
    mask = owned(spans, rows).view(n, tokens)
    assert (out[~mask] == 5).all() and (back[~mask] == 5).all()
    for t, edge in ((out, 1), (back, 2)):
        assert (t[..., :edge] == 5).all() and (t[..., width + edge:] == 5).all()
    e32 = float(torch.tensor(1e-6))
    w = torch.cat([gq.double().expand(hq, -1), gk.double().expand(hk, -1)])
    rt = ((dim + 8) / 2 + 4) * U  # (as of the smaller ones)
    for e in sorted({0, 1, n // 2, n - 1}):
        c = counts[e]
        v, d = (t[e, :c].double().unflatten(-1, (-1, dim)) for t in (x, dy))
        r = 1.0 / (v.square().mean(-1, keepdim=True) + e32).sqrt()
        hat, pos = v * r, torch.arange(c, device="cuda")
        want = turned(hat * w, pos, 10000.0)
        close(y[e, :c].unflatten(-1, (-1, dim)), want, pair_sum(hat * w) * (rt + 8 * U) + step(dtype) * want.abs() * 1.01 + tiny(dtype), "y")
        u, eu = turned(d, pos, 10000.0, back=True), pair_sum(d) * 8 * U
        q = u * w
        mean = (q * hat).mean(-1, keepdim=True)
        mean_err = (eu * w.abs() * hat.abs() + (q * hat).abs() * (rt + (dim + 8) * U)).mean(-1, keepdim=True)
        want = r * (q - hat * mean)
        tol = r * (w.abs() * eu + q.abs() * (rt + 4 * U) + hat.abs() * (mean_err + mean.abs() * (2 * rt + 4 * U)))
        close(dx[e, :c].unflatten(-1, (-1, dim)), want, tol + step(dtype) * want.abs() * 1.01 + tiny(dtype), "dx")
        each, err = u * hat, eu * hat.abs() + (u * hat).abs() * (rt + 2 * U)
        for which, heads in ((0, slice(0, hq)), (1, slice(hq, hq + hk))):
            s, a = each[:, heads].sum((0, 1)), each[:, heads].abs().sum((0, 1))
            close(g[e, which * dim:(which + 1) * dim], s, err[:, heads].sum((0, 1)) + (c * (hq + hk) + 8) * U * a + 1e-38, "G")


# ---- many examples: several launches ----------------------------------------------------------------

def test_heads_of_more_examples_than_a_launch_holds(lib):
    """Examples of one row each, and their rows again in longer examples that share them."""
    n, dim = (1 << 21) + 77, 4
    x, dy, gain = rand(1, n, 2 * dim), rand(2, n, 2 * dim), rand(3, dim, offset=1.0)
    h = lib.Handle()
    kw = dict(q_heads=1, k_heads=1, base=0.0)
    y = lib.cdgrab_headnorm(h, x.unsqueeze(1), gain, **kw).view(n, 2, dim)
    dx, g = lib.cdgrab_pergrad_headnorm(h, x.unsqueeze(1), dy.unsqueeze(1), gain, **kw)
    v, d = x.double().view(n, 2, dim), dy.double().view(n, 2, dim)
    w = torch.stack([gain.double(), torch.ones_like(gain).double()])
    hat = v / (v.square().mean(-1, keepdim=True) + float(torch.tensor(1e-6))).sqrt()
    rt = (dim + 12) * U
    close(y, hat * w, (hat * w).abs() * rt + 1e-40, "y")
    close(g.view(n, 2, dim), d * hat, (d * hat).abs() * rt + 1e-40, "G")
    r = 1.0 / (v.square().mean(-1, keepdim=True) + float(torch.tensor(1e-6))).sqrt()
    mean, size = (d * w * hat).mean(-1, keepdim=True), (d * w * hat).abs().mean(-1, keepdim=True)
    close(dx.view(n, 2, dim), r * (d * w - hat * mean), r * ((d * w).abs() + hat.abs() * (size + mean.abs())) * 3 * rt + 1e-40, "dx")
    first = torch.arange(n, device="cuda")  # examples of two rows, but for the last
    _, pairs = lib.cdgrab_pergrad_headnorm(h, x, dy, gain, want_dx=False, first=first, tokens=2, **kw)
    close(pairs[:-1], g[:-1].double() + g[1:].double(), (g[:-1].abs() + g[1:].abs()) * 4 * U + 1e-40, "G of two rows")
    assert torch.equal(pairs[-1], g[-1])


def test_embed_gradient_of_more_examples_than_a_launch_holds(lib):
    n, vocab = (1 << 21) + 77, 3
    ids = torch.randint(-1, vocab + 1, (n, 1), generator=torch.Generator().manual_seed(1)).int().cuda()
    dy = rand(2, n, 1, 2)
    g = lib.cdgrab_pergrad_embed(lib.Handle(), ids, dy, vocab).view(n, vocab, 2)
    assert torch.equal(g, (ids == torch.arange(vocab, device="cuda")).unsqueeze(2) * dy)


@pytest.mark.parametrize("width,examples", [(1500, 1900), (3, 25_000)])
def test_embed_gradients_of_long_examples_in_parts(lib, width, examples):
    """More keys and sums than the workspace holds at a time: examples of up to 2100 rows that share their rows."""
    rows, tokens, vocab = 2600, 2100, 2
    chunks = -(-tokens // 1024)
    assert examples * chunks * 1024 * (16 + width * 4 // 16) > 1 << 30
    gen = torch.Generator().manual_seed(3)
    ids = torch.randint(-1, vocab + 1, (rows,), generator=gen).int().cuda()
    dy = rand(4, rows, width, dtype=torch.float16)
    first = torch.randint(0, rows, (examples,), generator=gen)
    count = torch.randint(0, tokens + 1, (examples,), generator=gen)
    first[-1], count[-1] = 17, tokens
    first[0], count[0] = rows - 1, 0
    h = lib.Handle()
    kw = dict(first=first.cuda(), count=count.int().cuda(), tokens=tokens)
    g = lib.cdgrab_pergrad_embed(h, ids, dy, vocab, **kw).view(examples, vocab, width)
    for v in range(vocab):
        part = torch.where((ids == v).unsqueeze(1), dy.double(), 0.0)
        upto = torch.cat([torch.zeros(1, width, dtype=torch.float64, device="cuda"), part.cumsum(0)])
        size = torch.cat([torch.zeros(1, width, dtype=torch.float64, device="cuda"), part.abs().cumsum(0)])
        end = (first + count).clamp(max=rows).cuda()
        begin = first.cuda()
        for i in range(0, examples, 1000):
            a, b = begin[i:i + 1000], end[i:i + 1000]
            close(g[i:i + 1000, v], upto[b] - upto[a], (size[b] - size[a]) * (tokens + 2) * U + 1e-9, "G")
    assert torch.equal(g.flatten(1), lib.cdgrab_pergrad_embed(h, ids, dy, vocab, **kw))


# ---- attention: the order of pairs, long lists ------------------------------------------------------

@pytest.mark.parametrize("kind,n,tokens,hq,hk,dim,dtype", [("dense", 31, 400, 24, 6, 32, torch.bfloat16), ("padded", 41, 300, 24, 6, 24, torch.float16),
                                                           ("packed", 37, 513, 16, 1, 64, torch.bfloat16), ("dense", 13, 700, 30, 15, 40, torch.float32)])
def test_attention_pair_by_pair(lib, kind, n, tokens, hq, hk, dim, dtype):
    """Enough tiles for the order that goes pair by pair (example and head of keys), several tiles and heads of queries in each."""
    counts = [tokens - i * 7 % tokens if kind != "dense" else tokens for i in range(n)]
    spans, rows, kw = layout(kind, counts, tokens)
    assert -(-n * hk // 8) * 8 * -(-tokens // 128) * (hq // hk) >= 2048
    q, k, v, do = attention_inputs(5, spans, rows, hq, hk, dim, dtype)
    check_attention(lib, spans, rows, kw, kind, n, tokens, q, k, v, do, hq, hk)


def test_attention_of_a_list_of_more_than_a_thousand_tiles(lib):
    long, short, hq, hk, dim = 1030 * 128 + 5, 200, 2, 1, 8
    counts = [1 + i % 150 for i in range(short)] + [long] + [3, 129]
    n, tokens = len(counts), long
    spans, rows, kw = layout("packed", counts, tokens)
    tiles = -(-tokens // 128)
    assert tiles > 1024 and n >= 2 * (rows // 128 + n) // tiles + 64
    q, k, v, do = (t.contiguous() for t in attention_inputs(6, spans, rows, hq, hk, dim, torch.bfloat16))
    h = lib.Handle()
    kw = dict(kw, q_heads=hq, kv_heads=hk)
    o, lse = lib.cdgrab_attention(h, q, k, v, **kw)
    grads = lib.cdgrab_attention_backward(h, q, k, v, o, lse, do, **kw)
    for at, count in spans:  # the same numbers as of the example by itself
        part = [t[at:at + count].unsqueeze(0) for t in (q, k, v, do)]
        o1, l1 = lib.cdgrab_attention(h, *part[:3], q_heads=hq, kv_heads=hk)
        assert torch.equal(o[at:at + count], o1[0]) and torch.equal(lse[:, at:at + count], l1[:, 0])
        for got, want in zip(grads, lib.cdgrab_attention_backward(h, *part[:3], o1, l1, part[3], q_heads=hq, kv_heads=hk)):
            assert torch.equal(got[at:at + count], want[0])
    at = spans[short][0]
    scale = float(torch.tensor(dim ** -0.5))
    for row in (0, 1, 127, 128, 5000, long // 2, long - 2, long - 1):  # and some rows of the long one
        s = q[at + row].view(hq, dim).double() @ k[at:at + row + 1].double().t() * scale
        want = torch.softmax(s, 1) @ v[at:at + row + 1].double()
        # (weights and outputs rounded to bf16, an exponential's two steps, sums of row + 1)
        tol = torch.softmax(s, 1) @ v[at:at + row + 1].double().abs() * (2.0 ** -8 * 1.01 + (row + 100) * U) + want.abs() * 2.0 ** -8 * 1.01
        close(o[at + row].view(hq, dim), want, tol, "o")
        close(lse[:, at + row], torch.logsumexp(s, 1), (row + 100) * U * torch.ones(hq, device="cuda") + 8 * U * torch.logsumexp(s, 1).abs(), "lse")
