"""GPU tests of the sequence operators called as the header allows: from another stream than the handle's, on arrays beyond 4 GB, with
examples that lie outside the rows, at the smallest scale, with elements that are not finite where nothing reads them."""
import pytest
import torch

from test_gpu_sequence import TYPES, check_attention, lib, rand  # noqa: F401  (lib: the fixture)

pytestmark = pytest.mark.gpu


def calls(lib, h, s, at):
    """(what, its call) one after the other; a call may use what the ones before returned, in `s`."""
    kw = dict(at, q_heads=4, k_heads=2)
    att = dict(at, q_heads=4, kv_heads=2)
    yield "x", lambda: lib.cdgrab_embed(h, s["ids"], s["table"], scale=3.0, dtype=torch.bfloat16)
    yield "y", lambda: lib.cdgrab_headnorm(h, s["x"][:, :144], s["gq"], s["gk"], **kw)
    yield "o", lambda: lib.cdgrab_attention(h, s["y"][:, :96], s["y"][:, 96:], s["x"][:, 144:], **att)
    yield "d", lambda: lib.cdgrab_attention_backward(h, s["y"][:, :96], s["y"][:, 96:], s["x"][:, 144:], *s["o"], s["do"], **att)
    yield "dx", lambda: lib.cdgrab_pergrad_headnorm(h, s["x"][:, :144], s["do2"], s["gq"], s["gk"], **kw)
    yield "e", lambda: lib.cdgrab_pergrad_embed(h, s["ids"], s["do3"], 60, scale=3.0, **at)


def inputs(first, count, tokens, rows):
    gen = torch.Generator().manual_seed(3)
    s = {"ids": torch.randint(0, 60, (rows,), generator=gen).int().cuda(), "table": rand(1, 60, 192), "gq": rand(2, 24, offset=1.0),
         "gk": rand(3, 24, offset=1.0), "do": rand(4, rows, 96, scale=0.01, dtype=torch.bfloat16),
         "do2": rand(5, rows, 144, dtype=torch.bfloat16), "do3": rand(6, rows, 192, dtype=torch.bfloat16)}
    return s, dict(first=torch.tensor(first, dtype=torch.int64, device="cuda"), count=torch.tensor(count, dtype=torch.int32, device="cuda"),
                   tokens=tokens)


def flat(x):
    return [x] if torch.is_tensor(x) else list(x)


def test_calls_from_another_stream(lib):
    """The handle's stream is not the current one; memory that the current stream lets go of is used again at once."""
    s, at = inputs([0, 40, 40, 110], [40, 0, 65, 70], 70, 185)
    h = lib.Handle()
    want = {}
    for name, call in calls(lib, h, s, at):
        want[name] = s[name] = call()
    torch.cuda.synchronize()
    want = {name: [t.clone() for t in flat(x)] for name, x in want.items()}
    stream, now = torch.cuda.Stream(), torch.cuda.current_stream()
    h = lib.Handle(stream=stream)
    for _ in range(3):
        for name, call in calls(lib, h, s, at):
            junk = [torch.full_like(t, 7.0) for t in want[name]]  # (what outputs may be given)
            stream.wait_stream(now)
            del junk
            s[name] = call()
            now.wait_stream(stream)
            assert all(torch.equal(a, b) for a, b in zip(flat(s[name]), want[name])), name


def test_examples_outside_the_rows(lib):
    """What of an example lies before, behind or beyond `tokens` is left out; the others are as without it."""
    rows, tokens = 190, 70
    first = [-5, 30, rows + 3, rows - 9, 2 ** 62, 100, -2 ** 63, rows]
    count = [20, 40, 4, 100, 5, 2 ** 31 - 1, 3, 7]
    s, at = inputs(first, count, tokens, rows)
    h = lib.Handle()
    whole = [(0, 0), (30, 40), (0, 0), (rows - 9, 9), (0, 0), (100, 70), (0, 0), (0, 0)]
    t, bt = inputs([a for a, _ in whole], [c for _, c in whole], tokens, rows)
    for (name, call), (_, plain) in zip(calls(lib, h, s, at), calls(lib, h, t, bt)):
        s[name], t[name] = call(), plain()
        assert all(torch.equal(a, b) for a, b in zip(flat(s[name]), flat(t[name]))), name
    count[1] = -4
    whole[1] = (30, 0)
    s, at = inputs(first, count, tokens, rows)
    t, bt = inputs([a for a, _ in whole], [c for _, c in whole], tokens, rows)
    for (name, call), (_, plain) in zip(calls(lib, h, s, at), calls(lib, h, t, bt)):
        s[name], t[name] = call(), plain()
        assert all(torch.equal(a, b) for a, b in zip(flat(s[name]), flat(t[name]))), name


def test_examples_outside_the_rows_in_a_list(lib):
    """The same where a list of tiles is made: many examples, most of them without a row that is there."""
    rows, tokens, n = 1500, 1000, 400
    first = [(-1) ** i * (rows + i) for i in range(n)] + [0, 1000, 1390]
    count = [1000] * n + [1000, 390, 5000]
    q, k, v, do = (rand(i, rows, w, dtype=torch.bfloat16) for i, w in enumerate((64, 32, 32, 64)))
    h = lib.Handle()
    kw = dict(q_heads=2, kv_heads=1, tokens=tokens, first=torch.tensor(first).cuda(), count=torch.tensor(count, dtype=torch.int32).cuda())
    o, lse = lib.cdgrab_attention(h, q, k, v, **kw)
    grads = lib.cdgrab_attention_backward(h, q, k, v, o, lse, do, **kw)
    for at, c in ((0, 1000), (1000, 390), (1390, 110)):
        x = [t[at:at + c].unsqueeze(0) for t in (q, k, v, do)]
        o1, l1 = lib.cdgrab_attention(h, *x[:3], q_heads=2, kv_heads=1)
        assert torch.equal(o[at:at + c], o1[0]) and torch.equal(lse[:, at:at + c], l1[:, 0])
        for got, want in zip(grads, lib.cdgrab_attention_backward(h, *x[:3], o1, l1, x[3], q_heads=2, kv_heads=1)):
            assert torch.equal(got[at:at + c], want[0])


def test_rows_beyond_four_gigabytes(lib):
    """Everything is a stretch of the rows of one array of 2^18 elements and more a row; the last rows lie beyond 2^32 bytes."""
    rows, long = 8300, (1 << 18) + 8
    whole = torch.empty(rows, long, dtype=torch.bfloat16, device="cuda")
    hq, hk, dim, vocab, n = 4, 2, 24, 9, 3
    assert (rows - 100) * long * 2 > 1 << 32
    widths = {"q": hq * dim, "k": hk * dim, "v": hk * dim, "o": hq * dim, "do": hq * dim, "dq": hq * dim, "dk": hk * dim, "dv": hk * dim,
              "x": (hq + hk) * dim, "y": (hq + hk) * dim, "dy": (hq + hk) * dim, "dx": (hq + hk) * dim, "emb": 40, "demb": 40}
    far, near, at = {}, {}, 16
    for i, (name, w) in enumerate(widths.items()):
        far[name] = whole[:, at:at + w]
        at += w + 8 - w % 8 + (8 if i < 5 else 5)  # (whole pieces of sixteen bytes, and others)
        near[name] = rand(i, rows, w, dtype=torch.bfloat16)
        far[name].copy_(near[name])
    ids = torch.randint(-1, vocab + 1, (rows,), generator=torch.Generator().manual_seed(1)).int().cuda()
    table, gain = rand(90, vocab, 40), rand(91, dim, offset=1.0)
    span = dict(first=torch.tensor([100, 4000, rows - 700], device="cuda"), count=torch.tensor([300, 500, 700], dtype=torch.int32, device="cuda"),
                tokens=700)
    h = lib.Handle()
    got = []
    for s in (far, near):
        _, lse = lib.cdgrab_attention(h, s["q"], s["k"], s["v"], O=s["o"], q_heads=hq, kv_heads=hk, **span)
        lib.cdgrab_attention_backward(h, s["q"], s["k"], s["v"], s["o"], lse, s["do"], dQ=s["dq"], dK=s["dk"], dV=s["dv"], q_heads=hq,
                                      kv_heads=hk, **span)
        lib.cdgrab_headnorm(h, s["x"], gain, gain, q_heads=hq, k_heads=hk, Y=s["y"], **span)
        _, g = lib.cdgrab_pergrad_headnorm(h, s["x"], s["dy"], gain, gain, q_heads=hq, k_heads=hk, dX=s["dx"], **span)
        lib.cdgrab_embed(h, ids, table, Y=s["emb"])
        e = lib.cdgrab_pergrad_embed(h, ids, s["demb"], vocab, **span)
        got.append((lse, g, e))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    for name in widths:
        assert torch.equal(far[name], near[name]), name


def test_table_and_gradients_beyond_four_gigabytes(lib):
    """A table of 2^20 rows of 1100 and two examples' gradients of it: offsets beyond 2^32 bytes."""
    vocab, width = 1 << 20, 1100
    assert vocab * width * 4 > 1 << 32
    table = torch.zeros(vocab, width, device="cuda")
    ids = torch.tensor([[0, 5, vocab - 1, vocab - 1], [vocab // 2, vocab - 2, 5, vocab]], dtype=torch.int32, device="cuda")
    table[ids.flatten()[:-1].long()] = rand(1, 7, width)
    h = lib.Handle()
    y = lib.cdgrab_embed(h, ids, table)
    assert torch.equal(y[0], table[ids[0].long()]) and torch.equal(y[1, :3], table[ids[1, :3].long()]) and (y[1, 3] == 0).all()
    dy = rand(2, 2, 4, width)
    for long in (False, True):  # (examples that one workgroup looks through, and sorted ones)
        more = 3000 if long else 0
        i = torch.cat([ids, torch.full((2, more), -1, dtype=torch.int32, device="cuda")], 1)
        d = torch.cat([dy, torch.full((2, more, width), float("nan"), device="cuda")], 1)  # (of no id: not read)
        g = lib.cdgrab_pergrad_embed(h, i, d, vocab).view(2, vocab, width)
        assert torch.equal(g[0, 0], dy[0, 0]) and torch.equal(g[0, 5], dy[0, 1]) and torch.equal(g[0, -1], dy[0, 2] + dy[0, 3])
        assert torch.equal(g[1, vocab // 2], dy[1, 0]) and torch.equal(g[1, -2], dy[1, 1]) and torch.equal(g[1, 5], dy[1, 2])
        assert [int(x.any(1).sum()) for x in g] == [3, 3]
        del g


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_at_the_smallest_scale(lib, dtype):
    n, dim = 150, 40
    q, k, v, do = (rand(s, n, dim, dtype=dtype) for s in (1, 2, 3, 4))
    check_attention(lib, [(0, n)], n, {}, "dense", 1, n, q, k, v, do, 1, 1, scale=1e-30)
