"""GPU tests of attention where some examples share rows: what the others get."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    import paper_2302_00845_amd as p
    return p


def rand(seed, *shape, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64).to(dtype).cuda()


@pytest.mark.parametrize("shared,length,step", [(300, 900, 0), (300, 900, 1), (95, 1024, 0), (2000, 300, 3)])
@pytest.mark.parametrize("own", [[5, 129, 1, 300, 128, 40], [100, 900, 700]])
def test_examples_of_rows_of_their_own_among_others(lib, shared, length, step, own):
    """`shared` examples of `length` rows, each `step` rows behind the one before, and examples that share rows with none."""
    hq, hk, dim = 2, 1, 32
    first, count, at = [], [], 3
    for i in range(shared):
        first.append(at + i * step)
        count.append(length)
    at += (shared - 1) * step + length
    for c in own:
        first.append(at)
        count.append(c)
        at += c
    rows = at + 2
    order = torch.randperm(len(first), generator=torch.Generator().manual_seed(1))
    q, do, k, v = rand(1, rows, hq * dim), rand(2, rows, hq * dim), rand(3, rows, hk * dim), rand(4, rows, hk * dim)
    kw = dict(q_heads=hq, kv_heads=hk, tokens=max(count), first=torch.tensor(first)[order].cuda(),
              count=torch.tensor(count, dtype=torch.int32)[order].cuda())
    h = lib.Handle()
    o, lse = lib.cdgrab_attention(h, q, k, v, **kw)
    for at, c in list(zip(first, count))[shared:]:  # the same numbers as of the example by itself
        x = [t[at:at + c].unsqueeze(0) for t in (q, k, v, do)]
        o1, l1 = lib.cdgrab_attention(h, *x[:3], q_heads=hq, kv_heads=hk)
        assert torch.equal(o[at:at + c], o1[0]) and torch.equal(lse[:, at:at + c], l1[:, 0])
    grads = lib.cdgrab_attention_backward(h, q, k, v, o, lse, do, **kw)
    for at, c in list(zip(first, count))[shared:]:
        x = [t[at:at + c].unsqueeze(0) for t in (q, k, v, do)]
        o1, l1 = lib.cdgrab_attention(h, *x[:3], q_heads=hq, kv_heads=hk)
        for got, want in zip(grads, lib.cdgrab_attention_backward(h, *x[:3], o1, l1, x[3], q_heads=hq, kv_heads=hk)):
            assert torch.equal(got[at:at + c], want[0])
    assert (o[:3] == 0).all() and (o[-2:] == 0).all()


def test_recorded_calls_of_shared_rows(lib):
    """Whether examples share rows is seen when the recording is replayed."""
    n, length, hq, hk, dim = 200, 640, 2, 1, 32
    rows = n * 8 + 2 * length
    q, k, v = rand(1, rows, hq * dim), rand(2, rows, hk * dim), rand(3, rows, hk * dim)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    h = lib.Handle(stream=stream)
    with torch.cuda.stream(stream):
        first, count = torch.arange(n, device="cuda") * 8, torch.full((n,), 8, dtype=torch.int32, device="cuda")
        count[-1] = length
        kw = dict(q_heads=hq, kv_heads=hk, tokens=length, first=first, count=count)
        lib.cdgrab_attention(h, q, k, v, **kw)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            o, lse = lib.cdgrab_attention(h, q, k, v, **kw)
        apart, alike = first.clone(), torch.full_like(first, 16)
        alike[-1] = rows - length
        few, many = count.clone(), torch.full_like(count, length)
        for f, c, own in ((apart, few, 2), (alike, many, 1), (apart, few, 2), (alike, many, 1)):  # (`own`: the last ones share no rows)
            first.copy_(f)
            count.copy_(c)
            o.fill_(7.0)
            graph.replay()
            stream.synchronize()
            for at, rows_of in [(int(a), int(b)) for a, b in zip(f[-own:], c[-own:])]:
                x = [t[at:at + rows_of].unsqueeze(0) for t in (q, k, v)]
                assert torch.equal(o[at:at + rows_of], lib.cdgrab_attention(h, *x, q_heads=hq, kv_heads=hk)[0][0])
