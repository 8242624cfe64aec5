"""Host-side checks of the sequence operators that need no GPU: null handles, and what the binding makes of shapes, strides and spans
before it calls the library (with a stand-in for the library that records its arguments)."""
import os

import pytest
import torch


@pytest.fixture(scope="module")
def p():
    import paper_2302_00845_amd as pkg
    if not os.path.exists(pkg.library_path()):
        from paper_2302_00845_amd import build
        build.build_library(verbose=False)
    return pkg


class Recorder:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, [a._obj if type(a).__name__ == "CArgObject" else a for a in args]))
            return 0
        return call


class HostHandle:
    """What the binding uses of a Handle, on the CPU."""

    def __init__(self):
        self.device, self._h, self._lib, self.stream = torch.device("cpu"), None, Recorder(), None

    def _check(self, rc):
        assert rc == 0

    @property
    def last(self):
        return self._lib.calls[-1][1]


def test_null_handles(p):
    lib = p.load_library()
    assert lib.cdgrab_embed(None, 1, 1, 1, None, 0, None, 1, 1.0, 0, None, 1) == -1
    assert lib.cdgrab_pergrad_embed(None, None, 1, 1, 0, None, None, 1, 1.0, None, 1) == -1
    assert lib.cdgrab_headnorm(None, None, None, 0, None, 1, None, None, None, 1) == -1
    assert lib.cdgrab_pergrad_headnorm(None, None, None, 0, None, 1, None, 1, None, None, None, 1, None, 1) == -1
    assert lib.cdgrab_attention(None, None, 1, 1, 1, 0, 1.0, *[None, 1] * 4, None) == -1
    assert lib.cdgrab_attention_backward(None, None, 1, 1, 1, 0, 1.0, *[None, 1] * 4, None, *[None, 1] * 4) == -1


def test_embed(p):
    h = HostHandle()
    table, ids = torch.zeros(10, 50), torch.zeros(4, 6, dtype=torch.int32)
    y = p.cdgrab_embed(h, ids, table[:, 5:25], scale=2.0, dtype=torch.bfloat16)
    a = h.last
    assert y.shape == (4, 6, 20) and y.dtype == torch.bfloat16 and a[1:4] == [24, 10, 20]
    assert a[5:10] == [0, table.data_ptr() + 20, 50, 2.0, 1] and a[11] == 20
    for bad in (dict(ids=ids.long()), dict(table=table[0]), dict(table=table.bfloat16(), dtype=torch.float32), dict(dtype=torch.float64),
                dict(Y=torch.zeros(4, 6, 49)), dict(Y=torch.zeros(4, 6, 50), dtype=torch.float16), dict(table=table.t())):
        with pytest.raises((TypeError, ValueError)):
            p.cdgrab_embed(h, **{"ids": ids, "table": table, **bad})


def test_embed_gradient(p):
    h = HostHandle()
    ids, dy = torch.zeros(3, 5, dtype=torch.int32), torch.zeros(3, 5, 8)
    whole = torch.zeros(3, 100)
    g = p.cdgrab_pergrad_embed(h, ids, dy, 9, G_out=whole[:, 7:79])
    t = h.last[1]
    assert (t.examples, t.rows, t.tokens) == (3, 15, 5) and h.last[2:5] == [9, 8, 0] and h.last[9:] == [g.data_ptr(), 100]
    first = torch.zeros(7, dtype=torch.int64)
    assert p.cdgrab_pergrad_embed(h, ids.view(15), dy.view(15, 8), 2, first=first, tokens=4).shape == (7, 16)
    for args in ((ids[:2], dy, 9), (ids.long(), dy, 9), (ids, dy.double(), 9), (ids.view(15), dy.view(15, 8), 9)):
        with pytest.raises((TypeError, ValueError)):
            p.cdgrab_pergrad_embed(h, *args)
    with pytest.raises(ValueError):
        p.cdgrab_pergrad_embed(h, ids, dy, 9, G_out=whole)


def test_heads(p):
    h = HostHandle()
    x = torch.zeros(3, 5, 60, dtype=torch.float16)
    gain = torch.zeros(8)
    y = p.cdgrab_headnorm(h, x[..., 4:44], gain, None, q_heads=3, k_heads=2, eps=1e-4, base=500.0)
    t, s = h.last[1:3]
    assert (s.q_heads, s.k_heads, s.dim, s.base) == (3, 2, 8, 500.0) and abs(s.eps - 1e-4) < 1e-9 and t.rows == 15
    assert y.shape == (3, 5, 40) and h.last[3:6] == [2, x.data_ptr() + 8, 60] and h.last[6:8] == [gain.data_ptr(), None]
    dx, g = p.cdgrab_pergrad_headnorm(h, x, x, q_heads=6, k_heads=0, count=torch.zeros(3, dtype=torch.int32))
    assert dx.shape == x.shape and g.shape == (3, 20)
    assert p.cdgrab_pergrad_headnorm(h, x, x, q_heads=6, k_heads=0, want_dx=False)[0] is None
    for kw in (dict(q_heads=7, k_heads=0), dict(q_heads=0, k_heads=0), dict(q_heads=-1, k_heads=4),
               dict(q_heads=6, k_heads=0, gain_q=gain), dict(q_heads=6, k_heads=0, count=torch.zeros(2, dtype=torch.int32))):
        with pytest.raises(ValueError):
            p.cdgrab_headnorm(h, x, **kw)


def test_attention(p):
    h = HostHandle()
    qkv = torch.zeros(2, 7, 64, dtype=torch.bfloat16)
    q, k, v = qkv.split([32, 16, 16], -1)
    o, lse = p.cdgrab_attention(h, q, k, v, q_heads=4, kv_heads=2)
    a = h.last
    assert a[2:7] == [4, 2, 8, 1, 8 ** -0.5] and o.shape == q.shape and lse.shape == (4, 2, 7) and lse.dtype == torch.float32
    assert a[7:13] == [qkv.data_ptr(), 64, qkv.data_ptr() + 64, 64, qkv.data_ptr() + 96, 64] and a[14:] == [32, lse.data_ptr()]
    assert p.cdgrab_attention(h, q, k, v, q_heads=4, kv_heads=2, scale=0.5, want_lse=False)[1] is None and h.last[6] == 0.5
    dqkv = torch.zeros_like(qkv)
    parts = dqkv.split([32, 16, 16], -1)
    p.cdgrab_attention_backward(h, q, k, v, o, lse, o, q_heads=4, kv_heads=2, dQ=parts[0], dK=parts[1], dV=parts[2])
    a = h.last
    assert a[15] == lse.data_ptr() and a[18:] == [dqkv.data_ptr(), 64, dqkv.data_ptr() + 64, 64, dqkv.data_ptr() + 96, 64]
    for kw in (dict(q_heads=4, kv_heads=3), dict(q_heads=3, kv_heads=1), dict(q_heads=0, kv_heads=0), dict(q_heads=4, kv_heads=4)):
        with pytest.raises(ValueError):
            p.cdgrab_attention(h, q, k, v, **kw)
    for bad in (dict(K=k.float()), dict(V=v[:1]), dict(O=o.float()), dict(count=torch.zeros(2, dtype=torch.int64))):
        with pytest.raises((TypeError, ValueError)):
            p.cdgrab_attention(h, **{"Q": q, "K": k, "V": v, "q_heads": 4, "kv_heads": 2, **bad})
    with pytest.raises(ValueError):
        p.cdgrab_attention_backward(h, q, k, v, o, lse[:3], o, q_heads=4, kv_heads=2)
