"""Host-side checks of the layer operators that need no GPU: null handles, and what the binding makes of shapes, strides and
spans before it calls the library (with a stand-in for the library that records its arguments)."""
import ctypes
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
    assert lib.cdgrab_layernorm(None, 1, 1, 0, None, 1, None, None, 1e-5, None, 1) == -1
    assert lib.cdgrab_pergrad_layernorm(None, None, 1, 0, None, 1, None, 1, None, 1e-5, None, 1, 1, None, 1) == -1
    assert lib.cdgrab_pergrad_linear(None, None, 1, 1, 0, None, 1, None, 1, 1, None, 1) == -1
    assert lib.cdgrab_orthogonalize(None, 1, 1, 1, 0, None, 1, 1, 5, None, None, 1, 1) == -1
    assert lib.cdgrab_train_epoch_softmax_orthogonal(None, 1, 2, 1, 1, None, None, None, None, None, 0.1, 0.9, 5, None, None, None,
                                                     None, None) == -1


def test_rows_and_strides(p):
    h = HostHandle()
    x = torch.zeros(4, 6, 50, dtype=torch.bfloat16)
    y = p.cdgrab_layernorm(h, x[..., 5:25])
    assert y.shape == (4, 6, 20) and y.is_contiguous()
    assert h.last[1:6] == [24, 20, 1, x.data_ptr() + 10, 50] and h.last[10] == 20
    p.cdgrab_layernorm(h, x[1])  # one example's rows
    assert h.last[1:6] == [6, 50, 1, x[1].data_ptr(), 50]
    p.cdgrab_layernorm(h, x[:, 2])  # one row of each example
    assert h.last[1:6] == [4, 50, 1, x[:, 2].data_ptr(), 300]


@pytest.mark.parametrize("make,error", [
    (lambda x: x.transpose(1, 2), ValueError), (lambda x: x[..., ::2], ValueError), (lambda x: x[:, :3], ValueError),
    (lambda x: x[::2], ValueError),  # (rows one distance apart within an example, another between them)
    (lambda x: x.double(), TypeError), (lambda x: x.to(torch.int32), TypeError), (lambda x: x[0, 0], ValueError),
    (lambda x: x[:1, :1].expand(4, 6, 50), ValueError)])
def test_rows_that_are_refused(p, make, error):
    with pytest.raises(error):
        p.cdgrab_layernorm(HostHandle(), make(torch.zeros(4, 6, 50)))


def test_spans(p):
    h = HostHandle()
    x, d = torch.zeros(3, 5, 8), torch.zeros(3, 5, 2)
    g = p.cdgrab_pergrad_linear(h, x, d)
    t = h.last[1]
    assert (t.examples, t.rows, t.tokens, t.first, t.count) == (3, 15, 5, None, None) and g.shape == (3, 18)
    count = torch.zeros(3, dtype=torch.int32)
    p.cdgrab_pergrad_linear(h, x, d, count=count, with_bias=False)
    assert h.last[1].count == count.data_ptr() and h.last[9] == 0
    first = torch.zeros(7, dtype=torch.int64)
    g = p.cdgrab_pergrad_linear(h, x.view(15, 8), d.view(15, 2), first=first, count=torch.zeros(7, dtype=torch.int32), tokens=4)
    t = h.last[1]
    assert (t.examples, t.rows, t.tokens, t.first) == (7, 15, 4, first.data_ptr()) and g.shape == (7, 18)
    for kw in ({"first": first}, {"first": first.int(), "tokens": 4}, {"first": first.view(1, 7), "tokens": 4},
               {"count": count.long()}, {"count": count[:2]}, {"tokens": 6}):
        with pytest.raises((ValueError, TypeError)):
            p.cdgrab_pergrad_linear(h, x, d, **kw)
    with pytest.raises(ValueError):
        p.cdgrab_pergrad_linear(h, x.view(15, 8), d.view(15, 2))
    for bad in (d[:2], d.half(), d.view(15, 2)):
        with pytest.raises(ValueError):
            p.cdgrab_pergrad_linear(h, x, bad)


def test_gradient_rows(p):
    h = HostHandle()
    x, dy = torch.zeros(3, 5, 8), torch.zeros(3, 5, 8)
    whole = torch.zeros(3, 100)
    dx, g = p.cdgrab_pergrad_layernorm(h, x, dy, G_out=whole[:, 7:23])
    assert g.data_ptr() == whole.data_ptr() + 28 and h.last[13] == g.data_ptr() and h.last[14] == 100 and dx.shape == x.shape
    assert p.cdgrab_pergrad_layernorm(h, x, dy, want_dx=False, with_bias=False)[1].shape == (3, 8) and h.last[10] is None
    assert p.cdgrab_pergrad_layernorm(h, x, dy, want_grads=False)[1] is None and h.last[13] is None
    for bad in (whole[:, :15], whole[:2, :16], whole[:, :16].double(), whole[:, :32:2]):
        with pytest.raises((ValueError, TypeError)):
            p.cdgrab_pergrad_layernorm(h, x, dy, G_out=bad)
    with pytest.raises(ValueError):
        p.cdgrab_pergrad_layernorm(h, x, dy, gain=torch.zeros(9))


def test_matrices(p):
    h = HostHandle()
    m = torch.zeros(4, 30, 50)
    o = p.cdgrab_orthogonalize(h, m[1:3, 2:22, 5:15], steps=3, coeffs=(1.5, -0.5, 0))
    a = h.last
    assert o.shape == (2, 20, 10) and a[1:5] == [2, 20, 10, 0] and a[6:8] == [50, 1500] and a[11:13] == [10, 200] and a[8] == 3
    assert isinstance(a[9], ctypes.Array) and list(a[9]) == [1.5, -0.5, 0.0]
    p.cdgrab_orthogonalize(h, m[0, :1])
    assert h.last[1:4] == [1, 1, 50] and h.last[9] is None
    for bad in (m.transpose(1, 2), m[0, 0], m.double()):
        with pytest.raises((ValueError, TypeError)):
            p.cdgrab_orthogonalize(h, bad)
    with pytest.raises(ValueError):
        p.cdgrab_orthogonalize(h, m, out=torch.zeros(4, 50, 30))
